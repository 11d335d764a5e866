// Kernels for cache rows of 4-bit blocks (S3_MXFP4, s3kv_fp4.h) of libs3kv, gfx950: the append that rounds new rows, and
// decode attention over the exactly widened codes (section 2.1, in fp32), for any number of query heads per cached head.
//
// Attention.  A wave streams tiles of 32 rows of one unit: 128 or 256 elements of a row, i.e. one head of 128 or 256, or two
// neighbouring heads of 64.  Both products run on the matrix cores (v_mfma_f32_16x16x32_bf16: e2m1 codes under a power of two are
// exact in bf16) with up to 16 query heads as columns, also for a single one: 17 bits hold four elements, so the vector ALU
// would need more instructions for them than the memory leaves time for.
//   S^T = K Q^T   A operand: lane (r, g) holds block g (32 elements, one scale) of row r as it lies in memory, a 16-byte load;
//                 the four products of a unit of 128 take a word of it each, Q^T in the same element order.  An fp16 query is
//                 the exact sum of two bf16 parts, two products.
//   O^T += V^T P^T  A operand: lane (m, g) holds elements 8m .. 8m+7 (256: 16m ..) of the eight rows 4g .. 4g+3 and 16+4g ..
//                 16+4g+3 of the tile, one word a row: after widening, pairs of rows are brought together by byte permutes, and
//                 output tile i gets the elements 8m + i.  No row passes through LDS.  The accumulator layout of S^T is the B
//                 operand of P^T as it is.  Weights enter as two bf16 parts (2^-17 of a weight off, below a rounding of a 16-bit
//                 output by 2^5 and more) or, for 32-bit outputs, as three (exact to fp32).
// The exponent reference of a column follows its maximum lazily (a tile's scores may exceed it by 8 in log2 units), so most
// tiles need no exchange between lanes.  Four waves of a workgroup split an item's rows, meet in LDS, and chunks of a context
// meet through memory as in the other kernels.
#include "s3kv_fp4.h"

// grid (n, 2): block (b, which) rounds one new row of H*D 16-bit elements into row off+pos; a thread has eight elements.
template <int ACT>
__global__ void __launch_bounds__(256) append_fp4_kernel(char *kplane, char *vplane, const int64_t *slot_off, const int32_t *pos,
                                                         const char *k_new, const char *v_new, int32_t row_elems, int64_t n_tokens,
                                                         int32_t max_len) {
    const int b = blockIdx.x;
    const int64_t off = slot_off[b];
    const int64_t p = pos[b];
    if (off < 0 || p < 0 || p >= max_len || off + p >= n_tokens) return;  // never leave the arena
    const char *src = (blockIdx.y ? v_new : k_new) + (int64_t)b * row_elems * 2;
    const int codes = row_elems / 2, row = (codes + row_elems / 32 + 15) & ~15;
    char *dst = (blockIdx.y ? vplane : kplane) + (off + p) * (int64_t)row;
    for (int i = threadIdx.x; i < row_elems / 8; i += 256) {  // (a block's four threads are neighbours and stay together)
        float x[8];
        widen8<ACT>(*(const u32x4 *)(src + (int64_t)i * 16), x);
        unsigned most = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) most = fp4_magnitude(x[e], most);
        most = group_max<4>(most);
        const unsigned byte = fp4_scale_byte<ACT>(__builtin_bit_cast(float, most));
        *(unsigned *)(dst + i * 4) = fp4_codes8(x, byte);
        if ((i & 3) == 0) *(unsigned char *)(dst + codes + i / 4) = (unsigned char)byte;
    }
    for (int i = codes + row_elems / 32 + threadIdx.x; i < row; i += 256) dst[i] = 0;
}

// A tile of 32 rows of a unit of W elements as a lane loads it.
template <int W>
struct Fp4Tile {
    static constexpr int T = W / 128;
    u32x4 k[2][T];       // rows r and 16 + r, block g (and 4 + g)
    unsigned ks[2][T];   // their scale bytes
    unsigned v[8][T];    // rows 4g + 0..3, 16 + 4g + 0..3
    unsigned vs[8];
};

// Where a lane's pieces of a tile are, in bytes from its first row.
struct Fp4Offsets {
    unsigned k[2], ks[2], v[8], vs[8];
};

// Rows of one plane from `base` on, `rows` of them; what lies past them reads as zeros and costs no traffic (a scale of 0 under codes
// of 0: no NaN comes from there).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const char *base, int rows, int row_bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, max(rows, 0) * row_bytes, 0x00020000);
}

template <int W>
__device__ __forceinline__ void load_tile(Fp4Tile<W> &t, const char *kbase, const char *vbase, int rows, int row_bytes, const Fp4Offsets &o) {
    constexpr int T = W / 128;
    const __amdgpu_buffer_rsrc_t kr = rows_from(kbase, rows, row_bytes), vr = rows_from(vbase, rows, row_bytes);
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
        for (int h = 0; h < T; h++) {
            t.k[u][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kr, o.k[u] + 64 * h, 0, 2));
            t.ks[u][h] = __builtin_amdgcn_raw_buffer_load_b8(kr, o.ks[u] + 4 * h, 0, 0);
        }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        if constexpr (W == 256) {
            const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(vr, o.v[e], 0, 2));
            t.v[e][0] = w[0];
            t.v[e][1] = w[1];
        } else {
            t.v[e][0] = __builtin_amdgcn_raw_buffer_load_b32(vr, o.v[e], 0, 2);
        }
        t.vs[e] = __builtin_amdgcn_raw_buffer_load_b8(vr, o.vs[e], 0, 0);
    }
}

__device__ __forceinline__ f32x4 mfma_bf16(const bf16x8 a, const bf16x8 b, const f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 pack_words(const unsigned a, const unsigned b, const unsigned c, const unsigned d) {
    const u32x4 w = {a, b, c, d};
    return __builtin_bit_cast(bf16x8, w);
}

// Eight codes of one word, widened: the A operand's slots of a lane.
__device__ __forceinline__ bf16x8 widen_word(const unsigned w, const float scale) {
    return pack_words(__builtin_bit_cast(unsigned, fp4_widen2<0>(w, scale)), __builtin_bit_cast(unsigned, fp4_widen2<1>(w, scale)),
                      __builtin_bit_cast(unsigned, fp4_widen2<2>(w, scale)), __builtin_bit_cast(unsigned, fp4_widen2<3>(w, scale)));
}

// Two fp32 numbers as a word of two bf16 (nearest, ties to even); what that leaves of them stays in x0, x1.
__device__ __forceinline__ unsigned take_bf16_part(float &x0, float &x1) {
    const bf16x2 h = {(__bf16)x0, (__bf16)x1};
    const unsigned w = __builtin_bit_cast(unsigned, h);
    const unsigned lo = w << 16, hi = w & 0xFFFF0000u;
    x0 -= __builtin_bit_cast(float, lo);
    x1 -= __builtin_bit_cast(float, hi);
    return w;
}

template <int B>
__device__ __forceinline__ void widen_pairs(const unsigned (&v)[8], const float (&vs)[8], bf16x8 &lo, bf16x8 &hi) {
    unsigned x[8], l[4], h[4];
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = __builtin_bit_cast(unsigned, fp4_widen2<B>(v[e], vs[e]));
#pragma unroll
    for (int e = 0; e < 4; e++) {  // (element 2B of rows 2e, 2e+1), (element 2B+1 of them)
        l[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x05040100u);
        h[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x07060302u);
    }
    lo = pack_words(l[0], l[1], l[2], l[3]);
    hi = pack_words(h[0], h[1], h[2], h[3]);
}

// What one wave does with the rows of a unit.  NH: heads of a unit (2 only for D = 64); NP: bf16 parts of a weight.
template <int ACT, int D, int NH, int NP>
struct Fp4Wave {
    static constexpr int W = D == 256 ? 256 : 128, T = W / 128;
    static constexpr int QP = ACT == S3_F16 ? 2 : 1;  // bf16 parts of a query
    static constexpr int QB = 16 / NH;                // columns of a head
    static constexpr int Q_BYTES = QP * T * 4 * 1024;  // of the queries in LDS

    const AttnArgs &a;
    char *q_lds;  // the queries, as the B operand takes them: [part][half][word][lane]
    int lane, r, g;
    int code_bytes, row_bytes;
    int kh0, qb, per_head;  // first cached head, block of query heads, query heads of a cached head in it
    bool second;            // the unit has two heads
    int ksub, vsub, qsub, kblk, vel, khead, vhead, qhead;
    int ko, kso, vo, vso;
    bool column, q_here;
    Fp4Offsets at_row;
    float m, l;
    f32x4 acc[8 * T];

    __device__ __forceinline__ Fp4Wave(const AttnArgs &args, char *lds) : a(args), q_lds(lds) {
        lane = threadIdx.x & 63;
        r = lane & 15;
        g = lane >> 4;
        code_bytes = fp4_code_bytes(a.H, D);
        row_bytes = fp4_row_bytes(a.H, D);
    }

    // Which heads: of the A operand's lanes (K: block group g; V: elements of lane m = r), of the B operand's columns.
    __device__ __forceinline__ void set_column(int col) {
        const int unit = a.nqb == 1 ? col : col / a.nqb;
        qb = col - unit * a.nqb;
        kh0 = unit * NH;
        second = NH == 2 && kh0 + 1 < a.H;
        per_head = min(a.group - qb * QB, QB);
        ksub = NH == 2 ? g >> 1 : 0;
        vsub = qsub = NH == 2 ? r >> 3 : 0;
        khead = kh0 + (second ? ksub : 0);
        vhead = kh0 + (second ? vsub : 0);
        kblk = D == 64 ? g & 1 : g;                             // (+ 4 for the second half of 256)
        vel = D == 256 ? 16 * r : D == 64 ? 8 * (r & 7) : 8 * r;  // first element of the V words
        ko = khead * (D / 2) + kblk * 16;
        kso = code_bytes + khead * (D / 32) + kblk;
        vo = vhead * (D / 2) + vel / 2;
        vso = code_bytes + vhead * (D / 32) + vel / 32;
        const int qi = (r % QB) + qb * QB;
        qhead = (kh0 + qsub) * a.group + qi;
        column = qi < a.group && (NH == 1 || qsub == 0 || second);
        q_here = column && (D != 64 || (NH == 2 ? ksub == qsub : g < 2));
#pragma unroll
        for (int u = 0; u < 2; u++) {
            at_row.k[u] = (16 * u + r) * row_bytes + ko;
            at_row.ks[u] = (16 * u + r) * row_bytes + kso;
        }
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const int row = (e & 3) + 4 * g + 16 * (e >> 2);
            at_row.v[e] = row * row_bytes + vo;
            at_row.vs[e] = row * row_bytes + vso;
        }
    }

    // Sequence b's queries into LDS (fp16: two exact bf16 parts); nothing folded in yet.
    __device__ __forceinline__ void begin(int b) {
        u32x4 w[T][4];
#pragma unroll
        for (int h = 0; h < T; h++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                w[h][i] = (u32x4){0u, 0u, 0u, 0u};
                if (q_here) w[h][i] = *(const u32x4 *)(a.q + (((int64_t)b * a.Hq + qhead) * D + h * 128 + kblk * 32 + i * 8) * 2);
            }
#pragma unroll
        for (int h = 0; h < T; h++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (QP == 1) {
                    put_query(0, h, i, w[h][i]);
                } else {
                    float x[8];
                    widen8<ACT>(w[h][i], x);
#pragma unroll
                    for (int part = 0; part < QP; part++) {
                        u32x4 p;
#pragma unroll
                        for (int e = 0; e < 4; e++) p[e] = take_bf16_part(x[2 * e], x[2 * e + 1]);
                        put_query(part, h, i, p);
                    }
                }
            }
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 8 * T; i++) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void put_query(int part, int h, int i, const u32x4 w) {
        *(u32x4 *)(q_lds + (((part * T + h) * 4 + i) * 64 + lane) * 16) = w;
    }
    __device__ __forceinline__ bf16x8 query(int part, int h, int i) const {
        return __builtin_bit_cast(bf16x8, *(const u32x4 *)(q_lds + (((part * T + h) * 4 + i) * 64 + lane) * 16));
    }

    __device__ __forceinline__ void load(Fp4Tile<W> &t, const char *kp, const char *vp, int rows) const {
        load_tile<W>(t, kp, vp, rows, row_bytes, at_row);
    }

    // What a tile holds is folded into (m, l, acc); rows: those of the tile and behind it (fewer than 32: the last tile).
    __device__ __forceinline__ void fold(const Fp4Tile<W> &t, int rows) {
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < T; h++) {
            const float scale[2] = {fp4_scale(t.ks[0][h]), fp4_scale(t.ks[1][h])};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                bf16x8 q[QP];
#pragma unroll
                for (int part = 0; part < QP; part++) q[part] = query(part, h, i);
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    const bf16x8 k8 = widen_word(t.k[u][h][i], scale[u]);
#pragma unroll
                    for (int part = 0; part < QP; part++) s[u] = mfma_bf16(k8, q[part], s[u]);
                }
            }
        }
        if (NH == 2 && __builtin_amdgcn_ballot_w64(t.ks[0][0] == 255u || t.ks[1][0] == 255u)) {
            // a block that reads as NaN must not reach the other head's columns (NaN times their zeros)
#pragma unroll
            for (int u = 0; u < 2; u++) {
                f32x4 c[2];
#pragma unroll
                for (int sub = 0; sub < 2; sub++) {
                    c[sub] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bf16x8 k8 = widen_word(ksub == sub ? t.k[u][0][i] : 0u, ksub == sub ? fp4_scale(t.ks[u][0]) : 1.f);
#pragma unroll
                        for (int part = 0; part < QP; part++) c[sub] = mfma_bf16(k8, query(part, 0, i), c[sub]);
                    }
                }
                s[u] = qsub ? c[1] : c[0];
            }
        }
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float one = s[e >> 2][e & 3];
            p[e] = one;
        }
        if (rows < 32) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (16 * (e >> 2) + 4 * g + (e & 3) >= rows) p[e] = -INFINITY;
        }
        const float mx = fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7]))) * a.scale_log2e;
        if (__builtin_amdgcn_ballot_w64(mx > m + 8.f)) {  // (also where there is no reference yet)
            const float mn = fmaxf(m, max_over_rows(mx));
            const float alpha = fast_exp2(m - exp_reference(mn));
            l *= alpha;
#pragma unroll
            for (int i = 0; i < 8 * T; i++) acc[i] *= alpha;
            m = mn;
        }
        const float ref = exp_reference(m);
#pragma unroll
        for (int e = 0; e < 8; e++) p[e] = fast_exp2(fmaf(p[e], a.scale_log2e, -ref));
        l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        bf16x8 pw[NP];
#pragma unroll
        for (int part = 0; part < NP; part++) {
            unsigned w[4];
#pragma unroll
            for (int e = 0; e < 4; e++) w[e] = take_bf16_part(p[2 * e], p[2 * e + 1]);
            pw[part] = pack_words(w[0], w[1], w[2], w[3]);
        }
        float vs[8];
#pragma unroll
        for (int e = 0; e < 8; e++) vs[e] = fp4_scale(t.vs[e]);
#pragma unroll
        for (int h = 0; h < T; h++) {
            unsigned v[8];
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = t.v[e][h];
            fold_pairs<0>(v, vs, pw, h);
            fold_pairs<1>(v, vs, pw, h);
            fold_pairs<2>(v, vs, pw, h);
            fold_pairs<3>(v, vs, pw, h);
        }
    }
    template <int B>
    __device__ __forceinline__ void fold_pairs(const unsigned (&v)[8], const float (&vs)[8], const bf16x8 (&pw)[NP], int h) {
        bf16x8 lo, hi;
        widen_pairs<B>(v, vs, lo, hi);
#pragma unroll
        for (int part = 0; part < NP; part++) {
            acc[8 * h + 2 * B] = mfma_bf16(lo, pw[part], acc[8 * h + 2 * B]);
            acc[8 * h + 2 * B + 1] = mfma_bf16(hi, pw[part], acc[8 * h + 2 * B + 1]);
        }
    }

    // A decode step's new row, still 16-bit, as the last of a tile's `rows` rows: its blocks are rounded by the lanes that use them and
    // written to the arena (row `row`) by those that own the bytes.
    __device__ __forceinline__ void take_new_row(Fp4Tile<W> &t, int b, int64_t row, int rows) const {
        const int64_t at = row * row_bytes;
        const bool k_own = r == 0 && (D != 64 || (NH == 2 ? ksub == 0 || second : g < 2));
        const bool v_own = g == 0 && (D != 64 || (NH == 2 ? vsub == 0 || second : r < 8));
        const char *ksrc = a.k_new + (((int64_t)b * a.H + khead) * D + kblk * 32) * 2;
        const char *vsrc = a.v_new + (((int64_t)b * a.H + vhead) * D + vel) * 2;
#pragma unroll
        for (int h = 0; h < T; h++) {
            float x[4][8];
            unsigned most = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                widen8<ACT>(*(const u32x4 *)(ksrc + h * 256 + i * 16), x[i]);
#pragma unroll
                for (int e = 0; e < 8; e++) most = fp4_magnitude(x[i][e], most);
            }
            const unsigned byte = fp4_scale_byte<ACT>(__builtin_bit_cast(float, most));
            u32x4 c;
#pragma unroll
            for (int i = 0; i < 4; i++) c[i] = fp4_codes8(x[i], byte);
            if (k_own) {
                *(u32x4 *)(a.kplane + at + ko + 64 * h) = c;
                *(unsigned char *)(a.kplane + at + kso + 4 * h) = (unsigned char)byte;
            }
#pragma unroll
            for (int u = 0; u < 2; u++)
                if (16 * u + r >= rows - 1) {
                    t.k[u][h] = c;
                    t.ks[u][h] = byte;
                }
        }
        float x[T][8];
        unsigned most = 0;
#pragma unroll
        for (int h = 0; h < T; h++) {
            widen8<ACT>(*(const u32x4 *)(vsrc + h * 16), x[h]);
#pragma unroll
            for (int e = 0; e < 8; e++) most = fp4_magnitude(x[h][e], most);
        }
        most = group_max<4 / T>(most);
        const unsigned byte = fp4_scale_byte<ACT>(__builtin_bit_cast(float, most));
#pragma unroll
        for (int h = 0; h < T; h++) {
            const unsigned c = fp4_codes8(x[h], byte);
            if (v_own) *(unsigned *)(a.vplane + at + vo + 4 * h) = c;
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (16 * (e >> 2) + 4 * g + (e & 3) >= rows - 1) t.v[e][h] = c;
        }
        if (v_own && vel % 32 == 0) *(unsigned char *)(a.vplane + at + vso) = (unsigned char)byte;
        const int used = code_bytes + a.H * (D / 32);
        if (kh0 + NH >= a.H && lane < row_bytes - used) {  // zeros up to a multiple of 16 bytes
            a.kplane[at + used + lane] = 0;
            a.vplane[at + used + lane] = 0;
        }
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (16 * (e >> 2) + 4 * g + (e & 3) >= rows - 1) t.vs[e] = byte;
    }

    // Four neighbouring elements of this lane's column, i < 2T, rr < 4: elements 8T * (4g + rr) + 4i .. + 3 of the unit.
    __device__ __forceinline__ f32x4 sums4(int rr, int i) const {
        f32x4 o;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float one = acc[4 * i + e][rr];
            o[e] = one;
        }
        return o;
    }
};

// The new lengths, and a zero output row for empty or refused contexts, by the workgroups in turn.
template <int D>
__device__ __forceinline__ void publish_lengths(const AttnArgs &a, const BatchView &bv) {
    for (int b = blockIdx.x; b < a.n; b += gridDim.x) {
        if (a.len_out && threadIdx.x == 0) a.len_out[b] = a.cur_len[b] + 1;
        if (bv.len[b] == 0) {
            const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int e = threadIdx.x; e < a.Hq * D / 8; e += 256) store_out8(a.out, a.out_dtype, ((int64_t)b * a.Hq * D / 8 + e) * 8, z);
        }
    }
}

// Few (context, column) pairs: an item is a chunk of a context for a column, its rows shared out over the four waves of a workgroup,
// which meet in LDS; chunks meet through memory.
template <int ACT, int D, int NH, int NP>
__global__ void __launch_bounds__(256, 2) attn_fp4_team_kernel(const AttnArgs a) {
    typedef Fp4Wave<ACT, D, NH, NP> Wave;
    constexpr int W = Wave::W, T = Wave::T, QB = Wave::QB, TS = 4;
    constexpr int STRIDE = W + 4;  // floats of a column in LDS
    extern __shared__ __align__(16) char dyn_lds[];  // the batch view, the queries, then the waves' sums of the columns in use
    __shared__ int wave_sums[S3_MAX_CLASSES * S3_MAX_WAVES];
    __shared__ float comb_m[TS][16], comb_l[TS][16];
    __shared__ int last_of_context;
    const int ts = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (scalar: row ranges and buffers with it)
    const BatchView bv = build_batch_view<false>(a, dyn_lds, wave_sums);
    char *queries = dyn_lds + ((batch_view_bytes(a.n, a.ncls) + 15) & ~(size_t)15);
    float *comb = (float *)(queries + Wave::Q_BYTES);
    publish_lengths<D>(a, bv);
    Wave w(a, queries);  // (the waves have the same queries: each writes all of them, so none waits for another)
    const int row_bytes = w.row_bytes;
    // Work in the order of eighths: workgroup b (XCD b % 8) takes the chunks whose number leaves the same remainder, so that the
    // columns of a chunk, whose bytes share cache lines, are on one XCD's L2.
    const int64_t total = (int64_t)((bv.total + 7) / 8) * 8 * a.columns;
    for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
        const int64_t y = at >> 3;
        const int64_t chunk_no = (y / a.columns) * 8 + (at & 7);
        if (chunk_no >= bv.total) continue;
        const int col = (int)(y % a.columns);
        const Item it = uniform_item(decode_item(a, bv, chunk_no, 1));
        const int start = it.c * it.clen, end = min(it.len, start + it.clen);
        const int per = (end - start + TS - 1) / TS;
        const int j0 = min(end, start + ts * per), j1 = min(end, j0 + per);
        const bool has_new = a.k_new != nullptr && j1 == it.len && j0 < j1;
        w.set_column(col);
        const char *kp = a.kplane + (it.off + j0) * (int64_t)row_bytes, *vp = a.vplane + (it.off + j0) * (int64_t)row_bytes;
        const int64_t step = 32 * (int64_t)row_bytes, new_row = it.off + it.len - 1;
        // Two tiles' registers in turn, so that the next tile's loads are out while one is folded in.
        Fp4Tile<W> t0, t1;
        w.load(t0, kp, vp, j1 - j0);
        w.begin(it.b);
        for (int left = j1 - j0; left > 0; left -= 64) {
            w.load(t1, kp + step, vp + step, left - 32);
            if (has_new && left <= 32) w.take_new_row(t0, it.b, new_row, left);
            w.fold(t0, left);
            if (left <= 32) break;
            kp += 2 * step;
            vp += 2 * step;
            w.load(t0, kp, vp, left - 64);
            if (has_new && left <= 64) w.take_new_row(t1, it.b, new_row, left - 32);
            w.fold(t1, left - 32);
        }

        // the four waves meet: columns in use, compact (head, query)
        const int slot = w.qsub * w.per_head + (w.r % QB), n_cols = (w.second ? 2 : 1) * w.per_head;
        const float l = sum_over_rows(w.l);
        if (w.column && w.g == 0) {
            comb_m[ts][slot] = w.m;
            comb_l[ts][slot] = l;
        }
        if (w.column) {
#pragma unroll
            for (int rr = 0; rr < 4; rr++)
#pragma unroll
                for (int i = 0; i < 2 * T; i++)
                    *(f32x4 *)(comb + ((size_t)ts * n_cols + slot) * STRIDE + 8 * T * (4 * w.g + rr) + 4 * i) = w.sums4(rr, i);
        }
        __syncthreads();
        // a thread: eight elements of one column
        const int slices = n_cols * (D / 8);
        for (int i = threadIdx.x; i < slices; i += 256) {
            const int c = i / (D / 8), dl = i % (D / 8), sub = NH == 2 && c >= w.per_head ? 1 : 0;
            const int h = (w.kh0 + sub) * a.group + w.qb * QB + (c - sub * w.per_head);
            float mm = -INFINITY, ll = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < TS; x++) mm = fmaxf(mm, comb_m[x][c]);
            const float ref = exp_reference(mm);
#pragma unroll
            for (int x = 0; x < TS; x++) {
                const float wt = fast_exp2(comb_m[x][c] - ref);
                ll += wt * comb_l[x][c];
                const float *src = comb + ((size_t)x * n_cols + c) * STRIDE + sub * 64 + dl * 8;
                const f32x4 x0 = *(const f32x4 *)src, x1 = *(const f32x4 *)(src + 4);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    o[e] += wt * x0[e];
                    o[4 + e] += wt * x1[e];
                }
            }
            if (it.nchunks <= 1) {
                const float inv = 1.f / ll;
#pragma unroll
                for (int e = 0; e < 8; e++) o[e] *= inv;
                store_out8(a.out, a.out_dtype, ((int64_t)it.b * a.Hq + h) * D + dl * 8, o);
            } else {  // a chunk of a longer context: the partial goes out with write-through stores
                const int64_t pi = (int64_t)(it.slot0 + it.c) * a.Hq + h;
                if (dl == 0) put_partial2<true>((float *)a.part_ml + 2 * pi, (f32x2){mm, ll});
                float *pa = a.part_acc + pi * D + dl * 8;
                put_partial4<true>(pa, (f32x4){o[0], o[1], o[2], o[3]});
                put_partial4<true>(pa + 4, (f32x4){o[4], o[5], o[6], o[7]});
            }
        }
        if (it.nchunks > 1) {
            // every wave's partial stores are complete before the count, which the first wave makes for all
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __syncthreads();
            if (ts == 0) {
                const bool last = chunk_arrived(a, arrival_counter(a, it.b, a.columns, col), it.nchunks);
                if (w.lane == 0) last_of_context = last;
            }
            __syncthreads();
            if (last_of_context) {
                if (a.merge_sync) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
                for (int i = threadIdx.x; i < slices; i += 256) {
                    const int c = i / (D / 8), dl = i % (D / 8), sub = NH == 2 && c >= w.per_head ? 1 : 0;
                    merge_chunks<D, true>(a, it.slot0, a.Hq, it.b, (w.kh0 + sub) * a.group + w.qb * QB + (c - sub * w.per_head), dl, it.nchunks);
                }
            }
        }
        __syncthreads();  // LDS is used again by the next item
    }
}

// Many (context, column) pairs: the tiles of all contexts laid end to end are cut into equal shares, one a wave and column, so that
// waves end together whatever the lengths, and no wave waits for another.  A share runs through whole contexts, which it finishes by
// itself, and at either end through a part of one that others share: such a piece goes to memory (share u's piece of context b to slot
// u + b: along the shares either u or b grows, so no two meet), is counted, and whoever counts the last piece of a context merges them.
// Contexts of few tiles are not cut: a share takes those that begin in it.
#define S3_FP4_UNCUT 8
template <int ACT, int D, int NH, int NP>
__global__ void __launch_bounds__(256, 2) attn_fp4_share_kernel(const AttnArgs a) {
    typedef Fp4Wave<ACT, D, NH, NP> Wave;
    constexpr int W = Wave::W, T = Wave::T, QB = Wave::QB;
    extern __shared__ __align__(16) char dyn_lds[];  // the batch view in tiles, then the waves' queries
    __shared__ int wave_sums[3 * S3_MAX_WAVES];
    int longest = 0;
    const BatchView bv = build_tile_view<32>(a, dyn_lds, wave_sums, longest);
    char *queries = dyn_lds + ((batch_view_bytes(a.n, 1) + 15) & ~(size_t)15);
    publish_lengths<D>(a, bv);
    const int ts = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Neighbouring columns, whose bytes share cache lines, are on neighbouring waves, and those on one XCD (workgroup b is on XCD b % 8).
    const int rank = (gridDim.x & 7) == 0 ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;
    const int place = rank * 4 + ts;
    const int share = place / a.columns, col = place - share * a.columns;
    const int total = __builtin_amdgcn_readfirstlane(bv.total);
    const bool cut = __builtin_amdgcn_readfirstlane(longest) > 32 * S3_FP4_UNCUT;
    const int size = max((total + a.wave_shares - 1) / a.wave_shares, 1);
    if (share >= a.wave_shares || share * (int64_t)size >= total) return;
    int t0 = share * size, t1 = min(total, t0 + size);
    int b = __builtin_amdgcn_readfirstlane(find_sequence(bv.pre, a.n, t0));  // the context that holds tile t0
    if (!cut) {  // from the first context that begins at t0 or behind it to the last that begins in front of t1
        if (__builtin_amdgcn_readfirstlane(bv.pre[b]) < t0) b++;
        t0 = __builtin_amdgcn_readfirstlane(bv.pre[b]);
        if (t0 >= t1) return;
        t1 = __builtin_amdgcn_readfirstlane(bv.pre[find_sequence(bv.pre, a.n, t1 - 1) + 1]);
    }
    Wave w(a, queries + ts * Wave::Q_BYTES);
    w.set_column(col);
    const int row_bytes = w.row_bytes;
    Pending head = {0, 0, 0}, tail = {0, 0, 0};  // pieces of the contexts that the share's borders cut

    // the loader: context, its first tile, rows from the tile to load on (0: the share is loaded)
    struct Cursor {
        int b, begin, end;  // tiles of context b
        int tile, len;
        int64_t off;
    };
    const auto open = [&](Cursor &c, int tile) {  // the context that holds `tile`, from context c.b on
        while (true) {
            c.end = __builtin_amdgcn_readfirstlane(bv.pre[c.b + 1]);
            if (tile < c.end) break;
            c.b++;
        }
        c.begin = __builtin_amdgcn_readfirstlane(bv.pre[c.b]);
        c.len = __builtin_amdgcn_readfirstlane(bv.len[c.b]);
        c.off = uniform64(bv.off[c.b]);
        c.tile = tile;
    };
    const auto load = [&](Fp4Tile<W> &t, const Cursor &c, bool there) {
        const int64_t row = c.off + (int64_t)(c.tile - c.begin) * 32;
        w.load(t, a.kplane + row * row_bytes, a.vplane + row * row_bytes, there ? c.len - (c.tile - c.begin) * 32 : 0);
    };
    const auto finish = [&](const Cursor &c) {  // the share's part of context c.b is folded in
        const int first = max(c.begin, t0), last = min(c.end, t1);
        const float l = sum_over_rows(w.l);
        const bool mine = w.column && (D != 64 || (NH == 2 ? (w.g >> 1) == w.qsub : w.g < 2));
        const int e0 = 8 * T * 4 * w.g - (NH == 2 ? 64 * w.qsub : 0);  // this lane's first element of its head
        if (first == c.begin && last == c.end) {
            const float inv = 1.f / l;
            if (mine) {
#pragma unroll
                for (int rr = 0; rr < 4; rr++)
#pragma unroll
                    for (int i = 0; i < T; i++) {
                        const f32x4 lo = w.sums4(rr, 2 * i), hi = w.sums4(rr, 2 * i + 1);
                        const float o[8] = {lo[0] * inv, lo[1] * inv, lo[2] * inv, lo[3] * inv, hi[0] * inv, hi[1] * inv, hi[2] * inv, hi[3] * inv};
                        store_out8(a.out, a.out_dtype, ((int64_t)c.b * a.Hq + w.qhead) * D + e0 + 8 * T * rr + 8 * i, o);
                    }
            }
            return;
        }
        const int u0 = c.begin / size, u1 = (c.end - 1) / size;
        const Pending p = {c.b, u0, u1 - u0 + 1};
        if (first == t0) head = p;
        else tail = p;
        if (mine) {
            const int64_t pi = (int64_t)(share + c.b) * a.Hq + w.qhead;
            if (e0 == 0) put_partial2<true>((float *)a.part_ml + 2 * pi, (f32x2){w.m, l});
            float *pa = a.part_acc + pi * D + e0;
#pragma unroll
            for (int rr = 0; rr < 4; rr++)
#pragma unroll
                for (int i = 0; i < 2 * T; i++) put_partial4<true>(pa + 8 * T * rr + 4 * i, w.sums4(rr, i));
        }
    };
    // one tile: the next one's loads leave, then this one is folded in
    Cursor now;
    now.b = b;
    open(now, t0);
    const auto advance = [&](const Cursor &c, Fp4Tile<W> &t) {
        Cursor n = c;
        const bool there = c.tile + 1 < t1;
        if (there) {
            if (c.tile + 1 < c.end) n.tile++;
            else open(n, c.tile + 1);
        }
        load(t, n, there);
        return n;
    };
    const auto one = [&](Fp4Tile<W> &t, const Cursor &c, int next_b) {
        const int rows = c.len - (c.tile - c.begin) * 32;
        if (a.k_new != nullptr && rows <= 32) w.take_new_row(t, c.b, c.off + c.len - 1, rows);
        w.fold(t, rows);
        const bool last = c.tile + 1 == t1;
        if (last || c.tile + 1 == c.end) {
            finish(c);
            if (!last) w.begin(next_b);
        }
    };
    Fp4Tile<W> ta, tb;
    load(ta, now, true);
    w.begin(now.b);
    while (true) {
        Cursor next = advance(now, tb);
        one(ta, now, next.b);
        if (now.tile + 1 >= t1) break;
        now = advance(next, ta);
        one(tb, next, now.b);
        if (next.tile + 1 >= t1) break;
    }
    if (head.count + tail.count == 0) return;
    const unsigned who = pieces_arrived(a, head, tail, a.columns, col);
#pragma unroll 1
    for (int k = 0; k < 2; k++) {
        if (!(who >> k & 1)) continue;
        const Pending p = {k ? tail.b : head.b, k ? tail.first : head.first, k ? tail.count : head.count};
        const int slices = (w.second ? 2 : 1) * w.per_head * (D / 8);
        for (int i = w.lane; i < slices; i += 64) {
            const int c = i / (D / 8), dl = i % (D / 8), sub = NH == 2 && c >= w.per_head ? 1 : 0;
            merge_chunks<D, true>(a, p.first + p.b, a.Hq, p.b, (w.kh0 + sub) * a.group + w.qb * QB + (c - sub * w.per_head), dl, p.count);
        }
    }
}

template <int ACT, int NP, bool SHARES>
static attn_fn pick_fp4(int d, int nh) {
    if (SHARES) {
        if (d == 64) return nh == 2 ? attn_fp4_share_kernel<ACT, 64, 2, NP> : attn_fp4_share_kernel<ACT, 64, 1, NP>;
        return d == 128 ? attn_fp4_share_kernel<ACT, 128, 1, NP> : d == 256 ? attn_fp4_share_kernel<ACT, 256, 1, NP> : nullptr;
    }
    if (d == 64) return nh == 2 ? attn_fp4_team_kernel<ACT, 64, 2, NP> : attn_fp4_team_kernel<ACT, 64, 1, NP>;
    return d == 128 ? attn_fp4_team_kernel<ACT, 128, 1, NP> : d == 256 ? attn_fp4_team_kernel<ACT, 256, 1, NP> : nullptr;
}

attn_fn s3i_pick_fp4(int act, int d, int heads_per_unit, bool wide_out, bool shares, int *query_bytes) {
    *query_bytes = (shares ? 4 : 1) * (act == S3_F16 ? 2 : 1) * (d == 256 ? 2 : 1) * 4096;
    if (act == S3_F16) {
        if (wide_out) return shares ? pick_fp4<S3_F16, 3, true>(d, heads_per_unit) : pick_fp4<S3_F16, 3, false>(d, heads_per_unit);
        return shares ? pick_fp4<S3_F16, 2, true>(d, heads_per_unit) : pick_fp4<S3_F16, 2, false>(d, heads_per_unit);
    }
    if (wide_out) return shares ? pick_fp4<S3_BF16, 3, true>(d, heads_per_unit) : pick_fp4<S3_BF16, 3, false>(d, heads_per_unit);
    return shares ? pick_fp4<S3_BF16, 2, true>(d, heads_per_unit) : pick_fp4<S3_BF16, 2, false>(d, heads_per_unit);
}

append_fp8_fn s3i_pick_append_fp4(int act) {
    return act == S3_F16 ? append_fp4_kernel<S3_F16> : act == S3_BF16 ? append_fp4_kernel<S3_BF16> : nullptr;
}
