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

template <int D, int NH>
struct Fp4Lane {  // byte offsets of a lane within a row
    int k, ks, v, vs;
};

template <int W>
__device__ __forceinline__ unsigned load_v_words(const char *p, unsigned (&v)[W / 128]) {
    if constexpr (W == 256) {
        const u32x2 w = __builtin_nontemporal_load((const u32x2 *)p);
        v[0] = w[0];
        v[1] = w[1];
    } else {
        v[0] = __builtin_nontemporal_load((const unsigned *)p);
    }
    return 0;
}

// rows: how many rows of the tile there are (32 but for the last tile: rows past the end read the last one again).
template <int W, bool FULL>
__device__ __forceinline__ void load_tile(Fp4Tile<W> &t, const char *kbase, const char *vbase, int row_bytes, int rows, int ko, int kso, int vo,
                                          int vso) {
    constexpr int T = W / 128;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const int row = FULL ? 16 * u + r : min(16 * u + r, rows - 1);
        const unsigned at = (unsigned)(row * row_bytes);
#pragma unroll
        for (int h = 0; h < T; h++) {
            t.k[u][h] = __builtin_nontemporal_load((const u32x4 *)(kbase + at + ko + 64 * h));
            t.ks[u][h] = *(const unsigned char *)(kbase + at + kso + 4 * h);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const int want = (e & 3) + 4 * g + 16 * (e >> 2);
        const int row = FULL ? want : min(want, rows - 1);
        const unsigned at = (unsigned)(row * row_bytes);
        load_v_words<W>(vbase + at + vo, t.v[e]);
        t.vs[e] = *(const unsigned char *)(vbase + at + vso);
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

// NH: heads of a unit (2 only for D = 64); QP: bf16 parts of a query; NP: bf16 parts of a weight.
template <int ACT, int D, int NH, int NP>
__global__ void __launch_bounds__(256, 2) attn_fp4_kernel(const AttnArgs a) {
    constexpr int W = D == 256 ? 256 : 128, T = W / 128, TS = 4;
    constexpr int QP = ACT == S3_F16 ? 2 : 1;
    constexpr int QB = 16 / NH;              // columns of a head
    constexpr int STRIDE = W + 4;            // floats of a column in LDS
    extern __shared__ __align__(16) char dyn_lds[];  // the batch view, then the waves' sums of the columns in use
    __shared__ int wave_sums[S3_MAX_CLASSES * S3_MAX_WAVES];
    __shared__ float comb_m[TS][16], comb_l[TS][16];
    __shared__ int last_of_context;
    const int lane = threadIdx.x & 63, ts = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const BatchView bv = build_batch_view<false>(a, dyn_lds, wave_sums);
    float *comb = (float *)(dyn_lds + ((batch_view_bytes(a.n, a.ncls) + 15) & ~(size_t)15));
    // the new lengths, and a zero output row for empty or refused contexts, by the workgroups in turn
    for (int b = blockIdx.x; b < a.n; b += gridDim.x) {
        if (a.len_out && threadIdx.x == 0) a.len_out[b] = a.cur_len[b] + 1;
        if (bv.len[b] == 0) {
            const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int e = threadIdx.x; e < a.Hq * D / 8; e += 256) store_out8(a.out, a.out_dtype, ((int64_t)b * a.Hq * D / 8 + e) * 8, z);
        }
    }
    const int code_bytes = fp4_code_bytes(a.H, D), row_bytes = fp4_row_bytes(a.H, D);
    // Work in the order of eighths: workgroup b (XCD b % 8) takes the chunks whose number leaves the same remainder, so that the
    // columns of a chunk, whose bytes share cache lines, are on one XCD's L2.
    const int64_t total = (int64_t)((bv.total + 7) / 8) * 8 * a.columns;
    for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
        const int64_t y = at >> 3;
        const int64_t chunk_no = (y / a.columns) * 8 + (at & 7);
        if (chunk_no >= bv.total) continue;
        const int col = (int)(y % a.columns);
        const Item it = uniform_item(decode_item(a, bv, chunk_no, 1));
        const int unit = col / a.nqb, qb = col - unit * a.nqb;
        const int start = it.c * it.clen, end = min(it.len, start + it.clen);
        const int per = (end - start + TS - 1) / TS;
        const int j0 = min(end, start + ts * per), j1 = min(end, j0 + per);
        const bool has_new = a.k_new != nullptr && j1 == it.len && j0 < j1;

        // which heads: of the A operand's lanes (K: block group g; V: elements of lane m = r), of the B operand's columns
        const int ksub = NH == 2 ? g >> 1 : 0, vsub = NH == 2 ? r >> 3 : 0, qsub = NH == 2 ? r >> 3 : 0;
        const int kh0 = unit * NH;
        const bool second = NH == 2 && kh0 + 1 < a.H;
        const int khead = kh0 + (second ? ksub : 0), vhead = kh0 + (second ? vsub : 0);
        const int kblk = D == 64 ? g & 1 : g;                // (+ 4 for the second half of 256)
        const int vel = D == 256 ? 16 * r : D == 64 ? 8 * (r & 7) : 8 * r;  // first element of the V words
        const int ko = khead * (D / 2) + kblk * 16, kso = code_bytes + khead * (D / 32) + kblk;
        const int vo = vhead * (D / 2) + vel / 2, vso = code_bytes + vhead * (D / 32) + vel / 32;
        const int qi = (r % QB) + qb * QB, qhead = (kh0 + qsub) * a.group + qi;
        const bool column = qi < a.group && (NH == 1 || qsub == 0 || second);
        const bool q_here = column && (D != 64 || (NH == 2 ? ksub == qsub : g < 2));

        bf16x8 q[QP][T][4];
#pragma unroll
        for (int h = 0; h < T; h++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                u32x4 w = {0u, 0u, 0u, 0u};
                if (q_here) w = *(const u32x4 *)(a.q + (((int64_t)it.b * a.Hq + qhead) * D + h * 128 + kblk * 32 + i * 8) * 2);
                if (QP == 1) {
                    q[0][h][i] = __builtin_bit_cast(bf16x8, w);
                } else {
                    float x[8];
                    widen8<ACT>(w, x);
                    unsigned p[QP][4];
#pragma unroll
                    for (int part = 0; part < QP; part++)
#pragma unroll
                        for (int e = 0; e < 4; e++) p[part][e] = take_bf16_part(x[2 * e], x[2 * e + 1]);
#pragma unroll
                    for (int part = 0; part < QP; part++) q[part][h][i] = pack_words(p[part][0], p[part][1], p[part][2], p[part][3]);
                }
            }

        float m = -INFINITY, l = 0.f;
        f32x4 acc[8 * T];
#pragma unroll
        for (int i = 0; i < 8 * T; i++) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};

        const char *kp = a.kplane + (it.off + j0) * (int64_t)row_bytes, *vp = a.vplane + (it.off + j0) * (int64_t)row_bytes;
        // what a tile holds is folded into (m, l, acc); rows: 32, or fewer in the last tile
        auto fold = [&](const Fp4Tile<W> &t, int rows, bool full) {
            f32x4 s[2];
#pragma unroll
            for (int u = 0; u < 2; u++) {
                f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < T; h++) {
                    const float scale = fp4_scale(t.ks[u][h]);
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bf16x8 k8 = widen_word(t.k[u][h][i], scale);
#pragma unroll
                        for (int part = 0; part < QP; part++) c = mfma_bf16(k8, q[part][h][i], c);
                    }
                }
                s[u] = c;
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
                            for (int part = 0; part < QP; part++) c[sub] = mfma_bf16(k8, q[part][0][i], c[sub]);
                        }
                    }
                    s[u] = qsub ? c[1] : c[0];
                }
            }
            float p[8], mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                p[e] = s[e >> 2][e & 3] * a.scale_log2e;
                if (!full && 16 * (e >> 2) + 4 * g + (e & 3) >= rows) p[e] = -INFINITY;
                mx = fmaxf(mx, p[e]);
            }
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
            for (int e = 0; e < 8; e++) {
                p[e] = fast_exp2(p[e] - ref);
                l += p[e];
            }
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
                bf16x8 lo, hi;
#define S3_FP4_PAIR(B)                                                                            \
    widen_pairs<B>(v, vs, lo, hi);                                                                \
    _Pragma("unroll") for (int part = 0; part < NP; part++) {                                     \
        acc[8 * h + 2 * B] = mfma_bf16(lo, pw[part], acc[8 * h + 2 * B]);                         \
        acc[8 * h + 2 * B + 1] = mfma_bf16(hi, pw[part], acc[8 * h + 2 * B + 1]);                 \
    }
                S3_FP4_PAIR(0)
                S3_FP4_PAIR(1)
                S3_FP4_PAIR(2)
                S3_FP4_PAIR(3)
#undef S3_FP4_PAIR
            }
        };
        Fp4Tile<W> t0, t1;
        const int rows_all = j1 - j0, full_tiles = max(0, rows_all - (has_new ? 1 : 0)) / 32;
        const int tail = rows_all - 32 * full_tiles;  // 0 .. 32 rows, the new one among them
        if (full_tiles > 0) {
            load_tile<W, true>(t0, kp, vp, row_bytes, 32, ko, kso, vo, vso);
            for (int i = 0; i < full_tiles; i += 2) {
                if (i + 1 < full_tiles) load_tile<W, true>(t1, kp + (int64_t)(i + 1) * 32 * row_bytes, vp + (int64_t)(i + 1) * 32 * row_bytes, row_bytes, 32, ko, kso, vo, vso);
                fold(t0, 32, true);
                if (i + 1 >= full_tiles) break;
                if (i + 2 < full_tiles) load_tile<W, true>(t0, kp + (int64_t)(i + 2) * 32 * row_bytes, vp + (int64_t)(i + 2) * 32 * row_bytes, row_bytes, 32, ko, kso, vo, vso);
                fold(t1, 32, true);
            }
        }
        if (tail > 0) {
            const int64_t skip = (int64_t)full_tiles * 32 * row_bytes;
            load_tile<W, false>(t0, kp + skip, vp + skip, row_bytes, tail, ko, kso, vo, vso);
            if (has_new) {
                // The new row, still 16-bit: its blocks are rounded by the lanes that use them and written to the arena by those
                // that own the bytes; rows tail-1 and beyond of the tile read it.
                const int64_t row = (it.off + it.len - 1) * (int64_t)row_bytes;
                const bool k_own = r == 0 && (D != 64 || (NH == 2 ? ksub == 0 || second : g < 2));
                const bool v_own = g == 0 && (D != 64 || (NH == 2 ? vsub == 0 || second : r < 8));
                const char *ks = a.k_new + (((int64_t)it.b * a.H + khead) * D + kblk * 32) * 2;
                const char *vsrc = a.v_new + (((int64_t)it.b * a.H + vhead) * D + vel) * 2;
#pragma unroll
                for (int h = 0; h < T; h++) {
                    float x[4][8];
                    unsigned most = 0;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        widen8<ACT>(*(const u32x4 *)(ks + h * 256 + i * 16), x[i]);
#pragma unroll
                        for (int e = 0; e < 8; e++) most = fp4_magnitude(x[i][e], most);
                    }
                    const unsigned byte = fp4_scale_byte<ACT>(__builtin_bit_cast(float, most));
                    u32x4 c;
#pragma unroll
                    for (int i = 0; i < 4; i++) c[i] = fp4_codes8(x[i], byte);
                    if (k_own) {
                        *(u32x4 *)(a.kplane + row + ko + 64 * h) = c;
                        *(unsigned char *)(a.kplane + row + kso + 4 * h) = (unsigned char)byte;
                    }
#pragma unroll
                    for (int u = 0; u < 2; u++)
                        if (16 * u + r >= tail - 1) {
                            t0.k[u][h] = c;
                            t0.ks[u][h] = byte;
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
                    if (v_own) *(unsigned *)(a.vplane + row + vo + 4 * h) = c;
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (16 * (e >> 2) + 4 * g + (e & 3) >= tail - 1) t0.v[e][h] = c;
                }
                if (v_own && vel % 32 == 0) *(unsigned char *)(a.vplane + row + vso) = (unsigned char)byte;
                const int used = code_bytes + a.H * (D / 32);
                if (kh0 + NH >= a.H && lane < row_bytes - used) {  // zeros up to a multiple of 16 bytes
                    a.kplane[row + used + lane] = 0;
                    a.vplane[row + used + lane] = 0;
                }
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (16 * (e >> 2) + 4 * g + (e & 3) >= tail - 1) t0.vs[e] = byte;
            }
            fold(t0, tail, false);
        }

        // the four waves meet: columns in use, compact (head, query)
        const int per_head = min(a.group - qb * QB, QB);
        const int slot = qsub * per_head + (r % QB), n_cols = (second ? 2 : 1) * per_head;
        l = sum_over_rows(l);
        if (column && g == 0) {
            comb_m[ts][slot] = m;
            comb_l[ts][slot] = l;
        }
        if (column) {
#pragma unroll
            for (int rr = 0; rr < 4; rr++)
#pragma unroll
                for (int h = 0; h < 2 * T; h++) {
                    // elements 8T * (4g + rr) + 4h .. + 3 of the unit
                    f32x4 o;
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const float one = acc[4 * h + e][rr];
                        o[e] = one;
                    }
                    *(f32x4 *)(comb + ((size_t)ts * n_cols + slot) * STRIDE + 8 * T * (4 * g + rr) + 4 * h) = o;
                }
        }
        __syncthreads();
        // a thread: eight elements of one column
        const int slices = n_cols * (D / 8);
        for (int i = threadIdx.x; i < slices; i += 256) {
            const int c = i / (D / 8), dl = i % (D / 8), sub = NH == 2 && c >= per_head ? 1 : 0;
            const int h = (kh0 + sub) * a.group + qb * QB + (c - sub * per_head);
            float mm = -INFINITY, ll = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < TS; w++) mm = fmaxf(mm, comb_m[w][c]);
            const float ref = exp_reference(mm);
#pragma unroll
            for (int w = 0; w < TS; w++) {
                const float wt = fast_exp2(comb_m[w][c] - ref);
                ll += wt * comb_l[w][c];
                const float *src = comb + ((size_t)w * n_cols + c) * STRIDE + sub * 64 + dl * 8;
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
                if (lane == 0) last_of_context = last;
            }
            __syncthreads();
            if (last_of_context) {
                if (a.merge_sync) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
                for (int i = threadIdx.x; i < slices; i += 256) {
                    const int c = i / (D / 8), dl = i % (D / 8), sub = NH == 2 && c >= per_head ? 1 : 0;
                    merge_chunks<D, true>(a, it.slot0, a.Hq, it.b, (kh0 + sub) * a.group + qb * QB + (c - sub * per_head), dl, it.nchunks);
                }
            }
        }
        __syncthreads();  // LDS is used again by the next item
    }
}

template <int ACT, int NP>
static attn_fn pick_fp4(int d, int nh) {
    if (d == 64) return nh == 2 ? attn_fp4_kernel<ACT, 64, 2, NP> : attn_fp4_kernel<ACT, 64, 1, NP>;
    if (d == 128) return attn_fp4_kernel<ACT, 128, 1, NP>;
    if (d == 256) return attn_fp4_kernel<ACT, 256, 1, NP>;
    return nullptr;
}

attn_fn s3i_pick_fp4(int act, int d, int heads_per_unit, bool wide_out) {
    if (act == S3_F16) return wide_out ? pick_fp4<S3_F16, 3>(d, heads_per_unit) : pick_fp4<S3_F16, 2>(d, heads_per_unit);
    if (act == S3_BF16) return wide_out ? pick_fp4<S3_BF16, 3>(d, heads_per_unit) : pick_fp4<S3_BF16, 2>(d, heads_per_unit);
    return nullptr;
}

append_fp8_fn s3i_pick_append_fp4(int act) {
    return act == S3_F16 ? append_fp4_kernel<S3_F16> : act == S3_BF16 ? append_fp4_kernel<S3_BF16> : nullptr;
}
