// Kernels for cache rows of 4-bit blocks (S3_MXFP4, s3kv_fp4.h) of libs3kv, gfx950: the append that rounds new rows, and
// decode attention over the exactly widened codes (section 2.1, in fp32), for any number of query heads per cached head.
//
// Attention.  A wave streams tiles of 32 rows of one unit: 128 or 256 elements of a row, i.e. one head or two or four neighbouring ones.
// Both products run on the matrix cores (v_mfma_f32_16x16x32: e2m1 codes under a power of two are exact in bf16, and in fp16 but for far
// scales) with up to 16 query heads as columns, also for a single one: 17 bits hold four elements, so the vector ALU would need more
// instructions for them than the memory leaves time for.
//   S^T = K Q^T   A operand: lane (r, g) holds block g (32 elements, one scale) of row r as it lies in memory; the four products of a
//                 unit of 128 take a word of it each, Q^T in the same element order.  Codes are widened to bf16, beside fp16 queries to
//                 fp16, so that queries enter as they are; blocks whose scale fp16 does not hold go by way of bf16 parts of the query
//                 (special_scores).
//   O^T += V^T P^T  A operand: lane (m, g) holds elements 8m .. 8m+7 (256: 16m ..) of the eight rows 4g .. 4g+3 and 16+4g ..
//                 16+4g+3 of the tile, one word a row: after widening, pairs of rows are brought together by byte permutes, and
//                 output tile i gets the elements 8m + i.  The accumulator layout of S^T is the B operand of P^T as it is.  Weights enter
//                 as two bf16 parts (2^-17 of a weight off, below a rounding of a 16-bit output by 2^5 and more) or, for 32-bit
//                 outputs, as three (exact to fp32).
// The exponent reference of a column follows its maximum lazily (a tile's scores may exceed it by 8 in log2 units), so most tiles need no
// exchange between lanes.  Rows are read once and go from memory straight into LDS; what bounds long contexts is that stream, what bounds
// short ones the chain from launch to the first rows (some 6 us), and, for contexts cut in pieces, the meeting of the pieces.  Measured: 512
// contexts of 512-4096 rows, 32q/8kv x 128, bf16: 218 us, 5.9 TB/s; 256 of 32-1000: 43 us; 1 of 30000: 18 us.
#include "s3kv_fp4.h"

// grid (n, 2): block (b, which) rounds one new row of `columns` 16-bit elements into row off+pos; a thread has eight elements.
template <int ACT>
__global__ void __launch_bounds__(256) append_fp4_kernel(const AttnArgs a) {
    const int b = blockIdx.x, elems = a.columns;
    const int64_t off = a.slot_off[b];
    const int64_t p = a.cur_len[b];
    if (off < 0 || p < 0 || p >= a.max_len || off + p >= a.n_tokens) return;  // never leave the arena
    const char *src = (blockIdx.y ? a.v_new : a.k_new) + (int64_t)b * elems * 2;
    const int scales = elems / 32, scale_row = (scales + 15) & ~15;
    char *codes = (blockIdx.y ? a.vplane : a.kplane) + (off + p) * (int64_t)(elems / 2);
    char *scale = (blockIdx.y ? a.vscale : a.kscale) + (off + p) * (int64_t)scale_row;
    for (int i = threadIdx.x; i < elems / 8; i += 256) {  // (a block's four threads are neighbours and stay together)
        float x[8];
        widen8<ACT>(*(const u32x4 *)(src + (int64_t)i * 16), x);
        unsigned most = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) most = fp4_magnitude(x[e], most);
        most = group_max<4>(most);
        const unsigned byte = fp4_scale_byte<ACT>(__builtin_bit_cast(float, most));
        *(unsigned *)(codes + i * 4) = fp4_codes8(x, byte);
        if ((i & 3) == 0) scale[i / 4] = (char)byte;
    }
    for (int i = scales + threadIdx.x; i < scale_row; i += 256) scale[i] = 0;
}

// A tile of 32 rows of a unit of W elements as the matrix cores take it from a lane.
template <int W>
struct Fp4Tile {
    static constexpr int T = W / 128;
    u32x4 k[2][T];       // rows r and 16 + r, block g (and 4 + g)
    unsigned ks[2][T];   // their scale bytes
    unsigned v[8][T];    // rows 4g + 0..3, 16 + 4g + 0..3
    unsigned vs[8];
};

// Tiles on their way.  Rows go from memory straight into LDS (global_load_lds: lane l's bytes land behind lane l-1's), sixteen bytes a
// lane with the lanes of a row next to each other: 64 or 128 bytes of a row are one or two cache lines' worth of a load, where loads
// in operand order (lanes of a quad on four rows) kept the address unit busy for 42 cycles each and the kernel at half its rate.  A
// wave has its own ring of tiles and waits by the number of loads issued behind the one it needs (they complete in order), so no
// wave waits for another.
//   K   row R at R * W/2, its 16-byte pieces exchanged by XOR with R / 4 (256: R / 2), so that the sixteen rows a read takes one piece
//       of lie in different banks
//   V   row 16u + 4g + j at row place 16u + 4j + g: the rows that a read takes words of together are neighbours
//   S   the rows' scale bytes, K then V
template <int W>
struct Fp4Ring {
    static constexpr int T = W / 128, ROW = W / 2, LOADS = 2 * T, PER_LOAD = 32 / LOADS;  // loads of a tile and plane, rows of one
    static constexpr int STAGE = 2 * 32 * ROW + 64 * 4 * T, TILE_LOADS = 2 * LOADS + T;
    static constexpr int DEEP = W == 256 ? 2 : 3;  // tiles of a ring of attn_fp4_share_kernel (at most 3: see its waits)
};
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void glb_void;

template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// A tile out of LDS.  The reads and their wait are one block of machine code: to the compiler, every read of LDS would depend on all
// loads into it that are in flight.
__device__ __forceinline__ void read_tile(Fp4Tile<128> &t, unsigned k, unsigned ks, unsigned v, unsigned vs) {
    asm volatile(
        "ds_read_b128 %0, %20\n\t"
        "ds_read_b128 %1, %20 offset:1024\n\t"
        "ds_read_u8 %2, %21\n\t"
        "ds_read_u8 %3, %21 offset:64\n\t"
        "ds_read_b32 %4, %22\n\t"
        "ds_read_b32 %5, %22 offset:256\n\t"
        "ds_read_b32 %6, %22 offset:512\n\t"
        "ds_read_b32 %7, %22 offset:768\n\t"
        "ds_read_b32 %8, %22 offset:1024\n\t"
        "ds_read_b32 %9, %22 offset:1280\n\t"
        "ds_read_b32 %10, %22 offset:1536\n\t"
        "ds_read_b32 %11, %22 offset:1792\n\t"
        "ds_read_u8 %12, %23\n\t"
        "ds_read_u8 %13, %23 offset:4\n\t"
        "ds_read_u8 %14, %23 offset:8\n\t"
        "ds_read_u8 %15, %23 offset:12\n\t"
        "ds_read_u8 %16, %23 offset:64\n\t"
        "ds_read_u8 %17, %23 offset:68\n\t"
        "ds_read_u8 %18, %23 offset:72\n\t"
        "ds_read_u8 %19, %23 offset:76\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(t.k[0][0]), "=&v"(t.k[1][0]), "=&v"(t.ks[0][0]), "=&v"(t.ks[1][0]), "=&v"(t.v[0][0]), "=&v"(t.v[1][0]), "=&v"(t.v[2][0]),
          "=&v"(t.v[3][0]), "=&v"(t.v[4][0]), "=&v"(t.v[5][0]), "=&v"(t.v[6][0]), "=&v"(t.v[7][0]), "=&v"(t.vs[0]), "=&v"(t.vs[1]),
          "=&v"(t.vs[2]), "=&v"(t.vs[3]), "=&v"(t.vs[4]), "=&v"(t.vs[5]), "=&v"(t.vs[6]), "=&v"(t.vs[7])
        : "v"(k), "v"(ks), "v"(v), "v"(vs)
        : "memory");
}
__device__ __forceinline__ void read_tile(Fp4Tile<256> &t, unsigned k, unsigned k2, unsigned ks, unsigned ks2, unsigned v, unsigned vs) {
    u32x2 w[8];
    asm volatile(
        "ds_read_b128 %0, %24\n\t"
        "ds_read_b128 %1, %25\n\t"
        "ds_read_b128 %2, %24 offset:2048\n\t"
        "ds_read_b128 %3, %25 offset:2048\n\t"
        "ds_read_u8 %4, %26\n\t"
        "ds_read_u8 %5, %29\n\t"
        "ds_read_u8 %6, %26 offset:128\n\t"
        "ds_read_u8 %7, %29 offset:128\n\t"
        "ds_read_b64 %8, %27\n\t"
        "ds_read_b64 %9, %27 offset:512\n\t"
        "ds_read_b64 %10, %27 offset:1024\n\t"
        "ds_read_b64 %11, %27 offset:1536\n\t"
        "ds_read_b64 %12, %27 offset:2048\n\t"
        "ds_read_b64 %13, %27 offset:2560\n\t"
        "ds_read_b64 %14, %27 offset:0xc00\n\t"
        "ds_read_b64 %15, %27 offset:3584\n\t"
        "ds_read_u8 %16, %28\n\t"
        "ds_read_u8 %17, %28 offset:8\n\t"
        "ds_read_u8 %18, %28 offset:16\n\t"
        "ds_read_u8 %19, %28 offset:24\n\t"
        "ds_read_u8 %20, %28 offset:128\n\t"
        "ds_read_u8 %21, %28 offset:136\n\t"
        "ds_read_u8 %22, %28 offset:144\n\t"
        "ds_read_u8 %23, %28 offset:152\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(t.k[0][0]), "=&v"(t.k[0][1]), "=&v"(t.k[1][0]), "=&v"(t.k[1][1]), "=&v"(t.ks[0][0]), "=&v"(t.ks[0][1]), "=&v"(t.ks[1][0]),
          "=&v"(t.ks[1][1]), "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(w[4]), "=&v"(w[5]), "=&v"(w[6]), "=&v"(w[7]),
          "=&v"(t.vs[0]), "=&v"(t.vs[1]), "=&v"(t.vs[2]), "=&v"(t.vs[3]), "=&v"(t.vs[4]), "=&v"(t.vs[5]), "=&v"(t.vs[6]), "=&v"(t.vs[7])
        : "v"(k), "v"(k2), "v"(ks), "v"(v), "v"(vs), "v"(ks2)
        : "memory");
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const unsigned x = w[e][0], y = w[e][1];
        t.v[e][0] = x;
        t.v[e][1] = y;
    }
}

__device__ __forceinline__ f32x4 mfma_bf16(const bf16x8 a, const bf16x8 b, const f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f32x4 mfma_f16(const f16x8 a, const f16x8 b, const f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
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

__device__ __forceinline__ f16x8 widen_word_f16(const unsigned w, const float scale) {
    const u32x4 x = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3))};
    return __builtin_bit_cast(f16x8, x);
}

// Two fp32 numbers as a word of two bf16 (nearest, ties to even); what that leaves of them stays in x0, x1.
__device__ __forceinline__ unsigned take_bf16_part(float &x0, float &x1) {
    const unsigned w = round_bf16x2(x0, x1);
    const unsigned lo = w << 16, hi = w & 0xFFFF0000u;
    x0 -= __builtin_bit_cast(float, lo);
    x1 -= __builtin_bit_cast(float, hi);
    return w;
}

// Eight output elements; WIDE: of 32 bits.
template <bool WIDE>
__device__ __forceinline__ void put_out8(const AttnArgs &a, int64_t e, const float (&v)[8]) {
    if (WIDE) {
        f32x4 *to = (f32x4 *)((float *)a.out + e);
        to[0] = (f32x4){v[0], v[1], v[2], v[3]};
        to[1] = (f32x4){v[4], v[5], v[6], v[7]};
        return;
    }
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const f16x2 h = {(_Float16)v[2 * i], (_Float16)v[2 * i + 1]};
        const unsigned f16 = __builtin_bit_cast(unsigned, h), bf16 = round_bf16x2(v[2 * i], v[2 * i + 1]);
        w[i] = a.out_dtype == S3_F16 ? f16 : bf16;
    }
    *(u32x4 *)((uint16_t *)a.out + e) = w;
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

// What one wave does with the rows of a unit: NH neighbouring heads, 128 or 256 elements.  NP: bf16 parts of a weight.
template <int ACT, int D, int NH, int NP>
struct Fp4Wave {
    static constexpr int W = D * NH < 128 ? 128 : D * NH, T = W / 128;
    static_assert(W == 128 || W == 256, "a unit");
    static constexpr int QB = 16 / NH;                // columns of a head
    typedef Fp4Ring<W> Ring;

    const AttnArgs &a;
    char *ring;  // this wave's tiles on their way
    u32x4 q[T][4];  // the queries of this lane's column, of type ACT, as the B operand takes them
    int lane, r, g;
    int code_bytes, scale_bytes;  // of a row
    int kh0, qb, per_head;  // first cached head, block of query heads, query heads of a cached head in it
    int heads;              // of the unit that there are
    int qsub, qhead;        // this lane's column: its head of the unit, its query head
    bool column;            // the column is one
    float m, l;
    f32x4 acc[8 * T];

    __device__ __forceinline__ Fp4Wave(const AttnArgs &args, char *tiles) : a(args), ring(tiles) {
        lane = threadIdx.x & 63;
        r = lane & 15;
        g = lane >> 4;
        code_bytes = fp4_code_bytes(a.H, D);
        scale_bytes = fp4_scale_bytes(a.H, D);
    }

    // The element of the unit (of its first head, where the element's head is not there) that a lane's data begin with: K, block g of half
    // h; V, elements 8Tr ...
    __device__ __forceinline__ int there(int element) const { return NH == 1 ? element % D : element < heads * D ? element : element % D; }
    __device__ __forceinline__ int k_element(int h) const { return there(h * 128 + g * 32); }
    __device__ __forceinline__ int v_element() const { return there(8 * T * r); }
    __device__ __forceinline__ int k_head(int h) const { return NH == 1 ? 0 : (h * 128 + g * 32) / D; }

    __device__ __forceinline__ void set_column(int col) {
        const int unit = a.nqb == 1 ? col : col / a.nqb;
        qb = col - unit * a.nqb;
        kh0 = unit * NH;
        heads = min(NH, a.H - kh0);
        per_head = min(a.group - qb * QB, QB);
        qsub = NH == 1 ? 0 : r / QB;
        const int qi = r % QB + qb * QB;
        qhead = (kh0 + qsub) * a.group + qi;
        column = qi < a.group && qsub < heads;
        whole = offsets(31);
    }

    // Where a lane's pieces of a tile are, in bytes from the tile's first row; rows past `last` repeat that one, whose values they then
    // carry into the products with a weight of 0.
    struct Offsets {
        unsigned k[Ring::LOADS], v[Ring::LOADS], s[T];
    };
    __device__ __forceinline__ Offsets offsets(int last) const {
        Offsets o;
        constexpr int LPR = 64 / Ring::PER_LOAD;  // lanes a row
        const int base = kh0 * (D / 2), piece = lane % LPR;
        // (heads that are not there, and what a head of 64 alone leaves of a unit: pieces of the first)
        const int pieces = heads * (D / 32);
        const auto piece_at = [&](int p) { return p < pieces ? p : p & (D / 32 - 1); };
#pragma unroll
        for (int i = 0; i < Ring::LOADS; i++) {
            const int place = i * Ring::PER_LOAD + lane / LPR;
            const int swap = W == 256 ? (place >> 1) & 7 : (place >> 2) & 3;
            const int its = (place & 16) + 4 * (place & 3) + ((place >> 2) & 3);
            o.k[i] = min(place, last) * code_bytes + base + piece_at(piece ^ swap) * 16;
            o.v[i] = min(its, last) * code_bytes + base + piece_at(piece) * 16;
        }
        const int scales = kh0 * (D / 32) & ~3;
#pragma unroll
        for (int i = 0; i < T; i++) o.s[i] = W == 256 ? min(lane >> 1, last) * scale_bytes + scales + (lane & 1) * 4 : min(lane & 31, last) * scale_bytes + scales;
        return o;
    }

    Offsets whole;  // of a tile with all its rows

    // Issues the loads of a tile that begins at row `row` of the arena and of which `rows` rows (1 and more) are there.
    __device__ __forceinline__ void issue(char *stage, int64_t row, int rows) const {
        if (rows >= 32) issue(stage, row, whole);
        else issue(stage, row, offsets(rows - 1));
    }
    __device__ __forceinline__ void issue(char *stage, int64_t row, const Offsets &o) const {
        const char *kp = a.kplane + row * code_bytes, *vp = a.vplane + row * code_bytes;
        const char *ks = a.kscale + row * scale_bytes, *vs = a.vscale + row * scale_bytes;
        // Pieces of 128 bytes carry the streaming hint (512 contexts of 512-4096 rows, 32q/8kv x 128: 218 us with it, 249 without); of 64,
        // the other half of a cache line is another wave's, which finds it in L2 if the line was not given up at once (128 such contexts
        // by chunks: 113 us with the hint, 106 without).
        constexpr int HINT = W == 256 ? 2 : 0;
#pragma unroll
        for (int i = 0; i < Ring::LOADS; i++) __builtin_amdgcn_global_load_lds((glb_void *)(kp + o.k[i]), (lds_void *)(stage + i * 1024), 16, 0, HINT);
#pragma unroll
        for (int i = 0; i < Ring::LOADS; i++)
            __builtin_amdgcn_global_load_lds((glb_void *)(vp + o.v[i]), (lds_void *)(stage + 32 * Ring::ROW + i * 1024), 16, 0, HINT);
        char *s = stage + 64 * Ring::ROW;
        if constexpr (W == 256) {
            __builtin_amdgcn_global_load_lds((glb_void *)(ks + o.s[0]), (lds_void *)s, 4, 0, 0);
            __builtin_amdgcn_global_load_lds((glb_void *)(vs + o.s[1]), (lds_void *)(s + 256), 4, 0, 0);
        } else {
            __builtin_amdgcn_global_load_lds((glb_void *)((lane < 32 ? ks : vs) + o.s[0]), (lds_void *)s, 4, 0, 0);
        }
    }
    __device__ __forceinline__ void read(Fp4Tile<W> &t, const char *stage) const {
        const unsigned base = (unsigned)(uintptr_t)(lds_void *)stage, s = base + 64 * Ring::ROW;
        const int shift = W > D * NH ? 2 * (kh0 & 1) : 0;  // (a head of 64 alone: its scales within their word)
        // (of the second half of 256 elements: 4 bytes on; where its heads are not there, the first half's are read again)
        const unsigned ks = s + r * 4 * T + shift + k_element(0) / 32;
        const unsigned v = base + 32 * Ring::ROW + g * Ring::ROW + r * 4 * T;
        const unsigned vs = s + 128 * T + g * 16 * T + shift + v_element() / 32;
        if constexpr (W == 256) {
            const unsigned k = base + r * 128 + ((g ^ ((r >> 1) & 7)) * 16), k2 = base + r * 128 + (((4 + g) ^ ((r >> 1) & 7)) * 16);
            read_tile(t, k, k2, ks, s + r * 8 + k_element(1) / 32, v, vs);
        } else {
            read_tile(t, base + r * 64 + ((g ^ (r >> 2)) * 16), ks, v, vs);
        }
    }

    // Sequence b's queries; nothing folded in yet.
    __device__ __forceinline__ void begin(int b) {
#pragma unroll
        for (int h = 0; h < T; h++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                q[h][i] = (u32x4){0u, 0u, 0u, 0u};
                // (the queries of a column meet their own head's elements, zeros meet the others')
                if (column && (W > D * NH ? g < 2 : k_head(h) == qsub))
                    q[h][i] = *(const u32x4 *)(a.q + (((int64_t)b * a.Hq + qhead) * D + (h * 128 + g * 32) % D + i * 8) * 2);
            }
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 8 * T; i++) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    // Asks for the queries of a context to come, so that begin() finds them in L2: a word of every 64 bytes, into 256 bytes of LDS that
    // nobody reads.
    __device__ __forceinline__ void touch_queries(char *nowhere, int b) const {
        const int head = column ? qhead : kh0 * a.group + qb * QB;
#pragma unroll
        for (int h = 0; h < (D == 256 ? 2 : 1); h++)
            __builtin_amdgcn_global_load_lds((glb_void *)(a.q + (((int64_t)b * a.Hq + head) * D + (h * 128 + g * 32) % D) * 2), (lds_void *)nowhere, 4, 0, 0);
    }

    // Blocks that the products of fold() do not take: with several heads, those that read as NaN, which must not reach the other heads'
    // columns (NaN times their zeros); beside fp16 queries, those with a scale under which a code may be no fp16 number (below 104 half a
    // step is less than 2^-24).  Appended rows have those only where no number of a block reaches 7 * 2^-24, and 1 for zeros: under 0 and
    // 1 no number reaches 2^-123, and they count as zeros.
    __device__ __forceinline__ static bool special(unsigned byte) {
        return ACT == S3_F16 ? byte - 104u > 36u && byte > 1u : NH > 1 && byte == 255u;
    }
    // The scores of a tile with such blocks: head by head, widened to bf16 (fp16 queries are the exact sum of two bf16 parts).
    __device__ __forceinline__ void special_scores(const Fp4Tile<W> &t, f32x4 (&s)[2]) const {
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll 1
            for (int sub = 0; sub < heads; sub++) {
                f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < T; h++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bool its = NH == 1 || k_head(h) == sub;
                        const bf16x8 k8 = widen_word(its ? t.k[u][h][i] : 0u, its ? fp4_scale(t.ks[u][h]) : 1.f);
                        if (ACT == S3_BF16) {
                            c = mfma_bf16(k8, __builtin_bit_cast(bf16x8, q[h][i]), c);
                        } else {
                            u32x4 w = q[h][i];
                            asm volatile("" : "+v"(w));  // (taken apart here, and not kept in parts)
                            float x[8];
                            widen8<ACT>(w, x);
#pragma unroll
                            for (int part = 0; part < 2; part++) {
                                u32x4 p;
#pragma unroll
                                for (int e = 0; e < 4; e++) p[e] = take_bf16_part(x[2 * e], x[2 * e + 1]);
                                c = mfma_bf16(k8, __builtin_bit_cast(bf16x8, p), c);
                            }
                        }
                    }
                if (qsub == sub) s[u] = c;
            }
    }

    // What a tile holds is folded into (m, l, acc); rows: those of the tile and behind it (fewer than 32: the last tile).
    __device__ __forceinline__ void fold(const Fp4Tile<W> &t, int rows) {
        f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < T; h++) {
            const float scale[2] = {fp4_scale(t.ks[0][h]), fp4_scale(t.ks[1][h])};
#pragma unroll
            for (int i = 0; i < 4; i++) {
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    if (ACT == S3_BF16) s[u] = mfma_bf16(widen_word(t.k[u][h][i], scale[u]), __builtin_bit_cast(bf16x8, q[h][i]), s[u]);
                    else s[u] = mfma_f16(widen_word_f16(t.k[u][h][i], scale[u]), __builtin_bit_cast(f16x8, q[h][i]), s[u]);
                }
            }
        }
        if (ACT == S3_F16 || NH > 1) {
            bool any = false;
#pragma unroll
            for (int h = 0; h < T; h++) any = any || special(t.ks[0][h]) || special(t.ks[1][h]);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(any) != 0, 0)) special_scores(t, s);
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

    // A decode step's new row, still 16-bit, as the last of `rows` rows of a tile whose loads have arrived: its blocks are rounded, written
    // to the arena (row `row`), and put in the places of the tile's rows from rows - 1 on, which hold what the arena held there.  A lane
    // has a block of K and one of V.
    __device__ __forceinline__ void take_new_row(char *stage, int b, int64_t row, int rows) const {
        constexpr int LPR = 64 / Ring::PER_LOAD;
        const int first = lane / LPR, piece = lane % LPR, pieces = heads * (D / 32);
        const int mine = piece < pieces ? piece : piece & (D / 32 - 1), base = kh0 * D + mine * 32;  // first element within the row
        const int shift = W > D * NH ? 2 * (kh0 & 1) : 0;
#pragma unroll 1
        for (int which = 0; which < 2; which++) {
            const char *src = (which ? a.v_new : a.k_new) + ((int64_t)b * a.H * D + base) * 2;
            float x[4][8];
            unsigned most = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                widen8<ACT>(*(const u32x4 *)(src + i * 16), x[i]);
#pragma unroll
                for (int e = 0; e < 8; e++) most = fp4_magnitude(x[i][e], most);
            }
            const unsigned byte = fp4_scale_byte<ACT>(__builtin_bit_cast(float, most));
            u32x4 c;
#pragma unroll
            for (int i = 0; i < 4; i++) c[i] = fp4_codes8(x[i], byte);
            char *scales = (which ? a.vscale : a.kscale) + row * scale_bytes;
            if (first == 0 && piece < pieces) {
                *(u32x4 *)((which ? a.vplane : a.kplane) + row * code_bytes + base / 2) = c;
                scales[base / 32] = (char)byte;
            }
            const int used = a.H * (D / 32);
            if (kh0 + NH >= a.H && lane < scale_bytes - used) scales[used + lane] = 0;  // zeros up to a multiple of 16 bytes
            char *tile = stage + which * 32 * Ring::ROW, *s = stage + 64 * Ring::ROW + which * 128 * T;
#pragma unroll
            for (int i = 0; i < Ring::LOADS; i++) {
                const int place = i * Ring::PER_LOAD + first;
                const int swap = W == 256 ? (place >> 1) & 7 : (place >> 2) & 3;
                const int its = which ? (place & 16) + 4 * (place & 3) + ((place >> 2) & 3) : place;
                if (its >= rows - 1) *(u32x4 *)(tile + place * Ring::ROW + (which ? piece : piece ^ swap) * 16) = c;
                if (place >= rows - 1 && piece < pieces) s[place * 4 * T + shift + piece] = (char)byte;
            }
        }
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

    // This lane's first element of its column's head (32T from there on are its own), and whether it has any.
    __device__ __forceinline__ int first_element() const { return 32 * T * g - D * qsub; }
    __device__ __forceinline__ bool delivers() const { return column && first_element() >= 0 && first_element() < D; }

    // The output rows of context b for this column; total: the weights' sum of the lane's column.
    __device__ __forceinline__ void deliver(int b, const float total) const {
        const float inv = 1.f / total;
        if (!delivers()) return;
#pragma unroll
        for (int rr = 0; rr < 4; rr++)
#pragma unroll
            for (int i = 0; i < T; i++) {
                const f32x4 lo = sums4(rr, 2 * i), hi = sums4(rr, 2 * i + 1);
                const float o[8] = {lo[0] * inv, lo[1] * inv, lo[2] * inv, lo[3] * inv, hi[0] * inv, hi[1] * inv, hi[2] * inv, hi[3] * inv};
                put_out8<NP == 3>(a, ((int64_t)b * a.Hq + qhead) * D + first_element() + 8 * T * rr + 8 * i, o);
            }
    }

    // A piece of a context, as the lanes hold it: 8T quads a lane, lanes that deliver side by side, so that a store covers whole lines
    // (written a row of the output at a time, 16 bytes here and there past the caches, the pieces of 1024 contexts of 512 rows, 16q/1kv x
    // 256, took as long as their rows: 75 us).
    __device__ __forceinline__ unsigned piece_lane() const {
        return ((qsub * per_head + r % QB) * (D / (32 * T)) + first_element() / (32 * T)) * 16;
    }
    __device__ __forceinline__ unsigned piece_quads() const { return heads * per_head * (D / (32 * T)) * 16; }  // bytes of one quad of all lanes
    __device__ __forceinline__ float *piece(int64_t slot) const { return a.part_acc + (slot * a.Hq + kh0 * a.group + qb * QB) * D; }
    __device__ __forceinline__ void put_piece(int64_t slot, const float total) const {
        if (!delivers()) return;
        if (first_element() == 0) put_partial2<true>((float *)a.part_ml + 2 * (slot * a.Hq + qhead), (f32x2){m, total});
        char *to = (char *)piece(slot) + piece_lane();
#pragma unroll
        for (int i = 0; i < 8 * T; i++) put_partial4<true>((float *)(to + i * piece_quads()), acc[i]);
    }
    // Merges the `count` pieces of context b in slots slot0, slot0 + 1, ... and delivers its rows.  (Two a memory round trip cost registers and
    // code that all contexts paid for: 64 contexts of 32-400 rows, 16 heads of 256, 34.7 us instead of 33.4.)
    __device__ __forceinline__ void merge_pieces(int64_t slot0, int b, int count) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 8 * T; i++) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        const unsigned bytes = heads * per_head * D * 4, at = delivers() ? piece_lane() : bytes;  // (past the end: zeros, no traffic)
        for (int c = 0; c < count; c++) {
            const int64_t slot = slot0 + c;
            const __amdgpu_buffer_rsrc_t mr = piece_buffer((const float *)a.part_ml + 2 * slot * a.Hq, a.Hq * 8), pr = piece_buffer(piece(slot), bytes);
            const f32x2 ml = piece_load2(mr, delivers() ? qhead * 8 : a.Hq * 8);
            f32x4 p[8 * T];
#pragma unroll
            for (int i = 0; i < 8 * T; i++) p[i] = piece_load4(pr, at + i * piece_quads());
            const float pm = ml[0], mn = fmaxf(m, pm), ref = exp_reference(mn);
            const float old = fast_exp2(m - ref), now = fast_exp2(pm - ref);
            l = l * old + ml[1] * now;
#pragma unroll
            for (int i = 0; i < 8 * T; i++) acc[i] = acc[i] * old + p[i] * now;
            m = mn;
        }
        deliver(b, l);
    }
};

// The new lengths, and a zero output row for empty or refused contexts, by the workgroups in turn.  The first context's entry is asked
// for when the kernel begins and used when it ends.
struct FirstEntry {
    int64_t off;
    int32_t raw;
};
__device__ __forceinline__ FirstEntry first_entry(const AttnArgs &a) {
    const int b = min((int)blockIdx.x, a.n - 1);
    return {a.slot_off[b], a.cur_len[b]};
}
template <int D, bool WIDE>
__device__ __forceinline__ void publish_lengths(const AttnArgs &a, FirstEntry e) {
    for (int b = blockIdx.x; b < a.n; b += gridDim.x) {
        if (b != (int)blockIdx.x) e = {a.slot_off[b], a.cur_len[b]};
        if (a.len_out && threadIdx.x == 0) a.len_out[b] = e.raw + 1;
        if (checked_len(a, e.off, e.raw) == 0) {
            const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int i = threadIdx.x; i < a.Hq * D / 8; i += blockDim.x) put_out8<WIDE>(a, ((int64_t)b * a.Hq * D / 8 + i) * 8, z);
        }
    }
}

// Folds chunks c0 .. c1-1 of a context (their pieces begin at piece p0, a row of Hq pieces a chunk) into (m, l, o), eight elements of a head.
template <int D>
__device__ __forceinline__ void merge_range(const AttnArgs &a, int64_t p0, int dl, int c0, int c1, float &m, float &l, float (&o)[8]) {
    for (; c0 < c1; c0 += 4) {
        const float *mp[4], *ap[4];
        f32x2 ml[4];
        f32x4 lo[4], hi[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int64_t at = p0 + (int64_t)min(c0 + u, c1 - 1) * a.Hq;
            mp[u] = (const float *)a.part_ml + 2 * at;
            ap[u] = a.part_acc + at * D + dl * 8;
        }
        get_partials<true>(mp, ap, ml, lo, hi);
        const float mn = fmaxf(fmaxf(m, fmaxf(ml[0][0], ml[1][0])), fmaxf(ml[2][0], ml[3][0]));  // (repeats do not change it)
        const float ref = exp_reference(mn), old = fast_exp2(m - ref);
        l *= old;
#pragma unroll
        for (int i = 0; i < 8; i++) o[i] *= old;
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const float w = c0 + u < c1 ? fast_exp2(ml[u][0] - ref) : 0.f;
            l += w * ml[u][1];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                o[i] += w * lo[u][i];
                o[4 + i] += w * hi[u][i];
            }
        }
        m = mn;
    }
}

// Few (context, column) pairs: an item is a chunk of a context for a column, its rows shared out over the four waves of a workgroup,
// which meet in LDS; chunks meet through memory.  Units of 128 elements: twice the items of 256, and latency is what counts here (64
// contexts of 32-400 rows, 32q/8kv x 128: 10 us; in equal shares 26).
template <int ACT, int D, int NH, int NP>
__global__ void __launch_bounds__(256, 2) attn_fp4_team_kernel(const AttnArgs a) {
    typedef Fp4Wave<ACT, D, NH, NP> Wave;
    constexpr int W = Wave::W, T = Wave::T, QB = Wave::QB, TS = 4;
    constexpr int STRIDE = W + 4;  // floats of a column in LDS
    extern __shared__ __align__(16) char dyn_lds[];  // the batch view, the waves' rings
    __shared__ int wave_sums[S3_MAX_CLASSES * S3_MAX_WAVES];
    __shared__ float comb_m[TS][16], comb_l[TS][16];
    __shared__ int last_of_context;
    const int ts = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // (scalar: row ranges and buffers with it)
    const FirstEntry entry = first_entry(a);
    const BatchView bv = build_batch_view<false, W == 256 ? 30 : 10>(a, dyn_lds, wave_sums);
    char *rings = dyn_lds + ((batch_view_bytes(a.n, a.ncls) + 15) & ~(size_t)15);
    // a wave's ring takes its sums of the columns in use when its rows are done: STRIDE floats a column
    constexpr int RING = 2 * Wave::Ring::STAGE;
    static_assert(16 * STRIDE * 4 <= RING, "a wave's sums fit its ring");
    Wave w(a, rings + ts * RING);
    // Work in the order of eighths: workgroup b (XCD b % 8) takes the chunks whose number leaves the same remainder, so that the
    // columns of a chunk, whose bytes share cache lines, are on one XCD's L2.
    const int64_t total = (int64_t)((bv.total + 7) / 8) * 8 * a.columns;
    // The list begins with the longest contexts, and every other round goes through the workgroups backwards: who had the longest has the
    // shortest next (79 contexts of 32-1000 rows, 16 heads of 256: 50.7 -> 45.7 us, 65 of 32q/8kv x 128: 19.0 -> 17.1).
    for (int64_t from = 0, back = 0; from < total; from += gridDim.x, back ^= 1) {
        const int64_t at = from + (back ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
        if (at >= total) continue;
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
        const int64_t first_row = it.off + j0;
        const int tiles = (j1 - j0 + 31) / 32;
        // a tile is on its way while the one before it is folded in
        if (tiles > 0) w.issue(w.ring, first_row, j1 - j0);
        w.begin(it.b);
        for (int i = 0; i < tiles; i++) {
            const int left = j1 - j0 - 32 * i;
            Fp4Tile<W> t;
            if (left > 32) {
                w.issue(w.ring + ((i + 1) & 1) * Wave::Ring::STAGE, first_row + 32 * (i + 1), left - 32);
                wait_loads<Wave::Ring::TILE_LOADS>();
            } else {
                wait_loads<0>();
            }
            char *stage = w.ring + (i & 1) * Wave::Ring::STAGE;
            if (has_new && left <= 32) w.take_new_row(stage, it.b, it.off + it.len - 1, left);
            w.read(t, stage);
            w.fold(t, left);
        }

        // the four waves meet: columns in use, compact (head, query)
        const int slot = w.qsub * w.per_head + (w.r % QB), n_cols = w.heads * w.per_head;
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
                    *(f32x4 *)((float *)w.ring + slot * STRIDE + 8 * T * (4 * w.g + rr) + 4 * i) = w.sums4(rr, i);
        }
        __syncthreads();
        // a thread: eight elements of one column
        const int slices = n_cols * (D / 8);
        for (int i = threadIdx.x; i < slices; i += 256) {
            const int c = i / (D / 8), dl = i % (D / 8), sub = NH == 1 ? 0 : c / w.per_head;
            const int h = (w.kh0 + sub) * a.group + w.qb * QB + (c - sub * w.per_head);
            float mm = -INFINITY, ll = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < TS; x++) mm = fmaxf(mm, comb_m[x][c]);
            const float ref = exp_reference(mm);
#pragma unroll
            for (int x = 0; x < TS; x++) {
                const float wt = fast_exp2(comb_m[x][c] - ref);
                ll += wt * comb_l[x][c];
                const float *src = (const float *)(rings + x * RING) + c * STRIDE + sub * D + dl * 8;
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
                put_out8<NP == 3>(a, ((int64_t)it.b * a.Hq + h) * D + dl * 8, o);
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
                const auto head_of = [&](int c) {
                    const int sub = NH == 1 ? 0 : c / w.per_head;
                    return (w.kh0 + sub) * a.group + w.qb * QB + (c - sub * w.per_head);
                };
                if (W == 256 || slices > 128 || it.nchunks <= 4) {
                    for (int i = threadIdx.x; i < slices; i += 256)
                        merge_chunks<D, true>(a, it.slot0, a.Hq, it.b, head_of(i / (D / 8)), i % (D / 8), it.nchunks);
                } else {
                    // Threads left over take chunks of their own, four at least, and meet in LDS (one context of 8034 rows, 32q/8kv x 128: 11.9 us
                    // instead of 13.7; of 30000: 18 instead of 21.9).  Not beside units of 256 elements, whose loop over the rows, short of
                    // registers, got a fifth slower by it.
                    const int parts = min(256 / slices, (it.nchunks + 3) / 4), per = (it.nchunks + parts - 1) / parts;
                    const int part = threadIdx.x / slices, i = threadIdx.x - part * slices, h = head_of(i / (D / 8)), dl = i % (D / 8);
                    float *at = (float *)rings;  // [parts][slices] of (max, sum, 8 values, 2 unused)
                    float mm = -INFINITY, ll = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    if (part < parts) {
                        merge_range<D>(a, (int64_t)it.slot0 * a.Hq + h, dl, part * per, min(it.nchunks, (part + 1) * per), mm, ll, o);
                        float *mine = at + threadIdx.x * 12;
                        *(f32x4 *)mine = (f32x4){mm, ll, 0.f, 0.f};
                        *(f32x4 *)(mine + 4) = (f32x4){o[0], o[1], o[2], o[3]};
                        *(f32x4 *)(mine + 8) = (f32x4){o[4], o[5], o[6], o[7]};
                    }
                    __syncthreads();
                    if (part == 0) {
                        for (int x = 1; x < parts; x++) {
                            const float *from = at + (x * slices + i) * 12;
                            const f32x4 ml = *(const f32x4 *)from, lo = *(const f32x4 *)(from + 4), hi = *(const f32x4 *)(from + 8);
                            const float mn = fmaxf(mm, ml[0]), ref = exp_reference(mn), old = fast_exp2(mm - ref), now = fast_exp2(ml[0] - ref);
                            ll = ll * old + ml[1] * now;
#pragma unroll
                            for (int e = 0; e < 4; e++) {
                                o[e] = o[e] * old + lo[e] * now;
                                o[4 + e] = o[4 + e] * old + hi[e] * now;
                            }
                            mm = mn;
                        }
                        const float inv = 1.f / ll;
#pragma unroll
                        for (int e = 0; e < 8; e++) o[e] *= inv;
                        put_out8<NP == 3>(a, ((int64_t)it.b * a.Hq + h) * D + dl * 8, o);
                    }
                }
            }
        }
        __syncthreads();  // LDS is used again by the next item
    }
    publish_lengths<D, NP == 3>(a, entry);
}

// Exclusive prefix sums of the contexts' tiles into pre[0..n], by the whole workgroup; returns the total (longest: the rows of the
// longest context).
// off_s, len_s: receive the contexts' offsets and rows, unless off_s is null.
__device__ __forceinline__ int tile_prefix(const AttnArgs &a, int *pre, int64_t *off_s, int *len_s, int *wave_sums, int &longest) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nwaves = blockDim.x >> 6;
    constexpr int E = 4;
    int total = 0;
    for (int base = 0; base < a.n; base += E * (int)blockDim.x) {
        int64_t off[E];
        int len[E], sum = 0, mx = 0;
        load_entries<E>(a, base + tid * E, off, len);
#pragma unroll
        for (int e = 0; e < E; e++) {
            sum += (len[e] + 31) >> 5;
            mx = max(mx, len[e]);
        }
        const int incl = wave_inclusive_scan(sum);
        mx = wave_max_nonneg(mx);
        if (lane == 63) {
            wave_sums[wave] = incl;
            wave_sums[S3_MAX_WAVES + wave] = mx;
        }
        __syncthreads();
        const int upto = wave_inclusive_scan(lane < nwaves ? wave_sums[lane] : 0);
        longest = max(longest, wave_max_nonneg(lane < nwaves ? wave_sums[S3_MAX_WAVES + lane] : 0));
        int run = total + incl - sum + (wave > 0 ? __builtin_amdgcn_readlane(upto, wave - 1) : 0);
        total += __builtin_amdgcn_readlane(upto, nwaves - 1);
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int b = base + tid * E + e;
            if (b < a.n) {
                pre[b] = run;
                if (off_s) {
                    off_s[b] = off[e];
                    len_s[b] = len[e];
                }
            }
            run += (len[e] + 31) >> 5;
        }
        if (tid == 0) pre[a.n] = total;
        __syncthreads();
    }
    return total;
}

// Many (context, column) pairs: the tiles of all contexts laid end to end are cut into equal shares, one a wave and column, so that
// waves end together whatever the lengths, and no wave waits for another.  A share runs through whole contexts, which it finishes by
// itself, and at either end through a part of one that others share: such a piece goes to memory (share u's piece of context b to slot
// u + b: along the shares either u or b grows, so no two meet), is counted, and whoever counts the last piece of a context merges them.
// Where no context has more than 8 tiles none is cut, a share takes those that begin in it: the meeting would cost more than uneven
// shares (100-250 rows: 256 contexts, 32q/8kv x 128: 24.8 us, cut 27.2; 1024 contexts, 16q/1kv x 256: 26.6 and 40.3; of up to 13 tiles the
// former is better cut, 30 and 33 us).
#define S3_FP4_UNCUT 8
template <int ACT, int D, int NH, int NP>
__device__ __forceinline__ void fp4_share(const AttnArgs &a) {
    typedef Fp4Wave<ACT, D, NH, NP> Wave;
    constexpr int W = Wave::W;
    extern __shared__ __align__(16) char dyn_lds[];  // the waves' rings; tiles in front of every context, [n + 1]; offsets and rows
    __shared__ int wave_sums[2 * S3_MAX_WAVES];
    constexpr int DEEP = Wave::Ring::DEEP;
    char *rings = dyn_lds;
    int *pre = (int *)(dyn_lds + 8 * DEEP * Wave::Ring::STAGE + 8 * 256);
    const bool known = a.n <= S3_FP4_KNOWN;  // offsets and rows of the contexts are in LDS too
    int64_t *off_s = (int64_t *)((char *)pre + (((a.n + 1) * 4 + 15) & ~15));
    int *len_s = (int *)(off_s + a.n);
    int longest = 0;
    const int total = tile_prefix(a, pre, known ? off_s : nullptr, len_s, wave_sums, longest);
    const int ts = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Neighbouring columns, whose bytes share cache lines, are on neighbouring waves, and those on one XCD (workgroup b is on XCD b % 8).
    const int rank = (gridDim.x & 7) == 0 ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;
    const int place = rank * 8 + ts;
    const int share = place / a.columns, col = place - share * a.columns;
    const bool cut = longest > 32 * S3_FP4_UNCUT;
    // A long context among short ones: its pieces, merged one behind the other, cost as much as its tiles when a share has about the root
    // of its tiles (0.4 of it measured best; 255 contexts of 10-60 rows and one of 16384, 32q/8kv x 128: 72 us instead of 174; all of 32-1000
    // rows: 43 us either way).
    const int size = max((total + a.wave_shares - 1) / a.wave_shares, __builtin_amdgcn_readfirstlane((int)(0.4f * sqrtf((float)(longest >> 5)) + 1.f)));
    if (share >= a.wave_shares || share * (int64_t)size >= total) return;
    int t0 = share * size, t1 = min(total, t0 + size);
    int b = __builtin_amdgcn_readfirstlane(find_sequence(pre, a.n, t0));  // the context that holds tile t0
    if (!cut) {  // from the first context that begins at t0 or behind it to the last that begins in front of t1
        if (__builtin_amdgcn_readfirstlane(pre[b]) < t0) b++;
        t0 = __builtin_amdgcn_readfirstlane(pre[b]);
        if (t0 >= t1) return;
        t1 = __builtin_amdgcn_readfirstlane(pre[find_sequence(pre, a.n, t1 - 1) + 1]);
    }
    Wave w(a, rings + ts * DEEP * Wave::Ring::STAGE);
    w.set_column(col);
    Pending head = {0, 0, 0}, tail = {0, 0, 0};  // pieces of the contexts that the share's borders cut

    // the loader: context, its first tile, rows from the tile to load on (0: the share is loaded)
    struct Cursor {
        int b, begin, end;  // tiles of context b
        int tile, len;
        int64_t off;
    };
    const auto open = [&](Cursor &c, int tile) {  // the context that holds `tile`, from context c.b on
        while (true) {
            c.end = __builtin_amdgcn_readfirstlane(pre[c.b + 1]);
            if (tile < c.end) break;
            c.b++;
        }
        c.begin = __builtin_amdgcn_readfirstlane(pre[c.b]);
        if (known) {
            c.off = uniform64(off_s[c.b]);
            c.len = __builtin_amdgcn_readfirstlane(len_s[c.b]);
        } else {  // (a context with tiles: it has been checked)
            c.off = uniform64(a.slot_off[c.b]);
            c.len = __builtin_amdgcn_readfirstlane(a.cur_len[c.b]) + a.len_add;
        }
        c.tile = tile;
    };
    const auto finish = [&](const Cursor &c) {  // the share's part of context c.b is folded in
        const int first = max(c.begin, t0), last = min(c.end, t1);
        const float l = sum_over_rows(w.l);
        if (first == c.begin && last == c.end) {
            w.deliver(c.b, l);
            return;
        }
        const int u0 = c.begin / size, u1 = (c.end - 1) / size;
        const Pending p = {c.b, u0, u1 - u0 + 1};
        if (first == t0) head = p;
        else tail = p;
        w.put_piece(share + c.b, l);
    };
    // the loader runs DEEP - 1 tiles ahead, across the contexts' borders
    Cursor now, ahead;
    now.b = b;
    open(now, t0);
    ahead = now;
    int put = 0, take = 0;  // places in the ring
    const auto issue = [&]() {
        const int begun = (ahead.tile - ahead.begin) * 32;
        w.issue(w.ring + put * Wave::Ring::STAGE, ahead.off + begun, ahead.len - begun);
        put = put + 1 == DEEP ? 0 : put + 1;
        if (ahead.tile + 1 < ahead.end) {
            ahead.tile++;
        } else if (ahead.tile + 1 < t1) {
            open(ahead, ahead.tile + 1);
            w.touch_queries(dyn_lds + 8 * DEEP * Wave::Ring::STAGE + ts * 256, ahead.b);
        } else {
            ahead.tile++;
        }
    };
#pragma unroll
    for (int i = 0; i < DEEP - 1; i++)
        if (ahead.tile < t1) issue();
    w.begin(now.b);
    while (true) {
        Fp4Tile<W> t;
        if (ahead.tile < t1) issue();
        const int behind = ahead.tile - 1 - now.tile;  // tiles issued behind the one that is folded in now
        if (behind >= 2) wait_loads<2 * Wave::Ring::TILE_LOADS>();
        else if (behind == 1) wait_loads<Wave::Ring::TILE_LOADS>();
        else wait_loads<0>();
        char *stage = w.ring + take * Wave::Ring::STAGE;
        const int rows = now.len - (now.tile - now.begin) * 32;
        if (a.k_new != nullptr && rows <= 32) w.take_new_row(stage, now.b, now.off + now.len - 1, rows);
        w.read(t, stage);
        take = take + 1 == DEEP ? 0 : take + 1;
        w.fold(t, rows);
        const int next = now.tile + 1;
        if (next == now.end || next == t1) {
            finish(now);
            if (next == t1) break;
            open(now, next);
            w.begin(now.b);
        } else {
            now.tile = next;
        }
    }
    if (head.count + tail.count == 0) return;
    const unsigned who = pieces_arrived(a, head, tail, a.columns, col);
#pragma unroll 1
    for (int k = 0; k < 2; k++) {
        if (!(who >> k & 1)) continue;
        const Pending p = {k ? tail.b : head.b, k ? tail.first : head.first, k ? tail.count : head.count};
        w.merge_pieces(p.first + p.b, p.b, p.count);
    }
}

template <int ACT, int D, int NH, int NP>
__global__ void __launch_bounds__(512, 2) attn_fp4_share_kernel(const AttnArgs a) {
    const FirstEntry e = first_entry(a);
    fp4_share<ACT, D, NH, NP>(a);
    publish_lengths<D, NP == 3>(a, e);
}

template <int ACT, int NP, bool SHARES>
static attn_fn pick_fp4(int d, int nh) {
    if (SHARES) {
        if (d == 64) return nh == 4 ? attn_fp4_share_kernel<ACT, 64, 4, NP> : nh == 2 ? attn_fp4_share_kernel<ACT, 64, 2, NP> : attn_fp4_share_kernel<ACT, 64, 1, NP>;
        if (d == 128 && nh == 2) return attn_fp4_share_kernel<ACT, 128, 2, NP>;
        return d == 128 ? attn_fp4_share_kernel<ACT, 128, 1, NP> : d == 256 ? attn_fp4_share_kernel<ACT, 256, 1, NP> : nullptr;
    }
    if (d == 64) return nh == 2 ? attn_fp4_team_kernel<ACT, 64, 2, NP> : attn_fp4_team_kernel<ACT, 64, 1, NP>;
    return d == 128 ? attn_fp4_team_kernel<ACT, 128, 1, NP> : d == 256 ? attn_fp4_team_kernel<ACT, 256, 1, NP> : nullptr;
}

attn_fn s3i_pick_fp4(int act, int d, int heads_per_unit, bool wide_out, bool shares, int *lds) {
    const bool wide = d * heads_per_unit == 256;
    const int stage = wide ? Fp4Ring<256>::STAGE : Fp4Ring<128>::STAGE;
    *lds = shares ? 8 * (stage * (wide ? Fp4Ring<256>::DEEP : Fp4Ring<128>::DEEP) + 256) : 4 * stage * 2;
    if (act == S3_F16) {
        if (wide_out) return shares ? pick_fp4<S3_F16, 3, true>(d, heads_per_unit) : pick_fp4<S3_F16, 3, false>(d, heads_per_unit);
        return shares ? pick_fp4<S3_F16, 2, true>(d, heads_per_unit) : pick_fp4<S3_F16, 2, false>(d, heads_per_unit);
    }
    if (wide_out) return shares ? pick_fp4<S3_BF16, 3, true>(d, heads_per_unit) : pick_fp4<S3_BF16, 3, false>(d, heads_per_unit);
    return shares ? pick_fp4<S3_BF16, 2, true>(d, heads_per_unit) : pick_fp4<S3_BF16, 2, false>(d, heads_per_unit);
}

append_fp4_fn s3i_pick_append_fp4(int act) {
    return act == S3_F16 ? append_fp4_kernel<S3_F16> : act == S3_BF16 ? append_fp4_kernel<S3_BF16> : nullptr;
}
