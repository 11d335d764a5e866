// Norms of queries and keys for each head, position rotation, and append, in one pass over the joined projection of new tokens
// (s3_qk_rotary, s3_kv_append_rotary), and cached rows read back as 16-bit numbers (s3_kv_fetch), gfx950.
//
// A head x of D elements is first divided by its root mean square, x * rsqrt(mean(x^2) + eps) * w (if w is given), then its pairs
// (a, b) turn by the angle t = rot_pos[axis] * inv_freq[pair]: (a cos t - b sin t, a sin t + b cos t).  Per element that is
// y = inv * (x * cw + x' * sw), where x' is the other element of the pair and cw, sw hold cosine, (signed) sine and norm weight:
// they depend on the token and the element only, so a wave works them out once, a pair a lane, and goes through the token's heads with
// them.
// All in fp32, rounded once to the type of the output or to the codes of the cache; angles in turns of 64 bits, since a far
// position times a frequency leaves few bits of the turn in 32.
//
// Bound by memory (every element is read once and written once); a token alone by latency.  A lane has eight elements of a head
// (16 bytes); in the half-split pairing the other elements of its pairs are a second load, of a cache line that a neighbouring
// lane of the same load reads, which is cheaper than moving eight numbers between lanes.  Measured: 32768 tokens, 32 + 8 heads of 128, bf16,
// three axes: 149 us, 4.5 TB/s read and written (a copy of 2 GiB: 4.9); 256 tokens: 5 us; 7.6 thousand prompt tokens into 4-bit rows: 22 us.
#include <math.h>

#include "s3kv_fp4.h"

#define S3_ROT_16BIT 0
#define S3_ROT_E4M3 1
#define S3_ROT_MXFP4 2
#define S3_ROT_NONE 3  // no cache: keys go to k_out

struct RotaryArgs {
    const char *q, *k, *v;
    char *q_out, *k_out;
    int64_t q_step, k_step, v_step, q_out_step, k_out_step;  // bytes from token to token
    char *kplane, *vplane, *kscale, *vscale;
    const int64_t *slot_off;
    const int32_t *pos, *rot_pos;  // rot_pos: [n_axes][n], null: pos on every axis
    const float *inv_freq, *q_weight, *k_weight;
    int64_t n_tokens;
    int32_t n, Hq, Hkv, max_len;
    int32_t rotary, interleaved, n_axes;
    float eps;
    int32_t parts;       // a token's heads are shared out over this many waves
    uint64_t axes[4];    // two bits a pair
};

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// sin and cos of 2 pi x, |x| <= 1/2: the nearest quarter of a turn, and Taylor's sums for the rest (at most pi/4; the terms left out
// are below 2^-29).  Their first two terms are in 64 bits, so that a result is off by little more than its one rounding: errors of these
// two are common to a token's heads, and rows of few bits show them as codes beside the nearest (with all in 32 bits, 25 thousand rows of
// 8-bit keys had 1.5 times the wrong codes).
__device__ __forceinline__ void sin_cos_turn(const double x, float &s, float &c) {
    const double quarter = rint(4.0 * x), t = fma(-0.25, quarter, x) * 6.283185307179586477, t2 = t * t;
    const float u = (float)t2;
    const float ps = (float)fma(t * t2, (double)(u * (1.f / 120 + u * (-1.f / 5040 + u * (1.f / 362880)))) - 1.0 / 6, t);
    const float pc = (float)fma(t2, (double)(u * (1.f / 24 + u * (-1.f / 720 + u * (1.f / 40320 + u * (-1.f / 3628800))))) - 0.5, 1.0);
    const int k = (int)quarter & 3;
    s = k & 1 ? pc : ps;
    c = k & 1 ? ps : pc;
    if (k & 2) s = -s;
    if (k == 1 || k == 2) c = -c;
}

template <int ACT>
__device__ __forceinline__ u32x4 round8(const float (&y)[8]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (ACT == S3_F16) {
            const f16x2 h = {(_Float16)y[2 * i], (_Float16)y[2 * i + 1]};
            const unsigned packed = __builtin_bit_cast(unsigned, h);
            w[i] = packed;
        } else {
            w[i] = round_bf16x2(y[2 * i], y[2 * i + 1]);
        }
    }
    return w;
}

// Eight elements (from element e of head h, x in fp32) of a row of the cache, its codes or numbers at `row`, 4-bit: its scales at `scale`.
template <int ACT, int D, int CACHE>
__device__ __forceinline__ void store_row8(char *row, char *scale, int heads, int h, int e, const float (&x)[8]) {
    if (CACHE == S3_ROT_16BIT) {
        *(u32x4 *)(row + (h * D + e) * 2) = round8<ACT>(x);
    } else if (CACHE == S3_ROT_E4M3) {
        u32x2 w;
        w[0] = quantize2_e4m3<true>(x[2], x[3], quantize2_e4m3<false>(x[0], x[1], 0u));
        w[1] = quantize2_e4m3<true>(x[6], x[7], quantize2_e4m3<false>(x[4], x[5], 0u));
        *(u32x2 *)(row + h * D + e) = w;
    } else if (CACHE == S3_ROT_MXFP4) {
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) most = fp4_magnitude(x[i], most);
        most = group_max<4>(most);
        const unsigned byte = fp4_scale_byte<ACT>(__builtin_bit_cast(float, most));
        *(unsigned *)(row + (h * D + e) / 2) = fp4_codes8(x, byte);
        if ((e & 31) == 0) scale[(h * D + e) / 32] = (char)byte;
        if (h == heads - 1 && e == D - 8)  // zeros up to a multiple of 16 bytes
            for (int i = heads * (D / 32); i < fp4_scale_bytes(heads, D); i++) scale[i] = 0;
    }
}

// Eight consecutive floats (PIECE: 16-byte aligned ones from w[at[0]] on) of a norm's weight.
template <bool PIECE>
__device__ __forceinline__ void load_weight8(const float *w, const int (&at)[8], float (&x)[8]) {
    if (PIECE) {
        const f32x4 lo = *(const f32x4 *)(w + at[0]), hi = *(const f32x4 *)(w + at[0] + 4);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            x[i] = lo[i];
            x[4 + i] = hi[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = w[at[i]];
    }
}

// PAIRS: where the other elements of a lane's pairs are: 0 in the lane (interleaved), 1 in one 16-byte piece (half of the elements that
// turn a multiple of 8), 2 anywhere.
template <int ACT, int D, int CACHE, int PAIRS>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
    constexpr int LPH = D == 96 ? 16 : D / 8;  // lanes a head (of 96: twelve of sixteen)
    constexpr int GH = 64 / LPH;               // heads a wave takes at once
    constexpr int P = (D / 2 + 63) / 64;       // pairs a lane works out
    __shared__ f32x2 turned[4][64 * P];        // cosine and sine of a wave's token, by pair
    const int lane = threadIdx.x & 63, sub = lane / LPH, e0 = (lane % LPH) * 8;
    const bool lane_ok = D != 96 || e0 < D;
    const int e = lane_ok ? e0 : 0;
    f32x2 *mine = turned[__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)];
    const int64_t row_bytes = CACHE == S3_ROT_MXFP4 ? fp4_code_bytes(a.Hkv, D) : (int64_t)a.Hkv * D * (CACHE == S3_ROT_E4M3 ? 1 : 2);
    const int half = a.rotary / 2;
    // turns per position and axis of the lane's pairs, whatever the token
    double rate[P];
    int axis[P];
#pragma unroll
    for (int i = 0; i < P; i++) {
        const int pair = lane + 64 * i;
        rate[i] = pair < half ? (double)a.inv_freq[pair] * 0.15915494309189533577 : 0.0;
        axis[i] = (int)(a.axes[(pair >> 5) & 3] >> (2 * (pair & 31))) & 3;
    }
    // the lane's elements: the pair of the first, which half of its pair it is, and where the other elements are
    const bool second = e >= half;  // (PAIRS 1: of all eight)
    int at[8], other[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int el = e + i;
        const bool turns = el < a.rotary;
        at[i] = !turns ? 0 : PAIRS == 0 ? el >> 1 : el >= half ? el - half : el;
        other[i] = !turns ? el : PAIRS == 0 ? el ^ 1 : el >= half ? el - half : el + half;
    }
    const int gq = (a.Hq + GH - 1) / GH, gk = (a.Hkv + GH - 1) / GH, groups = gq + gk + (CACHE == S3_ROT_NONE ? 0 : gk);
    const unsigned lane_at = (unsigned)(sub * D + e) * 2, other_at = (unsigned)(sub * D + other[0]) * 2;
    for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < (int64_t)a.n * a.parts; item += (int64_t)gridDim.x * 4) {
        const int64_t t = uniform64(a.parts == 1 ? item : item / a.parts);
        const int part = __builtin_amdgcn_readfirstlane((int)(item - t * a.parts));
        // this wave's groups of heads: part, part + parts, ... of the queries', the keys' and the values'
        u32x4 raw, raw_other = {0u, 0u, 0u, 0u};
        unsigned short one[8];
        const auto load = [&](int x) {
            const char *src = x < gq ? a.q + t * a.q_step + (int64_t)x * (GH * D * 2)
                            : x < gq + gk ? a.k + t * a.k_step + (int64_t)(x - gq) * (GH * D * 2)
                                          : a.v + t * a.v_step + (int64_t)(x - gq - gk) * (GH * D * 2);
            const int left = x < gq ? a.Hq - x * GH : a.Hkv - (x < gq + gk ? x - gq : x - gq - gk) * GH;
            raw = (u32x4){0u, 0u, 0u, 0u};
            if (lane_ok && sub < left) {
                raw = *(const u32x4 *)(src + lane_at);
                if (x < gq + gk) {
                    if (PAIRS == 1) raw_other = *(const u32x4 *)(src + other_at);
                    if (PAIRS == 2) {
#pragma unroll
                        for (int i = 0; i < 8; i++) one[i] = *(const unsigned short *)(src + (unsigned)(sub * D + other[i]) * 2);
                    }
                }
            }
        };
        load(part);
        int64_t row = 0, scale = 0;  // bytes into the planes
        int32_t p = 0;
        if (CACHE != S3_ROT_NONE) {
            const int64_t off = a.slot_off[t];
            p = a.pos[t];
            if (off < 0 || p < 0 || p >= a.max_len || off + p >= a.n_tokens) continue;  // never leave the arena
            row = (off + p) * row_bytes;
            scale = CACHE == S3_ROT_MXFP4 ? (off + p) * fp4_scale_bytes(a.Hkv, D) : 0;
        }
        float cs[8], sn[8];
        if (half > 0 && part < gq + gk) {
            int32_t where[4];
#pragma unroll
            for (int x = 0; x < 4; x++) where[x] = a.rot_pos ? a.rot_pos[(int64_t)min(x, a.n_axes - 1) * a.n + t] : p;
#pragma unroll
            for (int i = 0; i < P; i++) {
                double turn = (double)(axis[i] & 2 ? axis[i] & 1 ? where[3] : where[2] : axis[i] & 1 ? where[1] : where[0]) * rate[i];
                turn -= rint(turn);
                float s, c;
                sin_cos_turn(turn, s, c);
                mine[lane + 64 * i] = (f32x2){c, s};
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const f32x2 v = PAIRS == 1 ? mine[at[0] + i] : mine[at[i]];
                const bool turns = (PAIRS == 1 ? e : e + i) < a.rotary;
                const bool b = PAIRS == 0 ? i & 1 : PAIRS == 1 ? second : e + i >= half;
                cs[i] = turns ? v[0] : 1.f;
                sn[i] = turns ? b ? v[1] : -v[1] : 0.f;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                cs[i] = 1.f;
                sn[i] = 0.f;
            }
        }
        float cw[8], sw[8];
        int kind = -1;  // of the heads at hand: queries, keys, values
        for (int x = part; x < groups; x += a.parts) {
            const int now = x < gq ? 0 : x < gq + gk ? 1 : 2, heads = now == 0 ? a.Hq : a.Hkv;
            const int h = (now == 0 ? x : now == 1 ? x - gq : x - gq - gk) * GH + sub;
            const float *weight = now == 0 ? a.q_weight : a.k_weight;
            if (now != kind && now < 2) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    cw[i] = cs[i];
                    sw[i] = sn[i];
                }
                if (weight) {
                    float w[8], wo[8];
                    const int first[8] = {e, e + 1, e + 2, e + 3, e + 4, e + 5, e + 6, e + 7};
                    load_weight8<true>(weight, first, w);
                    if (PAIRS == 0) {
#pragma unroll
                        for (int i = 0; i < 8; i++) wo[i] = w[i ^ 1];
                    } else {
                        load_weight8<PAIRS == 1>(weight, other, wo);
                    }
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        cw[i] *= w[i];
                        sw[i] *= wo[i];
                    }
                }
            }
            kind = now;
            const u32x4 bits = raw;
            float v[8], vo[8], y[8];
            widen8<ACT>(raw, v);
            if (PAIRS == 1) widen8<ACT>(raw_other, vo);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if (PAIRS == 0) vo[i] = v[i ^ 1];
                if (PAIRS == 2) vo[i] = widen16<ACT>(one[i]);
            }
            if (x + a.parts < groups) load(x + a.parts);  // the next heads are on their way while these are turned
            const bool ok = lane_ok && h < heads;
            if (now == 2) {
                if (!ok) continue;
                if (CACHE == S3_ROT_16BIT) *(u32x4 *)(a.vplane + row + (h * D + e) * 2) = bits;
                else store_row8<ACT, D, CACHE>(a.vplane + row, a.vscale + scale, a.Hkv, h, e, v);
                continue;
            }
            float inv = 1.f;
            if (weight) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; i++) sum = fmaf(v[i], v[i], sum);
                sum = group_sum<LPH>(sum);
                inv = 1.f / sqrtf(sum * (1.f / D) + a.eps);
            }
#pragma unroll
            for (int i = 0; i < 8; i++) {
                // (elements that do not turn: infinities times a sine of 0 are kept out)
                const float its = (PAIRS == 1 ? e : e + i) < a.rotary ? vo[i] * inv * sw[i] : 0.f;
                y[i] = fmaf(v[i] * inv, cw[i], its);
            }
            if (!ok) continue;
            if (now == 0) *(u32x4 *)(a.q_out + t * a.q_out_step + (h * D + e) * 2) = round8<ACT>(y);
            else if (CACHE == S3_ROT_NONE) *(u32x4 *)(a.k_out + t * a.k_out_step + (h * D + e) * 2) = round8<ACT>(y);
            else store_row8<ACT, D, CACHE>(a.kplane + row, a.kscale + scale, a.Hkv, h, e, y);
        }
    }
}

typedef void (*rotary_fn)(const RotaryArgs);
template <int ACT, int D, int PAIRS>
static rotary_fn pick_cache(int cache) {
    if (cache == S3_ROT_16BIT) return rotary_kernel<ACT, D, S3_ROT_16BIT, PAIRS>;
    if (cache == S3_ROT_NONE) return rotary_kernel<ACT, D, S3_ROT_NONE, PAIRS>;
    if constexpr (D != 96) {
        if (cache == S3_ROT_E4M3) return rotary_kernel<ACT, D, S3_ROT_E4M3, PAIRS>;
        if (cache == S3_ROT_MXFP4) return rotary_kernel<ACT, D, S3_ROT_MXFP4, PAIRS>;
    }
    return nullptr;
}
template <int ACT, int D>
static rotary_fn pick_pairs(int cache, int pairs) {
    return pairs == 0 ? pick_cache<ACT, D, 0>(cache) : pairs == 1 ? pick_cache<ACT, D, 1>(cache) : pick_cache<ACT, D, 2>(cache);
}
template <int ACT>
static rotary_fn pick_rotary(int d, int cache, int pairs) {
    return d == 64 ? pick_pairs<ACT, 64>(cache, pairs) : d == 96 ? pick_pairs<ACT, 96>(cache, pairs) : d == 128 ? pick_pairs<ACT, 128>(cache, pairs)
         : d == 256 ? pick_pairs<ACT, 256>(cache, pairs) : nullptr;
}

// Checks the rule for heads of d elements and puts it into the arguments.
static bool take_rule(const s3_rotary *r, int d, RotaryArgs &a) {
    if (!r || r->rotary_dim < 0 || r->rotary_dim > d || (r->rotary_dim & 1) || r->n_axes < 1 || r->n_axes > 4) return false;
    if (r->interleaved != 0 && r->interleaved != 1) return false;
    if (r->rotary_dim > 0 && !r->inv_freq) return false;
    if (r->n_axes > 1 && r->rotary_dim > 0 && !r->axis_of_pair) return false;
    if ((r->q_weight || r->k_weight) && (!(r->eps >= 0.f) || !aligned16(r->q_weight) || !aligned16(r->k_weight))) return false;
    a.rotary = r->rotary_dim;
    a.interleaved = r->interleaved;
    a.n_axes = r->n_axes;
    a.eps = r->eps;
    a.inv_freq = r->inv_freq;
    a.q_weight = r->q_weight;
    a.k_weight = r->k_weight;
    for (int i = 0; i < 4; i++) a.axes[i] = 0;
    if (r->n_axes > 1)
        for (int i = 0; i < r->rotary_dim / 2; i++) {
            if (r->axis_of_pair[i] >= r->n_axes) return false;
            a.axes[i >> 5] |= (uint64_t)r->axis_of_pair[i] << (2 * (i & 31));
        }
    return true;
}

// Elements from token to token of `heads` heads of d -> bytes; 0: dense.  -1: refused.
static int64_t step_bytes(int64_t stride, int heads, int d) {
    if (stride == 0) return (int64_t)heads * d * 2;
    return stride < (int64_t)heads * d || (stride & 7) || stride > ((int64_t)1 << 40) ? -1 : stride * 2;
}

static int launch_rotary(RotaryArgs &a, int act, int d, int cache, int cus, void *stream) {
    const int pairs = a.interleaved || a.rotary == 0 ? 0 : a.rotary % 16 == 0 ? 1 : 2;
    rotary_fn fn = act == S3_F16 ? pick_rotary<S3_F16>(d, cache, pairs) : act == S3_BF16 ? pick_rotary<S3_BF16>(d, cache, pairs) : nullptr;
    if (!fn) return S3_ERR_INVALID;
    const int gh = d == 96 ? 4 : 512 / d, groups = (a.Hq + gh - 1) / gh + (a.Hkv + gh - 1) / gh * (cache == S3_ROT_NONE ? 1 : 2);
    // Few tokens: their heads are shared out over waves until there are some sixteen waves a compute unit, so that a launch is one
    // pass through memory deep; beyond, a wave keeps its token's angles for all of its heads.
    const int64_t waves = (int64_t)16 * cus;
    int64_t parts = a.n >= waves ? 1 : waves / a.n;
    if (parts > groups) parts = groups;
    a.parts = (int32_t)parts;
    int64_t blocks = ((int64_t)a.n * parts + 3) / 4;
    if (blocks > 8 * cus) blocks = 8 * cus;
    hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        s3i_set_hip_error("rotary_kernel", (int)e, hipGetErrorString(e));
        return S3_ERR_HIP;
    }
    return S3_OK;
}

extern "C" int s3_qk_rotary(const s3_rotary *rule, int32_t dtype, int32_t head_dim, int32_t n, const int32_t *rot_pos, const void *q,
                            int32_t n_heads, int64_t q_stride, const void *k, int32_t n_kv_heads, int64_t k_stride, void *q_out,
                            void *k_out, void *stream) {
    RotaryArgs a = {};
    if (dtype != S3_F16 && dtype != S3_BF16) return S3_ERR_INVALID;
    if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return S3_ERR_INVALID;
    if (n < 0 || n_heads < 0 || n_kv_heads < 0 || n_heads > 65536 || n_kv_heads > 65536 || !take_rule(rule, head_dim, a)) return S3_ERR_INVALID;
    a.Hq = q ? n_heads : 0;
    a.Hkv = k ? n_kv_heads : 0;
    a.q_step = a.q_out_step = step_bytes(q_stride, a.Hq, head_dim);
    a.k_step = a.k_out_step = step_bytes(k_stride, a.Hkv, head_dim);
    if (a.q_step < 0 || a.k_step < 0) return S3_ERR_INVALID;
    if ((a.Hq > 0 && (!q_out || !aligned16(q) || !aligned16(q_out))) || (a.Hkv > 0 && (!k_out || !aligned16(k) || !aligned16(k_out))))
        return S3_ERR_INVALID;
    if (n == 0 || a.Hq + a.Hkv == 0) return S3_OK;
    if (!rot_pos && a.rotary > 0) return S3_ERR_INVALID;
    a.q = (const char *)q;
    a.k = (const char *)k;
    a.q_out = (char *)q_out;
    a.k_out = (char *)k_out;
    a.rot_pos = rot_pos;
    a.n = n;
    int32_t cus = 0;
    const int rc = s3i_device_cus(&cus);
    if (rc != S3_OK) return rc;
    return launch_rotary(a, dtype, head_dim, S3_ROT_NONE, cus, stream);
}

extern "C" int s3_kv_append_rotary(s3_arena *ar, int32_t layer, int32_t n, const int32_t *slot_id, const int32_t *pos_host,
                                   const int64_t *slot_off, const int32_t *pos, const s3_rotary *rule, const int32_t *rot_pos,
                                   const void *q, int64_t q_stride, const void *k_new, int64_t k_stride, const void *v_new,
                                   int64_t v_stride, void *q_out, void *stream) {
    RotaryArgs a = {};
    if (!ar || !ar->base || layer < 0 || layer >= ar->cfg.n_layers || n < 0 || !take_rule(rule, ar->cfg.head_dim, a)) return S3_ERR_INVALID;
    const int d = ar->cfg.head_dim;
    a.Hq = q ? ar->cfg.n_heads : 0;
    a.Hkv = ar->cfg.n_kv_heads;
    a.q_step = step_bytes(q_stride, a.Hq, d);
    a.k_step = step_bytes(k_stride, a.Hkv, d);
    a.v_step = step_bytes(v_stride, a.Hkv, d);
    a.q_out_step = (int64_t)a.Hq * d * 2;
    if (a.q_step < 0 || a.k_step < 0 || a.v_step < 0) return S3_ERR_INVALID;
    if (n == 0) return S3_OK;
    if (!slot_off || !pos || !k_new || !v_new || !aligned16(k_new) || !aligned16(v_new)) return S3_ERR_INVALID;
    if (q && (!q_out || !aligned16(q) || !aligned16(q_out))) return S3_ERR_INVALID;
    if (q && q_out == q && a.q_step != a.q_out_step) return S3_ERR_INVALID;  // rows would overwrite others that are still to be read
    const int rc = s3i_check_slots_host(ar, n, slot_id, pos_host);
    if (rc != S3_OK) return rc;
    a.q = (const char *)q;
    a.k = (const char *)k_new;
    a.v = (const char *)v_new;
    a.q_out = (char *)q_out;
    a.kplane = ar->plane(layer, 0);
    a.vplane = ar->plane(layer, 1);
    if (ar->tail_bytes > 0) {
        a.kscale = ar->tails(layer, 0);
        a.vscale = ar->tails(layer, 1);
    }
    a.slot_off = slot_off;
    a.pos = pos;
    a.rot_pos = rot_pos;
    a.n_tokens = ar->n_tokens;
    a.n = n;
    a.max_len = ar->cfg.max_len;
    const int cache = ar->cfg.kv_dtype == S3_E4M3 ? S3_ROT_E4M3 : ar->cfg.kv_dtype == S3_MXFP4 ? S3_ROT_MXFP4 : S3_ROT_16BIT;
    return launch_rotary(a, ar->cfg.act_dtype, d, cache, ar->num_cus > 0 ? ar->num_cus : 256, stream);
}

// ---- cached rows as numbers ----------------------------------------------------------------------------------------
struct FetchArgs {
    const char *kplane, *vplane, *kscale, *vscale;
    const int64_t *slot_off;
    const int32_t *pos;
    char *k_out, *v_out;
    int64_t n_tokens, row_bytes, scale_bytes;
    int32_t n, elems, max_len;  // elems: of a row
};

// A thread: eight elements of a row, the same ones of every row it takes; a workgroup has as many rows at once as it has threads for.
// Bound by memory: 25 thousand rows of 8 heads of 128, 8-bit: 34 us, 4.6 TB/s read and written.
template <int ACT, int CACHE>
__global__ void __launch_bounds__(256) fetch_kernel(const FetchArgs a) {
    const char *plane = blockIdx.y ? a.vplane : a.kplane;
    char *out = blockIdx.y ? a.v_out : a.k_out;
    if (!out) return;
    const int pieces = a.elems / 8, rows = pieces < 256 ? 256 / pieces : 1;
    const int mine = threadIdx.x / pieces, first = (threadIdx.x - mine * pieces) * 8;
    if (mine >= rows) return;
    for (int64_t t = (int64_t)blockIdx.x * rows + mine; t < a.n; t += (int64_t)gridDim.x * rows) {
        const int64_t off = a.slot_off[t], p = a.pos[t];
        if (off < 0 || p < 0 || p >= a.max_len || off + p >= a.n_tokens) continue;  // never leave the arena
        const char *row = plane + (off + p) * a.row_bytes, *scales = (blockIdx.y ? a.vscale : a.kscale) + (off + p) * a.scale_bytes;
        char *dst = out + t * a.elems * 2;
        for (int e = first; e < a.elems; e += 2048) {
            u32x4 w;
            if (CACHE == S3_ROT_16BIT) {
                w = *(const u32x4 *)(row + e * 2);
            } else if (CACHE == S3_ROT_E4M3) {
                const u32x2 c = *(const u32x2 *)(row + e);
                float lo[4], hi[4];
                widen4_e4m3(c[0], lo);
                widen4_e4m3(c[1], hi);
                const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                w = round8<ACT>(x);  // (exact: four significant bits)
            } else {
                const unsigned c = *(const unsigned *)(row + e / 2);
                const float scale = fp4_scale(*(const unsigned char *)(scales + e / 32));
                const bf16x2 b[4] = {fp4_widen2<0>(c, scale), fp4_widen2<1>(c, scale), fp4_widen2<2>(c, scale), fp4_widen2<3>(c, scale)};
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; j++) x[j] = (float)b[j >> 1][j & 1];
                w = round8<ACT>(x);  // (exact but for powers of two that the type does not reach)
            }
            *(u32x4 *)(dst + e * 2) = w;
        }
    }
}

typedef void (*fetch_fn)(const FetchArgs);
template <int ACT>
static fetch_fn pick_fetch(int kv_dtype) {
    return kv_dtype == S3_E4M3 ? fetch_kernel<ACT, S3_ROT_E4M3> : kv_dtype == S3_MXFP4 ? fetch_kernel<ACT, S3_ROT_MXFP4> : fetch_kernel<ACT, S3_ROT_16BIT>;
}

extern "C" int s3_kv_fetch(s3_arena *ar, int32_t layer, int32_t n, const int64_t *slot_off, const int32_t *pos, void *k_out, void *v_out,
                           void *stream) {
    if (!ar || !ar->base || layer < 0 || layer >= ar->cfg.n_layers || n < 0) return S3_ERR_INVALID;
    if (n == 0) return S3_OK;
    if (!slot_off || !pos || (!k_out && !v_out) || !aligned16(k_out) || !aligned16(v_out)) return S3_ERR_INVALID;
    FetchArgs a;
    a.kplane = ar->plane(layer, 0);
    a.vplane = ar->plane(layer, 1);
    a.slot_off = slot_off;
    a.pos = pos;
    a.k_out = (char *)k_out;
    a.v_out = (char *)v_out;
    a.n_tokens = ar->n_tokens;
    a.row_bytes = ar->row_bytes;
    a.scale_bytes = ar->tail_bytes;
    a.kscale = ar->tail_bytes > 0 ? ar->tails(layer, 0) : nullptr;
    a.vscale = ar->tail_bytes > 0 ? ar->tails(layer, 1) : nullptr;
    a.n = n;
    a.elems = ar->cfg.n_kv_heads * ar->cfg.head_dim;
    a.max_len = ar->cfg.max_len;
    const int64_t cus = ar->num_cus > 0 ? ar->num_cus : 256;
    const int rows = a.elems / 8 < 256 ? 256 / (a.elems / 8) : 1;
    int64_t blocks = ((int64_t)n + rows - 1) / rows;
    if (blocks > 16 * cus) blocks = 16 * cus;
    fetch_fn fn = ar->cfg.act_dtype == S3_F16 ? pick_fetch<S3_F16>(ar->cfg.kv_dtype) : pick_fetch<S3_BF16>(ar->cfg.kv_dtype);
    hipLaunchKernelGGL(fn, dim3((unsigned)blocks, 2), dim3(256), 0, (hipStream_t)stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        s3i_set_hip_error("fetch_kernel", (int)e, hipGetErrorString(e));
        return S3_ERR_HIP;
    }
    return S3_OK;
}
