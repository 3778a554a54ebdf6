// The KV cache behind the radix tree: rotary positions and append, attention of one new token over the paged
// cache, eviction by accumulated attention weight.  See include/klpm_kv.h for the ABI.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cooperative_groups.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <atomic>
#include <type_traits>
#include <utility>

#include "klpm_kv.h"

#define FULL_MASK 0xffffffffu
#define KLPM_MAX_TOKENS (1 << 30)      // of a sequence: a token number plus a CTA's stride stays within 31 bits

namespace {

#define CK(call) do { cudaError_t e_ = (call); if (e_ != cudaSuccess) { \
    fprintf(stderr, "klpm: %s failed at %s:%d: %s\n", #call, __FILE__, __LINE__, cudaGetErrorString(e_)); return RT_ERR_CUDA; } } while (0)

// ------------------------------------------------------------------------------------------------
// element types: float values in and out, one rounding to the nearest when stored
// ------------------------------------------------------------------------------------------------
template <int DT> struct Elem;
template <> struct Elem<KV_F32> { using T = float; };
template <> struct Elem<KV_BF16> { using T = __nv_bfloat16; };
template <> struct Elem<KV_F16> { using T = __half; };
template <> struct Elem<KV_E4M3> { using T = __nv_fp8_e4m3; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_fp8_e4m3 x) { return (float)x; }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_fp8_e4m3 from_float<__nv_fp8_e4m3>(float x) { return __nv_fp8_e4m3(x); }   // saturates

inline int elem_size(int dtype) { return dtype == KV_F32 ? 4 : dtype == KV_E4M3 ? 1 : 2; }

// ------------------------------------------------------------------------------------------------
// argument checks
// ------------------------------------------------------------------------------------------------
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

rt_status check_cache(const kv_cache* c) {
    if (!c || !c->k || !c->v) return RT_ERR_INVALID;
    if (c->dtype != KV_BF16 && c->dtype != KV_F16 && c->dtype != KV_E4M3) return RT_ERR_INVALID;
    if (c->n_pages < 1 || c->n_heads < 1 || c->head_dim < 1 || c->page_size < 1) return RT_ERR_INVALID;
    if (c->page_size & (c->page_size - 1)) return RT_ERR_INVALID;
    if (c->page_size > KV_MAX_PAGE_SIZE || c->head_dim > KV_MAX_HEAD_DIM) return RT_ERR_TOO_LARGE;
    if ((int64_t)c->n_pages * c->page_size > 0x7fffffffLL || c->n_heads > 65535) return RT_ERR_TOO_LARGE;
    const int es = elem_size(c->dtype);
    if ((c->head_dim * es) % 16 || !aligned16(c->k) || !aligned16(c->v)) return RT_ERR_INVALID;
    const int32_t extent[3] = {c->n_pages, c->page_size, c->n_heads};
    for (int i = 0; i < 3; ++i) {
        if (extent[i] == 1) continue;
        if (c->k_stride[i] < c->head_dim || c->v_stride[i] < c->head_dim) return RT_ERR_INVALID;
        if ((c->k_stride[i] * es) % 16 || (c->v_stride[i] * es) % 16) return RT_ERR_INVALID;
    }
    if (c->dtype == KV_E4M3) {
        if (!(c->k_scale > 0) || !(c->v_scale > 0) || isinf(c->k_scale) || isinf(c->v_scale)) return RT_ERR_INVALID;
    } else if (c->k_scale != 1.0f || c->v_scale != 1.0f) return RT_ERR_INVALID;
    return RT_OK;
}

rt_status check_rows(const kv_rows* r, int32_t n) {
    if (!r || (n > 0 && !r->data)) return RT_ERR_INVALID;
    if (r->dtype != KV_BF16 && r->dtype != KV_F16 && r->dtype != KV_F32) return RT_ERR_INVALID;
    if (r->n_heads < 1) return RT_ERR_INVALID;
    if (r->n_heads > 65535) return RT_ERR_TOO_LARGE;
    if (reinterpret_cast<uintptr_t>(r->data) % elem_size(r->dtype)) return RT_ERR_INVALID;
    return RT_OK;
}

// Whether rows of len elements at i * s0 + j * s1, i < n0, j < n1, lie apart: nothing two threads write may be the same.  Two of them overlap where some
// |i s0 - j s1| < len; usually one dimension lies within the other's stride.
bool rows_apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t len) {
    using wide = __int128;
    if (len < 1 || n0 < 1 || n1 < 1) return true;
    wide a = s0 < 0 ? -(wide)s0 : s0, b = s1 < 0 ? -(wide)s1 : s1;
    if (n0 > 1 && a < len) return false;
    if (n1 > 1 && b < len) return false;
    if (n0 == 1 || n1 == 1) return true;
    if (a > b) { const wide t = a; a = b; b = t; const int64_t n = n0; n0 = n1; n1 = n; }            // a: the smaller stride, of n0 rows
    if (b >= (wide)(n0 - 1) * a + len) return true;
    for (int64_t j = 1; j < n1 && j * b < (wide)(n0 - 1) * a + len; ++j) {
        const wide i = j * b / a, over = j * b - i * a;       // the rows of the other dimension on either side
        if ((i < n0 && over < len) || (i + 1 < n0 && a - over < len)) return false;
    }
    return true;
}

// The cache as kernels see it: strides in bytes, dimensions of one entry with stride 0.
struct CacheDev {
    char *k, *v;
    int64_t ks[3], vs[3];
    int32_t n_pages, page_shift, n_heads, dim;
    float k_scale, v_scale;
};

CacheDev cache_dev(const kv_cache* c) {
    CacheDev d;
    const int es = elem_size(c->dtype);
    const int32_t extent[3] = {c->n_pages, c->page_size, c->n_heads};
    d.k = (char*)c->k; d.v = (char*)c->v;
    for (int i = 0; i < 3; ++i) {
        d.ks[i] = extent[i] == 1 ? 0 : c->k_stride[i] * es;
        d.vs[i] = extent[i] == 1 ? 0 : c->v_stride[i] * es;
    }
    d.n_pages = c->n_pages; d.n_heads = c->n_heads; d.dim = c->head_dim;
    d.page_shift = 0;
    while ((1 << d.page_shift) < c->page_size) ++d.page_shift;
    d.k_scale = c->k_scale; d.v_scale = c->v_scale;
    return d;
}

struct RowsDev { char* p; int64_t sr, sh; int32_t heads; };
RowsDev rows_dev(const kv_rows* r) {
    RowsDev d;
    if (!r) { d.p = nullptr; d.sr = d.sh = 0; d.heads = 0; return d; }
    const int es = elem_size(r->dtype);
    d.p = (char*)r->data; d.sr = r->stride[0] * es; d.sh = r->stride[1] * es; d.heads = r->n_heads;
    return d;
}
bool rows_aligned(const kv_rows* r) {
    const int es = elem_size(r->dtype);
    return aligned16(r->data) && (r->stride[0] * es) % 16 == 0 && (r->stride[1] * es) % 16 == 0;
}

// ------------------------------------------------------------------------------------------------
// rotary positions
// ------------------------------------------------------------------------------------------------
__global__ void rope_table_kernel(double* turns, int32_t rot, double theta, int32_t scaling, double scale, double original_len,
                                  double fast, double slow) {
    const int32_t i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= rot / 2) return;
    if (scaling == KV_ROPE_NTK) theta *= pow(scale, (double)rot / (rot - 2));
    double f = pow(theta, -2.0 * i / rot) / 6.283185307179586476925;
    if (scaling == KV_ROPE_LINEAR) f /= scale;
    if (scaling == KV_ROPE_YARN) {
        double keep = (original_len * f - slow) / (fast - slow);
        keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
        f *= keep + (1 - keep) / scale;
    }
    turns[i] = f;
}

struct AppendArgs {
    CacheDev c;
    RowsDev q, qo, k, v;
    const double* turns;          // NULL: no rotation
    const int32_t *pos, *slot;
    int32_t n, rot, interleaved;
    float factor;
    int32_t units;                // of a head: pairs, or 16 elements
    int32_t slices, tokens;       // of a CTA: threads that share a token's heads (in each of gridDim.y CTAs), tokens
};

// (a, b) -> (a cos - b sin, a sin + b cos) for the pairs of a head, angle = position x turns x 2 pi.  One thread handles one unit of a head -- a
// pair of elements, or (VEC) 8 pairs in 16 elements that two 16-byte loads bring -- of some of a token's heads.  A CTA works out the angles of its
// tokens once, in shared memory (64-bit products, a sine and a cosine each: with every thread at its own, 300 tokens of 12 heads took
// 4.5 us instead of 3.0).  Bound by HBM for many tokens (32,768 of 32 + 2 x 8 heads of 128, bf16: 137.7 us, 5.9 TB/s of what has to
// be read and written), by the launch and three dependent loads for few (1 token 2.4 us, 193 into an 8-bit cache 3.4 us).
template <int TX, int TC, bool VEC>
__global__ void __launch_bounds__(256) rope_append_kernel(const AppendArgs A) {
    using X = typename Elem<TX>::T;
    using C = typename Elem<TC>::T;
    constexpr int P = VEC ? 8 : 1;
    extern __shared__ float2 s_turned[];          // [tokens][rot / 2] cosine and sine
    const int tid = threadIdx.x, per = A.units * A.slices, half = A.turns ? A.rot / 2 : 0;
    const int64_t t0 = (int64_t)blockIdx.x * A.tokens;
    const int mine = tid / per, r = tid - mine * per;         // the token of this CTA's
    const int32_t slice = r / A.units, u = r - slice * A.units;
    for (int i = tid; i < A.tokens * half; i += 256) {
        const int which = i / half, pair = i - which * half;
        if (t0 + which >= A.n) break;
        // whole turns are taken off in 64 bits.  The product is off by half a step, 2^-25 of a turn at 2^31 positions of 1 / (2 pi) turns and less in proportion
        // nearer by; the rounding of the table's entry adds about as much, that of the rest to 32 bits 2^-26
        double t = (double)__ldg(A.pos + t0 + which) * __ldg(A.turns + pair);
        t -= rint(t);
        float sn, cs;
        sincospif(2.0f * (float)t, &sn, &cs);
        s_turned[i] = make_float2(cs * A.factor, sn * A.factor);
    }
    __syncthreads();
    const int64_t tok = t0 + mine;
    if (mine >= A.tokens || tok >= A.n) return;
    // The unit's elements: P from e0 and P from e1 on, half of the rotated elements (or half of the others) apart, so that neighbouring
    // threads are neighbours in memory.  Pairs are (e0 + j, e1 + j), or if interleaved neighbours in each of the two (VEC) or e0, e0 + 1.
    const int32_t rot_units = A.turns ? A.rot / (2 * P) : 0;
    const bool turn = u < rot_units;
    const int32_t v = turn ? u : u - rot_units, from = turn ? 0 : 2 * P * rot_units, size = turn ? A.rot : A.c.dim - from;
    const bool next = !VEC && turn && A.interleaved;
    const int32_t e0 = next ? 2 * v : from + v * P, e1 = next ? e0 + 1 : from + size / 2 + v * P;
    float cs[P], sn[P];
#pragma unroll
    for (int j = 0; j < P; ++j) { cs[j] = 1.0f; sn[j] = 0.0f; }
    if (turn) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int32_t pair = !VEC || !A.interleaved ? u * P + j : j < P / 2 ? e0 / 2 + j : e1 / 2 + j - P / 2;
            const float2 f = s_turned[mine * half + pair];
            cs[j] = f.x; sn[j] = f.y;
        }
    }
    const int32_t slot = __ldg(A.slot + tok);
    const int32_t page = slot >> A.c.page_shift, at = slot & ((1 << A.c.page_shift) - 1);
    const bool stored = slot >= 0 && page < A.c.n_pages;
    const int32_t heads = A.q.heads + A.k.heads + A.v.heads;
    for (int32_t h = blockIdx.y * A.slices + slice; h < heads; h += A.slices * gridDim.y) {
        const bool is_q = h < A.q.heads, is_v = h >= A.q.heads + A.k.heads;
        if (!is_q && !stored) break;
        const RowsDev& R = is_q ? A.q : is_v ? A.v : A.k;
        const int32_t hh = is_q ? h : is_v ? h - A.q.heads - A.k.heads : h - A.q.heads;
        const X* x = reinterpret_cast<const X*>(R.p + (int64_t)tok * R.sr + (int64_t)hh * R.sh);
        float a[P], b[P];
        if constexpr (VEC) {
            alignas(16) X xa[8], xb[8];
#pragma unroll
            for (int j = 0; j < (int)sizeof(X) / 2; ++j) {
                reinterpret_cast<int4*>(xa)[j] = reinterpret_cast<const int4*>(x + e0)[j];
                reinterpret_cast<int4*>(xb)[j] = reinterpret_cast<const int4*>(x + e1)[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) { a[j] = to_float(xa[j]); b[j] = to_float(xb[j]); }
        } else { a[0] = to_float(x[e0]); b[0] = to_float(x[e1]); }
        if (turn && !is_v) {
            if (VEC && A.interleaved) {
#pragma unroll
                for (int j = 0; j < P / 2; ++j) {
                    const float p0 = a[2 * j], p1 = a[2 * j + 1], q0 = b[2 * j], q1 = b[2 * j + 1];
                    a[2 * j] = p0 * cs[j] - p1 * sn[j];
                    a[2 * j + 1] = p0 * sn[j] + p1 * cs[j];
                    b[2 * j] = q0 * cs[P / 2 + j] - q1 * sn[P / 2 + j];
                    b[2 * j + 1] = q0 * sn[P / 2 + j] + q1 * cs[P / 2 + j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float p0 = a[j], p1 = b[j];
                    a[j] = p0 * cs[j] - p1 * sn[j];
                    b[j] = p0 * sn[j] + p1 * cs[j];
                }
            }
        }
        if (is_q) {
            X* y = reinterpret_cast<X*>(A.qo.p + (int64_t)tok * A.qo.sr + (int64_t)hh * A.qo.sh);
            if constexpr (VEC) {
                alignas(16) X ya[8], yb[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) { ya[j] = from_float<X>(a[j]); yb[j] = from_float<X>(b[j]); }
#pragma unroll
                for (int j = 0; j < (int)sizeof(X) / 2; ++j) {
                    reinterpret_cast<int4*>(y + e0)[j] = reinterpret_cast<int4*>(ya)[j];
                    reinterpret_cast<int4*>(y + e1)[j] = reinterpret_cast<int4*>(yb)[j];
                }
            } else { y[e0] = from_float<X>(a[0]); y[e1] = from_float<X>(b[0]); }
        } else {
            const int64_t* st = is_v ? A.c.vs : A.c.ks;
            C* y = reinterpret_cast<C*>((is_v ? A.c.v : A.c.k) + page * st[0] + at * st[1] + hh * st[2]);
            if constexpr (TC == KV_E4M3) {
                const float scale = is_v ? A.c.v_scale : A.c.k_scale;
#pragma unroll
                for (int j = 0; j < P; ++j) { a[j] = __fdiv_rn(a[j], scale); b[j] = __fdiv_rn(b[j], scale); }
            }
            if constexpr (VEC) {
                alignas(16) C ya[8], yb[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) { ya[j] = from_float<C>(a[j]); yb[j] = from_float<C>(b[j]); }
                using V = typename std::conditional<sizeof(C) == 1, int2, int4>::type;
                *reinterpret_cast<V*>(y + e0) = *reinterpret_cast<V*>(ya);
                *reinterpret_cast<V*>(y + e1) = *reinterpret_cast<V*>(yb);
            } else { y[e0] = from_float<C>(a[0]); y[e1] = from_float<C>(b[0]); }
        }
    }
}

template <int TX, int TC> void launch_append(const AppendArgs& A, bool vec, dim3 grid, size_t smem, cudaStream_t s) {
    if (vec) rope_append_kernel<TX, TC, true><<<grid, 256, smem, s>>>(A);
    else rope_append_kernel<TX, TC, false><<<grid, 256, smem, s>>>(A);
}

// ------------------------------------------------------------------------------------------------
// attention of one new token
//
// out_h = sum_t p_t v_t / sum_t p_t with p_t = 2^(s_t - m), s_t = scale log2(e) q_h . k_t and m the largest s_t seen so far; when m
// grows, what has been summed is multiplied by 2^(old m - new m).  Parts of a sequence are joined by the same rule.
//
// The floor is one read of the cache's rows (512 B per token and cache head at 128 elements of 16 bits, against a few flops per
// byte), so everything is laid out for loads in flight:
//   - Up to 16 query heads of a cache head (8 where heads have more than 128 elements: the sums are in registers) go through the tensor cores together
//     (mma.sync, 16 x 8 x 16): a tile of keys is read once for all of them.  More query heads are units of their own, which read it again.  Tokens,
//     then elements of the values, take the 16 rows of the operand that comes from shared memory, 8 heads the 8 columns.  tcgen05 has nothing to give here: its tiles would hold 128 rows for a few flops per byte that is read anyway.
//   - A warp works alone: its half tiles (keys, then values, of 16 or 32 tokens) come through a ring of its own in shared
//     memory (cp.async, 16 bytes a lane), with its own m and sums.  No barrier in the loop.  The warps of an SM hide what the
//     dependent steps of one take.  Up to 128 elements and 8 query heads there are 16 of them, with half tiles of 4 KB (2 KB: 64 elements in 8 bits) of which
//     two or four each are in flight; 8 warps with more query heads or wider heads (half tiles of 8 KB: 256 elements of 16 bits).
//   - All tiles of the batch, in the order (sequence, unit, tile), are cut into equal spans, one per warp of a grid that fills the
//     GPU once: ragged lengths leave no warp with more than another.  A row that is cut is joined by decode_join_kernel.
//     A unit is a cache head and up to 8 NT of its query heads.
//   - Probabilities enter the second product as the sum of two 16-bit numbers (off by 2^-16 of each at most with bf16, 2^-22 with f16, there nothing below
//     2^-39 of the row's largest), whose products go to the same sums; what divides them is summed before that.  One bf16 number would add as much error as the
//     output's own rounding has; a third would cost a third more products for what that rounding hides.  f16 probabilities are scaled
//     by 2^15 so that small ones keep their bits.  A bf16 query next to an 8-bit cache becomes f16, times a power of two per head that brings its largest
//     element next to 2^15: exact down to 2^-29 of that, nothing below 2^-39 of it.
// Measured (a graph of calls; MB are those that have to be read): 128 sequences of up to 16,384 tokens, 4.28 GB in 650 us, 6.6 TB/s, what a plain
// copy reaches; 33 of up to 8,191, 557 MB in 99 us, 10 us of which are start and join, with weights 115 us; 2 of 131,072 in 8 bits, 268 MB
// in 60 us: the conversions to f16 take as many instructions as everything else.
// ------------------------------------------------------------------------------------------------
struct DecodeArgs {
    CacheDev c;
    RowsDev q, out;
    const int32_t *table, *len;
    int64_t table_stride;
    int32_t n_seqs, group, max_tokens, window;
    int32_t head_tiles, units;         // units of a cache head, of a sequence
    int32_t q_words;                   // query rows may be read in words of 4 bytes
    float scale;
    float* lse;                        // nullable
    float* weight;                     // nullable
    int64_t ws[2];
    // workspace
    long long* tiles_before;           // [n_seqs + 1] tiles of the sequences before
    float* lse2;                       // [n_seqs, q heads] base-2 logarithm of the softmax's sum
    float* part;                       // [warps][2][8 NT][2 + DP]: m, sum, output of the two rows that a warp may share with others
    float* score;                      // [n_seqs, q heads, score_len] (with weight only)
    int64_t score_len;
    int32_t warps;
};

#define KLPM_DECODE_WARPS 4             // of a CTA
#define KLPM_DECODE_MIN_SPAN 2          // tiles
#define KLPM_SMS 148

template <int TQ_, int TC_, int DP_, int NT_> struct Dec {
    static constexpr int TQ = TQ_, TC = TC_, DP = DP_, NT = NT_;
    static constexpr bool E8 = TC == KV_E4M3;
    static constexpr bool HALF = E8 || TC == KV_F16;           // the products are of f16, else of bf16
    static constexpr bool SCALED = E8 && TQ == KV_BF16;        // the query becomes f16
    static constexpr int ROW = DP * (E8 ? 1 : 2);              // bytes of a row in shared memory
    static constexpr int CH = ROW / 16;
    static constexpr int TT = (E8 ? DP <= 128 : DP <= 64) ? 32 : 16;
    static constexpr int TILE = TT * ROW;                      // bytes of a half tile: keys or values
    static constexpr int CTAS = DP > 128 || NT > 1 ? 2 : 4;      // per SM: what the registers leave room for
    static constexpr int FIT = 192 * 1024 / (CTAS * KLPM_DECODE_WARPS * TILE);
    static constexpr int RING = FIT < 5 ? 3 : 5;               // half tiles (an odd number: what is loaded is what is used, some tiles ahead)
    static constexpr int WARP_SMEM = RING * TILE;
    static constexpr int SMEM = KLPM_DECODE_WARPS * WARP_SMEM;
    static constexpr int HEADS = 8 * NT;
    static constexpr int PART = HEADS * (2 + DP);
    static constexpr int KS = DP / 16;                         // steps of the first product, tiles of the output
};

__device__ __forceinline__ void token_range(const DecodeArgs& A, int32_t b, int32_t* lo, int32_t* hi) {
    int32_t n = __ldg(A.len + b);
    n = n < 0 ? 0 : n > A.max_tokens ? A.max_tokens : n;
    *hi = n;
    *lo = A.window > 0 && n > A.window ? n - A.window : 0;
}
template <int TT> __device__ __forceinline__ int32_t tiles_of(const DecodeArgs& A, int32_t b, int32_t* first) {
    int32_t lo, hi;
    token_range(A, b, &lo, &hi);
    *first = lo / TT;
    return hi > lo ? (hi + TT - 1) / TT - lo / TT : 0;
}
__device__ __forceinline__ long long span_of(long long total, int32_t warps) {
    const long long s = (total + warps - 1) / warps;
    return s < KLPM_DECODE_MIN_SPAN ? KLPM_DECODE_MIN_SPAN : s;
}

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int OFF> __device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {      // bytes 0: 16 zeros, nothing is read
    asm volatile("cp.async.cg.shared.global [%0 + %3], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes), "n"(OFF) : "memory");
}
template <int OFF> __device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0 + %2], [%1], 16;" :: "r"(dst), "l"(src), "n"(OFF) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }
template <int OFF> __device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4 + %5];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a), "n"(OFF) : "memory");
}
template <int OFF> __device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4 + %5];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a), "n"(OFF) : "memory");
}
template <int OFF> __device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4 + %5];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a), "n"(OFF) : "memory");
    return v;
}
template <int OFF> __device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2 + %3];" : "=r"(v.x), "=r"(v.y) : "r"(a), "n"(OFF) : "memory");
    return v;
}
// f(0), f(1), ... f(N - 1) with constants
template <class F, int... I> __device__ __forceinline__ void unrolled_(F& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, class F> __device__ __forceinline__ void unrolled(F f) { unrolled_(f, std::make_integer_sequence<int, N>()); }
template <bool HALF> __device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {          // of 16-bit elements, lane 4r + j holding columns 2j, 2j+1 of row r
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void e4m3_to_f16(uint32_t four, uint32_t* lo, uint32_t* hi) {           // exact; two values each
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(*lo) : "h"((unsigned short)four));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(*hi) : "h"((unsigned short)(four >> 16)));
}
// x and y as the sums of two 16-bit numbers each
template <bool HALF> __device__ __forceinline__ void split2(float x, float y, uint32_t* hi, uint32_t* lo) {
    if constexpr (HALF) {
        const __half2 h = __floats2half2_rn(x, y);
        const float2 f = __half22float2(h);
        const __half2 l = __floats2half2_rn(x - f.x, y - f.y);
        *hi = *reinterpret_cast<const uint32_t*>(&h); *lo = *reinterpret_cast<const uint32_t*>(&l);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        const float2 f = __bfloat1622float2(h);
        const __nv_bfloat162 l = __floats2bfloat162_rn(x - f.x, y - f.y);
        *hi = *reinterpret_cast<const uint32_t*>(&h); *lo = *reinterpret_cast<const uint32_t*>(&l);
    }
}
__device__ __forceinline__ float exp2_fast(float x) {        // 2 ulp; 2^-inf = 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Where chunk c of row r is, in 16-byte units.  Two-byte types: the eight rows of an ldmatrix lie in eight different 16-byte
// columns.  8-bit keys: lanes read chunks j, j < 4, of rows 2i and 2i+1 together; 8-bit values: chunks n, n+1 (or half chunks) of rows 0, 2, 4, 6.
// place(a + b, c) = (place(a, c) ^ (place(b, 0) - b rows)) + b rows for a multiple b of a power of two above a: addresses of a lane differ
// by constants.
template <class X, bool VALUE> __host__ __device__ constexpr int place(int r, int c) {
    if constexpr (!X::E8) return r * X::CH + (c ^ (r & 7));
    else if constexpr (X::CH == 4) return VALUE ? (r >> 1) * 8 + ((((r & 1) << 2) + c) ^ (((r >> 1) & 3) << 1)) : r * 4 + c;
    else if constexpr (!VALUE) return r * X::CH + (c ^ ((r & 1) << 2));
    else if constexpr (X::CH == 8) return r * 8 + (c ^ (((r >> 1) & 3) << 1));
    else return r * X::CH + (c ^ (((r >> 1) & 1) | (((r >> 2) & 1) << 2)));
}

// The element of a head that index k (0..15) of step ks of the first product stands for, in groups of two: lane column j holds
// k = 2j, 2j+1 (part 0) and 2j+8, 2j+9 (part 1).  8-bit keys: 16 consecutive elements per lane serve four steps.
template <class X> __device__ __forceinline__ int q_element(int ks, int j, int part) {
    if constexpr (X::E8) return (ks >> 2) * 64 + j * 16 + (ks & 3) * 4 + part * 2;
    else return ks * 16 + j * 2 + part * 8;
}
// The element that row r + 8e of output tile x stands for.
template <class X> __device__ __forceinline__ int out_element(int x, int r, int e) {
    if constexpr (X::E8) return r * (X::DP / 8) + 2 * x + e;
    else return x * 16 + r + 8 * e;
}

template <class X> struct Cursor {       // a tile of the batch: of sequence b, unit (cache head g, its query heads from 8 NT ht on)
    int32_t b, g, ht, tile, first, end, lo, hi;
    __device__ __forceinline__ void row(const DecodeArgs& A) {           // to the first tile of sequence b or of the next one that has any
        for (; b < A.n_seqs; ++b) {
            token_range(A, b, &lo, &hi);
            if (hi > lo) break;
        }
        first = lo / X::TT;
        end = (hi + X::TT - 1) / X::TT;
        tile = first;
    }
    __device__ __forceinline__ void next(const DecodeArgs& A) {
        if (++tile < end) return;
        tile = first;
        if (++ht < A.head_tiles) return;
        ht = 0;
        if (++g < A.c.n_heads) return;
        g = 0;
        ++b;
        row(A);
    }
    __device__ __forceinline__ int32_t head(const DecodeArgs& A) const { return g * A.group + ht * X::HEADS; }       // the first query head
};

// One warp computes `left` tiles of the batch from ci on.  finish(tile, begun, ended, heads, m, l, o) is called with what a row came to when the
// row or the span ends: begun and ended say whether the warp had the row's first and last tile.
template <class X, class F>
__device__ __forceinline__ void decode_span(const DecodeArgs& A, uint32_t ring, unsigned* s_there, Cursor<X> ci, long long left, F finish) {
    using Q = typename Elem<X::TQ>::T;
    constexpr int TT = X::TT, KS = X::DP / 16, TN = TT / 16, NT = X::NT, RING = X::RING;
    const int lane = threadIdx.x & 31;
    const int32_t chunks = A.c.dim * (X::E8 ? 1 : 2) / 16;
    Cursor<X> cc = ci;                                        // the tile that is computed next (ci: the one that is loaded next)
    long long to_load = left;
    const int32_t in_page = (1 << A.c.page_shift) - 1;
    const int my_row = lane / X::CH % TT, my_ch = lane % X::CH;
    // the page of token `lane` of the tile at ci; -1: nothing there
    auto page_of = [&]() -> int32_t {
        const int32_t t = ci.tile * TT + lane;
        int32_t p = -1;
        if (lane < TT && t >= ci.lo && t < ci.hi) p = __ldg(A.table + ci.b * A.table_stride + (t >> A.c.page_shift));
        return p < A.c.n_pages ? p : -1;                      // (negative: not there either)
    };
    int32_t page_next = page_of(), page = -1, at = 0, g_now = 0;           // (at: the lane's token's place in its page)
    int slot_in = 0, tile_in = 0;
    unsigned there_now = 0;                                   // which tokens of the tile that is being loaded are there
    auto copy_rows = [&](auto value) {
        constexpr bool VALUE = decltype(value)::value;
        constexpr int RPI = 32 / X::CH;                       // rows of one instruction
        const int64_t s0 = VALUE ? A.c.vs[0] : A.c.ks[0], s1 = VALUE ? A.c.vs[1] : A.c.ks[1];
        const char* base = (VALUE ? A.c.v : A.c.k) + g_now * (VALUE ? A.c.vs[2] : A.c.ks[2]) + my_ch * 16;
        const uint32_t to = ring + slot_in * X::TILE + place<X, VALUE>(my_row, my_ch) * 16;
        if (A.c.page_shift >= (TT == 32 ? 5 : 4) && there_now == (TT == 32 ? 0xffffffffu : 0xffffu)) {
            // the whole tile lies in one page
            const char* p = base + __shfl_sync(FULL_MASK, page, 0) * s0 + (__shfl_sync(FULL_MASK, at, 0) + my_row) * s1;
            if (my_ch < chunks)
                unrolled<TT / RPI>([&](auto i) {
                    constexpr int R = i.value * RPI, FLIP = place<X, VALUE>(R, 0) * 16 - R * X::ROW;
                    cp_async16<R * X::ROW>(to ^ FLIP, p);
                    p += RPI * s1;
                });
        } else {
            const int64_t mine = page < 0 ? 0 : page * s0 + at * s1;
            unrolled<TT / RPI>([&](auto i) {
                constexpr int R = i.value * RPI, FLIP = place<X, VALUE>(R, 0) * 16 - R * X::ROW;
                const char* p = base + __shfl_sync(FULL_MASK, mine, R + my_row);
                const int bytes = (there_now >> (R + my_row) & 1) << 4;
                if (my_ch < chunks) cp_async16<R * X::ROW>(to ^ FLIP, p, bytes);
            });
        }
        if (++slot_in == RING) slot_in = 0;
    };
    auto load_keys = [&]() {
        if (to_load > 0) {
            page = page_next;
            at = (ci.tile * TT + lane) & in_page;
            g_now = ci.g;
            there_now = __ballot_sync(FULL_MASK, page >= 0);
            if (lane == 0) s_there[tile_in & 7] = there_now;
            ++tile_in;
            if (to_load > 1) {
                ci.next(A);
                page_next = page_of();
            }
            copy_rows(std::false_type());
        }
        cp_async_commit();
    };
    auto load_values = [&]() {
        if (to_load > 0) {
            --to_load;
            copy_rows(std::true_type());
        }
        cp_async_commit();
    };

    const int r8 = lane >> 2, j = lane & 3;
    const float log2e = 1.4426950408889634f;
    // what the lane reads of a half tile.  Keys: tokens 0-15, two chunks; values: tokens 0-7 and 8-15 of two chunks
    const int in_keys = X::E8 ? place<X, false>(r8, j) * 16 : place<X, false>(lane & 15, lane >> 4) * 16;
    const int in_values = !X::E8 ? place<X, true>((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1) * 16
                        : X::CH == 4 ? place<X, true>(2 * j, r8 >> 1) * 16 + (r8 & 1) * 8 : place<X, true>(2 * j, r8 * (X::CH / 8)) * 16;
    uint32_t qb[NT][KS][2];
    float coef[NT][2], m[NT][2], l[NT][2], o[NT][KS][4];
    bool fresh = true, begun_here = false;
    int32_t heads = 0;
    int slot_out = 0, tile_out = 0;
    auto step = [&]() -> uint32_t {                           // the next half tile has arrived, and the one before it is no longer read
        cp_async_wait<RING - 2>();
        __syncwarp();
        const uint32_t a = ring + slot_out * X::TILE;
        if (++slot_out == RING) slot_out = 0;
        return a;
    };
    // (RING - 1) / 2 tiles ahead: the first rounds only load.  (One copy of the code: a small call runs through it once or twice, and what it
    // has to fetch of it counts)
    int ahead = (RING - 1) / 2;
    uint32_t ph[NT][TN][2], pl[NT][TN][2];
    for (;;) {
        const bool live = ahead == 0;
        if (live && fresh) {                                  // a row begins, or the span begins inside one
            fresh = false;
            begun_here = cc.tile == cc.first;
            heads = min(X::HEADS, A.group - cc.ht * X::HEADS);
            const char* qp = A.q.p + cc.b * A.q.sr + (int64_t)cc.head(A) * A.q.sh;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const bool have = n * 8 + r8 < heads;
                const uint16_t* q = reinterpret_cast<const uint16_t*>(qp + (n * 8 + r8) * A.q.sh);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const int d = q_element<X>(ks, j, part);
                        qb[n][ks][part] = !have || d >= A.c.dim ? 0u : A.q_words ? __ldg(reinterpret_cast<const uint32_t*>(q + d))
                                                                                : __ldg(q + d) | (uint32_t)__ldg(q + d + 1) << 16;
                    }
                float c = A.scale * A.c.k_scale * log2e;
                if constexpr (X::SCALED) {
                    float most = 0.0f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int part = 0; part < 2; ++part) {
                            const float x = fabsf(__uint_as_float(qb[n][ks][part] << 16)), y = fabsf(__uint_as_float(qb[n][ks][part] & 0xffff0000u));
                            if (x < INFINITY) most = fmaxf(most, x);
                            if (y < INFINITY) most = fmaxf(most, y);
                        }
                    most = fmaxf(most, __shfl_xor_sync(FULL_MASK, most, 1));
                    most = fmaxf(most, __shfl_xor_sync(FULL_MASK, most, 2));
                    int e = 0;
                    if (most > 0.0f) frexpf(most, &e);
                    // (-113: the largest elements, from 2^127 on, become 2^14 and more; with 110 the smallest, 2^-133, are f16's 2^-23.  64 bits, as
                    // the scale that goes with such queries may be subnormal)
                    e = max(-113, min(110, 15 - e));
                    const float up = ldexpf(1.0f, e);
                    c = (float)((double)A.scale * A.c.k_scale * 1.4426950408889634 * (double)ldexpf(1.0f, -e));
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int part = 0; part < 2; ++part) {
                            const __half2 h = __floats2half2_rn(__uint_as_float(qb[n][ks][part] << 16) * up, __uint_as_float(qb[n][ks][part] & 0xffff0000u) * up);
                            qb[n][ks][part] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                }
                coef[n][0] = __shfl_sync(FULL_MASK, c, 8 * j);           // of heads 2j and 2j+1
                coef[n][1] = __shfl_sync(FULL_MASK, c, 8 * j + 4);
#pragma unroll
                for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = 0.0f; }
#pragma unroll
                for (int x = 0; x < KS; ++x) o[n][x][0] = o[n][x][1] = o[n][x][2] = o[n][x][3] = 0.0f;
            }
        }
        // s = k . q, tokens x heads
        uint32_t sk = 0;
        if (live) sk = step();
        load_keys();
        if (live) {
        float s[NT][TN][4], s2[NT][1][4];                     // (one group of tokens: sums of every other step, shorter chains)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][t][i] = s2[n][0][i] = 0.0f;
        auto kq = [&](int t, int ks, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16816<X::HALF>(TN == 1 && ks & 1 ? s2[n][0] : s[n][t], a0, a1, a2, a3, qb[n][ks][0], qb[n][ks][1]);
        };
        const uint32_t key = sk + in_keys;
        if constexpr (X::E8) {
            unrolled<X::DP / 64>([&](auto h) {
                constexpr int hb = h.value;
                if (X::DP == 256 && hb == 3 && A.c.dim <= 192) return;              // (nothing but zeros)
                unrolled<TN>([&](auto u) {
                    constexpr int t = u.value, OFF = t * 16 * X::ROW + (hb >> 1) * 128;
                    const uint4 a = lds128<OFF>(key ^ (hb & 1) * 64), b = lds128<OFF + 8 * X::ROW>(key ^ (hb & 1) * 64);
                    const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        uint32_t f[4];
                        e4m3_to_f16(aw[y], &f[0], &f[2]);
                        e4m3_to_f16(bw[y], &f[1], &f[3]);
                        kq(t, hb * 4 + y, f[0], f[1], f[2], f[3]);
                    }
                });
            });
        } else {
            unrolled<KS>([&](auto k) {
                constexpr int ks = k.value;
                if (X::DP == 256 && ks / 4 == 3 && A.c.dim <= 192) return;          // (nothing but zeros)
                unrolled<TN>([&](auto u) {
                    uint32_t a[4];              // tokens 0-7 and 8-15 of elements 0-7, then of 8-15
                    ldmatrix4<u.value * 16 * X::ROW + ks / 4 * 128>(a, key ^ ks % 4 * 32);
                    kq(u.value, ks, a[0], a[1], a[2], a[3]);
                });
            });
        }
        // p = 2^(s - m): tokens r8 and r8 + 8 of heads 2j and 2j + 1
        const unsigned have = s_there[tile_out++ & 7];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][t][i] = (TN == 1 ? s[n][t][i] + s2[n][0][i] : s[n][t][i]) * coef[n][i & 1];
        if (have != (TT == 32 ? 0xffffffffu : 0xffffu)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < TN; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((have >> (t * 16 + (i >> 1) * 8 + r8)) & 1)) s[n][t][i] = -INFINITY;
        }
        bool grown = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) grown |= s[n][t][i] > m[n][i & 1];
        if (A.weight) {
            float* row = A.score + ((int64_t)cc.b * A.q.heads + cc.head(A)) * A.score_len + (int64_t)cc.tile * TT + r8;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < TN; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int hd = n * 8 + 2 * j + (i & 1);
                        if (hd < heads) row[hd * A.score_len + t * 16 + (i >> 1) * 8] = s[n][t][i];
                    }
        }
        if (__any_sync(FULL_MASK, grown)) {                   // rare after the first tiles of a row
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = m[n][e];
#pragma unroll
                    for (int t = 0; t < TN; ++t) top = fmaxf(top, fmaxf(s[n][t][e], s[n][t][e + 2]));
                    top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, 16));
                    const float f = m[n][e] == -INFINITY ? 0.0f : exp2_fast(m[n][e] - top);
                    m[n][e] = top;
                    l[n][e] *= f;
#pragma unroll
                    for (int x = 0; x < KS; ++x) { o[n][x][e] *= f; o[n][x][e + 2] *= f; }
                }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float base[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) base[e] = m[n][e] == -INFINITY ? 0.0f : m[n][e] - (X::HALF ? 15.0f : 0.0f);
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float p0 = exp2_fast(s[n][t][2 * i] - base[0]), p1 = exp2_fast(s[n][t][2 * i + 1] - base[1]);
                    l[n][0] += p0;
                    l[n][1] += p1;
                    uint32_t hi, lo;
                    split2<X::HALF>(p0, p1, &hi, &lo);
                    ph[n][t][i] = transpose8x8(hi);
                    pl[n][t][i] = transpose8x8(lo);
                }
        }
        }
        // o += v . p, elements x heads
        uint32_t sv = 0;
        if (live) sv = step();
        load_values();
        if (!live) { --ahead; continue; }
        auto vp = [&](int x, int t, const uint32_t (&a)[2][4]) {         // output tiles x, x + 1: the two products of one sum apart from one another
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint32_t (&p)[2] = half ? pl[n][t] : ph[n][t];
                        mma16816<X::HALF>(o[n][x + y], a[y][0], a[y][1], a[y][2], a[y][3], p[0], p[1]);
                    }
        };
        const uint32_t value = sv + in_values;
        if constexpr (X::E8) {
            unrolled<TN>([&](auto u) {
                constexpr int t = u.value, W = X::DP / 32;    // words of a lane's elements
                uint32_t v[4][W];                             // tokens 2j, 2j+1, 2j+8, 2j+9
                unrolled<4>([&](auto k) {
                    constexpr int i = k.value, OFF = (t * 16 + (i >> 1) * 8 + (X::CH == 4 ? 0 : i & 1)) * X::ROW;
                    if constexpr (X::CH == 4) {
                        const uint2 a = lds64<OFF>(value ^ (i & 1) * 64);
                        v[i][0] = a.x; v[i][1] = a.y;
                    } else {
                        unrolled<W / 4>([&](auto c) {
                            const uint4 a = lds128<OFF>(value ^ c.value * 16);
                            v[i][c.value * 4] = a.x; v[i][c.value * 4 + 1] = a.y; v[i][c.value * 4 + 2] = a.z; v[i][c.value * 4 + 3] = a.w;
                        });
                    }
                });
#pragma unroll
                for (int x = 0; x < KS; x += 2) {
                    // bytes 2x, 2x+1 of two tokens each: (token 0, token 1) of element 2x, then of 2x+1
                    uint32_t a[2][4];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint32_t sel = y ? 0x7362 : 0x5140;
                        const uint32_t c = __byte_perm(v[0][x / 2], v[1][x / 2], sel), d = __byte_perm(v[2][x / 2], v[3][x / 2], sel);
                        e4m3_to_f16(c, &a[y][0], &a[y][1]);
                        e4m3_to_f16(d, &a[y][2], &a[y][3]);
                    }
                    vp(x, t, a);
                }
            });
        } else {
            unrolled<KS / 2>([&](auto k) {
                constexpr int x = k.value * 2;
                if (X::DP == 256 && x / 4 == 3 && A.c.dim <= 192) return;
                unrolled<TN>([&](auto u) {
                    uint32_t a[2][4];           // elements 0-7 and 8-15 of tokens 0-7, then of 8-15
                    ldmatrix4_trans<u.value * 16 * X::ROW + x / 4 * 128>(a[0], value ^ x % 4 * 32);
                    ldmatrix4_trans<u.value * 16 * X::ROW + x / 4 * 128>(a[1], value ^ (x % 4 + 1) * 32);
                    vp(x, u.value, a);
                });
            });
        }
        // the row ends, or the span
        const bool row_ends = cc.tile + 1 == cc.end;
        if (row_ends || left == 1) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[n][e] += __shfl_xor_sync(FULL_MASK, l[n][e], 4);
                    l[n][e] += __shfl_xor_sync(FULL_MASK, l[n][e], 8);
                    l[n][e] += __shfl_xor_sync(FULL_MASK, l[n][e], 16);
                    m[n][e] -= X::HALF ? 15.0f : 0.0f;
                }
            finish(cc, begun_here, row_ends, heads, m, l, o);
            fresh = true;
        }
        if (--left == 0) break;
        cc.next(A);
    }
}

// Elements behind dim are 0 in shared memory throughout.
template <class X> __device__ __forceinline__ void clear_ring(const DecodeArgs& A, unsigned char* smem, int bytes) {
    if (A.c.dim * (X::E8 ? 1 : 2) / 16 < X::CH)
        for (int i = threadIdx.x; i < bytes / 16; i += blockDim.x) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
}
// What a warp has of a row, as its registers hold it: m and sums of the heads, then per (8 heads, 16 elements) a float4 per lane -- elements r8,
// r8 + 8 of the tile for heads 2j, 2j + 1.
template <class X> __device__ __forceinline__ void write_part(float* part, const float (&m)[X::NT][2], const float (&l)[X::NT][2], const float (&o)[X::NT][X::KS][4]) {
    const int lane = threadIdx.x & 31, j = lane & 3;
#pragma unroll
    for (int n = 0; n < X::NT; ++n) {
        if (lane < 4) {
            *reinterpret_cast<float2*>(part + n * 8 + 2 * j) = make_float2(m[n][0], m[n][1]);
            *reinterpret_cast<float2*>(part + X::HEADS + n * 8 + 2 * j) = make_float2(l[n][0], l[n][1]);
        }
#pragma unroll
        for (int x = 0; x < X::KS; ++x)
            reinterpret_cast<float4*>(part + 2 * X::HEADS)[(n * X::KS + x) * 32 + lane] = make_float4(o[n][x][0], o[n][x][1], o[n][x][2], o[n][x][3]);
    }
}
// The parts of a row joined for output tile x, by a warp: lane 4 r8 + j has elements r8, r8 + 8 of heads 2j, 2j + 1 of each group of eight.
template <class X> struct Joined {
    float m[X::NT][2], l[X::NT][2], o[X::NT][4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < X::NT; ++n) {
            m[n][0] = m[n][1] = -INFINITY;
            l[n][0] = l[n][1] = o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
        }
    }
    // parts k0, k0 + step, ... below parts; DEEP of them in flight together.  part(k): where part k is.
    template <int DEEP, class G> __device__ __forceinline__ void add(int x, int32_t k0, int32_t step, int32_t parts, G part) {
        const int lane = threadIdx.x & 31, j = lane & 3;
        for (; k0 < parts; k0 += step * DEEP) {
            float2 pm[DEEP][X::NT], pl[DEEP][X::NT];
            float4 po[DEEP][X::NT];
#pragma unroll
            for (int y = 0; y < DEEP; ++y) {
                const bool some = k0 + y * step < parts;
                const float* p = part(some ? k0 + y * step : k0);
#pragma unroll
                for (int n = 0; n < X::NT; ++n) {
                    pm[y][n] = *reinterpret_cast<const float2*>(p + n * 8 + 2 * j);
                    pl[y][n] = *reinterpret_cast<const float2*>(p + X::HEADS + n * 8 + 2 * j);
                    po[y][n] = reinterpret_cast<const float4*>(p + 2 * X::HEADS)[(n * X::KS + x) * 32 + lane];
                    if (!some) { pm[y][n] = make_float2(-INFINITY, -INFINITY); pl[y][n] = make_float2(0, 0); po[y][n] = make_float4(0, 0, 0, 0); }
                }
            }
#pragma unroll
            for (int n = 0; n < X::NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = m[n][e];
#pragma unroll
                    for (int y = 0; y < DEEP; ++y) top = fmaxf(top, e ? pm[y][n].y : pm[y][n].x);
                    const float base = top == -INFINITY ? 0.0f : top, f = exp2_fast(m[n][e] - base);
                    m[n][e] = top;
                    l[n][e] *= f; o[n][e] *= f; o[n][e + 2] *= f;
#pragma unroll
                    for (int y = 0; y < DEEP; ++y) {
                        const float pf = exp2_fast((e ? pm[y][n].y : pm[y][n].x) - base);
                        l[n][e] += pf * (e ? pl[y][n].y : pl[y][n].x);
                        o[n][e] += pf * (e ? po[y][n].y : po[y][n].x);
                        o[n][e + 2] += pf * (e ? po[y][n].w : po[y][n].z);
                    }
                }
        }
    }
    // to shared memory and, of what `others` warps have left there, back again
    __device__ __forceinline__ void put(float4* at) const {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int n = 0; n < X::NT; ++n) {
            at[(n * 2) * 32 + lane] = make_float4(m[n][0], m[n][1], l[n][0], l[n][1]);
            at[(n * 2 + 1) * 32 + lane] = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
        }
    }
    __device__ __forceinline__ void take(const float4* all, int others) {
        const int lane = threadIdx.x & 31;
        clear();
        for (int w = 0; w < others; ++w)
#pragma unroll
            for (int n = 0; n < X::NT; ++n) {
                const float4 a = all[(w * X::NT * 2 + n * 2) * 32 + lane], b = all[(w * X::NT * 2 + n * 2 + 1) * 32 + lane];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float pm = e ? a.y : a.x, top = fmaxf(m[n][e], pm), base = top == -INFINITY ? 0.0f : top;
                    const float f = exp2_fast(m[n][e] - base), pf = exp2_fast(pm - base);
                    m[n][e] = top;
                    l[n][e] = l[n][e] * f + pf * (e ? a.w : a.z);
                    o[n][e] = o[n][e] * f + pf * (e ? b.y : b.x);
                    o[n][e + 2] = o[n][e + 2] * f + pf * (e ? b.w : b.z);
                }
            }
    }
};
// Elements of output tile x that came out as NaN although the scores are numbers.  A value that is NaN makes them so, and they stay; but an infinite
// value times the second half of a probability, which may be 0 or negative, is no number either, while the sum of p_t v_t is infinite, and so is any value of a
// token whose score is -inf times its 0.  bad: the heads (h0 + bit) with such elements; norm: lane h's base-2 logarithm of the softmax's sum of head h.
//   - What is not finite among the values of tokens that take part says what an element is: NaN, the infinity if there is one sign of it, NaN with both.
//     The values alone are read, a token per lane; scores only of a group of tokens with something new, to leave out those of -inf.  It ends as soon as every
//     element is known to be NaN.
//   - Elements with nothing of that kind are summed again with whole probabilities.
// WARPS: of the CTA, which take turns with groups of tokens (all of them call this, behind a barrier); 1: a warp by itself.  8-bit values are finite or NaN, which is
// what comes out anyway.  A NaN at the end of a row: 2 sequences of 131,072 tokens (bf16, 2 cache heads of 128) 396 us instead of 70, one of 20,000 tokens 86 instead
// of 28, 200 of 2,000 172 instead of 87; a NaN value of a token whose score is -inf, which has the row summed again for every head: 20 ms, 2.9 and 2.5.
template <int WARPS> struct RepairShared {
    float sum[WARPS][16];
    unsigned flag[16][2];
};
template <class X, int WARPS>
__device__ __noinline__ void decode_repair(const DecodeArgs& A, int32_t b, int32_t h0, unsigned bad, float norm, int x, RepairShared<WARPS>* S) {
    using Q = typename Elem<X::TQ>::T;
    using C = typename Elem<X::TC>::T;
    static_assert(!X::E8 && sizeof(C) == 2 && X::HEADS <= 16);
    constexpr unsigned EXPONENT = X::HALF ? 0x7c00u : 0x7f80u, CARRY = 0x8000u - EXPONENT;
    constexpr int DEEP = 4;                                  // groups of 32 tokens in flight
    const int lane = threadIdx.x & 31, warp = WARPS > 1 ? threadIdx.x >> 5 : 0;
    const int32_t g = h0 / A.group, d0 = x * 16;
    const bool second = d0 + 8 < A.c.dim;                    // (dim is a multiple of 8)
    __syncwarp();
    unsigned want = 0;                                       // lane h: which of the tile's elements of head h are NaN
    for (unsigned rest = bad; rest; rest &= rest - 1) {
        const int hd = __ffs(rest) - 1;
        const Q* out = reinterpret_cast<const Q*>(A.out.p + b * A.out.sr + (int64_t)(h0 + hd) * A.out.sh);
        const float y = lane < 16 && d0 + lane < A.c.dim ? to_float(out[d0 + lane]) : 0.0f;
        const unsigned m = __ballot_sync(FULL_MASK, y != y);
        if (lane == hd) want = m;
    }
    int32_t lo, hi;
    token_range(A, b, &lo, &hi);
    auto page_of = [&](int32_t t) -> int32_t {
        const int32_t p = t < hi ? __ldg(A.table + b * A.table_stride + (t >> A.c.page_shift)) : -1;
        return p < A.c.n_pages ? p : -1;
    };
    auto load = [&](int32_t t, int32_t page, uint4 (&v)[2]) {
        v[0] = v[1] = make_uint4(0, 0, 0, 0);
        if (page < 0) return;
        const char* p = A.c.v + page * A.c.vs[0] + (t & ((1 << A.c.page_shift) - 1)) * A.c.vs[1] + g * A.c.vs[2] + d0 * 2;
        v[0] = *reinterpret_cast<const uint4*>(p);
        if (second) v[1] = *reinterpret_cast<const uint4*>(p + 16);
    };
    auto score = [&](int hd, int32_t t, int32_t page) -> float {           // of this lane's token, base 2
        const Q* q = reinterpret_cast<const Q*>(A.q.p + b * A.q.sr + (int64_t)(h0 + hd) * A.q.sh);
        const char* k = A.c.k + page * A.c.ks[0] + (t & ((1 << A.c.page_shift) - 1)) * A.c.ks[1] + g * A.c.ks[2];
        float s = 0.0f;
#pragma unroll 4
        for (int32_t d = 0; d < A.c.dim; d += 8) {
            alignas(16) C e[8];
            *reinterpret_cast<uint4*>(e) = *reinterpret_cast<const uint4*>(k + d * 2);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += to_float(q[d + i]) * to_float(e[i]);
        }
        return s * (A.scale * A.c.k_scale * 1.4426950408889634f);
    };
    // lane h: what is not finite among the values that head h attends to -- bits 0-15 of inf: +infinity, 16-31: -infinity, of nan: NaN
    unsigned inf = 0, nan = 0;
    auto open = [&]() { return want & ~(nan | (inf & inf >> 16)); };
    for (int32_t t0 = lo + warp * 32 * DEEP; t0 < hi; t0 += WARPS * 32 * DEEP) {
        int32_t page[DEEP];
        uint4 v[DEEP][2];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) page[i] = page_of(t0 + i * 32 + lane);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) load(t0 + i * 32 + lane, page[i], v[i]);
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const unsigned w[8] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w, v[i][1].x, v[i][1].y, v[i][1].z, v[i][1].w};
            unsigned any = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) any |= (w[j] & EXPONENT * 0x10001u) + CARRY * 0x10001u;
            if (!__any_sync(FULL_MASK, any & 0x80008000u)) continue;
            unsigned mine_inf = 0, mine_nan = 0;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const unsigned u = w[j >> 1] >> (j & 1) * 16 & 0xffffu;
                if ((u & EXPONENT) != EXPONENT) continue;
                if (u & (CARRY - 1)) mine_nan |= 1u << j;
                else mine_inf |= (u & 0x8000u ? 0x10000u : 1u) << j;
            }
            const unsigned all_inf = __reduce_or_sync(FULL_MASK, mine_inf), all_nan = __reduce_or_sync(FULL_MASK, mine_nan);
            const unsigned more = all_inf & ~inf;
            for (unsigned need = __ballot_sync(FULL_MASK, (more | more >> 16 | all_nan) & open()); need; need &= need - 1) {
                const int hd = __ffs(need) - 1;
                const bool there = (mine_inf | mine_nan) && score(hd, t0 + i * 32 + lane, page[i]) != -INFINITY;
                const unsigned a = __reduce_or_sync(FULL_MASK, there ? mine_inf : 0u), n = __reduce_or_sync(FULL_MASK, there ? mine_nan : 0u);
                if (lane == hd) { inf |= a; nan |= n; }
            }
        }
        if (!__any_sync(FULL_MASK, open())) break;
    }
    if constexpr (WARPS > 1) {
        if (threadIdx.x < 16) S->flag[threadIdx.x][0] = S->flag[threadIdx.x][1] = 0;
        __syncthreads();
        if (lane < 16 && inf) atomicOr(&S->flag[lane][0], inf);
        if (lane < 16 && nan) atomicOr(&S->flag[lane][1], nan);
        __syncthreads();
        if (lane < 16) { inf = S->flag[lane][0]; nan = S->flag[lane][1]; }
    }
    for (unsigned rest = bad; rest; rest &= rest - 1) {
        const int hd = __ffs(rest) - 1;
        const unsigned w = __shfl_sync(FULL_MASK, want, hd), f = __shfl_sync(FULL_MASK, inf, hd), n = __shfl_sync(FULL_MASK, nan, hd);
        const float lse2 = __shfl_sync(FULL_MASK, norm, hd);
        float y = 0.0f;
        if (w & ~(n | f | f >> 16)) {
            float o[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = 0.0f;
            for (int32_t t0 = lo + warp * 32; t0 < hi; t0 += WARPS * 32) {
                const int32_t t = t0 + lane, page = page_of(t);
                if (page < 0) continue;
                const float s = score(hd, t, page);
                if (s == -INFINITY) continue;
                const float p = exp2f(s - lse2);
                uint4 v[2];
                load(t, page, v);
                const unsigned u[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint16_t bits = (uint16_t)(u[j >> 1] >> (j & 1) * 16);
                    o[j] += p * to_float(*reinterpret_cast<const C*>(&bits));
                }
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                for (int d = 16; d; d >>= 1) o[j] += __shfl_xor_sync(FULL_MASK, o[j], d);
                if (lane == j) y = o[j];
            }
            if constexpr (WARPS > 1) {
                if (lane < 16) S->sum[warp][lane] = y;
                __syncthreads();
                y = 0.0f;
                for (int k = 0; k < WARPS && lane < 16; ++k) y += S->sum[k][lane];
                __syncthreads();
            }
        }
        const unsigned bit = 1u << (lane & 15);
        if ((f & bit) || (f >> 16 & bit)) y = f & bit ? INFINITY : -INFINITY;
        if (warp == 0 && lane < 16 && (w & bit) && !(n & bit) && !(f & f >> 16 & bit))
            reinterpret_cast<Q*>(A.out.p + b * A.out.sr + (int64_t)(h0 + hd) * A.out.sh)[d0 + lane] = from_float<Q>(y);
    }
    if constexpr (WARPS > 1) __syncthreads();
}
// The outputs of tile x of a unit whose parts are joined; what a warp writes here nobody else writes.  Returns the heads that decode_repair has to look at, and
// their logarithms of the softmax's sum in *norm.
template <class X> __device__ __forceinline__ unsigned write_joined(const DecodeArgs& A, const Joined<X>& J, int32_t b, int32_t h0, int32_t heads, int x, float* norm) {
    using Q = typename Elem<X::TQ>::T;
    const int lane = threadIdx.x & 31, r8 = lane >> 2, j = lane & 3;
    unsigned bad = 0;                                        // heads with a NaN among this lane's elements
#pragma unroll
    for (int n = 0; n < X::NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int hd = n * 8 + 2 * j + e;
            if (hd >= heads) continue;
            const float sum = J.l[n][e], f = sum == 0.0f ? 0.0f : A.c.v_scale / sum;
            Q* out = reinterpret_cast<Q*>(A.out.p + b * A.out.sr + (int64_t)(h0 + hd) * A.out.sh);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int d = out_element<X>(x, r8, i);
                const float y = sum == 0.0f ? 0.0f : J.o[n][i * 2 + e] * f;
                if (d < A.c.dim) out[d] = from_float<Q>(y);
                if (!X::E8 && d < A.c.dim && y != y && sum == sum) bad |= 1u << hd;
            }
            if (x == 0 && r8 == 0) {
                const int64_t row = (int64_t)b * A.q.heads + h0 + hd;
                const float y = sum == 0.0f ? -INFINITY : J.m[n][e] + log2f(sum);
                if (A.lse) A.lse[row] = y * 0.6931471805599453f;
                A.lse2[row] = y;
            }
        }
    if (X::E8) return 0;
    bad = __reduce_or_sync(FULL_MASK, bad);
    if (bad) {
#pragma unroll
        for (int n = 0; n < X::NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float y = __shfl_sync(FULL_MASK, J.m[n][e] + log2f(J.l[n][e]), (lane & 7) >> 1);
                if (lane >> 3 == n && (lane & 1) == e) *norm = y;
            }
    }
    return bad;
}

template <class X>
__global__ void __launch_bounds__(KLPM_DECODE_WARPS * 32, X::CTAS) decode_kernel(const __grid_constant__ DecodeArgs A) {
    using Q = typename Elem<X::TQ>::T;
    constexpr int TT = X::TT, KS = X::DP / 16, NT = X::NT;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long s_sum[KLPM_DECODE_WARPS];
    __shared__ int32_t s_b[KLPM_DECODE_WARPS];
    __shared__ long long s_rem[KLPM_DECODE_WARPS];
    __shared__ unsigned s_there[KLPM_DECODE_WARPS][8];         // which tokens of the tiles on their way are there
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    clear_ring<X>(A, smem, X::SMEM);
    // where each warp starts: every CTA adds up the tiles of all sequences
    const int32_t per = (A.n_seqs + KLPM_DECODE_WARPS * 32 - 1) / (KLPM_DECODE_WARPS * 32);
    const int32_t b0 = min(tid * per, A.n_seqs), b1 = min(b0 + per, A.n_seqs);
    long long mine = 0;
    int32_t first;
    for (int32_t b = b0; b < b1; ++b) mine += tiles_of<TT>(A, b, &first);
    long long before = mine;
    for (int d = 1; d < 32; d <<= 1) {
        const long long v = __shfl_up_sync(FULL_MASK, before, d);
        if (lane >= d) before += v;
    }
    if (lane == 31) s_sum[warp] = before;
    before -= mine;
    __syncthreads();
    long long total = 0;
    for (int w = 0; w < KLPM_DECODE_WARPS; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
    }
    if (blockIdx.x == 0) {
        long long at = before;
        for (int32_t b = b0; b < b1; ++b) { A.tiles_before[b] = at; at += tiles_of<TT>(A, b, &first); }
        if (tid == 0) A.tiles_before[A.n_seqs] = total;
    }
    total *= A.units;
    const long long span = span_of(total, A.warps);
    for (int w = 0; w < KLPM_DECODE_WARPS; ++w) {
        const long long pos = ((long long)w * gridDim.x + blockIdx.x) * span;
        if (pos < total && pos >= before * A.units && pos < (before + mine) * A.units) {
            long long rem = pos - before * A.units;
            int32_t b = b0;
            for (;; ++b) {
                const long long n = (long long)tiles_of<TT>(A, b, &first) * A.units;
                if (rem < n) break;
                rem -= n;
            }
            s_b[w] = b; s_rem[w] = rem;
        }
    }
    __syncthreads();
    const int32_t w = warp * gridDim.x + blockIdx.x;          // neighbouring spans on different SMs
    const long long pos = (long long)w * span;
    if (pos >= total) return;

    Cursor<X> ci;                                             // the tile that is loaded next
    ci.b = s_b[warp];
    ci.row(A);
    {
        const long long rem = s_rem[warp];
        const int32_t u = (int32_t)(rem / (ci.end - ci.first));
        ci.g = u / A.head_tiles; ci.ht = u - ci.g * A.head_tiles;
        ci.tile = ci.first + (int32_t)(rem % (ci.end - ci.first));
    }
    bool first_piece = true;
    decode_span<X>(A, smem_addr(smem) + warp * X::WARP_SMEM, s_there[warp], ci, min(span, total - pos),
                   [&](const Cursor<X>& cc, bool begun, bool ended, int32_t heads, const float (&m)[NT][2], const float (&l)[NT][2], const float (&o)[NT][KS][4]) {
        if (!begun || !ended) {
            write_part<X>(A.part + ((int64_t)w * 2 + (first_piece ? 0 : 1)) * X::PART, m, l, o);
        } else {
            const int r8 = lane >> 2, j = lane & 3;
            const int32_t h0 = cc.head(A);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int hd = n * 8 + 2 * j + e;
                    if (hd >= heads) continue;
                    const float sum = l[n][e];
                    Q* out = reinterpret_cast<Q*>(A.out.p + cc.b * A.out.sr + (int64_t)(h0 + hd) * A.out.sh);
                    const float f = sum == 0.0f ? 0.0f : A.c.v_scale / sum;
#pragma unroll
                    for (int x = 0; x < KS; ++x)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int d = out_element<X>(x, r8, i);
                            if (d < A.c.dim) out[d] = from_float<Q>(sum == 0.0f ? 0.0f : o[n][x][i * 2 + e] * f);
                        }
                    if (r8 == 0) {
                        const int64_t row = (int64_t)cc.b * A.q.heads + h0 + hd;
                        const float y = sum == 0.0f ? -INFINITY : m[n][e] + log2f(sum);
                        if (A.lse) A.lse[row] = y * 0.6931471805599453f;
                        A.lse2[row] = y;
                    }
                }
        }
        first_piece = false;
    });
}

// Rows that were cut into parts, and rows with nothing to attend to.  An item is 16 elements of a unit, for WPR warps: a CTA where few rows
// have many parts each, a warp where many rows have few.  Four CTAs on an SM where the sums of 8 heads leave room (64 sequences, 2 cache heads: 18.4 us with four, 20.0
// with three); with 16 heads registers count for more (100 sequences: 40.0 us with two CTAs, 41.0 with three).
template <class X, int WPR>
__global__ void __launch_bounds__(WPR == 1 ? 256 : WPR * 32, WPR <= 8 && X::NT == 1 ? 4 : 1) decode_join_kernel(const __grid_constant__ DecodeArgs A) {
    using Q = typename Elem<X::TQ>::T;
    __shared__ float4 s_all[WPR > 1 ? WPR * X::NT * 2 * 32 : 1];
    __shared__ RepairShared<WPR> s_repair;
    __shared__ float s_norm[32];
    __shared__ unsigned s_bad;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t item = WPR > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 8 + warp, row = item / X::KS;
    const int x = (int)(item % X::KS);
    if (row >= (int64_t)A.n_seqs * A.units) return;
    const int32_t b = (int32_t)(row / A.units), u = (int32_t)(row % A.units), g = u / A.head_tiles, in = (u - g * A.head_tiles) * X::HEADS;
    const int32_t h0 = g * A.group + in, heads = min(X::HEADS, A.group - in);
    const long long t0 = A.tiles_before[b], tiles = A.tiles_before[b + 1] - t0;
    const long long span = span_of(A.tiles_before[A.n_seqs] * A.units, A.warps);
    const long long R = t0 * A.units + u * tiles, E = R + tiles;
    const int32_t w0 = (int32_t)(R / span), parts = tiles > 0 ? (int32_t)((E - 1) / span) - w0 + 1 : 0;
    if (parts == 1) {                                        // decode_kernel has written it; is there anything to repair?
        if constexpr (!X::E8) {
            if (WPR > 1 && warp) return;
            const int d = out_element<X>(x, lane & 7, (lane >> 3) & 1);
            unsigned bad = 0;
            const float norm = lane < heads ? A.lse2[(int64_t)b * A.q.heads + h0 + lane] : 0.0f;
            for (int32_t hd = 0; hd < heads; ++hd) {
                const Q* out = reinterpret_cast<const Q*>(A.out.p + b * A.out.sr + (int64_t)(h0 + hd) * A.out.sh);
                const float y = d < A.c.dim ? to_float(out[d]) : 0.0f;
                if (__any_sync(FULL_MASK, y != y)) bad |= 1u << hd;
            }
            bad &= __ballot_sync(FULL_MASK, norm == norm);
            if (bad) decode_repair<X, 1>(A, b, h0, bad, norm, x, nullptr);
        }
        return;
    }
    const int first = w0 * span == R ? 0 : 1;
    Joined<X> J;
    J.clear();
    J.template add<4>(x, WPR > 1 ? warp : 0, WPR, parts, [&](int k) { return A.part + ((int64_t)(w0 + k) * 2 + (k == 0 ? first : 0)) * X::PART; });
    if constexpr (WPR > 1) {
        J.put(s_all + warp * X::NT * 2 * 32);
        __syncthreads();
        if (warp == 0) J.take(s_all, WPR);
    }
    float norm = 0.0f;
    unsigned bad = 0;
    if (WPR == 1 || warp == 0) bad = write_joined<X>(A, J, b, h0, heads, x, &norm);
    if constexpr (!X::E8) {
        if constexpr (WPR > 1) {
            if (warp == 0) s_norm[lane] = norm;
            if (__syncthreads_or(bad)) {
                if (threadIdx.x == 0) s_bad = bad;
                __syncthreads();
                decode_repair<X, WPR>(A, b, h0, s_bad, s_norm[lane], x, &s_repair);
            }
        } else if (bad) decode_repair<X, 1>(A, b, h0, bad, norm, x, nullptr);
    }
}

// Small calls: a cluster of CTAs per row (sequence, unit), its tiles dealt out to all of the cluster's warps, whose results are joined through
// distributed shared memory: one kernel, no trip through the workspace.  Weights are added from the scores by the warps that made them.
#define KLPM_ROW_WARPS 8
#define KLPM_ROW_CTAS 16
template <class X>
__global__ void __launch_bounds__(KLPM_ROW_WARPS * 32, X::CTAS / 2) decode_row_kernel(const __grid_constant__ DecodeArgs A, int32_t lg) {       // 2^lg CTAs of a cluster
    using Q = typename Elem<X::TQ>::T;
    constexpr int TT = X::TT, KS = X::KS, NT = X::NT;
    static_assert(KLPM_ROW_WARPS == 8);
    static_assert(X::PART * 4 <= X::WARP_SMEM, "a warp's result lies in its ring");
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ unsigned s_there[KLPM_ROW_WARPS][8];
    __shared__ float4 s_all[KLPM_ROW_WARPS * NT * 2 * 32];
    __shared__ float s_lse2[X::HEADS];
    __shared__ RepairShared<KLPM_ROW_WARPS> s_repair;
    __shared__ float s_norm[KLPM_ROW_WARPS][32];
    __shared__ unsigned s_bad[KLPM_ROW_WARPS];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t ctas = 1 << lg, rank = blockIdx.x & (ctas - 1), row = blockIdx.x >> lg;
    Cursor<X> c;
    c.b = row / A.units;
    c.g = (row - c.b * A.units) / A.head_tiles; c.ht = row - c.b * A.units - c.g * A.head_tiles;
    token_range(A, c.b, &c.lo, &c.hi);
    c.first = c.lo / TT;
    c.end = c.hi > c.lo ? (c.hi + TT - 1) / TT : c.first;
    const int32_t tiles = c.end - c.first, warps = KLPM_ROW_WARPS << lg, per = (tiles + warps - 1) >> (lg + 3);
    const int32_t parts = per <= 1 ? tiles : (tiles + per - 1) / per;
    const int32_t g = c.g, h0 = c.head(A), heads = min(X::HEADS, A.group - c.ht * X::HEADS);
    clear_ring<X>(A, smem, KLPM_ROW_WARPS * X::WARP_SMEM);
    __syncthreads();
    const int32_t mine = warp * ctas + rank;                  // neighbouring parts on different SMs
    const int32_t from = c.first + mine * per, count = min(per, c.end - from);
    if (mine < parts) {
        c.tile = from;
        decode_span<X>(A, smem_addr(smem) + warp * X::WARP_SMEM, s_there[warp], c, count,
                       [&](const Cursor<X>&, bool, bool, int32_t, const float (&m)[NT][2], const float (&l)[NT][2], const float (&o)[NT][KS][4]) {
            cp_async_wait<0>();
            __syncwarp();
            write_part<X>(reinterpret_cast<float*>(smem + warp * X::WARP_SMEM), m, l, o);
        });
    }
    cluster.sync();
    // output tiles: as many of a CTA's warps to each as there are, a part of the parts to every warp
    auto part = [&](int k) { return reinterpret_cast<const float*>(cluster.map_shared_rank(smem, k & (ctas - 1)) + (k >> lg) * X::WARP_SMEM); };
    constexpr int LG_KS = X::KS == 4 ? 2 : X::KS == 8 ? 3 : 4;
    const int lg_share = parts <= 4 ? 0 : max(0, min(3, lg + 3 - LG_KS)), share = 1 << lg_share, mine_of = warp & (share - 1);
    const int per_cta = KLPM_ROW_WARPS >> lg_share;
    for (int x0 = rank * per_cta; x0 < X::KS; x0 += ctas * per_cta) {
        const int x = x0 + (warp >> lg_share);
        Joined<X> J;
        J.clear();
        if (x < X::KS) J.template add<4>(x, mine_of, share, parts, part);
        if (share > 1) {
            J.put(s_all + warp * NT * 2 * 32);
            __syncthreads();
            if (mine_of == 0) J.take(s_all + warp * NT * 2 * 32, share);
        }
        float norm = 0.0f;
        unsigned bad = 0;
        if (x < X::KS && mine_of == 0) bad = write_joined<X>(A, J, c.b, h0, heads, x, &norm);
        if constexpr (X::E8) {
            if (share > 1) __syncthreads();
        } else {
            if (share == 1) {
                if (bad) decode_repair<X, 1>(A, c.b, h0, bad, norm, x, nullptr);
            } else if (__syncthreads_or(bad)) {               // all of the CTA's warps, for one of its output tiles after the other
                s_norm[warp][lane] = norm;
                if (lane == 0) s_bad[warp] = bad;
                __syncthreads();
                for (int w = 0; w < KLPM_ROW_WARPS; w += share)
                    if (s_bad[w]) decode_repair<X, KLPM_ROW_WARPS>(A, c.b, h0, s_bad[w], s_norm[w][lane], x0 + (w >> lg_share), &s_repair);
            }
        }
    }
    if (A.weight) {                                           // (one unit per cache head)
        for (int hd = warp; hd < heads; hd += KLPM_ROW_WARPS) {
            float m = -INFINITY, l = 0.0f;
            for (int k = lane; k < parts; k += 32) m = fmaxf(m, part(k)[hd]);
            for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL_MASK, m, d));
            const float base = m == -INFINITY ? 0.0f : m;
            for (int k = lane; k < parts; k += 32) l += exp2_fast(part(k)[hd] - base) * part(k)[X::HEADS + hd];
            for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(FULL_MASK, l, d);
            if (lane == 0) s_lse2[hd] = l == 0.0f ? -INFINITY : m + log2f(l);
        }
        __syncthreads();
    }
    if (A.weight && mine < parts) {
        const int32_t t0 = max(c.lo, from * TT), t1 = min(c.hi, (from + count) * TT);
        const float* score = A.score + ((int64_t)c.b * A.q.heads + h0) * A.score_len;
        float* weight = A.weight + c.b * A.ws[0] + g * A.ws[1];
        for (int32_t t = t0 + lane; t < t1; t += 32) {
            float sum = 0.0f;
#pragma unroll 4
            for (int hd = 0; hd < heads; ++hd) {
                const float z = score[hd * A.score_len + t];
                if (z != -INFINITY) sum += exp2_fast(z - s_lse2[hd]);
            }
            if (sum != 0.0f) weight[t] += sum;
        }
    }
    cluster.sync();                                           // nobody leaves while its results are read
}

// What every token received, from the scores that decode_kernel kept: a warp takes a span of tiles of the batch, in the order (sequence,
// cache head, tile).  One thread adds up a token's heads, so that the order of the sum is fixed.
template <int TT>
__global__ void __launch_bounds__(256) decode_weight_kernel(const __grid_constant__ DecodeArgs A) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int32_t w = blockIdx.x * 8 + (threadIdx.x >> 5), warps = gridDim.x * 8;
    const long long total = A.tiles_before[A.n_seqs] * A.c.n_heads, span = span_of(total, warps);
    long long pos = w * span;
    const long long stop = min(pos + span, total);
    if (pos >= stop) return;
    // the sequence: tiles_before[b] * heads <= pos < tiles_before[b + 1] * heads, 32 places looked at side by side
    int32_t b = 0;
    for (int32_t width = A.n_seqs; width > 1;) {
        const int32_t step = (width + 31) / 32;
        const int32_t at = b + lane * step;
        const unsigned le = __ballot_sync(FULL_MASK, lane * step < width && A.tiles_before[at] * A.c.n_heads <= pos);
        const int k = 31 - __clz(le);                        // (lane 0 is always among them)
        b += k * step;
        width = min(step, width - k * step);
    }
    while (pos < stop) {
        const long long t0 = A.tiles_before[b], tiles = A.tiles_before[b + 1] - t0, in = pos - t0 * A.c.n_heads;
        if (in >= tiles * A.c.n_heads) { ++b; continue; }
        const int32_t g = (int32_t)(in / tiles);
        const long long at = in - g * tiles, n = min(tiles - at, stop - pos);
        int32_t lo, hi;
        token_range(A, b, &lo, &hi);
        const int32_t first = lo / TT, from = (int32_t)max((long long)lo, (first + at) * TT), to = (int32_t)min((long long)hi, (first + at + n) * TT);
        const float* score = A.score + ((int64_t)b * A.q.heads + g * A.group) * A.score_len;
        const float* norm = A.lse2 + (int64_t)b * A.q.heads + g * A.group;
        float* weight = A.weight + b * A.ws[0] + g * A.ws[1];
        constexpr int DEEP = 4;                              // tokens per lane whose loads are in flight together
        for (int32_t t = from; t < to; t += 32 * DEEP) {
            float sum[DEEP], old[DEEP];
#pragma unroll
            for (int x = 0; x < DEEP; ++x) {
                sum[x] = 0.0f;
                old[x] = t + 32 * x + lane < to ? weight[t + 32 * x + lane] : 0.0f;
            }
#pragma unroll 2
            for (int32_t i = 0; i < A.group; ++i) {
                const float z = norm[i];
                float s[DEEP];
#pragma unroll
                for (int x = 0; x < DEEP; ++x) s[x] = t + 32 * x + lane < to ? score[i * A.score_len + t + 32 * x + lane] : -INFINITY;
#pragma unroll
                for (int x = 0; x < DEEP; ++x)
                    if (s[x] != -INFINITY) sum[x] += exp2_fast(s[x] - z);      // (z is -inf only where every s is)
            }
#pragma unroll
            for (int x = 0; x < DEEP; ++x)
                if (sum[x] != 0.0f) weight[t + 32 * x + lane] = old[x] + sum[x];
        }
        pos += n;
    }
}

inline int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// The workspace of a call: what decode_kernel leaves for the kernels after it.
struct DecodeSpace { int64_t lse2, part, score, score_len, bytes; };
DecodeSpace decode_space(int64_t n_seqs, int64_t heads, int64_t max_tokens, int64_t warps, int64_t part, bool weight) {
    DecodeSpace s;
    s.lse2 = up256((n_seqs + 1) * 8);
    s.part = s.lse2 + up256(n_seqs * heads * 4);
    s.score = s.part + up256(warps * 2 * part * 4);
    s.score_len = (max_tokens + 31) / 32 * 32;
    s.bytes = s.score + (weight ? up256(n_seqs * heads * s.score_len * 4) : 0);
    return s;
}

// More than 48 KB of dynamic shared memory has to be asked for, once per kernel and device.
template <auto kernel> rt_status allow_smem(int bytes) {
    static std::atomic<uint64_t> asked{0};
    int dev = 0;
    CK(cudaGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (asked.load(std::memory_order_relaxed) & bit) return RT_OK;
    CK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    CK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    asked.fetch_or(bit, std::memory_order_relaxed);
    return RT_OK;
}

template <typename... P> rt_status launch_cluster(void (*kernel)(P...), unsigned grid, unsigned threads, int ctas, size_t smem, cudaStream_t s, P... args) {
    cudaLaunchConfig_t c = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ctas; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    c.gridDim = dim3(grid); c.blockDim = dim3(threads); c.dynamicSmemBytes = smem; c.stream = s; c.attrs = at; c.numAttrs = 1;
    CK(cudaLaunchKernelEx(&c, kernel, args...));
    return RT_OK;
}

template <typename... P> rt_status launch_after(void (*kernel)(P...), dim3 grid, unsigned threads, cudaStream_t s, P... args) {
    // its CTAs may be set up while the kernel before it in the stream still runs; griddepcontrol.wait in it waits for that one's end
    cudaLaunchConfig_t c = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    c.gridDim = grid; c.blockDim = dim3(threads); c.stream = s; c.attrs = at; c.numAttrs = 1;
    CK(cudaLaunchKernelEx(&c, kernel, args...));
    return RT_OK;
}

template <class X> rt_status launch_decode(DecodeArgs& A, char* work, cudaStream_t s) {
    A.warps = KLPM_SMS * X::CTAS * KLPM_DECODE_WARPS;
    A.head_tiles = (A.group + X::HEADS - 1) / X::HEADS;
    A.units = A.c.n_heads * A.head_tiles;
    const DecodeSpace W = decode_space(A.n_seqs, A.q.heads, A.max_tokens, A.warps, X::PART, A.weight != nullptr);
    A.tiles_before = (long long*)work; A.lse2 = (float*)(work + W.lse2); A.part = (float*)(work + W.part); A.score = (float*)(work + W.score);
    A.score_len = W.score_len;
    // the most tiles of a row: a window that begins inside a tile takes one more
    const long long seen = A.window > 0 && A.window < A.max_tokens ? (long long)A.window + X::TT : A.max_tokens;
    const long long tiles = seen / X::TT + 1, units = (long long)A.n_seqs * A.units;
    // CTAs of a cluster: until every warp has a tile or the GPU is full (by half with clusters of 8, by a quarter with 16, which have to
    // find their SMs in one GPC: 16 clusters of 16 take 16.6 us where as many of 8 take 10.3)
    int lg = 0;
    while ((1 << lg) < KLPM_ROW_CTAS && (KLPM_ROW_WARPS << lg) < tiles
           && (units << (lg + 1)) <= KLPM_SMS * (X::CTAS / 2) / (lg < 2 ? 1 : 1 << (lg - 1))) ++lg;
    // The other kernels start 3 to 7 us later, but deal out the tiles evenly; here the longest row counts, and every cluster more than the GPU holds
    // at once.  Over 40 calls of all kinds (here, there): 24 rows of 208 tiles, 6.5 a warp 17.7, 22.5 us; 8 of 755, 11.8 a warp 19.9, 19.1; 128
    // of 129 22.9, 19.3; 200 of 39 17.2, 21.2; 312 of 27 32.4, 29.3; 872 of 8 26.3, 22.0; 608 of 4 where 148 fit 37.5, 21.1.
    const long long load = units * tiles / A.warps;
    if (units <= KLPM_SMS * (X::CTAS / 2) && load <= 4 && tiles <= (long long)(KLPM_ROW_WARPS << lg) * (6 + load) && (!A.weight || A.head_tiles == 1)) {
        constexpr int bytes = KLPM_ROW_WARPS * X::WARP_SMEM;
        if (rt_status st = allow_smem<decode_row_kernel<X>>(bytes)) return st;
        return launch_cluster(decode_row_kernel<X>, (unsigned)(units << lg), KLPM_ROW_WARPS * 32, 1 << lg, bytes, s, A, (int32_t)lg);
    }
    const int64_t items = units * X::KS;
    if (items > 0x7fffffffLL) return RT_ERR_TOO_LARGE;
    rt_status st = allow_smem<decode_kernel<X>>(X::SMEM);
    if (st) return st;
    decode_kernel<X><<<KLPM_SMS * X::CTAS, KLPM_DECODE_WARPS * 32, X::SMEM, s>>>(A);
    CK(cudaGetLastError());
    // a unit has A.warps / units parts or so
    constexpr int MANY = 32 / X::NT;
    if (units * 64 <= A.warps) st = launch_after(decode_join_kernel<X, MANY>, dim3((unsigned)items), MANY * 32, s, A);
    else if (units * 16 <= A.warps) st = launch_after(decode_join_kernel<X, 8>, dim3((unsigned)items), 256, s, A);
    else st = launch_after(decode_join_kernel<X, 1>, dim3((unsigned)((items + 7) / 8)), 256, s, A);
    if (st || !A.weight) return st;
    return launch_after(decode_weight_kernel<X::TT>, dim3(KLPM_SMS * 4), 256, s, A);
}

// The instance for a call: DP = dim rounded up to 64, 128 or 256, 8 or 16 query heads per unit (8 for wide heads: the registers).
template <int TQ, int TC, int DP, class F> auto for_heads(int32_t group, F f) {
    if constexpr (DP <= 128)
        if (group > 8) return f(Dec<TQ, TC, DP, 2>());
    return f(Dec<TQ, TC, DP, 1>());
}
template <int TQ, int TC, class F> auto for_dim(int32_t dim, int32_t group, F f) {
    if (dim <= 64) return for_heads<TQ, TC, 64>(group, f);
    if (dim <= 128) return for_heads<TQ, TC, 128>(group, f);
    return for_heads<TQ, TC, 256>(group, f);
}
template <class F> auto for_decode(int tq, int tc, int32_t dim, int32_t group, F f) {
    if (tq == KV_BF16) return tc == KV_E4M3 ? for_dim<KV_BF16, KV_E4M3>(dim, group, f) : for_dim<KV_BF16, KV_BF16>(dim, group, f);
    return tc == KV_E4M3 ? for_dim<KV_F16, KV_E4M3>(dim, group, f) : for_dim<KV_F16, KV_F16>(dim, group, f);
}

// ------------------------------------------------------------------------------------------------
// eviction
// ------------------------------------------------------------------------------------------------
struct EvictArgs {
    CacheDev c;
    const float* weight;
    int64_t ws[2];
    const int32_t *table, *len, *new_table;
    int64_t table_stride, new_stride;
    int32_t n_seqs, max_tokens, keep, sinks, recent, new_len, row_bytes;
    int32_t* index;
    float* new_weight;
    int64_t nws[2];
    int32_t* new_lengths;
};

// What a token is ranked by, larger first: 0 = not there, then NaN, the numbers in their order, and what is kept in any case.
__device__ __forceinline__ unsigned evict_key(const EvictArgs& A, int32_t b, int32_t g, int32_t n, int32_t t) {
    const float w = __ldg(A.weight + b * A.ws[0] + g * A.ws[1] + t);
    const int32_t page = __ldg(A.table + b * A.table_stride + (t >> A.c.page_shift));
    const unsigned u = __float_as_uint(w == 0.0f ? 0.0f : w);
    unsigned k = u & 0x80000000u ? ~u : u | 0x80000000u;
    if (w != w) k = 1u;
    if (t < A.sinks || t >= n - A.recent) k = 0xffffffffu;
    return (unsigned)page < (unsigned)A.c.n_pages ? k : 0u;
}

// Copies `rows` kept rows of cache head g, keys and values: lane r holds where row r is (sk, sv) and goes (dk, dv; byte offsets, sk < 0: nothing
// to copy).  16 bytes a lane, four loads in flight (eight leave fewer warps on an SM: 32
// sequences of up to 8,191 tokens take 152.5 us then, else 150).
__device__ __forceinline__ void copy_kept(const EvictArgs& A, int rows, int64_t sk, int64_t sv, int64_t dk, int64_t dv) {
    const int lane = threadIdx.x & 31;
    const unsigned slots = A.row_bytes / 8;        // 16-byte pieces of a row's key and value together, at most 64
    const unsigned magic = (1u << 20) / slots + 1; // e * magic >> 20 = e / slots for e < 2^20 / slots
    constexpr int DEEP = 4;
    for (unsigned e0 = 0; e0 < rows * slots; e0 += 32 * DEEP) {
        int4 v[DEEP];
        char* to[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const unsigned e = e0 + i * 32 + lane;
            const unsigned r = e * magic >> 20, x = e - r * slots;
            const int64_t s0 = __shfl_sync(FULL_MASK, sk, r & 31), s1 = __shfl_sync(FULL_MASK, sv, r & 31);
            const int64_t d0 = __shfl_sync(FULL_MASK, dk, r & 31), d1 = __shfl_sync(FULL_MASK, dv, r & 31);
            const bool value = x >= slots / 2;
            to[i] = nullptr;
            if (r < rows && s0 >= 0) {
                to[i] = value ? A.c.v + d1 + (x - slots / 2) * 16 : A.c.k + d0 + x * 16;
                v[i] = *reinterpret_cast<const int4*>(value ? A.c.v + s1 + (x - slots / 2) * 16 : A.c.k + s0 + x * 16);
            }
        }
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if (to[i]) *reinterpret_cast<int4*>(to[i]) = v[i];
    }
}
// Where token t of sequence b is, and its place j in the new pages.
__device__ __forceinline__ void kept_row(const EvictArgs& A, int32_t b, int32_t g, int32_t t, int64_t j, int64_t* sk, int64_t* sv, int64_t* dk, int64_t* dv) {
    const int32_t in_page = (1 << A.c.page_shift) - 1;
    const int32_t from = __ldg(A.table + b * A.table_stride + (t >> A.c.page_shift));
    const int32_t to = __ldg(A.new_table + b * A.new_stride + (j >> A.c.page_shift));
    if ((unsigned)from >= (unsigned)A.c.n_pages || (unsigned)to >= (unsigned)A.c.n_pages) return;
    *sk = from * A.c.ks[0] + (t & in_page) * A.c.ks[1] + g * A.c.ks[2];
    *sv = from * A.c.vs[0] + (t & in_page) * A.c.vs[1] + g * A.c.vs[2];
    *dk = to * A.c.ks[0] + (j & in_page) * A.c.ks[1] + g * A.c.ks[2];
    *dv = to * A.c.vs[0] + (j & in_page) * A.c.vs[1] + g * A.c.vs[2];
}

// The kept tokens of a row (sequence, cache head), in order of position.  Latency-bound: the row is read once, then some ten steps wait for one
// another (256 rows of up to 8,191 tokens 22 us, 8 of 131,072 30 us, 8 of 1,000 6 us).  The key of the last one is found 11, 11 and 10 bits at a
// time from histograms; then everybody counts what lies before its part.  A row belongs to a cluster of CTAs that see each other's
// histograms through distributed shared memory, a contiguous part each, so that few long rows use many SMs.  HELD: the keys of a CTA's
// part stay in shared memory (4 bytes a token); beyond that they are made again from the weights for each pass.  COPY: it copies the rows too.
#define KLPM_EVICT_BINS 2048
#define KLPM_EVICT_HELD 49152          // keys a CTA holds (192 KB)
struct EvictShared {
    alignas(16) int32_t hist[3][KLPM_EVICT_BINS];
    int32_t warp_sum[32], warp_eq[32];
    int32_t bin, above, count, total;
    int32_t gt, eq;
};

template <int T, bool HELD, bool COPY>
__global__ void __launch_bounds__(T) evict_select_kernel(const EvictArgs A, int32_t ctas) {
    constexpr int WARPS = T / 32, PER = KLPM_EVICT_BINS / T;
    extern __shared__ __align__(16) unsigned s_key[];
    __shared__ EvictShared S;
    __shared__ int s_lane[COPY ? WARPS : 1][32];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t rank = blockIdx.x % ctas, row = blockIdx.x / ctas;
    const int32_t b = row / A.c.n_heads, g = row % A.c.n_heads;
    int32_t n = __ldg(A.len + b);
    for (int i = tid; i < 3 * KLPM_EVICT_BINS / 4; i += T) reinterpret_cast<int4*>(&S.hist[0][0])[i] = make_int4(0, 0, 0, 0);
    n = n < 0 ? 0 : n > A.max_tokens ? A.max_tokens : n;
    const int32_t part = ((n + ctas - 1) / ctas + 31) & ~31;
    const int32_t t0 = min((long long)rank * part, (long long)n), t1 = min(t0 + part, n);
    int32_t* index = A.index + (int64_t)row * A.keep;
    const float* w = A.weight + b * A.ws[0] + g * A.ws[1];
    float* nw = A.new_weight + b * A.nws[0] + g * A.nws[1];
    if (ctas > 1) cluster.barrier_arrive();
    __syncthreads();
    EvictShared* first = cluster.map_shared_rank(&S, 0);
    // keys, eight of a thread in flight, and the first histogram.  What many tokens have in common -- kept in any case, never looked
    // at -- is counted per warp: 32 additions to one word of shared memory would take turns
    constexpr int DEEP = 8;
    for (int32_t base = t0; base < t1; base += T * DEEP) {
        unsigned k[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const int32_t t = base + i * T + tid;
            k[i] = t < t1 ? evict_key(A, b, g, n, t) : 0u;
        }
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const int32_t t = base + i * T + tid;
            if (HELD && t < t1) s_key[t - t0] = k[i];
            const int held = __popc(__ballot_sync(FULL_MASK, k[i] == 0xffffffffu)), none = __popc(__ballot_sync(FULL_MASK, k[i] == 0x80000000u));
            if (lane == 0) {
                if (held) atomicAdd(&S.hist[0][KLPM_EVICT_BINS - 1], held);
                if (none) atomicAdd(&S.hist[0][0x80000000u >> 21], none);
            }
            if (k[i] && k[i] != 0xffffffffu && k[i] != 0x80000000u) atomicAdd(&S.hist[0][k[i] >> 21], 1);
        }
    }
    auto key = [&](int32_t t) -> unsigned { return t >= t1 ? 0u : HELD ? s_key[t - t0] : evict_key(A, b, g, n, t); };
    unsigned limit = 0;                        // kept: keys above it, and the first `want` that equal it
    int32_t want = 0, K = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        if (pass) {
            const int up = pass == 1 ? 21 : 10;
            for (int32_t t = t0 + tid; t < t1; t += T) {
                const unsigned k = key(t);
                if (k && (k >> up) == (limit >> up)) atomicAdd(&S.hist[pass][(k >> shift) & (pass == 1 ? 2047 : 1023)], 1);
            }
        }
        __syncthreads();
        if (ctas > 1) {
            if (pass == 0) cluster.barrier_wait();            // the first CTA's histograms are 0 by now
            if (rank) {
                for (int i = tid; i < KLPM_EVICT_BINS; i += T) {
                    const int32_t v = S.hist[pass][i];
                    if (v) atomicAdd(&first->hist[pass][i], v);
                }
            }
            cluster.sync();
        }
        if (rank == 0) {
            // bins from the top: thread 0 has the highest
            int32_t c[PER], mine = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                c[i] = S.hist[pass][KLPM_EVICT_BINS - 1 - (tid * PER + i)];
                mine += c[i];
            }
            int32_t upto = mine;
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t v = __shfl_up_sync(FULL_MASK, upto, d);
                if (lane >= d) upto += v;
            }
            if (lane == 31) S.warp_sum[warp] = upto;
            __syncthreads();
            const int32_t sums = lane < WARPS ? S.warp_sum[lane] : 0;
            upto += __reduce_add_sync(FULL_MASK, lane < warp ? sums : 0);
            const int32_t total = __reduce_add_sync(FULL_MASK, sums), wanted = pass ? want : min(A.keep, total);
            int32_t above = upto - mine;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (above < wanted && wanted <= above + c[i]) { S.bin = KLPM_EVICT_BINS - 1 - (tid * PER + i); S.above = above; S.count = c[i]; }
                above += c[i];
            }
            if (tid == 0) S.total = total;
        }
        if (ctas > 1) cluster.sync();
        else __syncthreads();
        const int32_t bin = first->bin, above = first->above, count = first->count;
        if (pass == 0) {
            const int32_t total = first->total;
            K = min(A.keep, total);
            want = K;
            if (K == total) { want = 0; break; }              // everything that is there is kept: keys above 0
        }
        limit |= (unsigned)bin << shift;
        want -= above;
        if (count == want) { limit = limit ? limit - 1 : 0u; want = 0; break; }      // the whole bin is kept
        if (ctas > 1) cluster.sync();                         // (the first CTA writes bin again)
        else __syncthreads();
    }
    // what lies before: in the warps and the CTAs with earlier tokens
    const int32_t per_warp = (part / 32 + WARPS - 1) / WARPS * 32;
    const int32_t a0 = min((long long)t0 + (long long)warp * per_warp, (long long)t1), a1 = min(a0 + per_warp, t1);
    int32_t gts = 0, eqs = 0;
    if (K > 0)
        for (int32_t t = a0; t < a1; t += 32) {
            const unsigned k = t + lane < a1 ? key(t + lane) : 0u;
            gts += __popc(__ballot_sync(FULL_MASK, k > limit));
            eqs += __popc(__ballot_sync(FULL_MASK, k == limit && k));
        }
    __syncthreads();
    if (lane == 0) { S.warp_sum[warp] = gts; S.warp_eq[warp] = eqs; }
    __syncthreads();
    const int32_t a = lane < WARPS ? S.warp_sum[lane] : 0, e0 = lane < WARPS ? S.warp_eq[lane] : 0;
    const int32_t all_gt = __reduce_add_sync(FULL_MASK, a), all_eq = __reduce_add_sync(FULL_MASK, e0);
    gts = __reduce_add_sync(FULL_MASK, lane < warp ? a : 0);
    eqs = __reduce_add_sync(FULL_MASK, lane < warp ? e0 : 0);
    if (tid == 0) { S.gt = all_gt; S.eq = all_eq; }
    if (ctas > 1) {
        cluster.sync();
        for (int r = 0; r < rank; ++r) { gts += *cluster.map_shared_rank(&S.gt, r); eqs += *cluster.map_shared_rank(&S.eq, r); }
        cluster.barrier_arrive();               // nobody leaves while its shared memory is read
    }
    constexpr int AHEAD = COPY ? 1 : 2;          // groups of 32 tokens whose weights are in flight
    for (int32_t base = a0; base < a1 && K > 0; base += 32 * AHEAD) {
        unsigned key_of[AHEAD];
        float weight_of[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int32_t t = base + 32 * i + lane;
            key_of[i] = t < a1 ? key(t) : 0u;
            weight_of[i] = key_of[i] && key_of[i] >= limit ? __ldg(w + t) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int32_t t = base + 32 * i;
            const unsigned k = key_of[i];
            const bool gt = k > limit, eq = k == limit && k;
            const unsigned bg = __ballot_sync(FULL_MASK, gt), be = __ballot_sync(FULL_MASK, eq), below = (1u << lane) - 1;
            const int32_t e = eqs + __popc(be & below), j = gts + __popc(bg & below) + min(e, want);
            const bool kept = gt || (eq && e < want);
            if (kept) {
                index[j] = t + lane;
                nw[j] = weight_of[i];
            }
            if constexpr (COPY) {
                const unsigned bk = __ballot_sync(FULL_MASK, kept);
                int64_t sk = -1, sv = 0, dk = 0, dv = 0;
                if (kept) {
                    kept_row(A, b, g, t + lane, j, &sk, &sv, &dk, &dv);
                    s_lane[warp][__popc(bk & below)] = lane;
                }
                __syncwarp();
                const int from = lane < __popc(bk) ? s_lane[warp][lane] : 0;         // the kept ones side by side
                __syncwarp();
                sk = __shfl_sync(FULL_MASK, sk, from); sv = __shfl_sync(FULL_MASK, sv, from);
                dk = __shfl_sync(FULL_MASK, dk, from); dv = __shfl_sync(FULL_MASK, dv, from);
                copy_kept(A, __popc(bk), sk, sv, dk, dv);
            }
            gts += __popc(bg);
            eqs += __popc(be);
        }
    }
    for (int32_t j = K + rank * T + tid; j < A.keep; j += ctas * T) index[j] = -1;
    for (int32_t j = K + rank * T + tid; j < A.new_len; j += ctas * T) nw[j] = 0.0f;
    if (g == 0 && rank == 0 && tid == 0) A.new_lengths[b] = K;
    if (ctas > 1) cluster.barrier_wait();
}

// The kept rows, keys and values: a warp looks up ROWS of them, one per lane, then copies them.  Bound by HBM (786 MB read and written for 32
// sequences in 127 us: 6.2 TB/s).
template <int ROWS>
__global__ void __launch_bounds__(256, 5) evict_copy_kernel(const EvictArgs A) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t id = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int32_t g = (int32_t)(id % A.c.n_heads), b = blockIdx.y;
    const int64_t j0 = id / A.c.n_heads * ROWS;
    if (j0 >= A.keep) return;
    const int64_t j = j0 + lane;
    int64_t sk = -1, sv = 0, dk = 0, dv = 0;
    if (lane < ROWS && j < A.keep) {
        const int32_t t = A.index[((int64_t)b * A.c.n_heads + g) * A.keep + j];
        if (t >= 0) kept_row(A, b, g, t, j, &sk, &sv, &dk, &dv);
    }
    copy_kept(A, ROWS, sk, sv, dk, dv);
}

template <int T, bool HELD, bool COPY> rt_status launch_select(const EvictArgs& A, int64_t rows, int ctas, size_t smem, cudaStream_t s) {
    if (rt_status st = allow_smem<evict_select_kernel<T, HELD, COPY>>(KLPM_EVICT_HELD * 4)) return st;
    return launch_cluster(evict_select_kernel<T, HELD, COPY>, (unsigned)(rows * ctas), T, ctas, smem, s, A, (int32_t)ctas);
}

}  // namespace

extern "C" {

rt_status kv_rope_table(double* d_turns, int32_t rot_dim, double theta, int32_t scaling, double scale, double original_len,
                        double beta_fast, double beta_slow, float* factor, void* stream) {
    if (!d_turns || rot_dim < 2 || rot_dim % 2 || !(theta > 0) || isinf(theta)) return RT_ERR_INVALID;
    if (rot_dim > KV_MAX_HEAD_DIM) return RT_ERR_TOO_LARGE;
    if (scaling < KV_ROPE_PLAIN || scaling > KV_ROPE_YARN) return RT_ERR_INVALID;
    if (scaling != KV_ROPE_PLAIN && (!(scale >= 1) || isinf(scale))) return RT_ERR_INVALID;
    if (scaling == KV_ROPE_NTK && rot_dim == 2) return RT_ERR_INVALID;
    if (scaling == KV_ROPE_YARN && (!(original_len > 0) || isinf(original_len) || !(beta_slow >= 0) || !(beta_fast > beta_slow) || isinf(beta_fast)))
        return RT_ERR_INVALID;
    if (factor) *factor = scaling == KV_ROPE_YARN ? (float)(0.1 * log(scale) + 1.0) : 1.0f;
    rope_table_kernel<<<1, KV_MAX_HEAD_DIM / 2, 0, (cudaStream_t)stream>>>(d_turns, rot_dim, theta, scaling, scale, original_len, beta_fast, beta_slow);
    CK(cudaGetLastError());
    return RT_OK;
}

rt_status kv_rope_append(const kv_cache* cache, const kv_rope* rope, const int32_t* d_positions, const int32_t* d_slots, int32_t n,
                         const kv_rows* q, const kv_rows* q_out, const kv_rows* k, const kv_rows* v, void* stream) {
    rt_status st = check_cache(cache);
    if (st) return st;
    if (n < 0) return RT_ERR_INVALID;
    if ((st = check_rows(k, n)) || (st = check_rows(v, n))) return st;
    if ((q != nullptr) != (q_out != nullptr)) return RT_ERR_INVALID;
    if (q && ((st = check_rows(q, n)) || (st = check_rows(q_out, n)))) return st;
    if (k->n_heads != cache->n_heads || v->n_heads != cache->n_heads || v->dtype != k->dtype) return RT_ERR_INVALID;
    if (q && (q->dtype != k->dtype || q_out->dtype != k->dtype || q->n_heads != q_out->n_heads)) return RT_ERR_INVALID;
    if (q && q->data == q_out->data && (q->stride[0] != q_out->stride[0] || q->stride[1] != q_out->stride[1])) return RT_ERR_INVALID;
    if (q && !rows_apart(n, q_out->stride[0], q_out->n_heads, q_out->stride[1], cache->head_dim)) return RT_ERR_INVALID;
    if (k->dtype != KV_F32 && cache->dtype != KV_E4M3 && cache->dtype != k->dtype) return RT_ERR_INVALID;
    if (rope) {
        if (!rope->d_turns || rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > cache->head_dim) return RT_ERR_INVALID;
        if (n > 0 && !d_positions) return RT_ERR_INVALID;
    }
    if (n > 0 && !d_slots) return RT_ERR_INVALID;
    if (n == 0) return RT_OK;
    AppendArgs A;
    A.c = cache_dev(cache);
    A.q = rows_dev(q); A.qo = rows_dev(q_out); A.k = rows_dev(k); A.v = rows_dev(v);
    A.turns = rope ? rope->d_turns : nullptr;
    A.rot = rope ? rope->rot_dim : 0;
    A.interleaved = rope ? rope->interleaved != 0 : 0;
    A.factor = rope ? rope->factor : 1.0f;
    A.pos = d_positions; A.slot = d_slots; A.n = n;
    const bool vec = A.c.dim % 16 == 0 && A.rot % 16 == 0 && rows_aligned(k) && rows_aligned(v) && (!q || (rows_aligned(q) && rows_aligned(q_out)));
    A.units = A.c.dim / (vec ? 16 : 2);
    const int32_t heads = A.q.heads + A.k.heads + A.v.heads;
    // Heads per thread: one while that leaves the GPU room, up to a quarter of them (12 of 48) where there is enough to do without.  48 heads of 128
    // elements with 1, 2, 3, 12 heads a thread: 300 tokens 5.3, 3.8, 4.3, 8.0 us; 1,000 11.9, 9.1, 7.3, 13.3; 12,000 113, 81, 62, 56
    const int64_t items = (int64_t)n * heads * (A.c.dim / 16);
    const int32_t limit = heads < 8 ? 2 : heads / 4, wanted = items < 90000 ? 1 : items < 170000 ? 2 : items < 1000000 ? 3 : limit;
    const int32_t each = wanted < limit ? wanted : limit;
    const int32_t all = (heads + each - 1) / each, most = 256 / A.units, groups = (all + most - 1) / most;
    A.slices = (all + groups - 1) / groups;
    A.tokens = 256 / (A.units * A.slices);
    const int64_t blocks = ((int64_t)n + A.tokens - 1) / A.tokens;
    if (blocks > 0x7fffffffLL || groups > 65535) return RT_ERR_TOO_LARGE;
    const size_t smem = (size_t)A.tokens * (A.rot / 2) * sizeof(float2);
    cudaStream_t s = (cudaStream_t)stream;
    const dim3 grid((unsigned)blocks, (unsigned)groups);
    switch (k->dtype * 4 + cache->dtype) {
        case KV_F32 * 4 + KV_BF16: launch_append<KV_F32, KV_BF16>(A, vec, grid, smem, s); break;
        case KV_F32 * 4 + KV_F16: launch_append<KV_F32, KV_F16>(A, vec, grid, smem, s); break;
        case KV_F32 * 4 + KV_E4M3: launch_append<KV_F32, KV_E4M3>(A, vec, grid, smem, s); break;
        case KV_BF16 * 4 + KV_BF16: launch_append<KV_BF16, KV_BF16>(A, vec, grid, smem, s); break;
        case KV_BF16 * 4 + KV_E4M3: launch_append<KV_BF16, KV_E4M3>(A, vec, grid, smem, s); break;
        case KV_F16 * 4 + KV_F16: launch_append<KV_F16, KV_F16>(A, vec, grid, smem, s); break;
        default: launch_append<KV_F16, KV_E4M3>(A, vec, grid, smem, s); break;
    }
    CK(cudaGetLastError());
    return RT_OK;
}

int64_t kv_decode_workspace(const kv_cache* cache, int32_t n_seqs, int32_t n_q_heads, int32_t max_pages, int32_t with_weight) {
    const rt_status st = check_cache(cache);
    if (st) return st;
    if (n_seqs < 0 || n_q_heads < 1 || max_pages < 0 || n_q_heads % cache->n_heads) return RT_ERR_INVALID;
    if (n_seqs > 65535 || n_q_heads > 65535 || (int64_t)max_pages * cache->page_size > KLPM_MAX_TOKENS) return RT_ERR_TOO_LARGE;
    if ((double)n_seqs * n_q_heads * ((double)max_pages * cache->page_size + 64) > 1e15) return RT_ERR_TOO_LARGE;
    // (the query's type is not known here: the larger of what either needs next to an 8-bit cache)
    int64_t bytes = 0;
    for (int tq = KV_BF16; tq <= KV_F16; ++tq) {
        if (cache->dtype != KV_E4M3 && cache->dtype != tq) continue;
        const int64_t n = for_decode(tq, cache->dtype, cache->head_dim, n_q_heads / cache->n_heads, [&](auto x) {
            using X = decltype(x);
            return decode_space(n_seqs, n_q_heads, (int64_t)max_pages * cache->page_size, KLPM_SMS * X::CTAS * KLPM_DECODE_WARPS, X::PART, with_weight != 0).bytes;
        });
        bytes = n > bytes ? n : bytes;
    }
    return bytes;
}

rt_status kv_decode(const kv_cache* cache, const kv_rows* q, const kv_rows* out, int32_t n_seqs, const int32_t* d_page_table,
                    int64_t table_stride, int32_t max_pages, const int32_t* d_lengths, float scale, int32_t window, float* d_lse,
                    float* d_weight, const int64_t* weight_stride, void* d_workspace, int64_t workspace_bytes, void* stream) {
    rt_status st = check_cache(cache);
    if (st) return st;
    if (n_seqs < 0 || max_pages < 0 || window < 0 || !(scale == scale) || isinf(scale)) return RT_ERR_INVALID;
    if ((st = check_rows(q, n_seqs)) || (st = check_rows(out, n_seqs))) return st;
    if (q->dtype == KV_F32 || out->dtype != q->dtype || out->n_heads != q->n_heads || (n_seqs > 0 && q->data == out->data)) return RT_ERR_INVALID;
    if (cache->dtype != KV_E4M3 && cache->dtype != q->dtype) return RT_ERR_INVALID;
    if (q->n_heads % cache->n_heads) return RT_ERR_INVALID;
    if (n_seqs > 65535 || (int64_t)max_pages * cache->page_size > KLPM_MAX_TOKENS) return RT_ERR_TOO_LARGE;
    if (n_seqs > 0 && (!d_lengths || (max_pages > 0 && !d_page_table))) return RT_ERR_INVALID;
    if (table_stride < max_pages && n_seqs > 1) return RT_ERR_INVALID;
    if (!rows_apart(n_seqs, out->stride[0], out->n_heads, out->stride[1], cache->head_dim)) return RT_ERR_INVALID;
    if (d_weight && (!weight_stride || !rows_apart(n_seqs, weight_stride[0], cache->n_heads, weight_stride[1], (int64_t)max_pages * cache->page_size)))
        return RT_ERR_INVALID;
    const int64_t need = kv_decode_workspace(cache, n_seqs, q->n_heads, max_pages, d_weight != nullptr);
    if (need < 0) return (rt_status)need;
    if (need > 0 && (!d_workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(d_workspace) % 256)) return RT_ERR_INVALID;
    if (n_seqs == 0) return RT_OK;
    DecodeArgs A;
    A.c = cache_dev(cache); A.q = rows_dev(q); A.out = rows_dev(out);
    A.table = d_page_table; A.len = d_lengths; A.table_stride = table_stride; A.n_seqs = n_seqs;
    A.group = q->n_heads / cache->n_heads; A.max_tokens = max_pages * cache->page_size; A.window = window; A.scale = scale;
    A.lse = d_lse;
    A.q_words = reinterpret_cast<uintptr_t>(q->data) % 4 == 0 && q->stride[0] % 2 == 0 && q->stride[1] % 2 == 0;
    A.weight = A.max_tokens > 0 ? d_weight : nullptr;
    A.ws[0] = d_weight ? weight_stride[0] : 0; A.ws[1] = d_weight ? weight_stride[1] : 0;
    return for_decode(q->dtype, cache->dtype, cache->head_dim, A.group, [&](auto x) {
        return launch_decode<decltype(x)>(A, (char*)d_workspace, (cudaStream_t)stream);
    });
}

rt_status kv_evict(const kv_cache* cache, const float* d_weight, const int64_t* weight_stride, int32_t n_seqs,
                   const int32_t* d_page_table, int64_t table_stride, int32_t max_pages, const int32_t* d_lengths,
                   const int32_t* d_new_table, int64_t new_stride, int32_t new_pages, int32_t keep, int32_t sinks, int32_t recent,
                   int32_t* d_index, float* d_new_weight, const int64_t* new_weight_stride, int32_t new_weight_len,
                   int32_t* d_new_lengths, void* stream) {
    rt_status st = check_cache(cache);
    if (st) return st;
    if (n_seqs < 0 || max_pages < 0 || new_pages < 0 || keep < 1 || sinks < 0 || recent < 0) return RT_ERR_INVALID;
    if ((int64_t)sinks + recent > keep || new_weight_len < keep || (int64_t)new_pages * cache->page_size < keep) return RT_ERR_INVALID;
    if (n_seqs > 65535 || (int64_t)max_pages * cache->page_size > KLPM_MAX_TOKENS) return RT_ERR_TOO_LARGE;
    if (keep > KLPM_MAX_TOKENS || new_weight_len > KLPM_MAX_TOKENS) return RT_ERR_TOO_LARGE;
    if (n_seqs > 1 && (table_stride < max_pages || new_stride < new_pages)) return RT_ERR_INVALID;
    if (!weight_stride || !new_weight_stride) return RT_ERR_INVALID;
    if (!rows_apart(n_seqs, new_weight_stride[0], cache->n_heads, new_weight_stride[1], new_weight_len)) return RT_ERR_INVALID;
    if (n_seqs > 0 && (!d_lengths || !d_new_table || !d_index || !d_new_weight || !d_new_lengths)) return RT_ERR_INVALID;
    if (n_seqs > 0 && max_pages > 0 && (!d_page_table || !d_weight || d_weight == d_new_weight)) return RT_ERR_INVALID;
    if (n_seqs == 0) return RT_OK;
    EvictArgs A;
    A.c = cache_dev(cache);
    A.weight = d_weight; A.ws[0] = weight_stride[0]; A.ws[1] = weight_stride[1];
    A.table = d_page_table; A.len = d_lengths; A.new_table = d_new_table; A.table_stride = table_stride; A.new_stride = new_stride;
    A.n_seqs = n_seqs; A.max_tokens = max_pages * cache->page_size; A.keep = keep; A.sinks = sinks; A.recent = recent;
    A.new_len = new_weight_len; A.row_bytes = cache->head_dim * elem_size(cache->dtype);
    A.index = d_index; A.new_weight = d_new_weight; A.nws[0] = new_weight_stride[0]; A.nws[1] = new_weight_stride[1];
    A.new_lengths = d_new_lengths;
    cudaStream_t s = (cudaStream_t)stream;
    const int64_t rows = (int64_t)n_seqs * cache->n_heads;
    // Few kept rows are copied by the CTA that selects them: up to 32 KB of a row's keys and values that costs the GPU no more than the other kernel,
    // and the host a launch less (64 of 175 tokens, 7 sequences: 9.4 us and 10.1 of the host, else 8.2 and 11.9); 128 KB take 17 us, else 9.9.
    const bool copy = A.max_tokens <= 1024 && (int64_t)keep * A.row_bytes * 2 <= 32 * 1024;
    // CTAs per row: as many as it takes to hold the keys, and more of them while rows leave SMs idle (8 rows of 131,072: 46 us with 8 CTAs, 49 with 16, 67
    // with 4; 4,257 tokens: 13.0 us with 2 or more, 15.0 us with one)
    int ctas = 1;
    while (ctas < 8 && ((int64_t)ctas * KLPM_EVICT_HELD < A.max_tokens || (rows * ctas * 2 <= KLPM_SMS && A.max_tokens / ctas > 2048))) ctas *= 2;
    const int64_t part = ((A.max_tokens + ctas - 1) / ctas + 31) & ~31LL;
    // rows of a warp of the copy: 8 while that leaves every warp of the GPU at most one turn
    const int rpw = rows * keep <= (int64_t)KLPM_SMS * 64 * 8 ? 8 : 32;
    const int64_t blocks = ((int64_t)((keep + rpw - 1) / rpw) * cache->n_heads + 7) / 8;
    if (rows * ctas > 0x7fffffffLL || blocks > 0x7fffffffLL) return RT_ERR_TOO_LARGE;
    const size_t held = (size_t)part * 4;
    if (copy) return launch_select<256, true, true>(A, rows, ctas, held, s);
    // (1,024 threads: 2,016 tokens 24.8 us instead of 27.7; 256: 1,008 tokens 9.9 us instead of 10.5)
    if (part > KLPM_EVICT_HELD) st = launch_select<1024, false, false>(A, rows, ctas, 0, s);
    else st = part > 1024 ? launch_select<1024, true, false>(A, rows, ctas, held, s) : launch_select<256, true, false>(A, rows, ctas, held, s);
    if (st) return st;
    const dim3 grid((unsigned)blocks, (unsigned)n_seqs);
    return rpw == 8 ? launch_after(evict_copy_kernel<8>, grid, 256, s, A) : launch_after(evict_copy_kernel<32>, grid, 256, s, A);
}

}  // extern "C"
