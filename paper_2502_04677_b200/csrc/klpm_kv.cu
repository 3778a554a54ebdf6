// The KV cache behind the radix tree: rotary positions and append, attention of one new token over the paged
// cache, eviction by accumulated attention weight.  See include/klpm_kv.h for the ABI.
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

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
    int32_t units, slices;        // per token: units of a head (pairs, or 16 elements), threads that share its heads
};

// One thread handles one unit of a head -- a pair of elements, or (VEC) 8 pairs in 16 elements that two 16-byte loads bring --
// of every `slices`-th head of a token, so that the angles of its pairs are worked out once.
template <int TX, int TC, bool VEC>
__global__ void __launch_bounds__(256) rope_append_kernel(const AppendArgs A) {
    using X = typename Elem<TX>::T;
    using C = typename Elem<TC>::T;
    constexpr int P = VEC ? 8 : 1;
    const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int32_t per = A.units * A.slices;
    const int32_t tok = (int32_t)(gid / per);
    if (tok >= A.n) return;
    const int32_t r = (int32_t)(gid - (int64_t)tok * per);
    const int32_t slice = r / A.units, u = r - slice * A.units;
    // where the unit's elements are: lo[0..P) and hi[0..P) of the pairs (interleaved: 2P elements in a row)
    const int32_t rot_units = A.turns ? A.rot / (2 * P) : 0;
    const bool turn = u < rot_units;
    const bool pairs_apart = turn && !A.interleaved;
    const int32_t e0 = pairs_apart ? u * P : u * 2 * P;
    const int32_t e1 = pairs_apart ? A.rot / 2 + u * P : e0 + P;
    float cs[P], sn[P];
#pragma unroll
    for (int j = 0; j < P; ++j) { cs[j] = 1.0f; sn[j] = 0.0f; }
    if (turn) {
        const double p = (double)__ldg(A.pos + tok);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            // whole turns are taken off in 64 bits: what is left of a far position is exact to 2^-31 * 2^-22 of a turn and better
            double t = p * __ldg(A.turns + u * P + j);
            t -= rint(t);
            float s, c;
            sincospif(2.0f * (float)t, &s, &c);
            cs[j] = c * A.factor; sn[j] = s * A.factor;
        }
    }
    const int32_t slot = __ldg(A.slot + tok);
    const int32_t page = slot >> A.c.page_shift, at = slot & ((1 << A.c.page_shift) - 1);
    const bool stored = slot >= 0 && page < A.c.n_pages;
    const int32_t heads = A.q.heads + A.k.heads + A.v.heads;
    for (int32_t h = slice; h < heads; h += A.slices) {
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
            if (A.interleaved) {
                float y[2 * P];
#pragma unroll
                for (int j = 0; j < P; ++j) { y[j] = a[j]; y[P + j] = b[j]; }
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float p0 = y[2 * j], p1 = y[2 * j + 1];
                    y[2 * j] = p0 * cs[j] - p1 * sn[j];
                    y[2 * j + 1] = p0 * sn[j] + p1 * cs[j];
                }
#pragma unroll
                for (int j = 0; j < P; ++j) { a[j] = y[j]; b[j] = y[P + j]; }
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

template <int TX, int TC> void launch_append(const AppendArgs& A, bool vec, unsigned grid, cudaStream_t s) {
    if (vec) rope_append_kernel<TX, TC, true><<<grid, 256, 0, s>>>(A);
    else rope_append_kernel<TX, TC, false><<<grid, 256, 0, s>>>(A);
}

// ------------------------------------------------------------------------------------------------
// attention of one new token
// ------------------------------------------------------------------------------------------------
struct DecodeArgs {
    CacheDev c;
    RowsDev q, out;
    const int32_t *table, *len;
    int64_t table_stride;
    int32_t n_seqs, group, max_tokens, window;
    float scale;
    float* lse;
    float* weight;
    int64_t ws[2];
};

__device__ __forceinline__ void token_range(const DecodeArgs& A, int32_t b, int32_t* lo, int32_t* hi) {
    int32_t n = __ldg(A.len + b);
    n = n < 0 ? 0 : n > A.max_tokens ? A.max_tokens : n;
    *hi = n;
    *lo = A.window > 0 && n > A.window ? n - A.window : 0;
}

// One warp per (sequence, query head), one token after the other: s_t, then the running maximum, sum and output.
template <int TQ, int TC>
__global__ void __launch_bounds__(128) decode_kernel(const DecodeArgs A) {
    using Q = typename Elem<TQ>::T;
    using C = typename Elem<TC>::T;
    const int lane = threadIdx.x & 31;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (id >= (int64_t)A.n_seqs * A.q.heads) return;
    const int32_t b = (int32_t)(id / A.q.heads), h = (int32_t)(id % A.q.heads), g = h / A.group;
    const Q* q = reinterpret_cast<const Q*>(A.q.p + b * A.q.sr + h * A.q.sh);
    float x[KV_MAX_HEAD_DIM / 32], o[KV_MAX_HEAD_DIM / 32];
    for (int j = 0; j < KV_MAX_HEAD_DIM / 32; ++j) {
        const int d = lane + 32 * j;
        x[j] = d < A.c.dim ? to_float(q[d]) : 0.0f;
        o[j] = 0.0f;
    }
    int32_t lo, hi;
    token_range(A, b, &lo, &hi);
    float m = -INFINITY, l = 0.0f;
    for (int32_t t = lo; t < hi; ++t) {
        const int32_t page = __ldg(A.table + b * A.table_stride + (t >> A.c.page_shift));
        if ((unsigned)page >= (unsigned)A.c.n_pages) continue;
        const int32_t at = t & ((1 << A.c.page_shift) - 1);
        const C* k = reinterpret_cast<const C*>(A.c.k + page * A.c.ks[0] + at * A.c.ks[1] + g * A.c.ks[2]);
        const C* v = reinterpret_cast<const C*>(A.c.v + page * A.c.vs[0] + at * A.c.vs[1] + g * A.c.vs[2]);
        float s = 0.0f;
        for (int j = 0; j < KV_MAX_HEAD_DIM / 32; ++j) if (lane + 32 * j < A.c.dim) s += x[j] * to_float(k[lane + 32 * j]);
        for (int w = 16; w; w >>= 1) s += __shfl_xor_sync(FULL_MASK, s, w);
        s *= A.scale * A.c.k_scale;
        const float m1 = fmaxf(m, s);
        const float base = m1 == -INFINITY ? 0.0f : m1;
        const float f = expf(m - base), p = expf(s - base);
        m = m1;
        l = l * f + p;
        for (int j = 0; j < KV_MAX_HEAD_DIM / 32; ++j) if (lane + 32 * j < A.c.dim) o[j] = o[j] * f + p * to_float(v[lane + 32 * j]);
    }
    Q* out = reinterpret_cast<Q*>(A.out.p + b * A.out.sr + h * A.out.sh);
    const float r = l == 0.0f ? 0.0f : A.c.v_scale / l;
    for (int j = 0; j < KV_MAX_HEAD_DIM / 32; ++j) if (lane + 32 * j < A.c.dim) out[lane + 32 * j] = from_float<Q>(l == 0.0f ? 0.0f : o[j] * r);
    if (lane == 0) A.lse[id] = l == 0.0f ? -INFINITY : m + logf(l);
}

// One warp per (sequence, cache head, token): the scores once more, now that the sums are known.
template <int TQ, int TC>
__global__ void __launch_bounds__(128) decode_weight_kernel(const DecodeArgs A) {
    using Q = typename Elem<TQ>::T;
    using C = typename Elem<TC>::T;
    const int lane = threadIdx.x & 31;
    const int32_t t = blockIdx.x * 4 + (threadIdx.x >> 5), g = blockIdx.y, b = blockIdx.z;
    int32_t lo, hi;
    token_range(A, b, &lo, &hi);
    if (t < lo || t >= hi) return;
    const int32_t page = __ldg(A.table + b * A.table_stride + (t >> A.c.page_shift));
    if ((unsigned)page >= (unsigned)A.c.n_pages) return;
    const int32_t at = t & ((1 << A.c.page_shift) - 1);
    const C* k = reinterpret_cast<const C*>(A.c.k + page * A.c.ks[0] + at * A.c.ks[1] + g * A.c.ks[2]);
    float sum = 0.0f;
    for (int32_t h = g * A.group; h < (g + 1) * A.group; ++h) {
        const Q* q = reinterpret_cast<const Q*>(A.q.p + b * A.q.sr + h * A.q.sh);
        float s = 0.0f;
        for (int d = lane; d < A.c.dim; d += 32) s += to_float(q[d]) * to_float(k[d]);
        for (int w = 16; w; w >>= 1) s += __shfl_xor_sync(FULL_MASK, s, w);
        const float lse = A.lse[(int64_t)b * A.q.heads + h];
        if (lse != -INFINITY) sum += expf(s * A.scale * A.c.k_scale - lse);
    }
    if (lane == 0) A.weight[b * A.ws[0] + g * A.ws[1] + t] += sum;
}

template <int TQ, int TC> void launch_decode(const DecodeArgs& A, cudaStream_t s) {
    const int64_t warps = (int64_t)A.n_seqs * A.q.heads;
    decode_kernel<TQ, TC><<<(unsigned)((warps + 3) / 4), 128, 0, s>>>(A);
    if (A.weight) {
        const dim3 grid((A.max_tokens + 3) / 4, A.c.n_heads, A.n_seqs);
        decode_weight_kernel<TQ, TC><<<grid, 128, 0, s>>>(A);
    }
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
    if (t >= n) return 0u;
    const int32_t page = __ldg(A.table + b * A.table_stride + (t >> A.c.page_shift));
    if ((unsigned)page >= (unsigned)A.c.n_pages) return 0u;
    if (t < A.sinks || t >= n - A.recent) return 0xffffffffu;
    const float w = __ldg(A.weight + b * A.ws[0] + g * A.ws[1] + t);
    if (w != w) return 1u;
    const unsigned u = __float_as_uint(w == 0.0f ? 0.0f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

#define KLPM_EVICT_THREADS 1024
// One CTA per (sequence, cache head): the key of the last token that is kept is found 8 bits at a time, then the kept
// tokens are numbered in order of position.
__global__ void __launch_bounds__(KLPM_EVICT_THREADS) evict_select_kernel(const EvictArgs A) {
    __shared__ int32_t hist[256];
    __shared__ int32_t warp_sum[32];
    __shared__ int32_t s_bin, s_above, s_total;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t b = blockIdx.x / A.c.n_heads, g = blockIdx.x % A.c.n_heads;
    int32_t n = __ldg(A.len + b);
    n = n < 0 ? 0 : n > A.max_tokens ? A.max_tokens : n;
    int32_t* index = A.index + (int64_t)blockIdx.x * A.keep;
    float* nw = A.new_weight + b * A.nws[0] + g * A.nws[1];
    // how many there are
    int32_t mine = 0;
    for (int32_t t = tid; t < n; t += KLPM_EVICT_THREADS) mine += evict_key(A, b, g, n, t) != 0u;
    mine = __reduce_add_sync(FULL_MASK, mine);
    if (lane == 0) warp_sum[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        const int32_t v = __reduce_add_sync(FULL_MASK, warp_sum[lane]);
        if (lane == 0) s_total = v;
    }
    __syncthreads();
    const int32_t K = min(A.keep, s_total);
    unsigned prefix = 0, mask = 0;
    int32_t want = K;                              // how many of those with this prefix are kept
    for (int shift = 24; shift >= 0 && K > 0; shift -= 8) {
        for (int i = tid; i < 256; i += KLPM_EVICT_THREADS) hist[i] = 0;
        __syncthreads();
        for (int32_t t = tid; t < n; t += KLPM_EVICT_THREADS) {
            const unsigned k = evict_key(A, b, g, n, t);
            if (k != 0u && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int32_t above = 0;
            int bin = 255;
            for (; bin > 0 && above + hist[bin] < want; --bin) above += hist[bin];
            s_bin = bin; s_above = above;
        }
        __syncthreads();
        want -= s_above;
        prefix |= (unsigned)s_bin << shift;
        mask |= 255u << shift;
        __syncthreads();
    }
    int32_t gt0 = 0, eq0 = 0;
    for (int32_t base = 0; base < n && K > 0; base += KLPM_EVICT_THREADS) {
        const int32_t t = base + tid;
        const unsigned k = evict_key(A, b, g, n, t);
        const bool gt = k > prefix, eq = k == prefix;
        const unsigned bg = __ballot_sync(FULL_MASK, gt), be = __ballot_sync(FULL_MASK, eq), below = (1u << lane) - 1;
        if (lane == 0) warp_sum[warp] = __popc(bg) | __popc(be) << 16;
        __syncthreads();
        int32_t before = 0, all = 0;
        for (int w = 0; w < 32; ++w) { const int32_t v = warp_sum[w]; if (w < warp) before += v; all += v; }
        const int32_t gts = gt0 + (before & 0xffff) + __popc(bg & below), eqs = eq0 + (before >> 16) + __popc(be & below);
        if (gt || (eq && eqs < want)) {
            const int32_t j = gts + min(eqs, want);
            index[j] = t;
            nw[j] = __ldg(A.weight + b * A.ws[0] + g * A.ws[1] + t);
        }
        gt0 += all & 0xffff;
        eq0 += all >> 16;
        __syncthreads();
    }
    for (int32_t j = K + tid; j < A.keep; j += KLPM_EVICT_THREADS) index[j] = -1;
    for (int32_t j = K + tid; j < A.new_len; j += KLPM_EVICT_THREADS) nw[j] = 0.0f;
    if (g == 0 && tid == 0) A.new_lengths[b] = K;
}

// 16 bytes of a kept row per thread, keys and values.
__global__ void __launch_bounds__(256) evict_copy_kernel(const EvictArgs A) {
    const int32_t chunks = A.row_bytes / 16;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int32_t x = (int32_t)(id % chunks);
    const int64_t row = id / chunks;
    const int32_t g = (int32_t)(row % A.c.n_heads), b = blockIdx.y;
    const int64_t j = row / A.c.n_heads;
    if (j >= A.keep) return;
    const int32_t t = A.index[((int64_t)b * A.c.n_heads + g) * A.keep + j];
    if (t < 0) return;
    const int32_t in_page = (1 << A.c.page_shift) - 1;
    const int32_t from = __ldg(A.table + b * A.table_stride + (t >> A.c.page_shift));
    const int32_t to = __ldg(A.new_table + b * A.new_stride + (j >> A.c.page_shift));
    if ((unsigned)from >= (unsigned)A.c.n_pages || (unsigned)to >= (unsigned)A.c.n_pages) return;
    const int64_t sk = from * A.c.ks[0] + (t & in_page) * A.c.ks[1] + g * A.c.ks[2] + x * 16;
    const int64_t dk = to * A.c.ks[0] + (j & in_page) * A.c.ks[1] + g * A.c.ks[2] + x * 16;
    const int64_t sv = from * A.c.vs[0] + (t & in_page) * A.c.vs[1] + g * A.c.vs[2] + x * 16;
    const int64_t dv = to * A.c.vs[0] + (j & in_page) * A.c.vs[1] + g * A.c.vs[2] + x * 16;
    const int4 a = *reinterpret_cast<const int4*>(A.c.k + sk), c = *reinterpret_cast<const int4*>(A.c.v + sv);
    *reinterpret_cast<int4*>(A.c.k + dk) = a;
    *reinterpret_cast<int4*>(A.c.v + dv) = c;
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
    A.slices = n >= 1024 ? (heads < 4 ? heads : 4) : heads;
    const int64_t blocks = ((int64_t)n * A.units * A.slices + 255) / 256;
    if (blocks > 0x7fffffffLL) return RT_ERR_TOO_LARGE;
    cudaStream_t s = (cudaStream_t)stream;
    const unsigned grid = (unsigned)blocks;
    switch (k->dtype * 4 + cache->dtype) {
        case KV_F32 * 4 + KV_BF16: launch_append<KV_F32, KV_BF16>(A, vec, grid, s); break;
        case KV_F32 * 4 + KV_F16: launch_append<KV_F32, KV_F16>(A, vec, grid, s); break;
        case KV_F32 * 4 + KV_E4M3: launch_append<KV_F32, KV_E4M3>(A, vec, grid, s); break;
        case KV_BF16 * 4 + KV_BF16: launch_append<KV_BF16, KV_BF16>(A, vec, grid, s); break;
        case KV_BF16 * 4 + KV_E4M3: launch_append<KV_BF16, KV_E4M3>(A, vec, grid, s); break;
        case KV_F16 * 4 + KV_F16: launch_append<KV_F16, KV_F16>(A, vec, grid, s); break;
        default: launch_append<KV_F16, KV_E4M3>(A, vec, grid, s); break;
    }
    CK(cudaGetLastError());
    return RT_OK;
}

int64_t kv_decode_workspace(const kv_cache* cache, int32_t n_seqs, int32_t n_q_heads, int32_t max_pages, int32_t with_weight) {
    (void)with_weight;
    const rt_status st = check_cache(cache);
    if (st) return st;
    if (n_seqs < 0 || n_q_heads < 1 || max_pages < 0 || n_q_heads % cache->n_heads) return RT_ERR_INVALID;
    return ((int64_t)n_seqs * n_q_heads * 4 + 255) / 256 * 256;
}

rt_status kv_decode(const kv_cache* cache, const kv_rows* q, const kv_rows* out, int32_t n_seqs, const int32_t* d_page_table,
                    int64_t table_stride, int32_t max_pages, const int32_t* d_lengths, float scale, int32_t window, float* d_lse,
                    float* d_weight, const int64_t* weight_stride, void* d_workspace, int64_t workspace_bytes, void* stream) {
    rt_status st = check_cache(cache);
    if (st) return st;
    if (n_seqs < 0 || max_pages < 0 || window < 0 || !(scale == scale) || isinf(scale)) return RT_ERR_INVALID;
    if ((st = check_rows(q, n_seqs)) || (st = check_rows(out, n_seqs))) return st;
    if (q->dtype == KV_F32 || out->dtype != q->dtype || out->n_heads != q->n_heads) return RT_ERR_INVALID;
    if (cache->dtype != KV_E4M3 && cache->dtype != q->dtype) return RT_ERR_INVALID;
    if (q->n_heads % cache->n_heads) return RT_ERR_INVALID;
    if (n_seqs > 65535 || (int64_t)max_pages * cache->page_size > KLPM_MAX_TOKENS) return RT_ERR_TOO_LARGE;
    if (n_seqs > 0 && (!d_lengths || (max_pages > 0 && !d_page_table))) return RT_ERR_INVALID;
    if (table_stride < max_pages && n_seqs > 1) return RT_ERR_INVALID;
    if (d_weight && !weight_stride) return RT_ERR_INVALID;
    const int64_t need = kv_decode_workspace(cache, n_seqs, q->n_heads, max_pages, d_weight != nullptr);
    if (need < 0) return (rt_status)need;
    if (need > 0 && (!d_workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(d_workspace) % 256)) return RT_ERR_INVALID;
    if (n_seqs == 0) return RT_OK;
    DecodeArgs A;
    A.c = cache_dev(cache); A.q = rows_dev(q); A.out = rows_dev(out);
    A.table = d_page_table; A.len = d_lengths; A.table_stride = table_stride; A.n_seqs = n_seqs;
    A.group = q->n_heads / cache->n_heads; A.max_tokens = max_pages * cache->page_size; A.window = window; A.scale = scale;
    A.lse = d_lse ? d_lse : (float*)d_workspace;
    A.weight = A.max_tokens > 0 ? d_weight : nullptr;
    A.ws[0] = d_weight ? weight_stride[0] : 0; A.ws[1] = d_weight ? weight_stride[1] : 0;
    cudaStream_t s = (cudaStream_t)stream;
    switch (q->dtype * 4 + cache->dtype) {
        case KV_BF16 * 4 + KV_BF16: launch_decode<KV_BF16, KV_BF16>(A, s); break;
        case KV_BF16 * 4 + KV_E4M3: launch_decode<KV_BF16, KV_E4M3>(A, s); break;
        case KV_F16 * 4 + KV_F16: launch_decode<KV_F16, KV_F16>(A, s); break;
        default: launch_decode<KV_F16, KV_E4M3>(A, s); break;
    }
    CK(cudaGetLastError());
    return RT_OK;
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
    if (n_seqs > 0 && (!d_lengths || !d_new_table || !d_index || !d_new_weight || !d_new_lengths)) return RT_ERR_INVALID;
    if (n_seqs > 0 && max_pages > 0 && (!d_page_table || !d_weight)) return RT_ERR_INVALID;
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
    const int64_t blocks = ((int64_t)keep * cache->n_heads * (A.row_bytes / 16) + 255) / 256;
    if (rows > 0x7fffffffLL || blocks > 0x7fffffffLL) return RT_ERR_TOO_LARGE;
    evict_select_kernel<<<(unsigned)rows, KLPM_EVICT_THREADS, 0, s>>>(A);
    CK(cudaGetLastError());
    evict_copy_kernel<<<dim3((unsigned)blocks, (unsigned)n_seqs), 256, 0, s>>>(A);
    CK(cudaGetLastError());
    return RT_OK;
}

}  // extern "C"
