/*
 * Rotation of queries and keys by their positions, and the way of keys and values into a paged cache, from
 * one fused q/k/v row per token.
 *
 * A pair (a, b) of a head's values turns by position * frequency: (a cos - b sin, b cos + a sin).  The
 * angle in turns is the product of the position and the frequency in units of 2^-64 turns, modulo 2^64:
 * whole numbers, so that a far position keeps its fraction, and no table is read.  The frequency in turns
 * is off by 2^-52 of itself (the factor and the product) and by half a unit.  A block
 * computes the sines and cosines of its tokens once and every head takes them from shared memory.
 *
 * Bound by memory: 8192 tokens of 64 + 2 * 8 heads of 128 bf16 59 us (5.6 TB/s, 0.83 of a copy; the sines
 * come before a block's loads, which other blocks' hide in part), one token 2.4 us.  Blocks of 128 threads,
 * two tokens of 64 pairs each: 256 threads 60 us, 512 73; two, one and eight tokens a block of 256 64, 75
 * and 71.
 */
#include <cuda_fp8.h>

#include "cfa_ops.h"
#include "cfa_values.cuh"

using namespace cfa_dev;

namespace {

constexpr int kThreads = 128;
constexpr int kTokens = 8; /* of a block, at most */

template <typename CT, int N>
__device__ __forceinline__ void store_cache(CT *p, const float (&f)[N], float scale)
{
    if constexpr (sizeof(CT) == 1) {
        Pack<__nv_fp8_storage_t, N> q;
#pragma unroll
        for (int i = 0; i < N; ++i) /* rounded once from fp32; beyond 448 to 448 */
            q.v[i] = __nv_cvt_float_to_fp8(f[i] / scale, __NV_SATFINITE, __NV_E4M3);
        *reinterpret_cast<Pack<__nv_fp8_storage_t, N> *>(p) = q;
    } else {
        store_pack<CT, N>(p, f);
    }
}

struct Split {
    int units, turned; /* a head's units of 2 VEC values, those of them that turn */
    int tokens;        /* of a block */
    int heads;         /* of a block: heads, key heads, value heads in a row */
};

template <typename T, typename CT, int VEC>
__global__ void __launch_bounds__(kThreads, 12) cfa_append_kernel(const cfa_append_args a, const Split s)
{
    extern __shared__ float2 turn[]; /* [tokens][rotary_dim / 2] cos, sin */
    __shared__ int64_t page_of[kTokens];
    __shared__ int32_t place_of[kTokens];
    const int64_t first = (int64_t)blockIdx.x * s.tokens;
    const int n = (int)min((int64_t)s.tokens, a.tokens - first);
    const int head0 = blockIdx.y * s.heads, all = a.heads + 2 * a.kv_heads;
    const int heads = min(s.heads, all - head0);
    const int half = a.rotary_dim / 2;
    launch_in_turn();

    for (int i = threadIdx.x; i < n * half; i += kThreads) {
        const int t = i / half;
        const double f = __ldcg(a.frequencies + (i - t * half));
        const int64_t position = __ldcg(a.positions + first + t);
        double turns = fabs(f) * 0.15915494309189533577;
        turns -= floor(turns); /* of f's magnitude, since 1 less a little has no room for the little */
        uint64_t step = __double2ull_rn(turns * 18446744073709551616.0);
        if (f < 0.0) step = 0 - step;
        const int64_t angle = (int64_t)(step * (uint64_t)position); /* of 2^-64 turns, -1/2 .. 1/2 */
        float2 v;
        sincospif((float)angle * 1.0842021724855044e-19f, &v.y, &v.x);
        if (!isfinite(f)) v.x = v.y = NAN;
        turn[i] = make_float2(v.x * a.magnitude, v.y * a.magnitude);
    }
    if (threadIdx.x < n) {
        const int32_t slot = __ldcg(a.slots + first + threadIdx.x);
        const int32_t page = slot < 0 ? -1 : slot / a.page_size;
        page_of[threadIdx.x] = page < a.pages ? page : -1;
        place_of[threadIdx.x] = slot < 0 ? 0 : slot - page * a.page_size;
    }
    __syncthreads();

    const int per_token = heads * s.units;
    for (int i = threadIdx.x; i < n * per_token; i += kThreads) {
        const int t = i / per_token, j = i - t * per_token;
        const int head = head0 + j / s.units, u = j % s.units;
        const bool is_v = head >= a.heads + a.kv_heads;
        const bool turns = u < s.turned && !is_v;
        if (head < a.heads && !a.q) continue;
        const bool apart = turns && !(a.flags & CFA_APPEND_INTERLEAVED);
        /* where the unit's two halves lie in the head */
        const int lo = apart ? u * VEC : 2 * u * VEC, hi = apart ? half + lo : lo + VEC;
        const T *row = static_cast<const T *>(a.qkv) + (first + t) * a.qkv_stride +
                       (int64_t)head * a.head_dim;
        const Pack<T, VEC> p = load_pack<T, VEC>(row + lo), q = load_pack<T, VEC>(row + hi);
        float x[VEC], y[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            x[k] = to_f32(p.v[k]);
            y[k] = to_f32(q.v[k]);
        }
        if (turns) {
            const float2 *w = turn + t * half + u * VEC;
            if (apart || VEC == 1) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const float2 c = w[k];
                    const float v = x[k];
                    x[k] = v * c.x - y[k] * c.y;
                    y[k] = y[k] * c.x + v * c.y;
                }
            } else {
                if constexpr (VEC > 1) {
#pragma unroll
                    for (int k = 0; k < VEC; k += 2) {
                        float2 c = w[k / 2];
                        float v = x[k];
                        x[k] = v * c.x - x[k + 1] * c.y;
                        x[k + 1] = x[k + 1] * c.x + v * c.y;
                        c = w[VEC / 2 + k / 2];
                        v = y[k];
                        y[k] = v * c.x - y[k + 1] * c.y;
                        y[k + 1] = y[k + 1] * c.x + v * c.y;
                    }
                }
            }
        }
        if (head < a.heads) {
            T *to = static_cast<T *>(a.q) + (first + t) * a.q_stride + (int64_t)head * a.head_dim;
            store_pack<T, VEC>(to + lo, x);
            store_pack<T, VEC>(to + hi, y);
        } else if (page_of[t] >= 0) {
            CT *to = is_v ? static_cast<CT *>(a.v_cache) + page_of[t] * a.v_page_stride +
                                place_of[t] * a.v_token_stride +
                                (head - a.heads - a.kv_heads) * a.v_head_stride
                          : static_cast<CT *>(a.k_cache) + page_of[t] * a.k_page_stride +
                                place_of[t] * a.k_token_stride + (head - a.heads) * a.k_head_stride;
            const float scale = is_v ? a.v_scale : a.k_scale;
            store_cache<CT, VEC>(to + lo, x, scale);
            store_cache<CT, VEC>(to + hi, y, scale);
        }
    }
}

template <typename T, typename CT, int VEC>
cudaError_t launch(const cfa_append_args &a, cudaStream_t stream)
{
    const int half = a.rotary_dim / 2, all = a.heads + 2 * a.kv_heads;
    Split s;
    s.units = a.head_dim / (2 * VEC);
    s.turned = a.rotary_dim / (2 * VEC);
    s.tokens = 1;
    s.heads = all;
    /* Few tokens: their heads on as many blocks as give every thread one unit.  Many: so many tokens
     * that every thread computes one sine and cosine.  32 + 2 * 8 heads of 128, the first way and the
     * second: 512 tokens 5.1 and 6.3 us, 1024 7.3 and 7.7, 2048 13.2 and 16.0, 4096 23.6 and 21.7; 8 + 2
     * heads of 64: 512 2.7 and 3.4, 1024 3.5 and 3.8, 2048 5.0 and 4.5, 4096 6.9 and 6.6. */
    if (a.tokens < 1024) {
        s.heads = (kThreads + s.units - 1) / s.units;
        if (s.heads > all) s.heads = all;
    } else {
        s.tokens = half ? kThreads / half : kTokens;
        s.tokens = s.tokens < 1 ? 1 : s.tokens > kTokens ? kTokens : s.tokens;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.tokens + s.tokens - 1) / s.tokens),
                       (unsigned)((all + s.heads - 1) / s.heads));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(float2) * s.tokens * half;
    cfg.stream = stream;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    void *p[] = {const_cast<cfa_append_args *>(&a), &s};
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(&cfa_append_kernel<T, CT, VEC>), p);
}

template <typename T, typename CT> cudaError_t pick(const cfa_append_args &a, cudaStream_t stream)
{
    constexpr int kVec = 8;
    uint64_t grid = (uint64_t)(uintptr_t)a.qkv | (uintptr_t)a.q;
    if (a.tokens > 1) grid |= (uint64_t)(a.qkv_stride | a.q_stride) * sizeof(T);
    const uint64_t cgrid = (uint64_t)(uintptr_t)a.k_cache | (uintptr_t)a.v_cache |
                           (uint64_t)(a.k_page_stride | a.k_token_stride | a.k_head_stride |
                                      a.v_page_stride | a.v_token_stride | a.v_head_stride) * sizeof(CT);
    if (!(grid & 15) && !(cgrid & (kVec * sizeof(CT) - 1)) && a.head_dim % (2 * kVec) == 0 &&
        a.rotary_dim % (2 * kVec) == 0)
        return launch<T, CT, kVec>(a, stream);
    return launch<T, CT, 1>(a, stream);
}

template <typename T> cudaError_t pick(const cfa_append_args &a, cudaStream_t stream)
{
    if (a.cache_dtype == CFA_DTYPE_F8_E4M3) return pick<T, __nv_fp8_storage_t>(a, stream);
    return pick<T, T>(a, stream);
}

} // namespace

cudaError_t cfa_launch_append(const cfa_append_args *a, cudaStream_t stream)
{
    if (a->dtype == CFA_DTYPE_F16) return pick<__half>(*a, stream);
    return pick<__nv_bfloat16>(*a, stream);
}
