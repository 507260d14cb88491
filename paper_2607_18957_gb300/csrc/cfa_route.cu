/*
 * Choice of experts.  One warp a token: each lane holds every 32nd logit, the top_k come out one at
 * a time as the warp's largest key, a key being the fp32 value mapped onto unsigned integers of the
 * same order, with equal keys going to the lowest index.
 */
#include <math.h>

#include "cfa_device.cuh"
#include "cfa_ops.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace {

constexpr int kWarps = 4;
constexpr uint32_t kAll = 0xFFFFFFFFu;

/* Unsigned integers in the order of the floats; 0 for -inf and NaN, which no choice goes by. */
__device__ __forceinline__ uint32_t order_of(float v)
{
    if (!(v > -INFINITY)) return 0u;
    const uint32_t b = __float_as_uint(v == 0.0f ? 0.0f : v); /* -0 ties with 0 */
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float logit(const cfa_route_args &a, int64_t i)
{
    if (a.dtype == CFA_DTYPE_F32) return static_cast<const float *>(a.logits)[i];
    if (a.dtype == CFA_DTYPE_F16) return __half2float(static_cast<const __half *>(a.logits)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16 *>(a.logits)[i]);
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}

__device__ __forceinline__ float warp_add(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}

/* R: logits per lane. */
template <int R>
__global__ void __launch_bounds__(kWarps * 32) cfa_route_kernel(const cfa_route_args a)
{
    extern __shared__ float s_key[]; /* [warps][experts], with groups only */
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = (int64_t)blockIdx.x * kWarps + warp;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (t >= a.tokens) return;

    float v[R], key[R];
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int e = r * 32 + lane;
        v[r] = e < a.experts ? logit(a, t * a.logits_stride + e) : -INFINITY;
        nan |= v[r] != v[r];
        top = fmaxf(top, v[r]);
    }
    const bool softmax = a.scoring == CFA_SCORE_SOFTMAX;
    float norm = 1.0f;
    if (softmax) {
        top = warp_max(top);
        nan = __any_sync(kAll, nan);
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r * 32 + lane < a.experts) sum += v[r] > -INFINITY ? expf(v[r] - top) : 0.0f;
        norm = nan ? NAN : warp_add(sum);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int e = r * 32 + lane;
        float k = softmax ? v[r] : 1.0f / (1.0f + expf(-v[r]));
        if (a.bias && e < a.experts)
            k = (softmax ? expf(v[r] - top) / norm : k) + a.bias[e];
        key[r] = v[r] > -INFINITY ? k : -INFINITY;
    }

    if (a.groups > 1) {
        float *mine = s_key + warp * a.experts;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r * 32 + lane < a.experts) mine[r * 32 + lane] = key[r];
        __syncwarp();
        const int size = a.experts / a.groups;
        float first = -INFINITY, second = -INFINITY;
        if (lane < a.groups)
            for (int i = 0; i < size; ++i) {
                const float k = mine[lane * size + i];
                if (!(k > -INFINITY)) continue;
                if (k > first) {
                    second = first;
                    first = k;
                } else if (k > second) {
                    second = k;
                }
            }
        const float best = softmax || size == 1 ? first : first + second;
        /* a group is kept if fewer than top_groups come before it */
        int before = 0;
        for (int g = 0; g < a.groups; ++g) {
            const float o = __shfl_sync(kAll, best, g);
            const uint32_t x = order_of(o), y = order_of(best);
            before += x > y || (x == y && g < lane);
        }
        const uint32_t kept = __ballot_sync(kAll, lane < a.groups && before < a.top_groups);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int e = r * 32 + lane;
            if (e < a.experts && !(kept >> (e / size) & 1u)) key[r] = -INFINITY;
        }
    }

    uint32_t k[R];
#pragma unroll
    for (int r = 0; r < R; ++r) k[r] = order_of(key[r]);
    float chosen = -INFINITY; /* lane j: the logit of choice j */
    int id = -1;
    for (int j = 0; j < a.top_k; ++j) {
        uint32_t best = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) best = max(best, k[r]);
        best = __reduce_max_sync(kAll, best);
        if (best == 0) break; /* nothing left to choose */
        uint32_t e = kAll;
        float z = 0.0f;
#pragma unroll
        for (int r = R - 1; r >= 0; --r)
            if (k[r] == best) {
                e = r * 32 + lane;
                z = v[r];
            }
        const uint32_t win = __reduce_min_sync(kAll, e);
        z = __shfl_sync(kAll, z, win & 31u);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r * 32 + lane == win) k[r] = 0;
        if (lane == j) {
            chosen = z;
            id = (int)win;
        }
    }

    float w = 0.0f;
    const bool renormalize = a.flags & CFA_ROUTE_RENORMALIZE;
    if (softmax) {
        if (renormalize) {
            const float m = warp_max(chosen);
            w = id >= 0 ? expf(chosen - m) : 0.0f;
            w /= nan ? NAN : warp_add(w);
        } else {
            w = expf(chosen - top) / norm;
        }
    } else {
        w = id >= 0 ? 1.0f / (1.0f + expf(-chosen)) : 0.0f;
        if (renormalize) {
            const float sum = warp_add(w);
            w = sum > 0.0f ? w / sum : 0.0f;
        }
    }
    if (lane < a.top_k) {
        a.weights[t * a.top_k + lane] = id >= 0 ? w * a.scale : 0.0f;
        a.ids[t * a.top_k + lane] = id;
    }
}

template <int R> cudaError_t launch(const cfa_route_args &a, cudaStream_t stream)
{
    const unsigned grid = (unsigned)((a.tokens + kWarps - 1) / kWarps);
    const size_t smem = a.groups > 1 ? sizeof(float) * kWarps * a.experts : 0;
    cfa_launch_ctl ctl = {};
    ctl.flags = CFA_LAUNCH_EARLY;
    void *p[] = {const_cast<cfa_route_args *>(&a)};
    return cfa_dev::launch_ctl(reinterpret_cast<const void *>(&cfa_route_kernel<R>), grid,
                               kWarps * 32, smem, stream, ctl, p);
}

} // namespace

cudaError_t cfa_launch_route(const cfa_route_args *a, cudaStream_t stream)
{
    if (a->experts <= 32) return launch<1>(*a, stream);
    if (a->experts <= 64) return launch<2>(*a, stream);
    if (a->experts <= 128) return launch<4>(*a, stream);
    if (a->experts <= 256) return launch<8>(*a, stream);
    if (a->experts <= 512) return launch<16>(*a, stream);
    return launch<32>(*a, stream);
}
