/*
 * Norms between blocks: a = x or its norm times post_weight, times act(gate); h = residual + scale a;
 * y = norm(h) weight, norm(v) = v / sqrt(mean(v^2) + eps).
 *
 * A row lies in the registers of `lanes` threads, up to NV pieces of VEC values each, from its only
 * load to the stores; the sum of squares is the one thing that they exchange.  h is held in fp32 and y
 * is computed from that, not from h as it is stored.
 */
#include "cfa_ops.h"
#include "cfa_values.cuh"

using namespace cfa_dev;

namespace {

constexpr int kBlock = 128; /* threads, unless a row has more */
constexpr int kEarly = 8;   /* up to so many values per thread the gate and the weight are asked for with x */

/* a act(v) */
__device__ __forceinline__ float gated(float a, float v, int act)
{
    switch (act) {
    case CFA_ACT_RELU: return a * (v < 0.0f ? 0.0f : v); /* NaN stays */
    case CFA_ACT_GELU: return a * (0.5f * v * (1.0f + erff(v * 0.70710678118654752f)));
    case CFA_ACT_GELU_TANH:
        return a * (0.5f * v * (1.0f + tanhf(0.79788456080286536f * (v + 0.044715f * v * v * v))));
    case CFA_ACT_SILU:
        /* exp of a negative argument alone, since exp(-v) leaves fp32 before v / (1 + exp(-v)) does, and
         * as a square, one half of it behind a: exp(v) has lost bits where a v exp(v) has not yet */
        if (v < 0.0f) {
            const float half = expf(0.5f * v);
            return a * (v * half / (1.0f + half * half)) * half;
        }
        return a * (v / (1.0f + expf(-v)));
    default: return a * v;
    }
}

/* The sum over the row's threads (a power of two, neighbours), in the same order every time. */
__device__ __forceinline__ float row_sum(float v, int lanes, float *part)
{
    for (int o = min(lanes, 32) >> 1; o; o >>= 1) v += __shfl_xor_sync(kAllLanes, v, o);
    if (lanes <= 32) return v;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = lanes >> 5;
    if (lane == 0) part[warp] = v;
    __syncthreads();
    v = part[(warp & ~(warps - 1)) + (lane & (warps - 1))];
    for (int o = warps >> 1; o; o >>= 1) v += __shfl_xor_sync(kAllLanes, v, o);
    return v;
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(1024) cfa_norm_kernel(const cfa_norm_args a, int lanes)
{
    __shared__ float part[2][32];
    const int at = threadIdx.x & (lanes - 1);
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / lanes) + threadIdx.x / lanes;
    const bool here = row < a.tokens; /* every thread takes part in the sums */
    const int cols = (int)a.cols;
    const bool f32 = a.weight_dtype == CFA_DTYPE_F32;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
    const T *g = static_cast<const T *>(a.gate) + row * a.gate_stride;
    constexpr bool early = NV * VEC <= kEarly;
    launch_in_turn();

    Pack<T, VEC> px[NV], pr[NV], pg[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + at) * VEC;
        if (here && c < cols) px[i] = load_pack<T, VEC>(x + c);
    }
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * lanes + at) * VEC;
            if (here && c < cols) pr[i] = load_pack<T, VEC>(r + c);
        }
    }
    if (a.gate && early) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * lanes + at) * VEC;
            if (here && c < cols) pg[i] = load_pack<T, VEC>(g + c);
        }
    }
    float h[NV][VEC], w[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + at) * VEC;
        if (here && c < cols) {
            if (early) load_weight<T, VEC>(a.weight, f32, c, w[i]);
#pragma unroll
            for (int k = 0; k < VEC; ++k) h[i][k] = to_f32(px[i].v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k) h[i][k] = 0.0f;
        }
    }
    if (a.post_weight) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < VEC; ++k) sum += h[i][k] * h[i][k];
        const float unit = 1.0f / sqrtf(row_sum(sum, lanes, part[0]) / (float)cols + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * lanes + at) * VEC;
            if (here && c < cols) {
                float p[VEC];
                load_weight<T, VEC>(a.post_weight, f32, c, p);
#pragma unroll
                for (int k = 0; k < VEC; ++k) h[i][k] = h[i][k] * unit * (a.offset + p[k]);
            }
        }
    }
    if (a.gate) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * lanes + at) * VEC;
            if (here && c < cols) {
                if (!early) pg[i] = load_pack<T, VEC>(g + c);
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    h[i][k] = gated(h[i][k], to_f32(pg[i].v[k]), a.activation);
            }
        }
    }
    float sum = 0.0f;
    T *out = static_cast<T *>(a.h) + row * a.h_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + at) * VEC;
        if (here && c < cols) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                h[i][k] *= a.scale;
                if (a.residual) h[i][k] += to_f32(pr[i].v[k]);
            }
            if (a.h) store_pack<T, VEC>(out + c, h[i]);
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k) sum += h[i][k] * h[i][k];
    }
    const float unit = 1.0f / sqrtf(row_sum(sum, lanes, part[1]) / (float)cols + a.eps);
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + at) * VEC;
        if (here && c < cols) {
            if (!early) load_weight<T, VEC>(a.weight, f32, c, w[i]);
#pragma unroll
            for (int k = 0; k < VEC; ++k) h[i][k] = h[i][k] * unit * (a.offset + w[i][k]);
            store_pack<T, VEC>(y + c, h[i]);
        }
    }
}

template <typename T, int VEC, int NV>
cudaError_t launch(const cfa_norm_args &a, int lanes, cudaStream_t stream)
{
    const int threads = lanes > kBlock ? lanes : kBlock, rows = threads / lanes;
    cfa_launch_ctl ctl = {};
    ctl.flags = CFA_LAUNCH_EARLY;
    void *p[] = {const_cast<cfa_norm_args *>(&a), &lanes};
    return launch_ctl(reinterpret_cast<const void *>(&cfa_norm_kernel<T, VEC, NV>),
                      (unsigned)((a.tokens + rows - 1) / rows), threads, 0, stream, ctl, p);
}

template <typename T, int VEC> cudaError_t pick(const cfa_norm_args &a, cudaStream_t stream)
{
    const int64_t pieces = (a.cols + VEC - 1) / VEC;
    int lanes = 8;
    while (lanes < 1024 && lanes < pieces) lanes *= 2;
    if (lanes >= pieces) return launch<T, VEC, 1>(a, lanes, stream);
    if (2 * lanes >= pieces) return launch<T, VEC, 2>(a, lanes, stream);
    if constexpr (VEC <= 4)
        if (4 * lanes >= pieces) return launch<T, VEC, 4>(a, lanes, stream);
    if constexpr (VEC == 1)
        if (16 * lanes >= pieces) return launch<T, VEC, 16>(a, lanes, stream);
    return cudaErrorInvalidValue; /* rows of more than CFA_NORM_MAX_COLS are refused */
}

template <typename T> cudaError_t pick(const cfa_norm_args &a, cudaStream_t stream)
{
    constexpr int kVec = 16 / sizeof(T);
    uint64_t grid = (uint64_t)(uintptr_t)a.x | (uintptr_t)a.residual | (uintptr_t)a.gate |
                    (uintptr_t)a.weight | (uintptr_t)a.post_weight | (uintptr_t)a.y | (uintptr_t)a.h |
                    (uint64_t)a.cols * sizeof(T) | (uint64_t)a.gate_stride * sizeof(T);
    if (a.tokens > 1)
        grid |= (uint64_t)(a.x_stride | a.residual_stride | a.y_stride | a.h_stride) * sizeof(T);
    if ((grid & 15) == 0) return pick<T, kVec>(a, stream);
    return pick<T, 1>(a, stream);
}

} // namespace

cudaError_t cfa_launch_norm(const cfa_norm_args *a, cudaStream_t stream)
{
    if (a->dtype == CFA_DTYPE_F32) return pick<float>(*a, stream);
    if (a->dtype == CFA_DTYPE_F16) return pick<__half>(*a, stream);
    return pick<__nv_bfloat16>(*a, stream);
}
