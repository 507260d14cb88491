/*
 * y = act(x w^T + bias) + residual, for one weight or for a stack of them (cfa_matmul).
 *
 * The simplest form: a block owns 64 rows of x and 64 columns of y (of each half when gated),
 * stages 16 columns of x and w at a time in shared memory as fp32 and multiplies in fp32 registers.
 */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cfa_device.cuh"
#include "cfa_ops.h"

namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;

__device__ __forceinline__ float value(const void *p, int64_t i, int f16)
{
    return f16 ? __half2float(static_cast<const __half *>(p)[i])
               : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ float activate(float v, int act)
{
    switch (act) {
    case CFA_ACT_RELU: return v > 0.0f ? v : 0.0f;
    case CFA_ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
    case CFA_ACT_GELU_TANH:
        return 0.5f * v * (1.0f + tanhf(0.79788456080286536f * (v + 0.044715f * v * v * v)));
    case CFA_ACT_SILU: return v / (1.0f + expf(-v));
    default: return v;
    }
}

struct Args {
    cfa_matmul m;
};

__global__ void __launch_bounds__(kThreads) cfa_matmul_kernel(const Args args)
{
    const cfa_matmul &m = args.m;
    __shared__ float xs[kDepth][kTile + 1], ws[2][kDepth][kTile + 1];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int g = blockIdx.z;
    const int64_t begin = m.offs ? m.offs[g] : 0, end = m.offs ? m.offs[g + 1] : m.tokens;
    const int64_t t0 = begin + (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
    if (t0 >= end) return;
    const int64_t outs = m.gated ? m.w_rows / 2 : m.w_rows;
    const int64_t w0 = g * m.w_rows;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[2][4][4] = {};
    for (int64_t k0 = 0; k0 < m.cols; k0 += kDepth) {
        for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
            const int r = i / kDepth, c = i % kDepth;
            const int64_t k = k0 + c;
            const bool in = k < m.cols;
            xs[c][r] = in && t0 + r < end ? value(m.x, (t0 + r) * m.x_stride + k, m.f16) : 0.0f;
            const bool row = in && n0 + r < outs;
            ws[0][c][r] = row ? value(m.w, (w0 + n0 + r) * m.w_stride + k, m.f16) : 0.0f;
            if (m.gated)
                ws[1][c][r] =
                    row ? value(m.w, (w0 + outs + n0 + r) * m.w_stride + k, m.f16) : 0.0f;
        }
        __syncthreads();
        for (int c = 0; c < kDepth; ++c)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) {
                    acc[0][i][j] += xs[c][ty + 16 * i] * ws[0][c][tx + 16 * j];
                    if (m.gated) acc[1][i][j] += xs[c][ty + 16 * i] * ws[1][c][tx + 16 * j];
                }
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t t = t0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (t >= end || n >= outs) continue;
            float v = acc[0][i][j], u = acc[1][i][j];
            if (m.bias) {
                v += m.bias_f32 ? static_cast<const float *>(m.bias)[n] : value(m.bias, n, m.f16);
                if (m.gated)
                    u += m.bias_f32 ? static_cast<const float *>(m.bias)[outs + n]
                                    : value(m.bias, outs + n, m.f16);
            }
            v = activate(v, m.act);
            if (m.gated) v *= u;
            if (m.residual) {
                const int64_t at = t * m.r_stride + n;
                v += m.y_f32 ? static_cast<const float *>(m.residual)[at]
                             : value(m.residual, at, m.f16);
            }
            const int64_t at = t * m.y_stride + n;
            if (m.y_f32) static_cast<float *>(m.y)[at] = v;
            else if (m.f16) static_cast<__half *>(m.y)[at] = __float2half_rn(v);
            else static_cast<__nv_bfloat16 *>(m.y)[at] = __float2bfloat16_rn(v);
        }
}

} // namespace

cudaError_t cfa_launch_matmul(const cfa_matmul *m, int early, int release, cudaStream_t stream)
{
    (void)release;
    const int64_t outs = m->gated ? m->w_rows / 2 : m->w_rows;
    const dim3 grid((unsigned)((outs + kTile - 1) / kTile),
                    (unsigned)((m->tokens + kTile - 1) / kTile), (unsigned)m->n_groups);
    Args a = {*m};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = early ? 1 : 0;
    void *p[] = {&a};
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(&cfa_matmul_kernel), p);
}
