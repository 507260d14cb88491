/*
 * Tokens by expert: a stable counting sort of the (token, choice) pairs by the expert that each
 * names, the copy of the tokens' rows into that order, and the weighted sum of the products' rows
 * back into the tokens' order.  The order is fixed (by expert, then by pair), so nothing depends on
 * which block runs first.
 */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cfa_device.cuh"
#include "cfa_ops.h"

namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr int kThreads = 256;
constexpr int64_t kBlockPairs = 1024; /* pairs per block of the sort, at least */
constexpr int64_t kMostBlocks = 128;

__device__ __forceinline__ void wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void release()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__host__ __device__ inline int64_t block_pairs(int64_t pairs)
{
    const int64_t per = (pairs + kMostBlocks - 1) / kMostBlocks;
    return per > kBlockPairs ? (per + kThreads - 1) / kThreads * kThreads : kBlockPairs;
}

__device__ __forceinline__ int expert_of(const cfa_sort &s, int64_t p)
{
    const int64_t e = (int64_t)s.ids[p] - s.first;
    return e >= 0 && e < s.experts ? (int)e : -1;
}

/* hist[b][e]: pairs of block b that name expert e. */
__global__ void __launch_bounds__(kThreads) cfa_count_kernel(const cfa_sort s)
{
    extern __shared__ int32_t n[];
    for (int e = threadIdx.x; e < s.experts; e += kThreads) n[e] = 0;
    __syncthreads();
    wait_before();
    release();
    const int64_t per = block_pairs(s.pairs), p0 = blockIdx.x * per;
    const int64_t p1 = p0 + per < s.pairs ? p0 + per : s.pairs;
    for (int64_t p = p0 + threadIdx.x; p < p1; p += kThreads) {
        const int e = expert_of(s, p);
        if (e >= 0) atomicAdd(n + e, 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < s.experts; e += kThreads)
        s.hist[(int64_t)blockIdx.x * s.experts + e] = n[e];
}

/* Every block counts for itself where its rows begin: all pairs of lower experts, and those of the
 * same expert in the blocks before. */
__global__ void __launch_bounds__(kThreads) cfa_place_kernel(const cfa_sort s)
{
    extern __shared__ int32_t smem[];
    int32_t *total = smem, *next = smem + s.experts; /* next: row of the expert's next pair */
    __shared__ int32_t warp_sum[kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int blocks = (int)gridDim.x;
    for (int e = tid; e < s.experts; e += kThreads) total[e] = next[e] = 0;
    __syncthreads();
    wait_before();
    release();
    const int64_t per = block_pairs(s.pairs), p0 = blockIdx.x * per;
    const int64_t p1 = p0 + per < s.pairs ? p0 + per : s.pairs;
    if (blocks == 1) {
        for (int64_t p = tid; p < s.pairs; p += kThreads) {
            const int e = expert_of(s, p);
            if (e >= 0) atomicAdd(total + e, 1);
        }
    } else {
        for (int e = tid; e < s.experts; e += kThreads) {
            int32_t all = 0, before = 0;
            for (int b = 0; b < blocks; ++b) {
                const int32_t n = s.hist[(int64_t)b * s.experts + e];
                all += n;
                if (b < (int)blockIdx.x) before += n;
            }
            total[e] = all;
            next[e] = before;
        }
    }
    __syncthreads();
    /* exclusive sum of the totals over the experts, kThreads at a time */
    int32_t carry = 0;
    for (int e0 = 0; e0 < s.experts; e0 += kThreads) {
        const int e = e0 + tid;
        const int32_t n = e < s.experts ? total[e] : 0;
        int32_t x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t y = __shfl_up_sync(kAll, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        int32_t before = carry, all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += warp_sum[w];
            all += warp_sum[w];
        }
        if (e < s.experts) {
            next[e] += before + x - n;
            if (blockIdx.x == 0) s.offs[e] = before + x - n;
        }
        carry += all;
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) s.offs[s.experts] = carry;
    /* the pairs in order, one warp after another */
    for (int64_t q = p0; q < p1; q += kThreads) {
        const int64_t p = q + tid;
        const int e = p < p1 ? expert_of(s, p) : -1;
        const uint32_t same = __match_any_sync(kAll, e);
        const int rank = __popc(same & ((1u << lane) - 1u));
        int32_t row = -1;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp && e >= 0) row = next[e] + rank;
            __syncwarp();
            if (w == warp && e >= 0 && rank == 0) next[e] += __popc(same);
            if (q + w * 32 >= p1) break;
            __syncthreads();
        }
        __syncthreads();
        if (p < p1) {
            s.place[p] = row;
            if (row >= 0) s.token[row] = (int32_t)(p / s.top_k);
        }
    }
}

struct GatherArgs {
    const void *x;
    void *xs;
    const int32_t *token, *rows;
    int64_t x_stride, xs_stride, hidden;
    int vec; /* 16 bytes at a time */
};

/* One block a row, rows in turn. */
__global__ void __launch_bounds__(kThreads) cfa_gather_kernel(const GatherArgs g)
{
    wait_before();
    release();
    const int64_t rows = *g.rows;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const uint16_t *from = static_cast<const uint16_t *>(g.x) + g.token[r] * g.x_stride;
        uint16_t *to = static_cast<uint16_t *>(g.xs) + r * g.xs_stride;
        if (g.vec)
            for (int64_t i = threadIdx.x; i < g.hidden / 8; i += kThreads)
                reinterpret_cast<uint4 *>(to)[i] = reinterpret_cast<const uint4 *>(from)[i];
        else
            for (int64_t i = threadIdx.x; i < g.hidden; i += kThreads) to[i] = from[i];
    }
}

/* One block a token and kThreads columns; the choices are added in their order, in fp32. */
__global__ void __launch_bounds__(kThreads) cfa_combine_kernel(const cfa_combine c)
{
    wait_before();
    const int64_t t = blockIdx.x;
    for (int64_t h = threadIdx.x + (int64_t)blockIdx.y * kThreads; h < c.hidden;
         h += (int64_t)gridDim.y * kThreads) {
        float sum = 0.0f;
        for (int j = 0; j < c.top_k; ++j) {
            const int32_t row = c.place[t * c.top_k + j];
            if (row >= 0) sum += c.weights[t * c.top_k + j] * c.part[row * c.hidden + h];
        }
        const int64_t at = t * c.y_stride + h;
        if (c.f16) {
            if (c.residual)
                sum += __half2float(static_cast<const __half *>(c.residual)[t * c.r_stride + h]);
            static_cast<__half *>(c.y)[at] = __float2half_rn(sum);
        } else {
            if (c.residual)
                sum += __bfloat162float(
                    static_cast<const __nv_bfloat16 *>(c.residual)[t * c.r_stride + h]);
            static_cast<__nv_bfloat16 *>(c.y)[at] = __float2bfloat16_rn(sum);
        }
    }
}

struct RealignArgs {
    const uint16_t *from;
    uint16_t *to;
    int64_t from_stride, to_stride, rows, cols;
};

__global__ void __launch_bounds__(kThreads) cfa_realign_kernel(const RealignArgs a)
{
    wait_before();
    release();
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x)
        for (int64_t i = threadIdx.x; i < a.to_stride; i += kThreads)
            a.to[r * a.to_stride + i] = i < a.cols ? a.from[r * a.from_stride + i] : (uint16_t)0;
}

template <typename Args>
cudaError_t launch(void (*fn)(const Args), dim3 grid, size_t smem, cudaStream_t stream,
                   const Args &args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    void *p[] = {const_cast<Args *>(&args)};
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(fn), p);
}

} // namespace

int64_t cfa_sort_blocks(int64_t pairs)
{
    const int64_t per = block_pairs(pairs);
    return (pairs + per - 1) / per;
}

cudaError_t cfa_launch_sort(const cfa_sort *s, cudaStream_t stream)
{
    const unsigned blocks = (unsigned)cfa_sort_blocks(s->pairs);
    const size_t smem = sizeof(int32_t) * s->experts;
    cudaError_t e = cudaSuccess;
    if (blocks > 1) e = launch(cfa_count_kernel, dim3(blocks), smem, stream, *s);
    return e ? e : launch(cfa_place_kernel, dim3(blocks), 2 * smem, stream, *s);
}

cudaError_t cfa_launch_gather(const void *x, int64_t x_stride, int64_t hidden, const int32_t *token,
                              const int32_t *rows, int64_t most, void *xs, int64_t xs_stride,
                              cudaStream_t stream)
{
    GatherArgs g = {x, xs, token, rows, x_stride, xs_stride, hidden, 0};
    g.vec = (((uintptr_t)x | (uintptr_t)xs | (uint64_t)x_stride * 2 | (uint64_t)xs_stride * 2 |
              (uint64_t)hidden * 2) & 15u) == 0;
    return launch(cfa_gather_kernel, dim3((unsigned)(most < 1216 ? most : 1216)), 0, stream, g);
}

cudaError_t cfa_launch_combine(const cfa_combine *c, cudaStream_t stream)
{
    const unsigned y = (unsigned)((c->hidden + kThreads - 1) / kThreads);
    return launch(cfa_combine_kernel, dim3((unsigned)c->tokens, y < 64 ? y : 64), 0, stream, *c);
}

cudaError_t cfa_launch_realign(const void *from, int64_t from_stride, int64_t rows, int64_t cols,
                               void *to, int64_t to_stride, cudaStream_t stream)
{
    const RealignArgs a = {static_cast<const uint16_t *>(from), static_cast<uint16_t *>(to),
                           from_stride, to_stride, rows, cols};
    return launch(cfa_realign_kernel, dim3((unsigned)(rows < 4864 ? rows : 4864)), 0, stream, a);
}
