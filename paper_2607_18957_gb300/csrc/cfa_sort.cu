/*
 * Tokens by expert: a stable counting sort of the (token, choice) pairs by the expert that each
 * names, with the copy of the tokens' rows into that order, and the weighted sum of the products'
 * rows back in the tokens' order.  The order is fixed (by expert, then by pair), so nothing depends on
 * which block runs first.
 */
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cfa_device.cuh"
#include "cfa_ops.h"

namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;
constexpr int kThreads = 256;
constexpr int64_t kOnePass = 16384;   /* pairs that every block of the sort counts for itself */
constexpr int64_t kBlockPairs = 1024; /* pairs per count, at least, where there are more */
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

/* hist[b][e]: pairs of the b-th block of block_pairs that name expert e. */
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

struct PlaceArgs {
    cfa_sort s;
    const void *x;
    void *xs;
    int64_t x_stride, hidden;
    int32_t chunk;   /* pairs per block, at most kThreads */
    int32_t blocks;  /* of hist; 0: count here */
    int32_t vec;     /* rows can be copied 16 bytes at a time */
};

/* Adds pairs [p0, p1) to n, expert by expert. */
__device__ __forceinline__ void count(const cfa_sort &s, int64_t p0, int64_t p1, int32_t *n)
{
    for (int64_t p = p0 + threadIdx.x; p < p1; p += kThreads) {
        const int e = expert_of(s, p);
        if (e >= 0) atomicAdd(n + e, 1);
    }
}

/* Each block places its chunk of pairs and copies their tokens' rows of x there.  It counts for itself
 * where its rows begin: after all pairs of lower experts and those of the same expert before the
 * chunk.  (Up to 16,384 pairs that costs each block less than a launch that counts them once.) */
__global__ void __launch_bounds__(kThreads) cfa_place_kernel(const PlaceArgs a)
{
    extern __shared__ int32_t smem[];
    const cfa_sort &s = a.s;
    int32_t *before = smem, *rest = smem + s.experts; /* pairs before the chunk, all others */
    __shared__ int32_t warp_sum[kThreads / 32];
    __shared__ int32_t row_of[kThreads];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int e = tid; e < s.experts; e += kThreads) before[e] = rest[e] = 0;
    __syncthreads();
    wait_before();
    release();
    const int64_t p0 = (int64_t)blockIdx.x * a.chunk;
    const int64_t p1 = p0 + a.chunk < s.pairs ? p0 + a.chunk : s.pairs;
    if (a.blocks == 0) {
        count(s, 0, p0, before);
        count(s, p0, s.pairs, rest);
    } else { /* a chunk lies inside one block of the count */
        const int64_t per = block_pairs(s.pairs), mine = p0 / per;
        for (int e = tid; e < s.experts; e += kThreads) {
            int32_t lower = 0, upper = 0;
#pragma unroll 8
            for (int b = 0; b < a.blocks; ++b) {
                const int32_t n = s.hist[(int64_t)b * s.experts + e];
                if (b < mine) lower += n;
                else upper += n;
            }
            before[e] = lower;
            rest[e] = upper;
        }
        __syncthreads();
        /* what precedes the chunk in its own block moves over */
        for (int64_t p = mine * per + tid; p < p0; p += kThreads) {
            const int e = expert_of(s, p);
            if (e < 0) continue;
            atomicAdd(before + e, 1);
            atomicSub(rest + e, 1);
        }
    }
    __syncthreads();
    /* exclusive sum of the totals over the experts, kThreads at a time, onto before */
    int32_t carry = 0;
    for (int e0 = 0; e0 < s.experts; e0 += kThreads) {
        const int e = e0 + tid;
        const int32_t n = e < s.experts ? before[e] + rest[e] : 0;
        int32_t x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t y = __shfl_up_sync(kAll, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        int32_t lower = carry, all = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) lower += warp_sum[w];
            all += warp_sum[w];
        }
        if (e < s.experts) {
            before[e] += lower + x - n;
            if (blockIdx.x == 0) s.offs[e] = lower + x - n;
        }
        carry += all;
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) s.offs[s.experts] = carry;
    /* the chunk's pairs in order, one warp after another */
    const int64_t p = p0 + tid;
    const int e = p < p1 ? expert_of(s, p) : -1;
    const uint32_t same = __match_any_sync(kAll, e);
    const int rank = __popc(same & ((1u << lane) - 1u));
    int32_t row = -1;
    for (int w = 0; w * 32 < a.chunk; ++w) {
        if (w == warp && e >= 0) row = before[e] + rank;
        __syncwarp();
        if (w == warp && e >= 0 && rank == 0) before[e] += __popc(same);
        __syncthreads();
    }
    if (p < p1) s.place[p] = row;
    row_of[tid] = row;
    __syncthreads();
    /* their rows, a warp each */
    for (int64_t i = warp; i < p1 - p0; i += kThreads / 32) {
        const int64_t r = row_of[i];
        if (r < 0) continue;
        const uint16_t *from = static_cast<const uint16_t *>(a.x) + (p0 + i) / s.top_k * a.x_stride;
        uint16_t *to = static_cast<uint16_t *>(a.xs) + r * a.hidden;
        if (a.vec) {
            const uint4 *f = reinterpret_cast<const uint4 *>(from);
            uint4 *o = reinterpret_cast<uint4 *>(to);
            const int64_t n = a.hidden / 8;
            int64_t h = lane;
            for (; h + 96 < n; h += 128) {
                const uint4 v0 = f[h], v1 = f[h + 32], v2 = f[h + 64], v3 = f[h + 96];
                o[h] = v0;
                o[h + 32] = v1;
                o[h + 64] = v2;
                o[h + 96] = v3;
            }
            for (; h < n; h += 32) o[h] = f[h];
        } else {
            for (int64_t h = lane; h < a.hidden; h += 32) to[h] = from[h];
        }
    }
}

__device__ __forceinline__ float half_at(const void *p, int64_t i, int f16)
{
    return f16 ? __half2float(static_cast<const __half *>(p)[i])
               : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

/* Sum over the choices of a token, in their order and in fp32: N columns from h on. */
template <int N>
__device__ __forceinline__ void add_choices(const cfa_combine &c, int64_t t, int64_t h, float *sum)
{
#pragma unroll 4
    for (int j = 0; j < c.top_k; ++j) {
        const int64_t row = c.place[t * c.top_k + j];
        if (row < 0) continue;
        const float w = c.weights[t * c.top_k + j];
        const float *from = c.part + row * c.hidden + h;
        if constexpr (N == 8) {
            const float4 a = *reinterpret_cast<const float4 *>(from);
            const float4 b = *reinterpret_cast<const float4 *>(from + 4);
            sum[0] += w * a.x;
            sum[1] += w * a.y;
            sum[2] += w * a.z;
            sum[3] += w * a.w;
            sum[4] += w * b.x;
            sum[5] += w * b.y;
            sum[6] += w * b.z;
            sum[7] += w * b.w;
        } else {
            sum[0] += w * *from;
        }
    }
}

/* A thread takes eight columns of one token, or one where y or the residual is off the 16-byte grid. */
template <int N>
__global__ void __launch_bounds__(kThreads) cfa_combine_kernel(const cfa_combine c)
{
    wait_before();
    const int64_t per = c.hidden / N, i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= c.tokens * per) return;
    const int64_t t = i / per, h = (i - t * per) * N;
    float sum[N] = {};
    add_choices<N>(c, t, h, sum);
    const int64_t at = t * c.y_stride + h, from = t * c.r_stride + h;
    if constexpr (N == 8) {
        if (c.residual) {
            const uint4 r = *reinterpret_cast<const uint4 *>(
                static_cast<const uint16_t *>(c.residual) + from);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += half_at(&r, k, c.f16);
        }
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c.f16) {
                const __half2 v = __floats2half2_rn(sum[2 * k], sum[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t *>(&v);
            } else {
                const __nv_bfloat162 v = __floats2bfloat162_rn(sum[2 * k], sum[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t *>(&v);
            }
        }
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(c.y) + at) =
            make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        float v = sum[0];
        if (c.residual) v += half_at(c.residual, from, c.f16);
        if (c.f16) static_cast<__half *>(c.y)[at] = __float2half_rn(v);
        else static_cast<__nv_bfloat16 *>(c.y)[at] = __float2bfloat16_rn(v);
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
    if (pairs <= kOnePass) return 0;
    const int64_t per = block_pairs(pairs);
    return (pairs + per - 1) / per;
}

cudaError_t cfa_launch_sort(const cfa_sort *s, const void *x, int64_t x_stride, int64_t hidden,
                            void *xs, cudaStream_t stream)
{
    const size_t smem = sizeof(int32_t) * s->experts;
    PlaceArgs a = {*s, x, xs, x_stride, hidden, 0, (int32_t)cfa_sort_blocks(s->pairs), 0};
    /* chunks of a power of two, so that they do not straddle blocks: about two per SM */
    for (a.chunk = 1; a.chunk < kThreads && s->pairs > (int64_t)a.chunk * 512; a.chunk *= 2) {
    }
    a.vec = (((uintptr_t)x | (uintptr_t)xs | (uint64_t)x_stride * 2 | (uint64_t)hidden * 2) & 15u) ==
            0;
    cudaError_t e = cudaSuccess;
    if (a.blocks) e = launch(cfa_count_kernel, dim3((unsigned)a.blocks), smem, stream, *s);
    const unsigned grid = (unsigned)((s->pairs + a.chunk - 1) / a.chunk);
    return e ? e : launch(cfa_place_kernel, dim3(grid), 2 * smem, stream, a);
}

cudaError_t cfa_launch_combine(const cfa_combine *c, cudaStream_t stream)
{
    const bool wide = (((uintptr_t)c->y | (uintptr_t)c->residual | (uint64_t)c->y_stride * 2 |
                        (c->residual ? (uint64_t)c->r_stride * 2 : 0)) & 15u) == 0;
    const int64_t threads = c->tokens * (c->hidden / (wide ? 8 : 1));
    const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads));
    return wide ? launch(cfa_combine_kernel<8>, grid, 0, stream, *c)
                : launch(cfa_combine_kernel<1>, grid, 0, stream, *c);
}

cudaError_t cfa_launch_realign(const void *from, int64_t from_stride, int64_t rows, int64_t cols,
                               void *to, int64_t to_stride, cudaStream_t stream)
{
    const RealignArgs a = {static_cast<const uint16_t *>(from), static_cast<uint16_t *>(to),
                           from_stride, to_stride, rows, cols};
    return launch(cfa_realign_kernel, dim3((unsigned)(rows < 4864 ? rows : 4864)), 0, stream, a);
}
