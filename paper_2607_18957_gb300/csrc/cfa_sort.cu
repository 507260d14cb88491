/*
 * Tokens by expert: a stable counting sort of the (token, choice) pairs by the expert that each
 * names, with the copy of the tokens' rows into that order, and the weighted sum of the products'
 * rows back in the tokens' order.  The order is fixed (by expert, then by pair), so nothing depends on
 * which block runs first.  (The atomics only count.)
 *
 * With few pairs both are bound by their launch and by a chain of dependent loads: 3 us for the sort of
 * 48 pairs with rows of 5 KiB, 1.2 us for the sum of 16 tokens after its launch.  With many, by the
 * rows: 8192 rows of 8 KiB are placed in 20 us (100 MB, three quarters of what memory gives) and their
 * products summed in 45 (168 MB, half), beside 1.6 ms of products.
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

/* All loads of what other kernels write go past L1, which may hold what an older one read there. */
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
    const int64_t e = (int64_t)__ldcg(s.ids + p) - s.first;
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
    int64_t p = p0 + threadIdx.x;
    for (; p + 7 * kThreads < p1; p += 8 * kThreads) { /* eight loads under way at once */
        int e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = expert_of(s, p + i * kThreads);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (e[i] >= 0) atomicAdd(n + e[i], 1);
    }
    for (; p < p1; p += kThreads) {
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
                const int32_t n = __ldcg(s.hist + (int64_t)b * s.experts + e);
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
            for (; h + 7 * 32 < n; h += 8 * 32) {
                uint4 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = __ldcg(f + h + u * 32);
#pragma unroll
                for (int u = 0; u < 8; ++u) o[h + u * 32] = v[u];
            }
            for (; h < n; h += 32) o[h] = __ldcg(f + h);
        } else {
            for (int64_t h = lane; h < a.hidden; h += 32) to[h] = __ldcg(from + h);
        }
    }
}

__device__ __forceinline__ float half_of(unsigned short b, int f16)
{
    return f16 ? __half2float(__ushort_as_half(b)) : __bfloat162float(__ushort_as_bfloat16(b));
}

/* The rows and weights of up to kAhead choices of the token that piece i of `per` belongs to. */
constexpr int kAhead = 4;
struct Choices {
    int32_t row[kAhead];
    float w[kAhead];
    int64_t t, h;
};

template <int N>
__device__ __forceinline__ void choose(const cfa_combine &c, int64_t i, int64_t per, Choices &o)
{
    const bool in = i < c.tokens * per;
    o.t = in ? i / per : 0;
    o.h = in ? (i - o.t * per) * N : 0;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        o.row[j] = in && j < c.top_k ? __ldcg(c.place + o.t * c.top_k + j) : -1;
        o.w[j] = in && j < c.top_k ? __ldcg(c.weights + o.t * c.top_k + j) : 0.0f;
    }
}

template <int N>
__device__ __forceinline__ void add_row(const cfa_combine &c, int64_t row, int64_t h, float w,
                                        float (&sum)[N])
{
    if constexpr (N == 8) {
        const float4 *p = reinterpret_cast<const float4 *>(c.part + row * c.hidden + h);
        const float4 a = __ldcg(p), b = __ldcg(p + 1);
        sum[0] += w * a.x;
        sum[1] += w * a.y;
        sum[2] += w * a.z;
        sum[3] += w * a.w;
        sum[4] += w * b.x;
        sum[5] += w * b.y;
        sum[6] += w * b.z;
        sum[7] += w * b.w;
    } else {
        sum[0] += w * __ldcg(c.part + row * c.hidden + h);
    }
}

/* A thread takes eight columns of one token at a time, or one where y or the residual is off the 16-byte
 * grid, and adds the token's choices in their order, in fp32.  Where their rows lie and their weights it
 * reads a round ahead, and for the first before the launch's wait: both are there since the launch
 * before last.  (One piece per thread, in as many blocks as there are pieces, took twice as long on
 * 4096 tokens: every block waited for the two loads one after the other.) */
template <int N>
__global__ void __launch_bounds__(kThreads, 4) cfa_combine_kernel(const cfa_combine c)
{
    const int64_t per = c.hidden / N, all = c.tokens * per, step = (int64_t)gridDim.x * kThreads;
    int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    Choices now;
    choose<N>(c, i, per, now);
    wait_before();
    for (; i < all; i += step) {
        float sum[N] = {};
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (now.row[j] >= 0) add_row<N>(c, now.row[j], now.h, now.w[j], sum);
        const int64_t t = now.t, h = now.h;
        choose<N>(c, i + step, per, now);
        for (int j = kAhead; j < c.top_k; ++j) {
            const int64_t row = __ldcg(c.place + t * c.top_k + j);
            if (row >= 0) add_row<N>(c, row, h, __ldcg(c.weights + t * c.top_k + j), sum);
        }
        const int64_t at = t * c.y_stride + h, from = t * c.r_stride + h;
        if constexpr (N == 8) {
            if (c.residual) {
                const uint4 v = __ldcg(reinterpret_cast<const uint4 *>(
                    static_cast<const uint16_t *>(c.residual) + from));
                const unsigned short *b = reinterpret_cast<const unsigned short *>(&v);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += half_of(b[k], c.f16);
            }
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c.f16) {
                    const __half2 v = __floats2half2_rn(sum[2 * k], sum[2 * k + 1]);
                    o[k] = *reinterpret_cast<const uint32_t *>(&v);
                } else {
                    const __nv_bfloat162 v = __floats2bfloat162_rn(sum[2 * k], sum[2 * k + 1]);
                    o[k] = *reinterpret_cast<const uint32_t *>(&v);
                }
            }
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(c.y) + at) =
                make_uint4(o[0], o[1], o[2], o[3]);
        } else {
            if (c.residual)
                sum[0] += half_of(__ldcg(static_cast<const unsigned short *>(c.residual) + from),
                                  c.f16);
            if (c.f16) static_cast<__half *>(c.y)[at] = __float2half_rn(sum[0]);
            else static_cast<__nv_bfloat16 *>(c.y)[at] = __float2bfloat16_rn(sum[0]);
        }
    }
}

struct RealignMatrix {
    const uint16_t *from;
    uint16_t *to;
    int64_t from_stride, to_stride, rows, cols;
};
struct RealignArgs {
    RealignMatrix m[3];
};

/* 16 bytes that start `phase` bytes (an even number) into the 32 of a and b. */
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, uint32_t phase)
{
    const bool half = phase & 2u;
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (phase & 8u) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (phase & 4u) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (half) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

/* Rows onto the 16-byte grid, zeros behind the last column.  A warp takes 128 granules of a row at a
 * time, so that few long rows keep as many warps busy as many short ones: every lane loads the aligned
 * 16 bytes that its result starts in and has the next lane's for the rest.  Granules that are
 * not wholly inside the matrix go element by element. */
__global__ void __launch_bounds__(kThreads) cfa_realign_kernel(const RealignArgs all)
{
    wait_before();
    release();
    const RealignMatrix a = all.m[blockIdx.y];
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (kThreads / 32);
    const uintptr_t begin = (uintptr_t)a.from;
    const uintptr_t end = begin + 2 * ((a.rows - 1) * a.from_stride + a.cols);
    const auto granule = [&](uintptr_t at) {
        if (at >= begin && at + 16 <= end) return __ldcg(reinterpret_cast<const uint4 *>(at));
        uint32_t w[4] = {};
        for (int i = 0; i < 8; ++i) {
            const uintptr_t p = at + 2 * i;
            if (p >= begin && p + 2 <= end)
                w[i >> 1] |= (uint32_t)__ldcg(reinterpret_cast<const unsigned short *>(p))
                             << (16 * (i & 1));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    };
    const int64_t n = a.to_stride / 8, chunks = (n + 127) / 128;
    for (int64_t i = blockIdx.x * (int64_t)(kThreads / 32) + (threadIdx.x >> 5); i < a.rows * chunks;
         i += warps) {
        const int64_t r = i / chunks, c0 = (i - r * chunks) * 128;
        const uintptr_t row = (uintptr_t)(a.from + r * a.from_stride);
        const uint32_t phase = (uint32_t)(row & 15u);
        uint4 *to = reinterpret_cast<uint4 *>(a.to + r * a.to_stride);
        uint4 g[5];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t c = c0 + u * 32 + lane;
            g[u] = c < n ? granule(row - phase + 16 * c) : make_uint4(0, 0, 0, 0);
        }
        g[4] = make_uint4(0, 0, 0, 0);
        if (phase && lane == 0 && c0 + 128 < n + 1) g[4] = granule(row - phase + 16 * (c0 + 128));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t c = c0 + u * 32 + lane;
            uint4 v = g[u];
            if (phase) { /* the same for the whole warp */
                /* the granule behind the lane's: the next lane's, or lane 0's of the next round */
                const uint4 mine = lane == 0 ? g[u + 1] : g[u];
                uint4 next;
                next.x = __shfl_sync(kAll, mine.x, (lane + 1) & 31);
                next.y = __shfl_sync(kAll, mine.y, (lane + 1) & 31);
                next.z = __shfl_sync(kAll, mine.z, (lane + 1) & 31);
                next.w = __shfl_sync(kAll, mine.w, (lane + 1) & 31);
                if (c == n - 1) next = granule(row - phase + 16 * (c + 1));
                v = shifted(v, next, phase);
            }
            if (c >= n) continue;
            const int64_t left = a.cols - c * 8;
            if (left < 8) { /* zeros behind the last column */
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= left) w[i >> 1] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                v = make_uint4(w[0], w[1], w[2], w[3]);
            }
            to[c] = v;
        }
    }
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
    /* chunks of a power of two, so that they do not straddle blocks: two to four per SM, so that
     * enough rows are under way */
    for (a.chunk = 1; a.chunk < kThreads && s->pairs > (int64_t)a.chunk * 608; a.chunk *= 2) {
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
    const int64_t blocks = (c->tokens * (c->hidden / (wide ? 8 : 1)) + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)(blocks < 608 ? blocks : 608)); /* four per SM */
    return wide ? launch(cfa_combine_kernel<8>, grid, 0, stream, *c)
                : launch(cfa_combine_kernel<1>, grid, 0, stream, *c);
}

cudaError_t cfa_launch_realign(const cfa_rows *m, int n, cudaStream_t stream)
{
    RealignArgs a = {};
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        a.m[i] = {static_cast<const uint16_t *>(m[i].from), static_cast<uint16_t *>(m[i].to),
                  m[i].from_stride, m[i].to_stride, m[i].rows, m[i].cols};
        const int64_t pieces = m[i].rows * ((m[i].to_stride / 8 + 127) / 128);
        if (pieces > most) most = pieces;
    }
    const int64_t blocks = (most + kThreads / 32 - 1) / (kThreads / 32);
    return launch(cfa_realign_kernel, dim3((unsigned)(blocks < 1216 ? blocks : 1216), (unsigned)n),
                  0, stream, a);
}
