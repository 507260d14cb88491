/*
 * Log probabilities of given tokens, entropy and the largest logits of each row, in one pass over it.
 *
 * With m the row's largest logit and d = v - m: s = sum exp(scale d), w = sum exp(scale d) d, so that
 * log p = scale d - log s and the entropy is log s - scale w / s.  Every thread keeps the three for its own
 * part of the row (a running m; s and w follow when it grows) and they are joined in a fixed order.
 *
 * The largest: the top-th largest of the threads' own maxima is a bound below which no wanted logit lies,
 * and only the parts of threads whose maximum reaches it, about as many as logits are wanted, are looked
 * through again, by whole warps.  A logit's key is its value mapped onto integers of the same order and
 * its complemented index, so that keys are unique and equal values go to the lowest index.
 *
 * A row belongs to one block or to a cluster of blocks, whose results meet in the first one's shared
 * memory.
 */
#include <cooperative_groups.h>

#include "cfa_ops.h"
#include "cfa_values.cuh"

using namespace cfa_dev;
namespace cg = cooperative_groups;

namespace {

constexpr int kMaxWarps = 16, kMaxCluster = 8;
constexpr int kAhead = 4; /* loads of 16 bytes that a thread has in flight */

__device__ __forceinline__ uint32_t order_of(float v)
{
    if (v != v) v = -INFINITY; /* a row with NaN has no numbers, but its ids are of the row */
    const uint32_t b = __float_as_uint(v == 0.0f ? 0.0f : v); /* -0 ties with 0 */
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t o)
{
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

__device__ __forceinline__ uint64_t key_of(float v, uint32_t index)
{
    return (uint64_t)order_of(v) << 32 | (uint32_t)~index;
}

__device__ __forceinline__ float exp2_fast(float v) /* off by 2^-22; below 2^-126 zero */
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

struct Sums {
    float m, s, w; /* w in units of d */
};

/* The sums of two parts together.  A part without a logit above -inf has s = w = 0, or NaN. */
__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    Sums r;
    r.m = fmaxf(a.m, b.m);
    r.s = r.w = 0.0f;
    const Sums part[2] = {a, b};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (part[i].m == -INFINITY) {
            r.s += part[i].s;
            r.w += part[i].s;
        } else {
            const float d = part[i].m - r.m, e = exp2_fast(d * c);
            r.s += part[i].s * e;
            r.w += (part[i].w + fmaxf(d, -1e30f) * part[i].s) * e;
        }
    }
    return r;
}

/* The warp's 32 keys in descending order over its lanes, if they go down and then up, or up and then
 * down. */
template <typename K> __device__ __forceinline__ K bitonic_merge(K v, int lane)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const K other = __shfl_xor_sync(kAllLanes, v, o);
        v = (lane & o) ? min(v, other) : max(v, other);
    }
    return v;
}

template <typename K> __device__ __forceinline__ K warp_sort(K v, int lane)
{
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
        for (int o = size >> 1; o; o >>= 1) {
            const K other = __shfl_xor_sync(kAllLanes, v, o);
            v = ((lane & o) == 0) == ((lane & size) == 0) ? max(v, other) : min(v, other);
        }
    }
    return v;
}

/* The 32 largest of `lists` (a power of two) descending lists, one per warp, in every lane of warp 0.
 * All of the block's threads call it; room: [warps][32]. */
template <typename K> __device__ __forceinline__ K merge_lists(K v, int lists, K *room, int warp, int lane)
{
    for (int n = lists >> 1; n; n >>= 1) {
        if (warp >= n && warp < 2 * n) room[warp * 32 + lane] = v;
        __syncthreads();
        if (warp < n) v = bitonic_merge(max(v, room[(warp + n) * 32 + 31 - lane]), lane);
    }
    return v;
}

/* Puts key c, the same in all lanes, into the warp's descending list. */
__device__ __forceinline__ uint64_t insert(uint64_t list, uint64_t c, int lane)
{
    const int at = __popc(__ballot_sync(kAllLanes, list > c));
    const uint64_t up = __shfl_up_sync(kAllLanes, list, 1);
    return lane < at ? list : lane == at ? c : up;
}

/* The lanes' candidates among `top` best ones of the warp so far. */
__device__ __forceinline__ uint64_t offer(uint64_t list, uint64_t c, int top, int lane)
{
    uint64_t least = __shfl_sync(kAllLanes, list, top - 1);
    uint32_t who = __ballot_sync(kAllLanes, c > least);
    while (who) {
        const int from = __ffs(who) - 1;
        list = insert(list, __shfl_sync(kAllLanes, c, from), lane);
        least = __shfl_sync(kAllLanes, list, top - 1);
        who = __ballot_sync(kAllLanes, lane > from && c > least) & ~((2u << from) - 1u);
    }
    return list;
}

template <typename T>
__global__ void __launch_bounds__(kMaxWarps * 32, 2)
    cfa_logprobs_kernel(const cfa_logprobs_args a, int blocks /* of a row */)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ uint64_t lists[kMaxWarps * 32];
    __shared__ uint32_t maxima[kMaxWarps * 32];
    __shared__ Sums sums[kMaxWarps];
    __shared__ uint64_t cluster_lists[kMaxCluster * 32];
    __shared__ Sums cluster_sums[kMaxCluster];
    __shared__ uint32_t s_bound;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int rank = blocks > 1 ? (int)(blockIdx.x % blocks) : 0;
    const int64_t row = blockIdx.x / blocks;
    const float c = a.scale * 1.4426950408889634f;
    const T *x = static_cast<const T *>(a.logits) + row * a.stride;
    if (blocks > 1) cg::this_cluster().barrier_arrive(); /* its shared memory is there: waited for below */
    launch_in_turn();

    /* the row: `head` single values up to the 16-byte grid, pieces of VEC, `tail` single values */
    const int cols = (int)a.cols;
    int head = (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T);
    if (head > cols) head = cols;
    const int pieces = (cols - head) / VEC, tail = cols - head - pieces * VEC;
    const int step = blocks * blockDim.x, g = rank * blockDim.x + threadIdx.x;
    const T *body = x + head;

    const bool last = rank == 0 && threadIdx.x == 0; /* writes the row's numbers */
    const int token = last ? __ldcg(a.tokens + row) : -1;
    Sums mine = {-INFINITY, 0.0f, 0.0f};
    /* the thread's single values, -inf where it has none */
    float single[2] = {-INFINITY, -INFINITY};
    if (g < head) single[0] = to_f32(load_pack<T, 1>(x + g).v[0]);
    if (g < tail) single[1] = to_f32(load_pack<T, 1>(x + cols - tail + g).v[0]);

    auto add = [&](const float *v, int n) {
        float top = v[0];
#pragma unroll
        for (int i = 1; i < n; ++i) top = fmaxf(top, v[i]);
        if (top > mine.m) {
            if (mine.m > -INFINITY) {
                const float d = mine.m - top, e = exp2_fast(d * c);
                mine.w = (mine.w + fmaxf(d, -1e30f) * mine.s) * e;
                mine.s *= e;
            }
            mine.m = top;
        }
        if (mine.m > -INFINITY) {
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float d = v[i] - mine.m, e = exp2_fast(d * c);
                mine.s += e;
                mine.w += e * fmaxf(d, -1e30f);
            }
        } else {
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (v[i] != v[i]) mine.s = mine.w = NAN;
        }
    };
    int p = g;
    for (; p + (kAhead - 1) * step < pieces; p += kAhead * step) {
        Pack<T, VEC> q[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) q[i] = load_pack<T, VEC>(body + (int64_t)(p + i * step) * VEC);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            float v[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) v[k] = to_f32(q[i].v[k]);
            add(v, VEC);
        }
    }
    for (; p < pieces; p += step) {
        const Pack<T, VEC> q = load_pack<T, VEC>(body + (int64_t)p * VEC);
        float v[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] = to_f32(q.v[k]);
        add(v, VEC);
    }
    add(single, 2);
    float given = -INFINITY;
    if (token >= 0 && token < cols) given = to_f32(load_pack<T, 1>(x + token).v[0]);

    uint64_t best = 0; /* lane i of warp 0, in the end: the i-th largest */
    if (a.top > 0) {
        const uint32_t most = order_of(mine.m);
        const uint32_t sorted = merge_lists(warp_sort(most, lane), warps, maxima, warp, lane);
        if (warp == 0 && lane == a.top - 1) s_bound = sorted;
        __syncthreads();
        const uint32_t bound = s_bound;
        uint32_t who = __ballot_sync(kAllLanes, most >= bound);
        while (who) { /* the part of one thread after another, with all lanes */
            const int from = __ffs(who) - 1;
            who &= who - 1;
            const int theirs = g - lane + from;
            for (int q0 = theirs; q0 < pieces; q0 += 32 * step) {
                const int64_t q = q0 + (int64_t)lane * step;
                const bool in = q < pieces;
                Pack<T, VEC> v;
                if (in) v = load_pack<T, VEC>(body + q * VEC);
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    uint64_t key = 0;
                    if (in) key = key_of(to_f32(v.v[k]), (uint32_t)(head + q * VEC + k));
                    if ((uint32_t)(key >> 32) < bound) key = 0;
                    best = offer(best, key, a.top, lane);
                }
            }
            const float s0 = __shfl_sync(kAllLanes, single[0], from);
            const float s1 = __shfl_sync(kAllLanes, single[1], from);
            uint64_t key = 0;
            if (lane == 0 && theirs < head) key = key_of(s0, (uint32_t)theirs);
            if (lane == 1 && theirs < tail) key = key_of(s1, (uint32_t)(cols - tail + theirs));
            best = offer(best, key, a.top, lane);
        }
        best = merge_lists(best, warps, lists, warp, lane);
    }

    for (int o = 16; o; o >>= 1) {
        Sums other;
        other.m = __shfl_xor_sync(kAllLanes, mine.m, o);
        other.s = __shfl_xor_sync(kAllLanes, mine.s, o);
        other.w = __shfl_xor_sync(kAllLanes, mine.w, o);
        mine = join(lane & o ? other : mine, lane & o ? mine : other, c);
    }
    if (lane == 0) sums[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        mine = sums[0];
        for (int i = 1; i < warps; ++i) mine = join(mine, sums[i], c);
    }
    if (blocks > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.barrier_wait();
        if (warp == 0) {
            cluster.map_shared_rank(cluster_lists, 0)[rank * 32 + lane] = best;
            if (lane == 0) cluster.map_shared_rank(cluster_sums, 0)[rank] = mine;
        }
        cluster.sync();
        if (rank) return;
        if (a.top > 0) {
            best = merge_lists(warp < blocks ? cluster_lists[warp * 32 + lane] : 0, blocks, lists, warp,
                               lane);
        }
        if (warp == 0) {
            mine = cluster_sums[0];
            for (int i = 1; i < blocks; ++i) mine = join(mine, cluster_sums[i], c);
        }
    }
    if (warp) return;
    const float log_s = logf(mine.s);
    const bool none = mine.m == -INFINITY && mine.s == 0.0f; /* no logit above -inf */
    if (last) {
        float v = (given - mine.m) * a.scale - log_s;
        if (none) v = -INFINITY;
        if (token < 0) v = 0.0f;
        if (token >= cols) v = NAN;
        a.logprobs[row] = v;
        a.entropy[row] = none ? 0.0f : log_s - a.scale * (mine.w / mine.s);
    }
    if (lane < a.top) {
        const float v = value_of((uint32_t)(best >> 32));
        a.top_logprobs[row * a.top + lane] = none ? -INFINITY : (v - mine.m) * a.scale - log_s;
        a.top_ids[row * a.top + lane] = (int32_t) ~(uint32_t)best;
    }
}

template <typename T> cudaError_t launch(const cfa_logprobs_args &a, cudaStream_t stream)
{
    int blocks = kMaxCluster;
    while (blocks > 1 && (a.rows * blocks > 4 * 152 || a.cols < 4096 * (blocks / 2))) blocks /= 2;
    const int threads = blocks > 1 ? 512 : 256;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * blocks));
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = blocks > 1 ? 2 : 1;
    void *p[] = {const_cast<cfa_logprobs_args *>(&a), &blocks};
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void *>(&cfa_logprobs_kernel<T>), p);
}

} // namespace

cudaError_t cfa_launch_logprobs(const cfa_logprobs_args *a, cudaStream_t stream)
{
    if (a->dtype == CFA_DTYPE_F32) return launch<float>(*a, stream);
    if (a->dtype == CFA_DTYPE_F16) return launch<__half>(*a, stream);
    return launch<__nv_bfloat16>(*a, stream);
}
