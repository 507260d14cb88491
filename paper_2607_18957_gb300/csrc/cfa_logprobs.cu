/*
 * Log probabilities of given tokens, entropy and the largest logits of each row, in one pass over it.
 *
 * With m the row's largest logit and t = (v - m) scale log2(e): s = sum 2^t, w = sum 2^t t, so that
 * log p = t ln 2 - log s and the entropy is log s - ln 2 w / s.  Every thread keeps the three for its own
 * part of the row (a running m; s and w follow when it grows) and they are joined in a fixed order.
 *
 * The largest: each thread notes the largest of every batch of its loads (or of several).  Each warp's
 * ceil(top / warps)-th largest of its threads' own maxima has as many at or above it, so that no wanted logit
 * lies below the least of these, and only the batches that reach this bound, a few times as many as logits
 * are wanted, are looked through again.  What reaches it there is put into a list, and each of the list
 * counts how many are before it.  Should more reach it than the list holds (equal logits), the warps go
 * through their parts with sorted lists of their best instead, which are merged.  A logit's key is its
 * value mapped onto integers of the same order and its complemented index, so that keys are unique and
 * equal values go to the lowest index.
 *
 * A row belongs to one block or to a cluster of blocks, whose results meet in the first one's shared
 * memory.
 *
 * Bound by memory with fp32 logits (2048 rows of 128,256 163 us, 0.95 of a copy); with 16-bit ones, which come
 * twice as fast, by memory, exponentials and issue slots together (101 us, 5.2 TB/s).  Two values an
 * instruction for t and the sums, and the largest two at a time, took it there from 132 us; a ring in shared
 * memory in front of it was slower (98 us without the best, against 91).  One row with its 20 best 8.4 us.
 */
#include <cooperative_groups.h>

#include "cfa_ops.h"
#include "cfa_values.cuh"

using namespace cfa_dev;
namespace cg = cooperative_groups;

namespace {

constexpr int kMaxWarps = 16, kMaxCluster = 8, kMaxTop = CFA_LOGPROBS_MAX_TOP;
constexpr int kList = kMaxWarps * 32; /* logits that can reach the bound before the slower way is taken */
constexpr int kNotes = 16; /* a thread's, each of one or several batches */

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

/* The larger, NaN if one is. */
__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

constexpr float kLeast = -1000.0f; /* 2^t is 0 from there on, and 0 times t is to be 0 for -inf too */

struct Sums {
    float m, s, w;
};

/* s and w of a part whose largest logit is `from`, once it is `to` (finite c): a part without a logit above
 * -inf has s = w = 0, or NaN. */
__device__ __forceinline__ void lower(Sums &a, float to, float c)
{
    if (a.m > -INFINITY) {
        const float d = (a.m - to) * c, e = exp2_fast(d);
        a.w = (a.w + max_or_nan(d, kLeast) * a.s) * e;
        a.s *= e;
    } else {
        a.w = a.s;
    }
    a.m = to;
}

/* The sums of two parts together. */
__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    const float m = fmaxf(a.m, b.m);
    lower(a, m, c);
    lower(b, m, c);
    return {m, a.s + b.s, a.w + b.w};
}

/* The largest of N values that is not NaN, if there is any. */
template <int N> __device__ __forceinline__ float largest(const Pack<float, N> &q)
{
    float v = q.v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) v = fmaxf(v, q.v[i]);
    return v;
}
template <int N> __device__ __forceinline__ float largest(const Pack<__half, N> &q)
{
    const __half2 *p = reinterpret_cast<const __half2 *>(&q);
    __half2 v = p[0];
#pragma unroll
    for (int i = 1; i < N / 2; ++i) v = __hmax2(v, p[i]);
    return fmaxf(__low2float(v), __high2float(v));
}
template <int N> __device__ __forceinline__ float largest(const Pack<__nv_bfloat16, N> &q)
{
    const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&q);
    __nv_bfloat162 v = p[0];
#pragma unroll
    for (int i = 1; i < N / 2; ++i) v = __hmax2(v, p[i]);
    return fmaxf(__low2float(v), __high2float(v));
}

/* Two values side by side, for the instructions that take two at a time. */
struct Two {
    uint64_t v;
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void split(float &a, float &b) const
    {
        asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
    }
};
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c)
{
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(c.v) : "l"(a.v), "l"(b.v));
    return c;
}
__device__ __forceinline__ Two add_two(Two a, Two b)
{
    asm("add.rn.f32x2 %0, %0, %1;" : "+l"(a.v) : "l"(b.v));
    return a;
}

/* The least of N values that is not NaN, if that costs less than one operation a value. */
template <int N> __device__ __forceinline__ float least(const Pack<float, N> &) { return -INFINITY; }
template <int N> __device__ __forceinline__ float least(const Pack<__half, N> &q)
{
    const __half2 *p = reinterpret_cast<const __half2 *>(&q);
    __half2 v = p[0];
#pragma unroll
    for (int i = 1; i < N / 2; ++i) v = __hmin2(v, p[i]);
    return fminf(__low2float(v), __high2float(v));
}
template <int N> __device__ __forceinline__ float least(const Pack<__nv_bfloat16, N> &q)
{
    const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&q);
    __nv_bfloat162 v = p[0];
#pragma unroll
    for (int i = 1; i < N / 2; ++i) v = __hmin2(v, p[i]);
    return fminf(__low2float(v), __high2float(v));
}

/* sum 2^t and sum 2^t t of t = v c - mc; CLAMP: values can be -inf. */
template <bool CLAMP, typename T, int N, int M>
__device__ __forceinline__ void two_sums(const Pack<T, N> (&q)[M], float c, float mc, float &s, float &w)
{
    const Two c2(c, c), m2(-mc, -mc);
    Two s2(0.0f, 0.0f), w2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            Two d2 = fma_two(Two(to_f32(q[i].v[k]), to_f32(q[i].v[k + 1])), c2, m2);
            float d0, d1;
            d2.split(d0, d1);
            if (CLAMP) {
                d0 = max_or_nan(d0, kLeast);
                d1 = max_or_nan(d1, kLeast);
                d2 = Two(d0, d1);
            }
            const Two e2(exp2_fast(d0), exp2_fast(d1));
            s2 = add_two(s2, e2);
            w2 = fma_two(e2, d2, w2);
        }
    float a, b;
    s2.split(a, b);
    s = a + b;
    w2.split(a, b);
    w = a + b;
}

/* Adds n pieces, `step` apart, one value at a time: a part without a logit above -inf, or so large ones that
 * m c has no room for its rounding.  A call of its own, which reads
 * them again, so that the common way keeps its registers. */
template <typename T, int N>
__device__ __noinline__ Sums add_any(Sums a, const T *at, int64_t step, int n, float c)
{
    for (int i = 0; i < n; ++i) {
        const Pack<T, N> q = load_pack<T, N>(at + i * step * N);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float v = to_f32(q.v[k]);
            if (v > a.m) lower(a, v, c);
            if (a.m > -INFINITY) {
                const float d = max_or_nan((v - a.m) * c, kLeast), e = exp2_fast(d);
                a.s += e;
                a.w = fmaf(e, d, a.w);
            } else if (v != v) {
                a.s = a.w = v;
            }
        }
    }
    return a;
}

/* Adds pieces, `step` apart from `at` on, and returns the largest. */
template <typename T, int N, int M>
__device__ __forceinline__ float add(Sums &a, const Pack<T, N> (&q)[M], const T *at, int64_t step, float c)
{
    float top = largest(q[0]), low = least(q[0]);
#pragma unroll
    for (int i = 1; i < M; ++i) {
        top = fmaxf(top, largest(q[i]));
        low = fminf(low, least(q[i]));
    }
    const float m = fmaxf(a.m, top), mc = m * c;
    if (fabsf(mc) < 512.0f) {
        if (m > a.m) lower(a, m, c);
        /* t in one operation, off by what rounding m c leaves off, the same for all of them and at most
         * 2^-16: taken out of the sums to first order (the second is below 2^-33) */
        float s0, w0;
        if (sizeof(T) == 2 && low * c > -1e30f)
            two_sums<false>(q, c, mc, s0, w0);
        else
            two_sums<true>(q, c, mc, s0, w0);
        const float off = fmaf(m, c, -mc);
        a.s += fmaf(-0.69314718f * off, s0, s0);
        a.w += fmaf(-0.69314718f * off, w0, w0) - off * s0;
    } else {
        a = add_any<T, N>(a, at, step, M, c);
    }
    return top;
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

/* BATCH: loads of 16 bytes that a thread takes at a time */
template <typename T, int BATCH>
__global__ void __launch_bounds__(kMaxWarps * 32, 2)
    cfa_logprobs_kernel(const cfa_logprobs_args a, int blocks /* of a row */)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ uint64_t lists[kList], s_best[kMaxTop];
    __shared__ Sums sums[kMaxWarps];
    __shared__ uint64_t cluster_lists[kMaxCluster][kMaxTop];
    __shared__ Sums cluster_sums[kMaxCluster];
    __shared__ uint32_t s_bound[kMaxWarps], s_many, s_found;
    __shared__ uint16_t s_who[kList]; /* the notes that reach the bound */
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

    extern __shared__ uint4 room[]; /* the notes: [kNotes][threads] */
    T *const notes = reinterpret_cast<T *>(room) + threadIdx.x;
    const int top = a.top;
    const int64_t span = (int64_t)BATCH * step;
    const int batches = (int)((pieces + span - 1) / span); /* of the first thread, which has the most */
    const int of_note = (batches + kNotes - 1) / kNotes;
    int n = 0, note = 0;
    float noted = -INFINITY;
    for (int64_t p0 = g; p0 < pieces; p0 += span) {
        const T *at = body + p0 * VEC;
        if (p0 + (BATCH - 1) * (int64_t)step < pieces) {
            Pack<T, VEC> q[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) q[i] = load_pack<T, VEC>(at + (int64_t)i * step * VEC);
            noted = fmaxf(noted, add(mine, q, at, step, c));
        } else {
            for (int64_t p = p0; p < pieces; p += step, at += (int64_t)step * VEC) {
                const Pack<T, VEC> q[1] = {load_pack<T, VEC>(at)};
                noted = fmaxf(noted, add(mine, q, at, step, c));
            }
        }
        if (top > 0 && (++n == of_note || p0 + span >= pieces)) {
            notes[note * blockDim.x] = from_f32<T>(noted); /* a T's value */
            ++note;
            n = 0;
            noted = -INFINITY;
        }
    }
    if (g < head) mine = add_any<T, 1>(mine, x + g, 0, 1, c);
    if (g < tail) mine = add_any<T, 1>(mine, x + cols - tail + g, 0, 1, c);
    float given = -INFINITY;
    if (token >= 0 && token < cols) given = to_f32(load_pack<T, 1>(x + token).v[0]);

    const uint32_t own = order_of(mine.m);
    for (int o = 16; o; o >>= 1) {
        Sums other;
        other.m = __shfl_xor_sync(kAllLanes, mine.m, o);
        other.s = __shfl_xor_sync(kAllLanes, mine.s, o);
        other.w = __shfl_xor_sync(kAllLanes, mine.w, o);
        mine = join(lane & o ? other : mine, lane & o ? mine : other, c);
    }
    if (lane == 0) sums[warp] = mine;
    if (top > 0) {
        uint32_t left = own, reached = 0;
        for (int i = (top + warps - 1) / warps; i; --i) {
            reached = __reduce_max_sync(kAllLanes, left);
            if (lane == __ffs(__ballot_sync(kAllLanes, left == reached)) - 1) left = 0;
        }
        if (lane == 0) s_bound[warp] = reached;
    }
    if (threadIdx.x == 0) s_many = s_found = 0;
    __syncthreads();

    if (top > 0) {
        const uint32_t bound =
            __reduce_min_sync(kAllLanes, lane < warps ? s_bound[lane] : 0xFFFFFFFFu);
        auto put = [&](float v, uint32_t index) {
            if (order_of(v) < bound) return;
            const uint32_t n = atomicAdd(&s_found, 1u);
            if (n < kList) lists[n] = key_of(v, index);
        };
        if (own >= bound) {
            for (int i = 0; i < note; ++i)
                if (order_of(to_f32(notes[i * blockDim.x])) >= bound) {
                    const uint32_t n = atomicAdd(&s_many, 1u);
                    if (n < kList) s_who[n] = (uint16_t)(i * blockDim.x + threadIdx.x);
                }
            if (g < head) put(single[0], (uint32_t)g);
            if (g < tail) put(single[1], (uint32_t)(cols - tail + g));
        }
        __syncthreads();
        /* the pieces of those notes, one to a thread */
        const uint32_t many = s_many, of = of_note * BATCH;
        const int first = g - (int)threadIdx.x;
        if (many <= kList) {
#pragma unroll 2
            for (uint32_t i = threadIdx.x; i < many * of; i += blockDim.x) {
                const uint32_t who = s_who[i / of];
                const int64_t q = first + who % blockDim.x + (int64_t)(who / blockDim.x * of + i % of) * step;
                if (q >= pieces) continue;
                const Pack<T, VEC> v = load_pack<T, VEC>(body + q * VEC);
                const float most = largest(v);
                if (!(most == most) || order_of(most) >= bound) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) put(to_f32(v.v[k]), (uint32_t)(head + q * VEC + k));
                }
            }
        }
        if (threadIdx.x < kMaxTop) s_best[threadIdx.x] = 0;
        __syncthreads();
        const int found = (int)s_found;
        if (many <= kList && found <= kList) {
            for (int n = threadIdx.x; n < found; n += blockDim.x) {
                const uint64_t key = lists[n];
                int rank = 0;
                for (int i = 0; i < found; ++i) rank += lists[i] > key;
                if (rank < top) s_best[rank] = key;
            }
        } else {
            __syncthreads();
            uint64_t best = 0;
            auto give = [&](bool in, float v, uint32_t index) {
                best = offer(best, in && order_of(v) >= bound ? key_of(v, index) : 0, top, lane);
            };
            for (int64_t q0 = g - lane; q0 < pieces; q0 += step) {
                const int64_t q = q0 + lane;
                const bool in = q < pieces;
                Pack<T, VEC> v;
                if (in) v = load_pack<T, VEC>(body + q * VEC);
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    give(in, in ? to_f32(v.v[k]) : 0.0f, (uint32_t)(head + q * VEC + k));
            }
            if (warp == 0) { /* the single values, which the first threads of the row hold */
                give(g < head, single[0], (uint32_t)g);
                give(g < tail, single[1], (uint32_t)(cols - tail + g));
            }
            best = merge_lists(best, warps, lists, warp, lane);
            if (warp == 0 && lane < top) s_best[lane] = best;
        }
        __syncthreads();
    }
    if (warp == 0) {
        mine = sums[0];
        for (int i = 1; i < warps; ++i) mine = join(mine, sums[i], c);
    }
    if (blocks > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.barrier_wait();
        if (warp == 0) {
            if (lane < top) cluster.map_shared_rank(&cluster_lists[rank][0], 0)[lane] = s_best[lane];
            if (lane == 0) cluster.map_shared_rank(cluster_sums, 0)[rank] = mine;
        }
        cluster.sync();
        if (rank) return;
        if ((int)threadIdx.x < blocks * top) {
            const int list = threadIdx.x / top;
            const uint64_t key = cluster_lists[list][threadIdx.x - list * top];
            int before = 0;
            for (int i = 0; i < blocks; ++i) {
                int at = 0; /* the descending list's keys above this one */
#pragma unroll
                for (int o = kMaxTop; o; o >>= 1)
                    if (at + o <= top && cluster_lists[i][at + o - 1] > key) at += o;
                before += at;
            }
            if (key && before < top) s_best[before] = key;
        }
        if (warp == 0) {
            mine = cluster_sums[0];
            for (int i = 1; i < blocks; ++i) mine = join(mine, cluster_sums[i], c);
        }
        __syncthreads();
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
        a.entropy[row] = none ? 0.0f : log_s - 0.69314718f * (mine.w / mine.s);
    }
    if (lane < top) {
        const uint64_t best = s_best[lane];
        const float v = value_of((uint32_t)(best >> 32));
        a.top_logprobs[row * top + lane] = none ? -INFINITY : (v - mine.m) * a.scale - log_s;
        a.top_ids[row * top + lane] = (int32_t) ~(uint32_t)best;
    }
}

template <typename T> cudaError_t launch(const cfa_logprobs_args &a, cudaStream_t stream)
{
    /* So many threads to a row that the rows fill the SMs, but that each has some loads; a cluster of blocks
     * where one does not hold them.  Many rows get small blocks with more loads at a time, whose ends meet
     * others' streams (2048 rows of 128,256 bf16 logits: 128 threads of 8 loads 101 us, of 4 106, 256 threads
     * of 4 116; 116 rows of 18,319: one block of 512 to each 10.8 us, clusters of four 19.8). */
    const int64_t loads = a.cols * (int64_t)sizeof(T) / 16;
    int64_t threads_of_row = 152 * 1024 / a.rows;
    if (threads_of_row > loads / 4) threads_of_row = loads / 4;
    int blocks = 1, threads = 128;
    while (threads < 512 && 2 * threads <= threads_of_row) threads *= 2;
    while (blocks < kMaxCluster && 2 * blocks * threads <= threads_of_row) blocks *= 2;
    const void *fn = blocks > 1 ? reinterpret_cast<const void *>(&cfa_logprobs_kernel<T, 4>)
                                : reinterpret_cast<const void *>(&cfa_logprobs_kernel<T, 8>);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * blocks));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = a.top > 0 ? threads * kNotes * sizeof(T) : 0; /* 32 KiB at most */
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
    return cudaLaunchKernelExC(&cfg, fn, p);
}

} // namespace

cudaError_t cfa_launch_logprobs(const cfa_logprobs_args *a, cudaStream_t stream)
{
    if (a->dtype == CFA_DTYPE_F32) return launch<float>(*a, stream);
    if (a->dtype == CFA_DTYPE_F16) return launch<__half>(*a, stream);
    return launch<__nv_bfloat16>(*a, stream);
}
