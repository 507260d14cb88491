/*
 * Choice of experts.  One warp a token: each lane holds R neighbouring logits, so that a group of
 * experts lies in a few neighbouring lanes.  The top_k come out one at a time as the warp's largest
 * key, a key being the fp32 value mapped onto unsigned integers of the same order; every lane keeps
 * the best of its own.  Equal keys go to the lowest index.
 *
 * The lane that has just given its best needs the next one.  With few logits per lane it goes through
 * them alone; from kShared on its keys, which lie in shared memory, go one to a lane and the warp takes
 * their largest: the others would wait for that lane's loop anyway (4096 tokens over 128 experts, eight
 * choices: 4.9 -> 4.2 us when it was built, 3.5 now; 256 experts 7.3 -> 5.3, 4.0 now).
 *
 * Bound by the launch and by the chain of loads, exponentials and top_k warp reductions of one token,
 * and beyond some thousand tokens by the instructions of that chain; the bytes would take a tenth.
 * One token over 8 experts 1.5 us in a row of launches, 4099 tokens over 256 experts in 8 groups with a
 * bias 6.3 us, 16,384 tokens over 128 experts 9.7 us.  What made the difference there: neighbouring
 * logits in a lane instead of every 32nd (13.8 -> 8.1 us without a bias), the bias through L1 (3.2 us
 * less), and a warp brought together again before its shuffles (1.1 us less: lanes that a branch has
 * parted trade values one by one).
 */
#include <math.h>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cfa_device.cuh"
#include "cfa_ops.h"

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

__device__ __forceinline__ float from_bits(uint32_t b, int32_t dtype) /* of a 2-byte type */
{
    if (dtype == CFA_DTYPE_F16) return __half2float(__ushort_as_half((unsigned short)b));
    return __bfloat162float(__ushort_as_bfloat16((unsigned short)b));
}

/* The lane's R of n values, -inf behind the last.  (All loads go past L1: see cfa_matmul.cu.) */
template <int R>
__device__ __forceinline__ void load(int32_t dtype, int n, const void *row, int first, bool vec,
                                     float (&v)[R])
{
    if (dtype == CFA_DTYPE_F32) {
        const float *p = static_cast<const float *>(row) + first;
        if (R % 4 == 0 && vec) {
#pragma unroll
            for (int r = 0; r + 3 < R; r += 4) {
                const float4 q = __ldcg(reinterpret_cast<const float4 *>(p + r));
                v[r] = q.x;
                v[r + 1] = q.y;
                v[r + 2] = q.z;
                v[r + 3] = q.w;
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) v[r] = first + r < n ? __ldcg(p + r) : -INFINITY;
        }
    } else {
        const unsigned short *p = static_cast<const unsigned short *>(row) + first;
        if (R % 4 == 0 && vec) {
#pragma unroll
            for (int r = 0; r + 3 < R; r += 4) {
                const uint2 q = __ldcg(reinterpret_cast<const uint2 *>(p + r));
                v[r] = from_bits(q.x & 0xFFFFu, dtype);
                v[r + 1] = from_bits(q.x >> 16, dtype);
                v[r + 2] = from_bits(q.y & 0xFFFFu, dtype);
                v[r + 3] = from_bits(q.y >> 16, dtype);
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r)
                v[r] = first + r < n ? from_bits(__ldcg(p + r), dtype) : -INFINITY;
        }
    }
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

/* (first, second) of two values together with another two in descending order */
__device__ __forceinline__ void merge(float &first, float &second, float a, float b)
{
    const float low = fminf(first, a);
    first = fmaxf(first, a);
    second = fmaxf(fmaxf(second, b), low);
}

/* A group's place among the others by its two best keys.  An expert that cannot be chosen counts for
 * nothing in its group: the sum of the two best is the one key where only one expert is left (with -inf
 * in the sum the group would rank behind all others), and a group without any is last. */
__device__ __forceinline__ uint32_t rank_of(float first, float second, bool sum_two)
{
    return order_of(sum_two && second > -INFINITY ? first + second : first);
}

/* Which lanes' keys lie in a group that is kept; by lanes where every lane's keys lie in one group of
 * 2^n neighbouring lanes, otherwise through shared memory. */
template <int R>
__device__ __forceinline__ void keep_groups(const cfa_route_args &a, float (&key)[R], float *mine,
                                            int lane, bool sum_two)
{
    const int size = a.experts / a.groups, lanes = size / R;
    if (size == lanes * R && (lanes & (lanes - 1)) == 0) {
        float first = -INFINITY, second = -INFINITY;
#pragma unroll
        for (int r = 0; r < R; ++r) merge(first, second, key[r], -INFINITY);
        for (int o = 1; o < lanes; o <<= 1)
            merge(first, second, __shfl_xor_sync(kAll, first, o), __shfl_xor_sync(kAll, second, o));
        const uint32_t best = rank_of(first, second, sum_two);
        const int group = lane / lanes;
        int before = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t other = __shfl_sync(kAll, best, g * lanes);
            before += other > best || (other == best && g < group);
        }
        if (before >= a.top_groups) {
#pragma unroll
            for (int r = 0; r < R; ++r) key[r] = -INFINITY;
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (lane * R + r < a.experts) mine[lane * R + r] = key[r];
    __syncwarp();
    float first = -INFINITY, second = -INFINITY;
    if (lane < a.groups)
        for (int i = 0; i < size; ++i) merge(first, second, mine[lane * size + i], -INFINITY);
    const uint32_t best = rank_of(first, second, sum_two);
    int before = 0;
    for (int g = 0; g < a.groups; ++g) {
        const uint32_t other = __shfl_sync(kAll, best, g);
        before += other > best || (other == best && g < lane);
    }
    const uint32_t kept = __ballot_sync(kAll, lane < a.groups && before < a.top_groups);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int e = lane * R + r;
        if (e < a.experts && !(kept >> (e / size) & 1u)) key[r] = -INFINITY;
    }
}

/* The bias comes through L1, behind a fence that clears what L1 held before the launch's wait was over:
 * every warp reads the same few lines, which L2 hands out at 64 bytes a clock. */
template <int R>
__device__ __forceinline__ void load_bias(const float *bias, int first, int n, float (&b)[R])
{
    if (R % 4 == 0 && n == 32 * R && ((uintptr_t)bias & 15u) == 0) {
#pragma unroll
        for (int r = 0; r + 3 < R; r += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(bias + first + r);
            b[r] = q.x;
            b[r + 1] = q.y;
            b[r + 2] = q.z;
            b[r + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) b[r] = first + r < n ? bias[first + r] : 0.0f;
    }
}

/* The lane's R values side by side in shared memory. */
template <int R, typename T> __device__ __forceinline__ void put(T *to, const T (&v)[R])
{
    if constexpr (R % 4 == 0) {
        struct alignas(16) Four {
            T v[4];
        };
#pragma unroll
        for (int r = 0; r < R; r += 4)
            *reinterpret_cast<Four *>(to + r) = {v[r], v[r + 1], v[r + 2], v[r + 3]};
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) to[r] = v[r];
    }
}

constexpr int kShared = 4; /* from so many logits per lane on, keys and logits lie in shared memory too */

/* R: logits per lane. */
template <int R>
__global__ void __launch_bounds__(kWarps * 32) cfa_route_kernel(const cfa_route_args a)
{
    /* of each warp: [32 R] keys and [32 R] logits from kShared on; below, [experts] keys with groups */
    extern __shared__ __align__(16) uint32_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t *const s_key = smem + warp * (R >= kShared ? 64 * R : a.experts);
    float *const s_logit = reinterpret_cast<float *>(s_key + 32 * R);
    const int64_t t = (int64_t)blockIdx.x * kWarps + warp;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.bias) __threadfence();
    if (t >= a.tokens) return;

    const int es = a.dtype == CFA_DTYPE_F32 ? 4 : 2;
    const uint8_t *row = static_cast<const uint8_t *>(a.logits) + t * a.logits_stride * es;
    const bool vec = a.experts == 32 * R && ((uintptr_t)row & (uintptr_t)(4 * es - 1)) == 0;
    float v[R], key[R], b[R];
    load<R>(a.dtype, a.experts, row, lane * R, vec, v);
    if (a.bias) load_bias<R>(a.bias, lane * R, a.experts, b);
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        nan |= v[r] != v[r];
        top = fmaxf(top, v[r]);
    }
    const bool softmax = a.scoring == CFA_SCORE_SOFTMAX;
    const bool renormalize = a.flags & CFA_ROUTE_RENORMALIZE;
    float norm = 1.0f;
    if (softmax) {
        nan = __any_sync(kAll, nan);
        if (!renormalize || a.bias) { /* the sum over all of them counts */
            top = warp_max(top);
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r) sum += v[r] > -INFINITY ? expf(v[r] - top) : 0.0f;
            norm = nan ? NAN : warp_add(sum);
        }
    }
    if (!softmax) {
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = 1.0f / (1.0f + expf(-v[r]));
    } else if (a.bias) {
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = expf(v[r] - top) / norm;
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = v[r];
    }
    /* What cannot be chosen, NaN among it, is -inf from here on: fminf and fmaxf give the other one of
     * a NaN and a number, and a NaN key would count its group's best key twice.  (Without a bias a key
     * is NaN only where its logit is.) */
    if (a.bias) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            key[r] += b[r];
            if (!(key[r] > -INFINITY)) key[r] = -INFINITY;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (!(v[r] > -INFINITY)) key[r] = -INFINITY;
    if (a.groups > 1) keep_groups<R>(a, key, reinterpret_cast<float *>(s_key), lane, !softmax);

    uint32_t k[R], best = 0; /* the lane's best key, its place and its logit */
    int at = 0;
    float z = 0.0f;
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
        k[r] = order_of(key[r]);
        if (k[r] >= best) {
            best = k[r];
            at = r;
            z = v[r];
        }
    }
    float chosen = -INFINITY; /* lane j: the logit of choice j */
    int id = -1;
    if constexpr (R >= kShared) {
        __syncwarp();
        put<R>(s_key + lane * R, k);
        put<R>(s_logit + lane * R, v);
        __syncwarp();
    }
    for (int j = 0; j < a.top_k; ++j) {
        const uint32_t most = __reduce_max_sync(kAll, best);
        if (most == 0) break; /* nothing left to choose */
        const int win = __ffs(__ballot_sync(kAll, best == most)) - 1;
        if constexpr (R >= kShared) {
            /* the winner's keys, one to a lane, which alone reads and writes it: the best that is left */
            const int gone = __shfl_sync(kAll, at, win);
            if (lane == j) id = win * R + gone;
            const int own = win * R + (lane < R ? lane : 0);
            uint32_t left = lane < R && lane != gone ? s_key[own] : 0;
            if (lane == gone) s_key[own] = 0;
            const uint32_t next = __reduce_max_sync(kAll, left);
            const int place = __ffs(__ballot_sync(kAll, left == next)) - 1;
            if (lane == win) {
                best = next;
                at = place;
            }
            continue;
        }
        const int e = __shfl_sync(kAll, lane * R + at, win);
        const float logit = __shfl_sync(kAll, z, win);
        if (lane == j) {
            chosen = logit;
            id = e;
        }
        if (lane == win) {
            const int gone = at;
            best = 0;
#pragma unroll
            for (int r = R - 1; r >= 0; --r) {
                if (r == gone) k[r] = 0;
                if (k[r] >= best) {
                    best = k[r];
                    at = r;
                    z = v[r];
                }
            }
        }
    }

    if constexpr (R >= kShared) chosen = id >= 0 ? s_logit[id < 0 ? 0 : id] : -INFINITY;
    __syncwarp(); /* the lanes together, for the shuffles below */

    float w = 0.0f;
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
    const size_t smem = sizeof(float) * kWarps *
                        (R >= kShared ? 64 * R : a.groups > 1 ? a.experts : 0);
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
    if (a->experts <= 96) return launch<3>(*a, stream);
    if (a->experts <= 128) return launch<4>(*a, stream);
    if (a->experts <= 160) return launch<5>(*a, stream);
    if (a->experts <= 192) return launch<6>(*a, stream);
    if (a->experts <= 256) return launch<8>(*a, stream);
    if (a->experts <= 512) return launch<16>(*a, stream);
    return launch<32>(*a, stream);
}
