/*
 * What the kernels of a decoding step's operators share: values of each type to fp32 and back, 16 bytes
 * or one value at a time, sums over a block, the start behind the kernel before.  Loads go past L1, which
 * may hold what an older kernel read there (see launch_early in cfa_device.cuh).
 */
#pragma once

#include <math.h>

#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cfa_device.cuh"

namespace cfa_dev {

/* Lets kernel fn have so much shared memory, once per device (`done` has a bit for each that knows). */
inline cudaError_t allow_shared(const void *fn, int bytes, std::atomic<uint64_t> &done)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (!e) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

constexpr uint32_t kAllLanes = 0xFFFFFFFFu;

/* Before anything that an earlier kernel has written is read, and anything at all written: the earlier
 * kernels have ended.  From here on the next one may start (its own wait is for this kernel's end), not
 * before, so that a kernel that reads ahead of its wait reads nothing that these still write. */
__device__ __forceinline__ void launch_in_turn()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v)
{
    return __float2bfloat16_rn(v);
}

template <typename T, int N> struct alignas(sizeof(T) * N) Pack {
    T v[N];
};

/* N neighbouring values (N * sizeof(T) 16 bytes and p on that grid, or N = 1) */
template <typename T, int N> __device__ __forceinline__ Pack<T, N> load_pack(const T *p)
{
    Pack<T, N> q;
    if constexpr (N == 1) {
        q.v[0] = __ldcg(p);
    } else {
        static_assert(sizeof(q) == 16, "");
        *reinterpret_cast<uint4 *>(&q) = __ldcg(reinterpret_cast<const uint4 *>(p));
    }
    return q;
}

template <typename T, int N> __device__ __forceinline__ void store_pack(T *p, const float (&f)[N])
{
    Pack<T, N> q;
#pragma unroll
    for (int i = 0; i < N; ++i) q.v[i] = from_f32<T>(f[i]);
    *reinterpret_cast<Pack<T, N> *>(p) = q;
}

/* N values of a weight in T or fp32 */
template <typename T, int N>
__device__ __forceinline__ void load_weight(const void *w, bool f32, int64_t at, float (&f)[N])
{
    if (!f32) {
        const Pack<T, N> q = load_pack<T, N>(static_cast<const T *>(w) + at);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = to_f32(q.v[i]);
    } else if constexpr (N == 1) {
        f[0] = __ldcg(static_cast<const float *>(w) + at);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 q = __ldcg(reinterpret_cast<const float4 *>(static_cast<const float *>(w) + at + i));
            f[i] = q.x;
            f[i + 1] = q.y;
            f[i + 2] = q.z;
            f[i + 3] = q.w;
        }
    }
}

} // namespace cfa_dev
