/*
 * Norms between blocks: a = x or its norm times post_weight, times act(gate); h = residual + scale a;
 * y = norm(h) weight, norm(v) = v / sqrt(mean(v^2) + eps).
 *
 * A row lies in the registers of `lanes` threads, up to NV pieces of VEC values each, from its only
 * load to the stores; the sum of squares is the one thing that they exchange.  h is held in fp32 and y
 * is computed from that, not from h as it is stored.
 *
 * Bound by memory: 4096 rows of 8192 bf16 with a residual 43 us (6.2 TB/s, 0.92 of a copy), 1777 rows of
 * 2307 fp16 off the grid with a gate and both norms 20.4 us (2.0 TB/s: every block first brings both weights
 * into shared memory, one value at a time, for two or three rows, each a chain of two sums); one row of
 * 4096 2.2 us in a row of launches.
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
    case CFA_ACT_SILU: {
        /* exp of a negative argument alone, since exp(-v) leaves fp32 before v / (1 + exp(-v)) does, and
         * as a square, for v < 0 one half of it behind a: exp(v) has lost bits where a v exp(v) has not
         * yet */
        const float half = expf(-0.5f * fabsf(v)), side = v < 0.0f ? half : 1.0f;
        return a * __fdividef(v * side, 1.0f + half * half) * side;
    }
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

/* The same for a row of up to 32 threads, a power of two, or of a whole block, a multiple of 32. */
__device__ __forceinline__ float block_sum(float v, int lanes, float *part)
{
    for (int o = min(lanes, 32) >> 1; o; o >>= 1) v += __shfl_xor_sync(kAllLanes, v, o);
    if (lanes <= 32) return v;
    const int lane = threadIdx.x & 31;
    if (lane == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < lanes >> 5 ? part[lane] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAllLanes, v, o);
    return v;
}

template <typename T, int VEC, int NV, int MOST>
__global__ void __launch_bounds__(MOST, MOST == 1024 ? 1 : 2) cfa_norm_kernel(const cfa_norm_args a, int lanes)
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

template <typename T, int VEC, int NV, int MOST>
cudaError_t launch(const cfa_norm_args &a, int lanes, cudaStream_t stream)
{
    const int threads = lanes > kBlock ? lanes : kBlock, rows = threads / lanes;
    cfa_launch_ctl ctl = {};
    ctl.flags = CFA_LAUNCH_EARLY;
    void *p[] = {const_cast<cfa_norm_args *>(&a), &lanes};
    return launch_ctl(reinterpret_cast<const void *>(&cfa_norm_kernel<T, VEC, NV, MOST>),
                      (unsigned)((a.tokens + rows - 1) / rows), threads, 0, stream, ctl, p);
}

/* ---- many rows ----
 * Blocks go through the rows, and each thread has its pieces of the next ones under way to its own places
 * in shared memory (nobody else reads them, so that no barrier is needed for them).
 *
 * SHIFT: rows off the 16-byte grid, all matrices by as much.  Pieces then lie on the grid of the memory
 * instead of the row's, and the first and the last are partly of the row.  The weights, which are not off
 * by as much, lie in shared memory with every VEC-th value side by side: whatever a row is off by, the
 * lanes read neighbours. */
template <typename T, bool SHIFT> struct Stream {
    static constexpr int VEC = 16 / sizeof(T);

    /* Brings the 16 bytes at column c of a row, as far as they are of it or before it. */
    static __device__ __forceinline__ void bring(uint32_t to, const T *row, int c, int cols)
    {
        const int bytes = min(16, (cols - c) * (int)sizeof(T));
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(row + c), "r"(bytes)
                     : "memory");
    }

    /* Where shared memory has the values k = 0 .. VEC - 1 of the piece at column 0 of a row; VEC zeros lie
     * before a weight's first value, and `apart` is how far every VEC-th values are from the next. */
    static __device__ __forceinline__ void places(int off, int apart, int (&at)[VEC])
    {
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const int n = VEC - off + k;
            at[k] = n % VEC * apart + n / VEC;
        }
    }

    /* offset + values c .. c + VEC - 1 of a weight, piece `piece` of the row */
    static __device__ __forceinline__ void weight(const void *w, const T *held, const int (&at)[VEC],
                                                  int piece, bool f32, int c, float offset,
                                                  float (&f)[VEC])
    {
        if constexpr (SHIFT) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) f[k] = to_f32(held[at[k] + piece]);
        } else {
            load_weight<T, VEC>(w, f32, c, f);
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] += offset;
    }

    /* What has been brought, zeros for what is not of the row. */
    static __device__ __forceinline__ void take(const uint4 &q, int c, int cols, float (&f)[VEC])
    {
        Pack<T, VEC> p;
        *reinterpret_cast<uint4 *>(&p) = q;
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] = to_f32(p.v[k]);
        if (SHIFT && (c < 0 || c + VEC > cols)) {
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (c + k < 0 || c + k >= cols) f[k] = 0.0f;
        }
    }

    static __device__ __forceinline__ void hold(const void *w, T *held, int apart, int cols)
    {
        const T *v = static_cast<const T *>(w);
        auto put = [&](int c, T x) { held[(c + VEC) % VEC * apart + (c + VEC) / VEC] = x; };
        const int vectors = ((uintptr_t)w & 15) == 0 ? cols / VEC : 0;
#pragma unroll 2
        for (int i = threadIdx.x; i < vectors; i += blockDim.x) {
            const Pack<T, VEC> p = load_pack<T, VEC>(v + i * VEC);
#pragma unroll
            for (int k = 0; k < VEC; ++k) put(i * VEC + k, p.v[k]);
        }
#pragma unroll 4
        for (int c = vectors * VEC + threadIdx.x; c < cols; c += blockDim.x)
            put(c, load_pack<T, 1>(v + c).v[0]);
        for (int c = threadIdx.x; c < VEC; c += blockDim.x) put(c - VEC, from_f32<T>(0.0f));
        for (int c = cols + threadIdx.x; c < (apart - 1) * VEC; c += blockDim.x)
            put(c, from_f32<T>(0.0f));
    }

    static __device__ __forceinline__ void store(T *row, int c, int cols, const float (&f)[VEC])
    {
        if (!SHIFT || (c >= 0 && c + VEC <= cols)) {
            store_pack<T, VEC>(row + c, f);
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (c + k >= 0 && c + k < cols) row[c + k] = from_f32<T>(f[k]);
        }
    }
};

template <typename T, int NV, bool SHIFT>
__global__ void __launch_bounds__(1024) cfa_norm_rows_kernel(const cfa_norm_args a, int lanes, int stages)
{
    using S = Stream<T, SHIFT>;
    constexpr int VEC = S::VEC;
    extern __shared__ uint4 ring[]; /* [stages][x, residual, gate][NV][threads]; SHIFT: the weights */
    __shared__ float part[2][2][32];
    const int threads = blockDim.x, side = threads / lanes;
    const int at = lanes > 32 ? threadIdx.x : threadIdx.x & (lanes - 1);
    const int cols = (int)a.cols, parts = 1 + (a.residual != nullptr) + (a.gate != nullptr);
    const int gate_part = a.residual ? 2 : 1;
    const bool f32 = a.weight_dtype == CFA_DTYPE_F32;
    const int64_t step = (int64_t)gridDim.x * side;
    T *const held = reinterpret_cast<T *>(ring + stages * parts * NV * threads);
    const int apart = (cols + 2 * VEC - 1) / VEC + 1;
    T *const post = held + apart * VEC;
    launch_in_turn();

    /* where the piece i of a row begins */
    auto column = [&](const T *row, int i) {
        const int off = SHIFT ? (int)((uintptr_t)row & 15) / (int)sizeof(T) : 0;
        return (i * lanes + at) * VEC - off;
    };
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring + threadIdx.x);
    auto bring = [&](int64_t row, int stage) {
        if (row < a.tokens) {
            const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
            const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
            const T *g = static_cast<const T *>(a.gate) + row * a.gate_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = column(x, i);
                if (c >= cols) continue;
                const uint32_t to = mine + ((stage * parts) * NV + i) * threads * 16;
                S::bring(to, x, c, cols);
                if (a.residual) S::bring(to + NV * threads * 16, r, c, cols);
                if (a.gate) S::bring(to + gate_part * NV * threads * 16, g, c, cols);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int64_t row = (int64_t)blockIdx.x * side + (lanes > 32 ? 0 : threadIdx.x / lanes);
    for (int s = 0; s < stages - 1; ++s) bring(row + s * step, s);
    float w[NV][VEC]; /* SHIFT: of the row, else of all */
    int none[VEC] = {};
    if constexpr (SHIFT) {
        S::hold(a.weight, held, apart, cols);
        if (a.post_weight) S::hold(a.post_weight, post, apart, cols);
        __syncthreads();
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * lanes + at) * VEC;
            if (c < cols) S::weight(a.weight, held, none, 0, f32, c, a.offset, w[i]);
        }
    }
    const float per_col = 1.0f / (float)cols;
    int stage = 0, odd = 0;
    /* every thread of a block goes through as many rows: the sums want all of them */
    for (int64_t first = (int64_t)blockIdx.x * side; first < a.tokens; first += step, row += step) {
        const int ahead = stage ? stage - 1 : stages - 1;
        bring(row + (stages - 1) * step, ahead);
        if (stages == 2)
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        else if (stages == 3)
            asm volatile("cp.async.wait_group 2;" ::: "memory");
        else
            asm volatile("cp.async.wait_group 3;" ::: "memory");
        const bool here = row < a.tokens;
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const uint4 *q = ring + (stage * parts) * NV * threads + threadIdx.x;
        int c[NV], (&places)[VEC] = none;
#pragma unroll
        for (int i = 0; i < NV; ++i) c[i] = column(x, i);
        if (SHIFT) S::places((int)((uintptr_t)x & 15) / (int)sizeof(T), apart, places);
        float h[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (here && c[i] < cols) {
                S::take(q[i * threads], c[i], cols, h[i]);
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
            const float unit = rsqrtf(block_sum(sum, lanes, part[odd][0]) * per_col + a.eps);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (here && c[i] < cols) {
                    float v[VEC];
                    S::weight(a.post_weight, post, places, i * lanes + at, f32, c[i], a.offset, v);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) h[i][k] = h[i][k] * unit * v[k];
                }
        }
        if (a.gate) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (here && c[i] < cols) {
                    float v[VEC];
                    S::take(q[(gate_part * NV + i) * threads], c[i], cols, v);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) h[i][k] = gated(h[i][k], v[k], a.activation);
                }
        }
        if (SHIFT) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (here && c[i] < cols)
                    S::weight(a.weight, held, places, i * lanes + at, f32, c[i], a.offset, w[i]);
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (here && c[i] < cols) {
                if (a.residual) {
                    float v[VEC];
                    S::take(q[(NV + i) * threads], c[i], cols, v);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) h[i][k] = fmaf(h[i][k], a.scale, v[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) h[i][k] *= a.scale;
                }
                if (a.h) S::store(static_cast<T *>(a.h) + row * a.h_stride, c[i], cols, h[i]);
#pragma unroll
                for (int k = 0; k < VEC; ++k) sum += h[i][k] * h[i][k];
            }
        const float unit = rsqrtf(block_sum(sum, lanes, part[odd][1]) * per_col + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (here && c[i] < cols) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) h[i][k] = h[i][k] * unit * w[i][k];
                S::store(static_cast<T *>(a.y) + row * a.y_stride, c[i], cols, h[i]);
            }
        odd ^= 1;
        stage = stage + 1 == stages ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

constexpr int64_t kFewRows = 152; /* up to so many a block has no next row */
constexpr int kRoom = 220 << 10;  /* shared memory of an SM's blocks */
/* Threads that an SM wants: fewer stages are taken until it holds as many.  With 256, 512, 768 and 1024,
 * us: 4096 x 8192 bf16 with a residual 48.0, 48.0, 43.1, 43.1, with gate and both norms too 110, 110, 82, 82;
 * 8192 x 2048 fp32 with all 113, 76, 76, 76; 4096 x 4096 bf16 with a residual 24.3, 24.3, 24.3, 22.7, 1000 of
 * these rows 7.4, 7.4, 7.4, 7.9; 1777 x 2307 fp16 with all 20.4, 18.5, 20.1, 20.1. */
constexpr int kBusy = 768;

template <typename T, bool SHIFT>
cudaError_t launch_rows(const cfa_norm_args &a, cudaStream_t stream, bool *fits)
{
    constexpr int VEC = 16 / sizeof(T), NV = 16 / VEC;
    const int64_t pieces = (a.cols + (SHIFT ? VEC - 1 : 0) + VEC - 1) / VEC;
    int lanes = 8; /* a power of two up to a warp, then whole warps */
    while (lanes < 32 && lanes * NV < pieces) lanes *= 2;
    if (lanes * NV < pieces) lanes = (int)((pieces + 32 * NV - 1) / (32 * NV)) * 32;
    const int threads = lanes > 32 ? lanes : kBlock, side = threads / lanes;
    const int parts = 1 + (a.residual != nullptr) + (a.gate != nullptr);
    const int stage = parts * NV * threads * 16;
    const int weights = SHIFT ? (int)((a.cols + 2 * VEC - 1) / VEC + 1) * VEC * (int)sizeof(T) *
                                    (a.post_weight ? 2 : 1)
                              : 0;
    /* as many stages, up to four, as leave room for kBusy threads on an SM */
    int stages = 4, blocks = 0;
    for (;; --stages) {
        blocks = kRoom / (stages * stage + weights);
        if (blocks > 1024 / threads) blocks = 1024 / threads;
        if (stages == 2 || blocks * threads >= kBusy) break;
    }
    const int room = stages * stage + weights;
    *fits = lanes <= 1024 && blocks > 0 && !(SHIFT && a.weight_dtype != a.dtype);
    if (!*fits) return cudaSuccess;
    const int64_t most = (a.tokens + side - 1) / side;
    const void *fn = reinterpret_cast<const void *>(&cfa_norm_rows_kernel<T, NV, SHIFT>);
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_shared(fn, kRoom, done);
    if (e) return e;
    cfa_launch_ctl ctl = {};
    ctl.flags = CFA_LAUNCH_EARLY;
    void *p[] = {const_cast<cfa_norm_args *>(&a), &lanes, &stages};
    return launch_ctl(fn, (unsigned)(most < 152 * blocks ? most : 152 * blocks), threads, room, stream,
                      ctl, p);
}

template <typename T, int VEC> cudaError_t pick(const cfa_norm_args &a, cudaStream_t stream)
{
    constexpr int NV = 16 / VEC;
    const int64_t pieces = (a.cols + VEC - 1) / VEC;
    int lanes = 8;
    while (lanes < 1024 && lanes < pieces) lanes *= 2;
    if (a.tokens <= kFewRows && lanes >= pieces) return launch<T, VEC, 1, 1024>(a, lanes, stream);
    for (lanes = 8; lanes * NV < pieces;) lanes *= 2;
    if (lanes > 512) return launch<T, VEC, NV, 1024>(a, lanes, stream); /* CFA_NORM_MAX_COLS: 1024 */
    return launch<T, VEC, NV, 512>(a, lanes, stream);
}

template <typename T> cudaError_t pick(const cfa_norm_args &a, cudaStream_t stream)
{
    constexpr int kVec = 16 / sizeof(T);
    const uint64_t in = (uint64_t)(uintptr_t)a.x | (uintptr_t)a.residual | (uintptr_t)a.gate;
    const uint64_t out = (uint64_t)(uintptr_t)a.y | (uintptr_t)a.h;
    const uint64_t weights = (uint64_t)(uintptr_t)a.weight | (uintptr_t)a.post_weight;
    uint64_t strides = (uint64_t)(a.gate ? a.gate_stride : 0);
    if (a.tokens > 1)
        strides |= (uint64_t)(a.x_stride | (a.residual ? a.residual_stride : 0) | a.y_stride |
                              (a.h ? a.h_stride : 0));
    const bool grid = !((in | out | weights | strides * sizeof(T) | (uint64_t)a.cols * sizeof(T)) & 15);
    bool fits = false;
    cudaError_t e = cudaSuccess;
    if (a.tokens > kFewRows) {
        /* rows that begin on the grid and whose ends or strides are off it, by as much in all matrices */
        const uint64_t per = 16 / sizeof(T), d = (uint64_t)a.x_stride % per;
        const bool alike = !((in | out) & 15) && (uint64_t)a.y_stride % per == d &&
                           (!a.residual || (uint64_t)a.residual_stride % per == d) &&
                           (!a.gate || (uint64_t)a.gate_stride % per == d) &&
                           (!a.h || (uint64_t)a.h_stride % per == d);
        if (grid)
            e = launch_rows<T, false>(a, stream, &fits);
        else if (alike)
            e = launch_rows<T, true>(a, stream, &fits);
        if (e || fits) return e;
    }
    if (grid) return pick<T, kVec>(a, stream);
    return pick<T, 1>(a, stream);
}

} // namespace

cudaError_t cfa_launch_norm(const cfa_norm_args *a, cudaStream_t stream)
{
    if (a->dtype == CFA_DTYPE_F32) return pick<float>(*a, stream);
    if (a->dtype == CFA_DTYPE_F16) return pick<__half>(*a, stream);
    return pick<__nv_bfloat16>(*a, stream);
}
