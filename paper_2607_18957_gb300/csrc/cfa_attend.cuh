/*
 * Attention of new tokens over a paged cache: o = softmax(scale q K^T) V, each row over the keys that it
 * sees.
 *
 * The keys of a sequence are cut into slots of 16.  A tile is up to 8 NT rows (new tokens times the query
 * heads that share a key head) of one sequence and key head; the slots of all tiles in a row, sequence by
 * sequence, are split evenly over the warps of all blocks, whatever the sequences' lengths, so that the
 * work is even without the host knowing a length.  Where a warp's share begins or ends inside a tile its
 * sums are joined with its neighbours': in shared memory within a block, through the workspace and by a
 * second launch between blocks.  All joins go in a fixed order.
 *
 * A warp brings its slots into its own ring in shared memory (cp.async; rows that are not there are filled
 * with zeros and nothing is read for them) and needs no barrier with other warps.  Per slot it computes
 * S^T = K Q^T (16 keys by 8 NT rows), follows the rows' running maximum m and sum l, and adds V^T P^T to
 * O^T (dim by 8 NT rows): with the keys along the 16 of the matrix instruction and the rows along its 8, one
 * token of a group of 8 heads fills it.
 */
#pragma once

#include <cuda_fp8.h>

#include "cfa_ops.h"
#include "cfa_values.cuh"

namespace cfa_attend_dev {

using namespace cfa_dev;

constexpr int kBlocks = CFA_ATTEND_BLOCKS;
constexpr int kKeys = 16; /* of a slot */
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

template <int D, int NT, bool F8> struct Shape {
    static constexpr int kWarps = D > 128 ? 4 : 8;
    static constexpr int kTiles = D / 16;                     /* of 16 dims */
    static constexpr int kRows = 8 * NT;
    static constexpr int kRowBytes = D * (F8 ? 1 : 2);
    static constexpr int kPitch = kRowBytes + 16;             /* an odd number of 16 bytes: no conflicts */
    static constexpr int kStage = 2 * kKeys * kPitch;         /* keys, then values */
    static constexpr int kFloats = kTiles * NT * 4 * 32 + 2 * kRows; /* of a partial: O, m, l */
    static constexpr int kRoom = (232448 - 2048) / kWarps - kFloats * 4;
    static constexpr int kFit = kRoom / kStage;
    static constexpr int kStages = kFit > 6 ? 6 : kFit;
    static constexpr int kWarpBytes = kStages * kStage + kFloats * 4;
    static constexpr int kSmem = kWarps * kWarpBytes;
    static_assert(kStages >= 2 && kStages * kStage >= kFloats * 4 && kStage % 16 == 0 &&
                  kWarpBytes % 16 == 0 && D % 32 == 0, "");
};

using Work = cfa_attend_work;

/* A place in the row of slots. */
struct Place {
    int32_t b, tile, slot; /* sequence, tile of it, slot of the tile */
    int32_t slots, first;  /* of a tile; the first slot that any row sees */
    int32_t len, low;      /* keys of the sequence; the first one that any row sees */
};

__device__ __forceinline__ int clamped(const Work &w, int len)
{
    const int64_t most = (int64_t)w.a.max_pages * w.a.page_size;
    return len < 0 ? 0 : (int64_t)len < most ? len : (int)most;
}

/* The sequence's part of a place. */
__device__ __forceinline__ void enter(const Work &w, Place &p, int len)
{
    p.len = clamped(w, len);
    p.low = 0;
    if (w.a.window > 0) p.low = max(0, p.len - w.a.new_tokens + 1 - w.a.window);
    p.first = p.low / kKeys;
    p.slots = max(1, (p.len + kKeys - 1) / kKeys - p.first);
}

__device__ __forceinline__ int length_of(const Work &w, int b)
{
    return b < w.a.sequences ? __ldcg(w.a.lengths + b) : 0;
}

__device__ __forceinline__ void cp_async(uint32_t to, const void *from, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldmatrix(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ void ldmatrix_trans(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                                   uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, "
                 "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                            uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, "
                 "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack2(__nv_bfloat16, float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack2(__half, float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 unpack2(__nv_bfloat16, uint32_t v)
{
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v));
}
__device__ __forceinline__ float2 unpack2(__half, uint32_t v)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}

/* Probabilities enter the second product as sums of two 16-bit values: rounded to one alone they would put
 * the result off by as much as its own rounding does.  The first is cut off at least one of its units
 * below the probability, so that neither is 0 or negative and an infinite value stays what it is. */
template <int UNIT> __device__ __forceinline__ float below(float v)
{
    const uint32_t b = __float_as_uint(v);
    return __uint_as_float(max(b, 1u << UNIT) - (1u << UNIT)); /* NaN stays NaN */
}
__device__ __forceinline__ uint32_t split(__nv_bfloat16, float x, float y, uint32_t &low)
{
    const uint32_t a = __float_as_uint(below<16>(x)) & 0xFFFF0000u;
    const uint32_t b = __float_as_uint(below<16>(y)) & 0xFFFF0000u;
    low = pack2(__nv_bfloat16(), x - __uint_as_float(a), y - __uint_as_float(b));
    return __byte_perm(a, b, 0x7632);
}
__device__ __forceinline__ uint32_t split(__half, float x, float y, uint32_t &low)
{
    const __half a = __float2half_rz(below<13>(x)), b = __float2half_rz(below<13>(y));
    low = pack2(__half(), x - __half2float(a), y - __half2float(b));
    const __half2 v = __halves2half2(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
/* All probabilities and their sums are held 2^kUp times as large: fp16 has no smaller ones than 2^-24. */
template <typename P> constexpr float kUp = 0.0f;
template <> constexpr float kUp<__half> = 14.0f;

/* Two e4m3 values, the low 16 bits, as T.  All of them are values of both types. */
__device__ __forceinline__ uint32_t widen(__half, uint32_t v)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v & 0xFFFFu), __NV_E4M3);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t widen(__nv_bfloat16, uint32_t v)
{
    const uint32_t h = widen(__half(), v);
    const float2 f = unpack2(__half(), h);
    return pack2(__nv_bfloat16(), f.x, f.y);
}

__device__ __forceinline__ float exp2_fast(float v) /* off by 2^-22; below 2^-126 zero */
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

/* exp2 of the difference of two maxima, the second the larger: 0 where the first is of no key at all */
__device__ __forceinline__ float shrink(float m, float top)
{
    return exp2_fast(m - (top == -INFINITY ? 0.0f : top));
}

/* Where a row's results go: rows of a tile are the new tokens' heads of one key head. */
struct Row {
    int64_t token; /* of all sequences' new tokens */
    int32_t head;
    bool here;
};
__device__ __forceinline__ Row row_of(const Work &w, int b, int tile, int n, int rows)
{
    const int kv = tile / w.row_tiles, r = (tile - kv * w.row_tiles) * rows + n;
    const int i = r / w.group;
    Row x;
    x.here = i < w.a.new_tokens;
    x.token = (int64_t)b * w.a.new_tokens + i;
    x.head = kv * w.group + r - i * w.group;
    return x;
}

/* Writes 16 dims of a tile's rows: c is O^T as the matrix instruction leaves it, l its sums, m the
 * maxima in powers of two.  With an 8-bit cache the dims of a lane are 2 g and 2 g + 1 instead of g and g +
 * 8 (see below). */
template <typename T, int NT, bool F8>
__device__ __forceinline__ void finish(const Work &w, int b, int tile, int dims, int lane,
                                       const float (*c)[4], const float (*m)[2], const float (*l)[2],
                                       bool sums)
{
    using P = typename std::conditional<F8, __half, T>::type;
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const float u0 = l[nt][0] == 0.0f ? 0.0f : w.a.v_scale / l[nt][0];
        const float u1 = l[nt][1] == 0.0f ? 0.0f : w.a.v_scale / l[nt][1];
        float v[4] = {c[nt][0] * u0, c[nt][1] * u1, c[nt][2] * u0, c[nt][3] * u1};
        /* rows along the lanes: two dims side by side (F8: the pairs are of every second dim) */
        const uint32_t a0 = transposed(pack2(T(), v[0], v[1])), a1 = transposed(pack2(T(), v[2], v[3]));
        const Row r = row_of(w, b, tile, nt * 8 + g, 8 * NT);
        if (r.here) {
            T *o = static_cast<T *>(w.a.out) + r.token * w.a.out_stride +
                   (int64_t)r.head * w.a.head_dim + dims;
            if constexpr (F8) { /* a0: dims 4 t, 4 t + 2; a1: 4 t + 1, 4 t + 3 */
                uint2 q;
                q.x = __byte_perm(a0, a1, 0x5410);
                q.y = __byte_perm(a0, a1, 0x7632);
                *reinterpret_cast<uint2 *>(o + 4 * t) = q;
            } else {
                *reinterpret_cast<uint32_t *>(o + 2 * t) = a0;
                *reinterpret_cast<uint32_t *>(o + 8 + 2 * t) = a1;
            }
        }
        if (sums && w.a.lse && g < 2) {
            const Row s = row_of(w, b, tile, nt * 8 + 2 * t + g, 8 * NT);
            const float top = g ? m[nt][1] : m[nt][0], sum = g ? l[nt][1] : l[nt][0];
            if (s.here)
                w.a.lse[s.token * w.a.heads + s.head] =
                    sum == 0.0f ? -INFINITY : (top + (log2f(sum) - kUp<P>)) * kLn2;
        }
    }
}

template <typename T, int D, int NT, bool F8>
__global__ void __launch_bounds__(Shape<D, NT, F8>::kWarps * 32, 1) cfa_attend_kernel(const Work w)
{
    using S = Shape<D, NT, F8>;
    using P = typename std::conditional<F8, __half, T>::type; /* of the probabilities and values */
    constexpr int W = S::kWarps, MT = S::kTiles, ROWS = S::kRows, STAGES = S::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t s_sum[W];
    __shared__ Place s_at[W + 1];     /* the borders of the warps' shares */
    __shared__ uint8_t s_part[W][2];  /* which partials there are */
    __shared__ uint32_t s_ok[W][STAGES];
    const cfa_attend_args &a = w.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int64_t tiles = (int64_t)a.kv_heads * w.row_tiles; /* of a sequence */
    wait_for_earlier();

    /* ---- the block's and the warps' shares ---- */
    const int64_t per = (a.sequences + W * 32 - 1) / (W * 32);
    const int b0 = (int)min(tid * per, a.sequences), b1 = (int)min(b0 + per, a.sequences);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) {
        Place p;
        enter(w, p, length_of(w, b));
        mine += p.slots;
    }
    int64_t before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(kAllLanes, before, o);
        if (lane >= o) before += v;
    }
    if (lane == 31) s_sum[warp] = before;
    if (tid < W * 2) s_part[tid >> 1][tid & 1] = 0;
    __syncthreads();
    int64_t total = 0;
    before -= mine;
    for (int i = 0; i < W; ++i) {
        if (i < warp) before += s_sum[i];
        total += s_sum[i];
    }
    total *= tiles;
    const int64_t full = (total + W - 1) / W;
    const int blocks = full < kBlocks ? (int)full : kBlocks; /* that get any */
    if ((int)blockIdx.x >= blocks) {
        if (tid < 2) w.ends[blockIdx.x * 2 + tid] = -1;
        return;
    }
    const int64_t shares = (int64_t)blocks * W;
    const int64_t lo = before * tiles, hi = (before + mine) * tiles;
    for (int i = 0; i <= W; ++i) {
        /* total * share fits: total < 2^48 */
        const int64_t at = total * ((int64_t)blockIdx.x * W + i) / shares;
        const bool end = at == total;
        if (end ? tid == 0 : lo <= at && at < hi) {
            Place p;
            p.b = (int)a.sequences;
            p.tile = p.slot = p.slots = p.first = p.len = p.low = 0;
            if (!end) {
                int64_t from = lo;
                int b = b0;
                for (;; ++b) {
                    enter(w, p, length_of(w, b));
                    if (at < from + p.slots * tiles) break;
                    from += p.slots * tiles;
                }
                p.b = b;
                p.tile = (int)((at - from) / p.slots);
                p.slot = (int)((at - from) % p.slots);
            }
            s_at[i] = p;
        }
    }
    __syncthreads();
    const int64_t share = (int64_t)blockIdx.x * W + warp;
    int count = (int)(total * (share + 1) / shares - total * share / shares);

    /* ---- the warp's slots ---- */
    uint8_t *const ring = smem + warp * S::kWarpBytes;
    float *const held = reinterpret_cast<float *>(ring + STAGES * S::kStage); /* the first partial */
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    Place in = s_at[warp], out = in; /* of the loads, of the products */
    const uint8_t *const kc = static_cast<const uint8_t *>(a.k_cache);
    const uint8_t *const vc = static_cast<const uint8_t *>(a.v_cache);
    constexpr int ES = F8 ? 1 : 2;

    /* Each lane looks one key up, one slot ahead of the loads: its page's number, -1 if it is not there. */
    auto page_at = [&](const Place &p, int left) {
        const int key = (p.first + p.slot) * kKeys + (lane & 15);
        if (left <= 0 || key >= p.len || key < p.low) return -1;
        return __ldcg(a.pages + (int64_t)p.b * a.pages_stride + key / a.page_size);
    };
    auto advance = [&](Place &p) {
        if (++p.slot < p.slots) return;
        p.slot = 0;
        if (++p.tile < tiles) return;
        p.tile = 0;
        ++p.b;
        enter(w, p, length_of(w, p.b));
    };
    int to_load = count, page = page_at(in, to_load);
    auto load = [&](int stage) {
        if (to_load > 0) {
            const int key = (in.first + in.slot) * kKeys + (lane & 15), place = key % a.page_size;
            const int kv = in.tile / w.row_tiles;
            const bool ok = page >= 0 && page < a.cache_pages;
            const uint32_t all = __ballot_sync(kAllLanes, ok) & 0xFFFFu;
            const int64_t ko = ok ? (page * a.k_page_stride + place * a.k_token_stride +
                                     kv * a.k_head_stride) * ES : 0;
            const int64_t vo = ok ? (page * a.v_page_stride + place * a.v_token_stride +
                                     kv * a.v_head_stride) * ES : 0;
            constexpr int CH = S::kRowBytes / 16;
            const uint32_t to = ring_at + stage * S::kStage;
#pragma unroll
            for (int i = 0; i < kKeys * CH / 32; ++i) {
                const int n = i * 32 + lane, r = n / CH, c = n - r * CH;
                const int64_t at = __shfl_sync(kAllLanes, ko, r);
                cp_async(to + r * S::kPitch + c * 16, kc + at + c * 16, all >> r & 1u ? 16 : 0);
            }
#pragma unroll
            for (int i = 0; i < kKeys * CH / 32; ++i) {
                const int n = i * 32 + lane, r = n / CH, c = n - r * CH;
                const int64_t at = __shfl_sync(kAllLanes, vo, r);
                cp_async(to + (kKeys + r) * S::kPitch + c * 16, vc + at + c * 16,
                         all >> r & 1u ? 16 : 0);
            }
            if (lane == 0) s_ok[warp][stage] = all;
            --to_load;
            advance(in);
            page = page_at(in, to_load);
        }
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) load(i);

    uint32_t qf[MT][NT][2];
    float o[MT][NT][4], m[NT][2], l[NT][2];
    int hi_n[NT][2], hi_least = 0, hi_most = 0; /* keys below these are seen */
    const float unit = a.scale * kLog2e * a.k_scale;

    auto start = [&] { /* a tile */
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const Row r = row_of(w, out.b, out.tile, nt * 8 + g, ROWS);
            const T *q = static_cast<const T *>(a.q) + r.token * a.q_stride + (int64_t)r.head * D;
#pragma unroll
            for (int k = 0; k < MT; ++k) {
                qf[k][nt][0] = qf[k][nt][1] = 0;
                if (r.here) {
                    if constexpr (F8) { /* dims in the order in which the keys' bytes come */
                        const uint2 v = __ldcg(reinterpret_cast<const uint2 *>(q + k * 16 + 4 * t));
                        qf[k][nt][0] = v.x;
                        qf[k][nt][1] = v.y;
                    } else {
                        qf[k][nt][0] = __ldcg(reinterpret_cast<const uint32_t *>(q + k * 16 + 2 * t));
                        qf[k][nt][1] = __ldcg(reinterpret_cast<const uint32_t *>(q + k * 16 + 8 + 2 * t));
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[nt][j] = -INFINITY;
                l[nt][j] = 0.0f;
                const Row s = row_of(w, out.b, out.tile, nt * 8 + 2 * t + j, ROWS);
                hi_n[nt][j] = out.len - a.new_tokens + 1 +
                              min((int)(s.token - (int64_t)out.b * a.new_tokens), a.new_tokens - 1);
            }
        }
        const int r0 = (out.tile % w.row_tiles) * ROWS;
        hi_least = out.len - a.new_tokens + 1 + r0 / w.group;
        hi_most = out.len - a.new_tokens + 1 + min((r0 + ROWS - 1) / w.group, a.new_tokens - 1);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.0f;
    };
    /* l over the lanes that hold one row's keys */
    auto sum_up = [&] {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[nt][j] += __shfl_xor_sync(kAllLanes, l[nt][j], x);
    };
    auto keep = [&](float *to) { /* a partial */
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                *reinterpret_cast<float4 *>(to + ((i * NT + nt) * 32 + lane) * 4) =
                    make_float4(o[i][nt][0], o[i][nt][1], o[i][nt][2], o[i][nt][3]);
        if (g == 0) {
            float *ml = to + MT * NT * 128;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ml[nt * 8 + 2 * t + j] = m[nt][j];
                    ml[ROWS + nt * 8 + 2 * t + j] = l[nt][j];
                }
        }
    };

    int stage = 0;
    bool open_start = out.slot != 0; /* the tile has begun in another warp's share */
    if (count > 0) start();
    const uint32_t k_row = (lane & 15) * S::kPitch + (lane >> 4) * 16;
    const uint32_t v_row = F8 ? (kKeys + (lane & 15)) * S::kPitch + (lane >> 4) * 16
                              : (kKeys + (lane & 7) + (lane >> 4) * 8) * S::kPitch + (lane >> 3 & 1) * 16;
    for (; count > 0; --count) {
        cp_wait<STAGES - 2>();
        __syncwarp(); /* this stage is there for all lanes, and all have read the one before */
        load((stage + STAGES - 1) % STAGES);
        const uint32_t at = ring_at + stage * S::kStage, ok = s_ok[warp][stage];
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[nt][j] = 0.0f;
        if constexpr (F8) {
#pragma unroll
            for (int k = 0; k < MT; k += 2) {
                uint32_t r[4];
                ldmatrix(r, at + k_row + k * 16);
                const uint32_t f0[4] = {widen(T(), r[0]), widen(T(), r[1]), widen(T(), r[0] >> 16),
                                        widen(T(), r[1] >> 16)};
                const uint32_t f1[4] = {widen(T(), r[2]), widen(T(), r[3]), widen(T(), r[2] >> 16),
                                        widen(T(), r[3] >> 16)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<T>(s[nt], f0, qf[k][nt][0], qf[k][nt][1]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<T>(s[nt], f1, qf[k + 1][nt][0], qf[k + 1][nt][1]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < MT; ++k) {
                uint32_t f[4];
                ldmatrix(f, at + k_row + k * 32);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<T>(s[nt], f, qf[k][nt][0], qf[k][nt][1]);
            }
        }

        /* scores in powers of two, -inf for keys that a row does not see */
        const int base = (out.first + out.slot) * kKeys;
        /* keys that are there, but not for every row of the tile (one token's rows all see the same) */
        const bool mixed = a.new_tokens > 1 && ((base + kKeys > hi_least && base < out.len) ||
                                                (a.window > 0 && base < hi_most - a.window));
        const bool some = ok != 0xFFFFu || base + kKeys > hi_least ||
                          (a.window > 0 && base < hi_most - a.window);
        bool rise = false;
        float f[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[nt][j] *= unit;
                if (some) {
                    const int i = g + (j >> 1) * 8, key = base + i, top = hi_n[nt][j & 1];
                    const bool seen = (ok >> i & 1u) && key < top &&
                                      (a.window <= 0 || key >= top - a.window);
                    if (!seen) s[nt][j] = -INFINITY;
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float top = fmaxf(s[nt][j], s[nt][j + 2]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(kAllLanes, top, x));
                top = fmaxf(top, m[nt][j]);
                f[nt][j] = shrink(m[nt][j], top);
                rise |= top > m[nt][j];
                m[nt][j] = top;
                const float ref = (top == -INFINITY ? 0.0f : top) - kUp<P>;
                s[nt][j] = exp2_fast(s[nt][j] - ref);
                s[nt][j + 2] = exp2_fast(s[nt][j + 2] - ref);
                l[nt][j] = l[nt][j] * f[nt][j] + (s[nt][j] + s[nt][j + 2]);
            }
        }
        if (__any_sync(kAllLanes, rise)) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[i][nt][j] *= f[nt][j & 1];
        }
        uint32_t p[NT][2][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t low;
                const uint32_t high = split(P(), s[nt][2 * j], s[nt][2 * j + 1], low);
                p[nt][j][0] = transposed(high);
                p[nt][j][1] = transposed(low);
            }
        auto values = [&](int i, uint32_t (&v)[4], uint32_t (&r)[4]) { /* V^T of 16 dims */
            if constexpr (F8) {
                if (i % 2 == 0) ldmatrix_trans(r, at + v_row + i * 16);
                const uint32_t r0 = r[i % 2 * 2], r1 = r[i % 2 * 2 + 1];
                const uint32_t x0 = widen(P(), r0), y0 = widen(P(), r0 >> 16);
                const uint32_t x1 = widen(P(), r1), y1 = widen(P(), r1 >> 16);
                v[0] = __byte_perm(x0, y0, 0x5410); /* row g: dim 2 g, row g + 8: dim 2 g + 1 */
                v[1] = __byte_perm(x0, y0, 0x7632);
                v[2] = __byte_perm(x1, y1, 0x5410);
                v[3] = __byte_perm(x1, y1, 0x7632);
            } else {
                ldmatrix_trans(v, at + v_row + i * 32);
            }
        };
        uint32_t r[4] = {};
        if (!mixed) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                uint32_t v[4];
                values(i, v, r);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma<P>(o[i][nt], v, p[nt][0][0], p[nt][1][0]);
                    mma<P>(o[i][nt], v, p[nt][0][1], p[nt][1][1]);
                }
            }
        } else {
            /* Keys that some rows see and others do not: token by token, with the values that it does not
             * see taken out, since 0 times an infinity or NaN would come through. */
            for (int top = hi_least; top <= hi_most; ++top) {
                uint32_t mask[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int key = base + j * 8 + 2 * t;
                    const bool x = key < top && (a.window <= 0 || key >= top - a.window);
                    const bool y = key + 1 < top && (a.window <= 0 || key + 1 >= top - a.window);
                    mask[j] = (x ? 0x0000FFFFu : 0u) | (y ? 0xFFFF0000u : 0u);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    uint32_t v[4];
                    values(i, v, r);
                    v[0] &= mask[0];
                    v[1] &= mask[0];
                    v[2] &= mask[1];
                    v[3] &= mask[1];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float c[4] = {};
                        mma<P>(c, v, p[nt][0][0], p[nt][1][0]);
                        mma<P>(c, v, p[nt][0][1], p[nt][1][1]);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (hi_n[nt][j & 1] == top) o[i][nt][j] += c[j];
                    }
                }
            }
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;

        const bool ends = out.slot + 1 == out.slots;
        if (ends || count == 1) {
            sum_up();
            if (open_start) {
                keep(held);
                if (lane == 0) s_part[warp][0] = 1;
            } else if (!ends) {
                cp_wait<0>();
                __syncwarp();
                keep(reinterpret_cast<float *>(ring));
                if (lane == 0) s_part[warp][1] = 1;
            } else {
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    finish<T, NT, F8>(w, out.b, out.tile, i * 16, lane, o[i], m, l, i == 0);
            }
            if (count > 1) {
                advance(out);
                open_start = false;
                start();
            }
        } else {
            advance(out);
        }
    }
    cp_wait<0>();
    release_later();
    __syncthreads();

    /* ---- tiles that several warps have worked on: 16 dims to a warp ---- */
    const bool any0 = s_at[0].slot != 0, anyW = s_at[W].slot != 0;
    auto id = [&](const Place &p) { return p.slot ? (int64_t)p.b * tiles + p.tile : (int64_t)-1; };
    if (tid == 0) {
        w.ends[blockIdx.x * 2] = any0 ? id(s_at[0]) : -1;
        w.ends[blockIdx.x * 2 + 1] = anyW ? id(s_at[W]) : -1;
    }
    for (int e = 0; e <= W;) {
        const int64_t tile = id(s_at[e]);
        if (tile < 0) {
            ++e;
            continue;
        }
        int last = e; /* borders e .. last lie inside this tile */
        while (last < W && id(s_at[last + 1]) == tile) ++last;
        const bool outside = e == 0 || last == W;
        const int pb = s_at[e].b, pt = s_at[e].tile;
        for (int i = warp; i < MT; i += W) {
            float c[NT][4], top[NT][2], sum[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int j = 0; j < 4; ++j) c[nt][j] = 0.0f;
                top[nt][0] = top[nt][1] = -INFINITY;
                sum[nt][0] = sum[nt][1] = 0.0f;
            }
            for (int x = max(e - 1, 0); x <= min(last, W - 1); ++x) {
                const int which = x < e ? 1 : 0; /* the warp in which it begins holds it as its last */
                if (!s_part[x][which]) continue;
                const uint8_t *from = smem + x * S::kWarpBytes + (which ? 0 : STAGES * S::kStage);
                const float *part = reinterpret_cast<const float *>(from), *ml = part + MT * NT * 128;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float4 q =
                        *reinterpret_cast<const float4 *>(part + ((i * NT + nt) * 32 + lane) * 4);
                    const float v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float m1 = ml[nt * 8 + 2 * t + j], l1 = ml[ROWS + nt * 8 + 2 * t + j];
                        const float both = fmaxf(m1, top[nt][j]);
                        const float f0 = shrink(top[nt][j], both), f1 = shrink(m1, both);
                        top[nt][j] = both;
                        sum[nt][j] = sum[nt][j] * f0 + l1 * f1;
                        c[nt][j] = c[nt][j] * f0 + v[j] * f1;
                        c[nt][j + 2] = c[nt][j + 2] * f0 + v[j + 2] * f1;
                    }
                }
            }
            if (!outside) {
                finish<T, NT, F8>(w, pb, pt, i * 16, lane, c, top, sum, i == 0);
                continue;
            }
            float *to = w.parts + (int64_t)(blockIdx.x * 2 + (e == 0 ? 0 : 1)) * S::kFloats;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                *reinterpret_cast<float4 *>(to + ((i * NT + nt) * 32 + lane) * 4) =
                    make_float4(c[nt][0], c[nt][1], c[nt][2], c[nt][3]);
            if (i == 0 && g == 0) {
                float *ml = to + MT * NT * 128;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        ml[nt * 8 + 2 * t + j] = top[nt][j];
                        ml[ROWS + nt * 8 + 2 * t + j] = sum[nt][j];
                    }
            }
        }
        e = last + 1;
    }
}

constexpr int kJoinWarps = 8;

/* Tiles that several blocks have worked on: block (c, i) joins 16 dims of the tile that begins in block c
 * of the launch before and ends in a later one. */
template <typename T, int D, int NT, bool F8>
__global__ void __launch_bounds__(kJoinWarps * 32) cfa_attend_join_kernel(const Work w)
{
    using S = Shape<D, NT, F8>;
    __shared__ float4 s_c[kJoinWarps][NT][32];
    __shared__ float s_m[kJoinWarps][8 * NT], s_l[kJoinWarps][8 * NT];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int first = blockIdx.x, i = blockIdx.y;
    wait_for_earlier();
    const int64_t tile = __ldcg(w.ends + first * 2 + 1);
    if (tile < 0 || __ldcg(w.ends + first * 2) == tile) return;
    float c[NT][4], top[NT][2], sum[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c[nt][j] = 0.0f;
        top[nt][0] = top[nt][1] = -INFINITY;
        sum[nt][0] = sum[nt][1] = 0.0f;
    }
    auto join = [&](int nt, const float (&v)[4], const float (&m1)[2], const float (&l1)[2]) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float both = fmaxf(m1[j], top[nt][j]);
            const float f0 = shrink(top[nt][j], both), f1 = shrink(m1[j], both);
            top[nt][j] = both;
            sum[nt][j] = sum[nt][j] * f0 + l1[j] * f1;
            c[nt][j] = c[nt][j] * f0 + v[j] * f1;
            c[nt][j + 2] = c[nt][j + 2] * f0 + v[j + 2] * f1;
        }
    };
    int parts = 1;
    for (int x0 = first + 1; x0 < kBlocks; x0 += 32) { /* blocks that lie inside it */
        const int x = x0 + lane;
        const bool in = x < kBlocks && __ldcg(w.ends + x * 2) == tile;
        const uint32_t all = __ballot_sync(kAllLanes, in);
        parts += __popc(all);
        if (all != kAllLanes) break;
    }
    for (int x = warp; x < parts; x += kJoinWarps) {
        const float *part = w.parts + (int64_t)((first + x) * 2 + (x == 0 ? 1 : 0)) * S::kFloats;
        const float *ml = part + S::kTiles * NT * 128;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float4 q =
                __ldcg(reinterpret_cast<const float4 *>(part + ((i * NT + nt) * 32 + lane) * 4));
            const float2 m1 = __ldcg(reinterpret_cast<const float2 *>(ml + nt * 8 + 2 * t));
            const float2 l1 = __ldcg(reinterpret_cast<const float2 *>(ml + 8 * NT + nt * 8 + 2 * t));
            join(nt, {q.x, q.y, q.z, q.w}, {m1.x, m1.y}, {l1.x, l1.y});
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        s_c[warp][nt][lane] = make_float4(c[nt][0], c[nt][1], c[nt][2], c[nt][3]);
        if (g == 0) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s_m[warp][nt * 8 + 2 * t + j] = top[nt][j];
                s_l[warp][nt * 8 + 2 * t + j] = sum[nt][j];
            }
        }
    }
    __syncthreads();
    if (warp) return;
    for (int x = 1; x < kJoinWarps && x < parts; ++x)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float4 q = s_c[x][nt][lane];
            const int n = nt * 8 + 2 * t;
            join(nt, {q.x, q.y, q.z, q.w}, {s_m[x][n], s_m[x][n + 1]}, {s_l[x][n], s_l[x][n + 1]});
        }
    const int64_t tiles = (int64_t)w.a.kv_heads * w.row_tiles;
    finish<T, NT, F8>(w, (int)(tile / tiles), (int)(tile % tiles), i * 16, lane, c, top, sum, i == 0);
}

template <typename T, int D, int NT, bool F8> cudaError_t launch(const Work &w, cudaStream_t stream)
{
    using S = Shape<D, NT, F8>;
    const void *fn = reinterpret_cast<const void *>(&cfa_attend_kernel<T, D, NT, F8>);
    cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e) return e;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kBlocks);
    cfg.blockDim = dim3(S::kWarps * 32);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    void *p[] = {const_cast<Work *>(&w)};
    e = cudaLaunchKernelExC(&cfg, fn, p);
    if (e) return e;
    cfg.gridDim = dim3(kBlocks, S::kTiles);
    cfg.blockDim = dim3(kJoinWarps * 32);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelExC(
        &cfg, reinterpret_cast<const void *>(&cfa_attend_join_kernel<T, D, NT, F8>), p);
}

template <typename T, bool F8> cudaError_t launch_any(const Work &w, cudaStream_t stream)
{
    const int nt = w.nt;
    switch (w.a.head_dim) {
    case 64: return nt == 1 ? launch<T, 64, 1, F8>(w, stream) : launch<T, 64, 2, F8>(w, stream);
    case 96: return nt == 1 ? launch<T, 96, 1, F8>(w, stream) : launch<T, 96, 2, F8>(w, stream);
    case 128: return nt == 1 ? launch<T, 128, 1, F8>(w, stream) : launch<T, 128, 2, F8>(w, stream);
    case 256: return nt == 1 ? launch<T, 256, 1, F8>(w, stream) : launch<T, 256, 2, F8>(w, stream);
    default: return cudaErrorInvalidValue; /* refused before */
    }
}

} // namespace cfa_attend_dev
