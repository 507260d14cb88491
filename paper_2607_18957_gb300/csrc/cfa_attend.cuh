/*
 * Attention of new tokens over a paged cache: o = softmax(scale q K^T) V, each row over the keys that it
 * sees.
 *
 * The keys of a sequence are cut into slots of 32.  A tile is up to 8 NT rows (new tokens times the query
 * heads that share a key head) of one sequence and key head; the slots of all tiles in a row, sequence by
 * sequence, are split evenly over the warps of all blocks, whatever the sequences' lengths, so that the
 * work is even without the host knowing a length.  Where a warp's share begins or ends inside a tile its
 * sums are joined with its neighbours': in shared memory within a block, through the workspace between
 * blocks, by whichever of a tile's blocks comes last (none waits for another).  All joins go in a fixed
 * order.
 *
 * A warp brings its slots into its own ring in shared memory (cp.async; rows that are not there are filled
 * with zeros and nothing is read for them) and needs no barrier with other warps.  Per slot it computes
 * S^T = K Q^T (32 keys by 8 NT rows), follows the rows' running maximum m and sum l, and adds V^T P^T to
 * O^T (dim by 8 NT rows): with the keys along the 16 of the matrix instruction and the rows along its 8, one
 * token of a group of 8 heads fills it.
 *
 * Bound by memory where there are many keys: two sequences of 131,072 and 100,001 keys, 8 key heads of 128
 * bf16, 155 us (6.1 TB/s, 0.90 of a copy), 64 sequences of 1 to 8192 keys 55 us (4.6 TB/s).  What is missing:
 * 36 of the SMs get 12 % less of the memory than the others, and their equal shares end later; 3.5 us before
 * the first keys arrive, 3.5 for the joins between blocks.  Four tokens each of 24 sequences over 8-bit keys
 * 38 us (2.8 TB/s: by the latencies of its instructions, with two warps a scheduler).  1000 keys 9.8 us: the
 * chain of lengths, page table, keys and joins.
 */
#pragma once

#include <cuda_fp8.h>

#include "cfa_ops.h"
#include "cfa_values.cuh"

namespace cfa_attend_dev {

using namespace cfa_dev;

constexpr int kBlocks = CFA_ATTEND_BLOCKS;
constexpr int kLeast = 4; /* slots of a block, where there are few */
constexpr int kKeys = 32; /* of a slot, one to a lane when they are looked up */
constexpr int kHalves = kKeys / 16; /* of 16 keys, as the matrix instruction takes them */
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

template <int D, int NT, bool F8> struct Shape {
    static constexpr int kWarps = D > 128 && !F8 ? 4 : 8;
    static constexpr int kTiles = D / 16;                     /* of 16 dims */
    static constexpr int kRows = 8 * NT;
    static constexpr int kRowBytes = D * (F8 ? 1 : 2);
    static constexpr int kPitch = kRowBytes + 16;             /* an odd number of 16 bytes: no conflicts */
    static constexpr int kStage = 2 * kKeys * kPitch;         /* keys, then values */
    static constexpr int kFloats = kTiles * NT * 4 * 32 + 2 * kRows; /* of a partial: O, m, l */
    static constexpr int kRoom = (232448 - 7168) / kWarps - kFloats * 4;
    static constexpr int kFit = kRoom / kStage;
    static constexpr int kStages = kFit > 4 ? 4 : kFit;
    static constexpr int kWarpBytes = kStages * kStage + kFloats * 4;
    static constexpr int kSmem = kWarps * kWarpBytes;
    static_assert(kStages >= 1 && kStages * kStage >= kFloats * 4 && kStage % 16 == 0 &&
                  kWarpBytes % 16 == 0 && D % 32 == 0, "");
};

using Work = cfa_attend_work;

/* A place in the row of slots. */
struct Place {
    int32_t b, kv, part;   /* sequence, key head and which of its tiles of rows */
    int32_t slot;          /* of the tile */
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

/* Keys and values pass through L2 as the first to go: what the kernel comes back to (its code, the page
 * table, partials) stays there. */
__device__ __forceinline__ uint64_t passing()
{
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void cp_async(uint32_t to, const void *from, int bytes, uint64_t policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(to), "l"(from),
                 "r"(bytes), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void cp_async(uint32_t to, const void *from, uint64_t policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(to), "l"(from),
                 "l"(policy)
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
 * below the probability, so that neither is 0 or negative and an infinite value stays what it is (fp16: for
 * probabilities from 2^-28 of the largest on, whose cut is still one of its units). */
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
/* All probabilities and their sums are held 2^kUp times as large: fp16 has no smaller ones than 2^-24, nor
 * all of its bits below 2^-14. */
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

/* Whether an infinity or NaN is among kKeys rows of `pieces` 16 bytes in shared memory, a row to a lane. */
template <typename T, bool F8>
__device__ __forceinline__ bool any_special(uint32_t at, int lane, int pieces, int pitch)
{
    static_assert(kKeys == 32, "");
    /* adding the second to the exponent's bits (an 8-bit value: to all but the sign's) overflows */
    constexpr uint32_t BITS = F8 ? 0x7F7F7F7Fu : std::is_same<T, __half>::value ? 0x7C007C00u : 0x7F807F80u;
    constexpr uint32_t ONE = F8 ? 0x01010101u : std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
    uint32_t over = 0;
    for (int c = 0; c < pieces; ++c) {
        uint32_t q[4];
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3])
                     : "r"(at + lane * pitch + c * 16)
                     : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) over |= (q[i] & BITS) + ONE;
    }
    return __any_sync(kAllLanes, (over & (F8 ? 0x80808080u : 0x80008000u)) != 0);
}

/* exp2 of the difference of two maxima, the second the larger: 0 where the first is of no key at all */
__device__ __forceinline__ float shrink(float m, float top)
{
    return exp2_fast(m - (top == -INFINITY ? 0.0f : top));
}

/* Where a row's results go: rows of a tile are the new tokens' heads of one key head. */
struct Row {
    int32_t token, head; /* of the sequence's new tokens, of all heads */
    bool here;
};
__device__ __forceinline__ Row row_of(const Work &w, int kv, int part, int n, int rows)
{
    const uint32_t r = part * rows + n; /* below 2^19 */
    const uint32_t i = w.group == 1 ? r : __umulhi(r, w.group_inverse);
    Row x;
    x.here = (int)i < w.a.new_tokens;
    x.token = i;
    x.head = kv * w.group + (int)r - (int)i * w.group;
    return x;
}

/* Where a tile's results go, and its log sums, which it writes at once: m are the rows' maxima in powers
 * of two, l their sums. */
template <typename T, int NT, bool F8> struct Finish {
    T *o[NT];          /* the lane's row, NULL for none */
    float u[NT][2];    /* what its columns of O^T are multiplied by */

    __device__ __forceinline__ Finish(const Work &w, int b, int kv, int part, int lane, bool sums,
                                      const float (&m)[NT][2], const float (&l)[NT][2])
    {
        using P = typename std::conditional<F8, __half, T>::type;
        const int g = lane >> 2, t = lane & 3;
        const int64_t first = (int64_t)b * w.a.new_tokens;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int j = 0; j < 2; ++j) u[nt][j] = l[nt][j] == 0.0f ? 0.0f : w.a.v_scale / l[nt][j];
            const Row r = row_of(w, kv, part, nt * 8 + g, 8 * NT);
            o[nt] = r.here ? static_cast<T *>(w.a.out) + (first + r.token) * w.a.out_stride +
                                 (int64_t)r.head * w.a.head_dim
                           : nullptr;
            if (sums && w.a.lse && g < 2) {
                const Row s = row_of(w, kv, part, nt * 8 + 2 * t + g, 8 * NT);
                const float top = g ? m[nt][1] : m[nt][0], sum = g ? l[nt][1] : l[nt][0];
                if (s.here)
                    w.a.lse[(first + s.token) * w.a.heads + s.head] =
                        sum == 0.0f ? -INFINITY : (top + (log2f(sum) - kUp<P>)) * kLn2;
            }
        }
    }

    /* Writes 16 dims: c is O^T as the matrix instruction leaves it.  With an 8-bit cache the dims of a lane
     * are 2 g and 2 g + 1 instead of g and g + 8 (see below). */
    __device__ __forceinline__ void write(int dims, int lane, const float (*c)[4]) const
    {
        const int t = lane & 3;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            /* rows along the lanes: two dims side by side (F8: the pairs are of every second dim) */
            const uint32_t a0 = transposed(pack2(T(), c[nt][0] * u[nt][0], c[nt][1] * u[nt][1]));
            const uint32_t a1 = transposed(pack2(T(), c[nt][2] * u[nt][0], c[nt][3] * u[nt][1]));
            T *const to = o[nt];
            if (!to) continue;
            if constexpr (F8) { /* a0: dims 4 t, 4 t + 2; a1: 4 t + 1, 4 t + 3 */
                uint2 q;
                q.x = __byte_perm(a0, a1, 0x5410);
                q.y = __byte_perm(a0, a1, 0x7632);
                *reinterpret_cast<uint2 *>(to + dims + 4 * t) = q;
            } else {
                *reinterpret_cast<uint32_t *>(to + dims + 2 * t) = a0;
                *reinterpret_cast<uint32_t *>(to + dims + 8 + 2 * t) = a1;
            }
        }
    }
};

/* Sums of some of a tile's keys, to which others' are added. */
template <int MT, int NT> struct Joined {
    float c[MT][NT][4], top[NT][2], sum[NT][2];

    __device__ __forceinline__ Joined()
    {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[nt][j] = -INFINITY;
                sum[nt][j] = 0.0f;
#pragma unroll
                for (int i = 0; i < MT; ++i) c[i][nt][j] = c[i][nt][j + 2] = 0.0f;
            }
    }

    /* Adds a partial: of its dims those 16 of which (i & mask) == sub. */
    __device__ __forceinline__ void add(const float *part, int sub, int mask, int lane)
    {
        const int t = lane & 3;
        const float *ml = part + MT * NT * 128;
        float f0[NT][2], f1[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float2 m1 = *reinterpret_cast<const float2 *>(ml + nt * 8 + 2 * t);
            const float2 l1 = *reinterpret_cast<const float2 *>(ml + 8 * NT + nt * 8 + 2 * t);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float mj = j ? m1.y : m1.x, both = fmaxf(top[nt][j], mj);
                f0[nt][j] = shrink(top[nt][j], both);
                f1[nt][j] = shrink(mj, both);
                top[nt][j] = both;
                sum[nt][j] = sum[nt][j] * f0[nt][j] + (j ? l1.y : l1.x) * f1[nt][j];
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
            if ((i & mask) == sub) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float4 q = reinterpret_cast<const float4 *>(part)[(i * NT + nt) * 32 + lane];
                    const float v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        c[i][nt][j] = c[i][nt][j] * f0[nt][j & 1] + v[j] * f1[nt][j & 1];
                }
            }
    }
};

template <typename T, int D, int NT, bool F8>
__global__ void __launch_bounds__(Shape<D, NT, F8>::kWarps * 32, 1) cfa_attend_kernel(const Work w)
{
    using S = Shape<D, NT, F8>;
    using P = typename std::conditional<F8, __half, T>::type; /* of the probabilities and values */
    constexpr int W = S::kWarps, MT = S::kTiles, ROWS = S::kRows, STAGES = S::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    static_assert((W & (W - 1)) == 0, "");
    __shared__ uint32_t s_sum[W], s_before[W * 32];
    __shared__ int32_t s_len[W * 32];
    __shared__ Place s_at[W + 1];     /* the borders of the warps' shares */
    __shared__ int64_t s_id[W + 1];   /* the tile that a border lies inside, or -1 */
    __shared__ uint8_t s_part[W][2];  /* which partials there are */
    __shared__ int s_join[2][3];      /* whether to join a tile's parts, its first block, how many */
    __shared__ uint32_t s_ok[W][STAGES];              /* which keys of a slot are there */
    __shared__ const uint8_t *s_from[W][2][kKeys];    /* where they are, and their values; or NULL */
    const cfa_attend_args &a = w.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int64_t tiles = (int64_t)a.kv_heads * w.row_tiles; /* of a sequence */
    launch_in_turn();

    /* ---- the block's and the warps' shares ---- */
    const int per = (int)((a.sequences + W * 32 - 1) / (W * 32)); /* sequences of a thread */
    const int b0 = (int)min((int64_t)tid * per, a.sequences), b1 = (int)min((int64_t)b0 + per, a.sequences);
    uint32_t mine = 0; /* slots of a tile, summed over the sequences: below 2^31 */
    int len = 0;
    for (int b = b0; b < b1; ++b) {
        Place p;
        len = length_of(w, b);
        enter(w, p, len);
        mine += p.slots;
    }
    uint32_t before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(kAllLanes, before, o);
        if (lane >= o) before += v;
    }
    if (lane == 31) s_sum[warp] = before;
    if (tid < W * 2) s_part[tid >> 1][tid & 1] = 0;
    __syncthreads();
    uint32_t sum = 0;
    before -= mine;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (i < warp) before += s_sum[i];
        sum += s_sum[i];
    }
    s_before[tid] = before;
    s_len[tid] = len;
    __syncthreads();
    /* Blocks have equal shares but for one slot, and so have a block's warps; few slots go to as many
     * blocks as have kLeast of them. */
    const int64_t total = sum * tiles;
    const int blocks = total < kBlocks * kLeast ? (int)(total + kLeast - 1) / kLeast : kBlocks;
    if ((int)blockIdx.x >= blocks) return;
    int64_t each, rest; /* slots of a block, blocks with one more */
    if (total >> 32) {
        each = total / blocks;
        rest = total - each * blocks;
    } else {
        each = (uint32_t)total / (uint32_t)blocks;
        rest = (uint32_t)total - (uint32_t)each * (uint32_t)blocks;
    }
    const int64_t from = blockIdx.x * each + min((int64_t)blockIdx.x, rest);
    const int64_t size = each + (blockIdx.x < rest);
    /* Lane i, in every warp: the border between warps i - 1 and i. */
    Place in;
    {
        const int64_t at = from + (size * min(lane, W)) / W;
        in.b = (int)a.sequences;
        in.kv = in.part = in.slot = in.slots = in.first = in.len = in.low = 0;
        if (at < total) {
            /* the thread whose sequences it lies in: the last one with before * tiles <= at */
            const uint32_t q = at >> 32 ? (uint32_t)(at / tiles) : (uint32_t)at / (uint32_t)tiles;
            int k = 0;
#pragma unroll
            for (int o = W * 16; o; o >>= 1)
                if (s_before[k + o] <= q) k += o;
            int b = k * per;
            int64_t x = at - s_before[k] * tiles;
            for (enter(w, in, per == 1 ? s_len[k] : length_of(w, b)); x >= in.slots * tiles;
                 enter(w, in, length_of(w, b))) {
                x -= in.slots * tiles;
                ++b;
            }
            in.b = b;
            const int tile = (int)(x >> 32 ? x / in.slots : (uint32_t)x / (uint32_t)in.slots);
            in.slot = (int)(x - (int64_t)tile * in.slots);
            in.kv = tile;
            if (w.row_tiles > 1) {
                in.kv = tile / w.row_tiles;
                in.part = tile - in.kv * w.row_tiles;
            }
        }
        if (warp == 0 && lane <= W) {
            s_at[lane] = in;
            s_id[lane] = in.slot ? ((int64_t)in.b * a.kv_heads + in.kv) * w.row_tiles + in.part : -1;
        }
    }
    int *const place_words = reinterpret_cast<int *>(&in); /* the warp's own */
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Place) / 4); ++i)
        place_words[i] = __shfl_sync(kAllLanes, place_words[i], warp);
    int count = (int)((size * (warp + 1)) / W - (size * warp) / W);

    /* ---- the warp's slots ---- */
    uint8_t *const ring = smem + warp * S::kWarpBytes;
    float *const held = reinterpret_cast<float *>(ring + STAGES * S::kStage); /* the first partial */
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    Place out = in; /* `in` is where the loads are, `out` where the products are */
    const uint8_t *const kc = static_cast<const uint8_t *>(a.k_cache);
    const uint8_t *const vc = static_cast<const uint8_t *>(a.v_cache);
    constexpr int ES = F8 ? 1 : 2;

    /* Each lane looks one key up, one slot ahead of the loads: its page's number, -1 if it is not there,
     * and its place in the page. */
    int to_load = count, page, place = 0;
    auto look_up = [&] {
        const int key = (in.first + in.slot) * kKeys + lane;
        page = -1;
        if (to_load > 0 && key < in.len && key >= in.low) {
            const int n = key / a.page_size;
            place = key - n * a.page_size;
            page = __ldcg(a.pages + (int64_t)in.b * a.pages_stride + n);
        }
    };
    auto advance = [&](Place &p) {
        if (++p.slot < p.slots) return;
        p.slot = 0;
        if (++p.part < w.row_tiles) return;
        p.part = 0;
        if (++p.kv < a.kv_heads) return;
        p.kv = 0;
        ++p.b;
        enter(w, p, length_of(w, p.b));
    };
    /* A slot's keys or values, 16 bytes a lane: neighbouring lanes take a row's pieces. */
    const uint64_t policy = passing();
    auto bring = [&](uint32_t to, const uint8_t *const *from, bool all, const uint8_t *any) {
        constexpr int CH = S::kRowBytes / 16;
        constexpr int SIDE = CH % 8 == 0 ? 8 : CH % 4 == 0 ? 4 : 2, ROWS = 32 / SIDE;
        static_assert(CH % SIDE == 0, "");
        const int c0 = lane % SIDE, r0 = lane / SIDE;
        to += r0 * S::kPitch + c0 * 16;
        if (all) {
#pragma unroll
            for (int i = 0; i < kKeys / ROWS; ++i) {
                const uint8_t *at = from[i * ROWS + r0] + c0 * 16;
#pragma unroll
                for (int c = 0; c < CH; c += SIDE)
                    cp_async(to + i * ROWS * S::kPitch + c * 16, at + c * 16, policy);
            }
        } else {
#pragma unroll 2
            for (int i = 0; i < kKeys / ROWS; ++i) {
                const uint8_t *at = from[i * ROWS + r0];
                const int bytes = at ? 16 : 0;
                at = (at ? at : any) + c0 * 16;
#pragma unroll
                for (int c = 0; c < CH; c += SIDE)
                    cp_async(to + i * ROWS * S::kPitch + c * 16, at + c * 16, bytes, policy);
            }
        }
    };
    bool due = false, whole = false; /* values are to be asked for; all of them are there */
    look_up();
    auto load_keys = [&](int stage) {
        due = to_load > 0;
        if (due) {
            const bool ok = page >= 0 && page < a.cache_pages;
            const uint32_t there = __ballot_sync(kAllLanes, ok);
            s_from[warp][0][lane] =
                ok ? kc + (page * a.k_page_stride + place * a.k_token_stride + in.kv * a.k_head_stride) * ES
                   : nullptr;
            s_from[warp][1][lane] =
                ok ? vc + (page * a.v_page_stride + place * a.v_token_stride + in.kv * a.v_head_stride) * ES
                   : nullptr;
            if (lane == 0) s_ok[warp][stage] = there;
            __syncwarp();
            whole = there == kAllLanes;
            bring(ring_at + stage * S::kStage, s_from[warp][0], whole, kc);
            --to_load;
            advance(in);
            look_up();
        }
        cp_commit();
    };
    auto load_values = [&](int stage) { /* of the slot whose keys have been asked for last */
        if (due) bring(ring_at + stage * S::kStage + kKeys * S::kPitch, s_from[warp][1], whole, vc);
        cp_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
        load_keys(i);
        load_values(i);
        __syncwarp();
    }

    uint32_t qf[MT][NT][2];
    float o[MT][NT][4], m[NT][2], l[NT][2];
    int hi_n[NT][2], hi_least = 0, hi_most = 0; /* keys below these are seen */
    /* Scores stay as the products leave them until they are exponents; a scale below 0 turns q round. */
    /* (the least that fp32 has, not 0: -inf marks what is not seen, and is to stay that) */
    const float unit = a.scale == 0.0f ? 1.0f : fmaxf(fabsf(a.scale) * kLog2e * a.k_scale, 1.4e-45f);
    const uint32_t q_and = a.scale == 0.0f ? 0u : 0xFFFFFFFFu, q_xor = a.scale < 0.0f ? 0x80008000u : 0u;

    auto start = [&] { /* a tile */
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const Row r = row_of(w, out.kv, out.part, nt * 8 + g, ROWS);
            const T *q = static_cast<const T *>(a.q) +
                         ((int64_t)out.b * a.new_tokens + r.token) * a.q_stride + (int64_t)r.head * D;
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
            if (a.scale <= 0.0f) {
#pragma unroll
                for (int k = 0; k < MT; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j) qf[k][nt][j] = (qf[k][nt][j] & q_and) ^ q_xor;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[nt][j] = -INFINITY;
                l[nt][j] = 0.0f;
                const Row s = row_of(w, out.kv, out.part, nt * 8 + 2 * t + j, ROWS);
                hi_n[nt][j] = out.len - a.new_tokens + 1 + min(s.token, a.new_tokens - 1);
            }
        }
        hi_least = out.len - a.new_tokens + 1 + row_of(w, 0, out.part, 0, ROWS).token;
        hi_most = out.len - a.new_tokens + 1 +
                  min(row_of(w, 0, out.part, ROWS - 1, ROWS).token, a.new_tokens - 1);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.0f;
    };
    /* l over the lanes that hold one row's keys, m in powers of two */
    auto sum_up = [&] {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) m[nt][j] *= unit;
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
        cp_wait<2 * STAGES - 1>();
        __syncwarp(); /* the keys are there for all lanes */
        const uint32_t at = ring_at + stage * S::kStage, ok = s_ok[warp][stage];
        float s[kHalves][NT][4];
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[h][nt][j] = 0.0f;
#pragma unroll
        for (int k = 0; k < MT; k += F8 ? 2 : 1) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                uint32_t r[4];
                ldmatrix(r, at + k_row + h * 16 * S::kPitch + k * (F8 ? 16 : 32));
                if constexpr (F8) {
                    const uint32_t f0[4] = {widen(T(), r[0]), widen(T(), r[1]), widen(T(), r[0] >> 16),
                                            widen(T(), r[1] >> 16)};
                    const uint32_t f1[4] = {widen(T(), r[2]), widen(T(), r[3]), widen(T(), r[2] >> 16),
                                            widen(T(), r[3] >> 16)};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma<T>(s[h][nt], f0, qf[k][nt][0], qf[k][nt][1]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma<T>(s[h][nt], f1, qf[k + 1][nt][0], qf[k + 1][nt][1]);
                } else {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma<T>(s[h][nt], r, qf[k][nt][0], qf[k][nt][1]);
                }
            }
        }
        __syncwarp(); /* all lanes have read them */
        load_keys(stage);

        /* -inf for keys that a row does not see */
        const int base = (out.first + out.slot) * kKeys;
        /* keys that are there, but not for every row of the tile (one token's rows all see the same) */
        const bool mixed = a.new_tokens > 1 && ((base + kKeys > hi_least && base < out.len) ||
                                                (a.window > 0 && base < hi_most - a.window));
        const bool some = ok != 0xFFFFFFFFu || base + kKeys > hi_least ||
                          (a.window > 0 && base < hi_most - a.window);
        if (some) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = h * 16 + g + (j >> 1) * 8, key = base + i, top = hi_n[nt][j & 1];
                        const bool seen = (ok >> i & 1u) && key < top &&
                                          (a.window <= 0 || key >= top - a.window);
                        if (!seen) s[h][nt][j] = -INFINITY;
                    }
        }
        bool rise = false;
        float f[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float top = fmaxf(s[0][nt][j], s[0][nt][j + 2]);
#pragma unroll
                for (int h = 1; h < kHalves; ++h)
                    top = fmaxf(top, fmaxf(s[h][nt][j], s[h][nt][j + 2]));
                f[nt][j] = top;
            }
#pragma unroll
        for (int x = 4; x < 32; x <<= 1)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    f[nt][j] = fmaxf(f[nt][j], __shfl_xor_sync(kAllLanes, f[nt][j], x));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float top = fmaxf(f[nt][j], m[nt][j]);
                const float ref = top == -INFINITY ? 0.0f : top * unit;
                f[nt][j] = exp2_fast(m[nt][j] * unit - ref);
                rise |= top > m[nt][j];
                m[nt][j] = top;
                float sum = 0.0f;
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    s[h][nt][j] = exp2_fast(fmaf(s[h][nt][j], unit, kUp<P> - ref));
                    s[h][nt][j + 2] = exp2_fast(fmaf(s[h][nt][j + 2], unit, kUp<P> - ref));
                    sum += s[h][nt][j] + s[h][nt][j + 2];
                }
                l[nt][j] = l[nt][j] * f[nt][j] + sum;
            }
        if (__any_sync(kAllLanes, rise)) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[i][nt][j] *= f[nt][j & 1];
        }
        /* Values of 8 bits for a result in bf16: fp16's 11 bits of a probability do. */
        constexpr bool TWO = !F8 || std::is_same<T, __half>::value;
        uint32_t p[kHalves][NT][2][2];
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float x = s[h][nt][2 * j], y = s[h][nt][2 * j + 1];
                    uint32_t low;
                    const uint32_t high = TWO ? split(P(), x, y, low) : pack2(P(), x, y);
                    p[h][nt][j][0] = transposed(high);
                    p[h][nt][j][1] = TWO ? transposed(low) : 0;
                }
        auto values = [&](int i, int h, uint32_t (&v)[4], uint32_t (&r)[4]) { /* V^T of 16 dims */
            const uint32_t from = at + v_row + h * 16 * S::kPitch;
            if constexpr (F8) {
                if (i % 2 == 0) ldmatrix_trans(r, from + i * 16);
                const uint32_t r0 = r[i % 2 * 2], r1 = r[i % 2 * 2 + 1];
                const uint32_t x0 = widen(P(), r0), y0 = widen(P(), r0 >> 16);
                const uint32_t x1 = widen(P(), r1), y1 = widen(P(), r1 >> 16);
                v[0] = __byte_perm(x0, y0, 0x5410); /* row g: dim 2 g, row g + 8: dim 2 g + 1 */
                v[1] = __byte_perm(x0, y0, 0x7632);
                v[2] = __byte_perm(x1, y1, 0x5410);
                v[3] = __byte_perm(x1, y1, 0x7632);
            } else {
                ldmatrix_trans(v, from + i * 32);
            }
        };
        cp_wait<2 * STAGES - 1>();
        __syncwarp();
        uint32_t r[kHalves][4] = {};
        /* 0 times a value that a row does not see is 0, unless that is an infinity or NaN */
        if (!mixed || !any_special<T, F8>(at + kKeys * S::kPitch, lane, S::kRowBytes / 16, S::kPitch)) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    uint32_t v[4];
                    values(i, h, v, r[h]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma<P>(o[i][nt], v, p[h][nt][0][0], p[h][nt][1][0]);
                        if (TWO) mma<P>(o[i][nt], v, p[h][nt][0][1], p[h][nt][1][1]);
                    }
                }
        } else {
            /* token by token, with the values that it does not see taken out */
            for (int top = hi_least; top <= hi_most; ++top)
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    uint32_t mask[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int key = base + h * 16 + j * 8 + 2 * t;
                        const bool x = key < top && (a.window <= 0 || key >= top - a.window);
                        const bool y = key + 1 < top && (a.window <= 0 || key + 1 >= top - a.window);
                        mask[j] = (x ? 0x0000FFFFu : 0u) | (y ? 0xFFFF0000u : 0u);
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        uint32_t v[4];
                        values(i, h, v, r[h]);
                        v[0] &= mask[0];
                        v[1] &= mask[0];
                        v[2] &= mask[1];
                        v[3] &= mask[1];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float c[4] = {};
                            mma<P>(c, v, p[h][nt][0][0], p[h][nt][1][0]);
                            if (TWO) mma<P>(c, v, p[h][nt][0][1], p[h][nt][1][1]);
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (hi_n[nt][j & 1] == top) o[i][nt][j] += c[j];
                        }
                    }
                }
        }
        __syncwarp();
        load_values(stage);
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
                const Finish<T, NT, F8> to(w, out.b, out.kv, out.part, lane, true, m, l);
#pragma unroll
                for (int i = 0; i < MT; ++i) to.write(i * 16, lane, o[i]);
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
    __syncthreads();

    /* ---- tiles that several warps have worked on ----
     * Borders inside the same tile make a group; groups go to the warps, the dims of one to as many warps
     * as there are for it. */
    {
        const int64_t id = lane <= W ? s_id[lane] : -1;
        const uint32_t same = __match_any_sync(kAllLanes, id);
        const uint32_t first_of = __ballot_sync(kAllLanes, id >= 0 && lane == __ffs(same) - 1);
        const uint32_t held0 = __ballot_sync(kAllLanes, lane < W && s_part[min(lane, W - 1)][0]);
        const uint32_t held1 = __ballot_sync(kAllLanes, lane < W && s_part[min(lane, W - 1)][1]);
        const int groups = __popc(first_of);
        int split = W; /* warps of a group, a power of two */
        while (split > 1 && (split * groups > W || split > MT)) split >>= 1;
        for (int n = warp / split; n < groups; n += W / split) {
            const int e = __fns(first_of, 0, n + 1);
            const int last = 31 - __clz(__shfl_sync(kAllLanes, same, e));
            const bool outside = e == 0 || last == W;
            Joined<MT, NT> all;
            for (int x = max(e - 1, 0); x <= min(last, W - 1); ++x) {
                /* the warp in which the tile begins holds it as its last */
                const bool begins = x < e;
                if (!((begins ? held1 : held0) >> x & 1u)) continue;
                all.add(reinterpret_cast<const float *>(smem + x * S::kWarpBytes +
                                                        (begins ? 0 : STAGES * S::kStage)),
                        warp & (split - 1), split - 1, lane);
            }
            if (!outside) {
                const Place p = s_at[e];
                const Finish<T, NT, F8> to(w, p.b, p.kv, p.part, lane, (warp & (split - 1)) == 0, all.top,
                                           all.sum);
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    if ((i & (split - 1)) == (warp & (split - 1))) to.write(i * 16, lane, all.c[i]);
                continue;
            }
            float *to = w.parts + (int64_t)(blockIdx.x * 2 + (e == 0 ? 0 : 1)) * S::kFloats;
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if ((i & (split - 1)) == (warp & (split - 1))) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        reinterpret_cast<float4 *>(to)[(i * NT + nt) * 32 + lane] = make_float4(
                            all.c[i][nt][0], all.c[i][nt][1], all.c[i][nt][2], all.c[i][nt][3]);
                }
            if ((warp & (split - 1)) == 0 && g == 0) {
                float *ml = to + MT * NT * 128;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        ml[nt * 8 + 2 * t + j] = all.top[nt][j];
                        ml[ROWS + nt * 8 + 2 * t + j] = all.sum[nt][j];
                    }
            }
        }
    }

    /* ---- tiles that several blocks have worked on ----
     * A block says that its part is there, and looks whether all others of the tile's are: the last one
     * finds them, and joins (so may several that come at a time: they write the same).  Its mark is this
     * call's own number, which nothing else in the workspace holds, and is taken back by whoever joins,
     * when all have been set, so that the next call (or the next run of a captured one) finds none. */
    const bool outer[2] = {s_id[0] >= 0, s_id[W] >= 0 && s_id[W] != s_id[0]};
    if (!outer[0] && !outer[1]) return;
    __syncthreads();
    if (warp < 2 && outer[warp]) {
        /* the tile's slots are those from `begin` on; lane 0: its first block, lane 1: its last */
        const Place &p = s_at[warp * W];
        const int64_t begin = from + (warp ? size : 0) - p.slot;
        const int64_t x = lane == 0 ? begin : begin + p.slots - 1, big = rest * (each + 1);
        int block;
        if (total >> 32)
            block = (int)(x < big ? x / (each + 1) : rest + (x - big) / each);
        else
            block = x < big ? (uint32_t)x / (uint32_t)(each + 1)
                            : (uint32_t)rest + (uint32_t)(x - big) / (uint32_t)each;
        const int f = __shfl_sync(kAllLanes, block, 0), l = __shfl_sync(kAllLanes, block, 1);
        if (lane == 0) {
            __threadfence(); /* the block's partials before its mark */
            __stcg(w.marks + blockIdx.x * 2 + warp, w.number);
            __threadfence(); /* its mark before the look at the others' */
        }
        __syncwarp();
        bool all = true;
        for (int y = f + lane; y <= l; y += 32) {
            unsigned long long mark;
            asm volatile("ld.acquire.gpu.global.u64 %0, [%1];"
                         : "=l"(mark)
                         : "l"(w.marks + y * 2 + (y == f ? 1 : 0))
                         : "memory");
            all &= mark == w.number;
        }
        all = __all_sync(kAllLanes, all);
        if (lane == 0) {
            s_join[warp][0] = all;
            s_join[warp][1] = f;
            s_join[warp][2] = l - f + 1;
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        if (!outer[which] || !s_join[which][0]) continue;
        const int f = s_join[which][1], parts = s_join[which][2];
        const Place p = s_at[which * W];
        for (int i = warp; i < MT; i += W) {
            constexpr int AHEAD = 8 / NT; /* parts that are asked for at a time */
            float c[NT][4], top[NT][2], sum[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    top[nt][j] = -INFINITY;
                    sum[nt][j] = c[nt][j] = c[nt][j + 2] = 0.0f;
                }
            for (int x0 = 0; x0 < parts; x0 += AHEAD) {
                float4 q[AHEAD][NT];
                float2 m1[AHEAD][NT], l1[AHEAD][NT];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int x = x0 + k;
                    const float *part =
                        w.parts + (int64_t)((f + x) * 2 + (x == 0 ? 1 : 0)) * S::kFloats;
                    const float *ml = part + MT * NT * 128;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        q[k][nt] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        m1[k][nt] = make_float2(-INFINITY, -INFINITY);
                        l1[k][nt] = make_float2(0.0f, 0.0f);
                        if (x < parts) {
                            q[k][nt] = __ldcg(reinterpret_cast<const float4 *>(part) +
                                              (i * NT + nt) * 32 + lane);
                            m1[k][nt] = __ldcg(reinterpret_cast<const float2 *>(ml + nt * 8 + 2 * t));
                            l1[k][nt] =
                                __ldcg(reinterpret_cast<const float2 *>(ml + ROWS + nt * 8 + 2 * t));
                        }
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float both = top[nt][j];
#pragma unroll
                        for (int k = 0; k < AHEAD; ++k) both = fmaxf(both, j ? m1[k][nt].y : m1[k][nt].x);
                        const float f0 = shrink(top[nt][j], both);
                        top[nt][j] = both;
                        sum[nt][j] *= f0;
                        c[nt][j] *= f0;
                        c[nt][j + 2] *= f0;
#pragma unroll
                        for (int k = 0; k < AHEAD; ++k) {
                            const float f1 = shrink(j ? m1[k][nt].y : m1[k][nt].x, both);
                            sum[nt][j] += (j ? l1[k][nt].y : l1[k][nt].x) * f1;
                            c[nt][j] += (j ? q[k][nt].y : q[k][nt].x) * f1;
                            c[nt][j + 2] += (j ? q[k][nt].w : q[k][nt].z) * f1;
                        }
                    }
            }
            const Finish<T, NT, F8> to(w, p.b, p.kv, p.part, lane, i == 0, top, sum);
            to.write(i * 16, lane, c);
        }
        if (warp == 0)
            for (int x = lane; x < parts; x += 32)
                __stcg(w.marks + (f + x) * 2 + (x == 0 ? 1 : 0), 0ull);
    }
}

template <typename T, int D, int NT, bool F8> cudaError_t launch(const Work &w, cudaStream_t stream)
{
    using S = Shape<D, NT, F8>;
    const void *fn = reinterpret_cast<const void *>(&cfa_attend_kernel<T, D, NT, F8>);
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_shared(fn, S::kSmem, done);
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
    return cudaLaunchKernelExC(&cfg, fn, p);
}

template <typename T, bool F8> cudaError_t launch_any(const Work &w, cudaStream_t stream)
{
    const int nt = w.nt;
    switch (w.a.head_dim) {
    case 64: return nt == 1 ? launch<T, 64, 1, F8>(w, stream) : launch<T, 64, 2, F8>(w, stream);
    case 96: return nt == 1 ? launch<T, 96, 1, F8>(w, stream) : launch<T, 96, 2, F8>(w, stream);
    case 128: return nt == 1 ? launch<T, 128, 1, F8>(w, stream) : launch<T, 128, 2, F8>(w, stream);
    case 256: return launch<T, 256, 1, F8>(w, stream);
    default: return cudaErrorInvalidValue; /* refused before */
    }
}

} // namespace cfa_attend_dev
