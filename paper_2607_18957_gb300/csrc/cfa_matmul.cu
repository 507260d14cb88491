/*
 * y = act(x w^T + bias) + residual, for one weight or for a stack of them (cfa_matmul), on the
 * tensor cores (tcgen05).
 *
 * The weight's rows lie along the accumulator's lanes (M, 128 per SM) and the tokens along its
 * columns (N, 16 to 256).  So a few tokens cost a few columns while the weight streams through at
 * memory speed, ragged groups only shorten N, and a warp of the epilogue holds 32 neighbouring
 * output columns of one token, which it stores side by side.
 *
 * A CTA has six warps: four for the epilogue (each owns 32 lanes of tensor memory), one that asks
 * the TMA for tiles of 64 columns of w and x, and one that issues the products.  Tiles come in a ring
 * of shared-memory stages; the accumulator is double buffered, so that the epilogue of one output
 * tile runs under the products of the next.  CTAs are persistent and take output tiles in turn.
 *
 * PAIR: two CTAs work on one tile of 256 weight rows (cta_group::2): each holds half of the rows and
 * half of the tokens, so each operand is loaded once per pair.
 * split: with few output tiles a cluster of CTAs shares one, each over its part of the columns of w;
 * the partial sums meet in shared memory and are added in the order of the CTAs.
 * Gated: the stage holds 16 gate rows, then the 16 up rows that belong to them, and so on, so both
 * values of an output lie in one warp, 16 lanes apart.
 *
 * Every wait has a limit.  One that runs out sets the status word that cfa_op_status reads; its CTA
 * then issues nothing more, lets its loads in flight end (again with a limit) and frees its tensor
 * memory.
 */
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "cfa_device.cuh"
#include "cfa_ops.h"

namespace {

constexpr int kThreads = 192;
constexpr int kLoader = 4, kIssuer = 5;  /* warps; 0 to 3 are the epilogue's */
constexpr uint32_t kRows = 128;          /* weight rows per CTA */
constexpr uint32_t kDepth = 64;          /* columns of w and x per stage: one 128-byte swizzle row */
constexpr uint32_t kRowBytes = kDepth * 2;
constexpr uint32_t kMaxStages = 12;
constexpr uint32_t kSmem = 232448;       /* all that a CTA may have: one CTA per SM, so that the
                                            tensor memory is never asked for twice at once */
constexpr uint32_t kBand = 16;           /* token tiles that share a weight tile in turn */
constexpr uint32_t kSpinLimit = 1u << 20;    /* polls of a wait */
constexpr uint32_t kDrainLimit = 1u << 16;   /* polls for loads in flight after one ran out */

struct Args {
    CUtensorMap wmap, xmap;
    cfa_matmul m;
    int64_t outs;        /* columns of y */
    uint32_t bn;         /* token tile */
    uint32_t stages;
    uint32_t steps;      /* of kDepth columns */
    uint32_t f_tiles;    /* feature tiles per group */
    uint32_t split;      /* CTAs per output tile along the columns */
    uint32_t tmem_cols;
    uint32_t release;
};

__device__ int g_status; /* 1: a wait ran out, 2: and so did the wait for the loads in flight */

/* What precedes the stages in shared memory. */
struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem;
    int dead;
    int32_t total; /* output tiles */
    int32_t first[CFA_EXPERTS_MAX + 1]; /* output tiles before each group's */
    int32_t row[CFA_EXPERTS_MAX + 1];   /* rows of x before each group's */
};

__device__ __forceinline__ uint32_t smem_addr(const void *p)
{
    return (uint32_t)__cvta_generic_to_shared(p);
}

__device__ __forceinline__ void mbar_init(uint64_t *bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count)
                 : "memory");
}

__device__ __forceinline__ void mbar_expect_tx(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)),
                 "r"(bytes)
                 : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint64_t *bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done)
                 : "r"(smem_addr(bar)), "r"(parity)
                 : "memory");
    return done != 0;
}

/* Waits for phase `parity`; false if the limit ran out here or in another warp of the CTA. */
__device__ __forceinline__ bool mbar_wait(uint64_t *bar, uint32_t parity, Shared *s)
{
    for (uint32_t k = 0; k < kSpinLimit; ++k) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((k & 1023u) == 1023u && *(volatile int *)&s->dead) return false;
    }
    *(volatile int *)&s->dead = 1;
    return false;
}

/* The address of the same variable in CTA `rank` of the cluster. */
__device__ __forceinline__ uint32_t map_to(uint32_t addr, uint32_t rank)
{
    uint32_t out;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"(addr), "r"(rank));
    return out;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

template <bool PAIR>
__device__ __forceinline__ void load_w(uint32_t dst, const CUtensorMap *map, int32_t k, int32_t row,
                                       int32_t group, uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                     "l"(map), "r"(k), "r"(row), "r"(group), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                     "l"(map), "r"(k), "r"(row), "r"(group), "r"(bar)
                     : "memory");
}

template <bool PAIR>
__device__ __forceinline__ void load_gated(uint32_t dst, const CUtensorMap *map, int32_t k,
                                           int32_t row, int32_t group, uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                     "l"(map), "r"(k), "r"(row), "r"(0), "r"(group), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                     "l"(map), "r"(k), "r"(row), "r"(0), "r"(group), "r"(bar)
                     : "memory");
}

template <bool PAIR>
__device__ __forceinline__ void load_x(uint32_t dst, const CUtensorMap *map, int32_t k, int32_t row,
                                       uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(k), "r"(row), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(k), "r"(row), "r"(bar)
                     : "memory");
}

/* Shared-memory matrix of rows of 128 bytes, 128-byte swizzle, 8-row groups 1024 bytes apart. */
__device__ __forceinline__ uint64_t matrix(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

/* fp32 accumulator, both operands bf16 or both f16, rows of the contraction contiguous. */
__device__ __forceinline__ uint32_t instruction(int f16, uint32_t m, uint32_t n)
{
    const uint32_t type = f16 ? 0u : 1u;
    return (1u << 4) | (type << 7) | (type << 10) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t inst, uint32_t add)
{
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                     "l"(a), "l"(b), "r"(inst), "r"(add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                     "l"(a), "l"(b), "r"(inst), "r"(add)
                     : "memory");
}

/* Arrives on the barrier (of both CTAs of a pair) once all products issued so far are done. */
template <bool PAIR> __device__ __forceinline__ void commit(uint64_t *bar)
{
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster"
                     ".multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)), "h"((uint16_t)3)
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster"
                     ".b64 [%0];" ::"r"(smem_addr(bar))
                     : "memory");
}

__device__ __forceinline__ void fence_before()
{
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void fence_after()
{
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

/* 16 columns of the warp's 32 lanes. */
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[16])
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                   "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ float value(const void *p, int64_t i, int f16)
{
    return f16 ? __half2float(static_cast<const __half *>(p)[i])
               : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ float activate(float v, int act)
{
    switch (act) {
    case CFA_ACT_RELU: return v < 0.0f ? 0.0f : v;
    case CFA_ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
    case CFA_ACT_GELU_TANH:
        return 0.5f * v * (1.0f + tanhf(0.79788456080286536f * (v + 0.044715f * v * v * v)));
    case CFA_ACT_SILU: return v / (1.0f + expf(-v));
    default: return v;
    }
}

/* One output tile: group, first weight feature of the CTA (pair), first row of x, rows. */
struct Tile {
    int32_t group, row, rows;
    int64_t feature;
};

/* Tiles are numbered group after group; within a group in bands of kBand token tiles, in a band
 * feature after feature, so that neighbours in time share the weight tile and the tokens of a band
 * stay in L2. */
__device__ __forceinline__ Tile tile_at(const Args &a, const Shared *s, int32_t t, int32_t *group,
                                        uint32_t features)
{
    int32_t g = *group;
    while (t >= s->first[g + 1]) ++g;
    *group = g;
    const uint32_t local = (uint32_t)(t - s->first[g]);
    const int32_t rows = s->row[g + 1] - s->row[g];
    const uint32_t tiles = ((uint32_t)rows + a.bn - 1) / a.bn;
    const uint32_t band = local / (kBand * a.f_tiles), rest = local - band * kBand * a.f_tiles;
    const uint32_t left = tiles - band * kBand, width = left < kBand ? left : kBand;
    const uint32_t f = rest / width, n = band * kBand + rest % width;
    Tile o;
    o.group = g;
    o.feature = (int64_t)f * features;
    o.row = s->row[g] + (int32_t)(n * a.bn);
    o.rows = min((int32_t)a.bn, rows - (int32_t)(n * a.bn));
    return o;
}

/* Stores up to 16 tokens' values of one output column: activation, bias, residual, rounding.
 * Gated: lanes 0-15 hold gate values and lanes 16-31 the up values of the same 16 columns; of two
 * tokens the lower half finishes the first and the upper half the second. */
template <bool GATED>
__device__ __forceinline__ void finish(const Args &a, float (&v)[16], int64_t row, int n, int64_t col,
                                       bool in, float bias, float bias_up)
{
    const cfa_matmul &m = a.m;
    if constexpr (GATED) {
        const bool upper = threadIdx.x & 16;
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            if (j >= n) break;
            const float give = upper ? v[j] : v[j + 1];
            const float got = __shfl_xor_sync(0xFFFFFFFFu, give, 16);
            const float gate = upper ? got : v[j], up = upper ? v[j + 1] : got;
            const int mine = j + (upper ? 1 : 0);
            if (!in || mine >= n) continue;
            float o = activate(gate + bias, m.act) * (up + bias_up);
            if (m.residual) {
                const int64_t at = (row + mine) * m.r_stride + col;
                o += m.y_f32 ? static_cast<const float *>(m.residual)[at]
                             : value(m.residual, at, m.f16);
            }
            const int64_t at = (row + mine) * m.y_stride + col;
            if (m.y_f32) static_cast<float *>(m.y)[at] = o;
            else if (m.f16) static_cast<__half *>(m.y)[at] = __float2half_rn(o);
            else static_cast<__nv_bfloat16 *>(m.y)[at] = __float2bfloat16_rn(o);
        }
    } else {
        if (!in) return;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if (j >= n) break;
            float o = activate(v[j] + bias, m.act);
            if (m.residual) {
                const int64_t at = (row + j) * m.r_stride + col;
                o += m.y_f32 ? static_cast<const float *>(m.residual)[at]
                             : value(m.residual, at, m.f16);
            }
            const int64_t at = (row + j) * m.y_stride + col;
            if (m.y_f32) static_cast<float *>(m.y)[at] = o;
            else if (m.f16) static_cast<__half *>(m.y)[at] = __float2half_rn(o);
            else static_cast<__nv_bfloat16 *>(m.y)[at] = __float2bfloat16_rn(o);
        }
    }
}

/* After a wait that ran out: lets the loads in flight end, as far as a limit allows.  Of a pair, the
 * first CTA's barriers count the loads of both; the second only gives its own the same time. */
__device__ void drain(const Args &a, Shared *s, uint32_t issued, bool second)
{
    int word = 1;
    const uint32_t most = issued < a.stages ? issued : a.stages;
    for (uint32_t l = issued - most; l < issued; ++l) {
        bool done = false;
        for (uint32_t k = 0; !done && k < kDrainLimit; ++k)
            done = mbar_try_wait(s->full + l % a.stages, (l / a.stages) & 1u);
        if (!done && !second) word = 2;
    }
    atomicMax(&g_status, word);
}

template <bool PAIR, bool GATED>
__global__ void __launch_bounds__(kThreads, 1) cfa_matmul_kernel(const __grid_constant__ Args a)
{
    extern __shared__ uint8_t raw[];
    Shared *s = reinterpret_cast<Shared *>(raw);
    const uint32_t ring = (smem_addr(raw) + (uint32_t)sizeof(Shared) + 1023u) & ~1023u;
    const uint32_t x_rows = PAIR ? a.bn / 2 : a.bn;
    const uint32_t w_bytes = kRows * kRowBytes, x_bytes = x_rows * kRowBytes;
    const uint32_t stage = w_bytes + x_bytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool cluster = PAIR || a.split > 1;
    const uint32_t rank = cluster ? cluster_rank() : 0;
    const uint32_t ctas = PAIR ? 2 : a.split; /* that share a tile */
    const uint32_t features = (PAIR ? 2 : 1) * (GATED ? kRows / 2 : kRows);
    const cfa_matmul &m = a.m;

    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < a.stages; ++i) {
            mbar_init(s->full + i, 1);
            mbar_init(s->empty + i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s->acc_full + i, 1);
            mbar_init(s->acc_empty + i, PAIR ? 8 : 4);
        }
        s->dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuer) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                             smem_addr(&s->tmem)),
                         "r"(a.tmem_cols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                             smem_addr(&s->tmem)),
                         "r"(a.tmem_cols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.release) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 0) { /* the groups' rows and tiles */
        int32_t tiles = 0;
        for (int32_t g0 = 0; g0 < m.n_groups; g0 += 32) {
            const int32_t g = g0 + lane;
            int32_t r0 = 0, r1 = 0, n = 0;
            if (g < m.n_groups) {
                r0 = m.offs ? m.offs[g] : 0;
                r1 = m.offs ? m.offs[g + 1] : (int32_t)m.tokens;
                n = (int32_t)(((uint32_t)(r1 - r0) + a.bn - 1) / a.bn * a.f_tiles);
            }
            int32_t sum = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int32_t before = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= o) sum += before;
            }
            if (g < m.n_groups) {
                s->first[g] = tiles + sum - n;
                s->row[g] = r0;
                s->row[g + 1] = r1;
            }
            tiles += __shfl_sync(0xFFFFFFFFu, sum, 31);
            __syncwarp();
        }
        if (lane == 0) s->first[m.n_groups] = s->total = tiles;
    }
    fence_before();
    __syncthreads();
    if (cluster) cluster_sync();
    fence_after();
    const uint32_t tmem = s->tmem;
    const int32_t total = s->total;
    const int32_t stride = (int32_t)(gridDim.x / ctas), begin = (int32_t)(blockIdx.x / ctas);
    /* this CTA's part of the columns */
    const uint32_t k0 = PAIR ? 0 : rank * a.steps / a.split;
    const uint32_t k1 = PAIR ? a.steps : (rank + 1) * a.steps / a.split;
    const bool sync_tiles = !PAIR && a.split > 1;
    bool ok = true;

    if (warp == kLoader) {
        uint32_t at = 0, phase = 1; /* stage; an empty ring counts as released once */
        uint32_t issued = 0;
        int32_t group = 0;
        if (lane == 0) asm volatile("fence.proxy.async.global;" ::: "memory");
        for (int32_t t = begin; t < total; t += stride) {
            if (lane == 0) {
                const Tile o = tile_at(a, s, t, &group, features);
                /* rows of x for this CTA: of a pair, each holds half of the columns in use */
                uint32_t half = 0;
                if constexpr (PAIR) half = rank * (((uint32_t)o.rows + 31u) / 32u * 16u);
                const int32_t row = o.row + (int32_t)half;
                const int32_t f = (int32_t)o.feature + (int32_t)(rank * (GATED ? 64u : 128u)) *
                                                           (PAIR ? 1 : 0);
                for (uint32_t k = k0; k < k1; ++k) {
                    ok = ok && mbar_wait(s->empty + at, phase, s);
                    if (!ok) break;
                    const uint32_t dst = ring + at * stage;
                    uint32_t bar = smem_addr(s->full + at);
                    if constexpr (PAIR) bar = map_to(bar, 0);
                    if (!PAIR || rank == 0)
                        mbar_expect_tx(s->full + at, PAIR ? 2 * stage : stage);
                    const int32_t c = (int32_t)(k * kDepth);
                    if constexpr (GATED) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            load_gated<PAIR>(dst + q * 32 * kRowBytes, &a.wmap, c, f + 16 * q,
                                             o.group, bar);
                    } else {
                        load_w<PAIR>(dst, &a.wmap, c, f, o.group, bar);
                    }
                    load_x<PAIR>(dst + w_bytes, &a.xmap, c, row, bar);
                    ++issued;
                    if (++at == a.stages) {
                        at = 0;
                        phase ^= 1;
                    }
                }
            }
            __syncwarp();
            if (sync_tiles) {
                cluster_sync();
                cluster_sync();
            }
        }
        if (lane == 0 && *(volatile int *)&s->dead) drain(a, s, issued, PAIR && rank);
    } else if (warp == kIssuer) {
        const bool issues = lane == 0 && (!PAIR || rank == 0);
        uint32_t at = 0, phase = 0, buf = 0, buf_phase = 1;
        int32_t group = 0;
        for (int32_t t = begin; t < total; t += stride) {
            if (issues) {
                const Tile o = tile_at(a, s, t, &group, features);
                const uint32_t unit = PAIR ? 32u : 16u;
                const uint32_t inst = instruction(m.f16, PAIR ? 256u : 128u,
                                                  ((uint32_t)o.rows + unit - 1) / unit * unit);
                const uint32_t d = tmem + buf * a.bn;
                ok = ok && mbar_wait(s->acc_empty + buf, buf_phase, s);
                fence_after();
                for (uint32_t k = k0; k < k1; ++k) {
                    ok = ok && mbar_wait(s->full + at, phase, s);
                    if (!ok) break;
                    fence_after();
                    const uint32_t src = ring + at * stage;
                    const uint64_t da = matrix(src), db = matrix(src + w_bytes);
#pragma unroll
                    for (uint32_t q = 0; q < kDepth / 16; ++q) /* 32 bytes further in the row */
                        mma<PAIR>(d, da + q * 2, db + q * 2, inst, k > k0 || q > 0);
                    commit<PAIR>(s->empty + at);
                    if (++at == a.stages) {
                        at = 0;
                        phase ^= 1;
                    }
                }
                if (ok) commit<PAIR>(s->acc_full + buf);
                if (buf) buf_phase ^= 1;
                buf ^= 1;
            }
            __syncwarp();
            if (sync_tiles) {
                cluster_sync();
                cluster_sync();
            }
        }
    } else {
        uint32_t buf = 0, buf_phase = 0;
        int32_t group = 0;
        const uint32_t lanes = (uint32_t)warp * 32u << 16;
        float *partial = reinterpret_cast<float *>(
            raw + (ring - smem_addr(raw)) + a.stages * stage); /* [bn][128], split > 1 */
        for (int32_t t = begin; t < total; t += stride) {
            const Tile o = tile_at(a, s, t, &group, features);
            int64_t col = o.feature + (GATED ? warp * 16 + (lane & 15) : warp * 32 + lane);
            if constexpr (PAIR) col += rank * (GATED ? 64 : 128);
            const bool in = col < a.outs;
            float bias = 0.0f, bias_up = 0.0f;
            if (m.bias && in) {
                bias = m.bias_f32 ? static_cast<const float *>(m.bias)[col]
                                  : value(m.bias, col, m.f16);
                if (GATED)
                    bias_up = m.bias_f32 ? static_cast<const float *>(m.bias)[a.outs + col]
                                         : value(m.bias, a.outs + col, m.f16);
            }
            ok = ok && mbar_wait(s->acc_full + buf, buf_phase, s);
            ok = __all_sync(0xFFFFFFFFu, ok);
            fence_after();
            const uint32_t src = tmem + lanes + buf * a.bn;
            float v[16];
            if (!sync_tiles) {
                for (int32_t c = 0; ok && c < o.rows; c += 16) {
                    __syncwarp();
                    tmem_load(src + c, v);
                    finish<GATED>(a, v, o.row + c, o.rows - c, col, in, bias, bias_up);
                }
            } else {
                for (int32_t c = 0; ok && c < o.rows; c += 16) {
                    tmem_load(src + c, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        partial[(c + j) * kRows + warp * 32 + lane] = v[j];
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) {
                const uint32_t bar = smem_addr(s->acc_empty + buf);
                asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                                 PAIR ? map_to(bar, 0) : bar)
                             : "memory");
            }
            if (buf) buf_phase ^= 1;
            buf ^= 1;
            if (sync_tiles) {
                cluster_sync();
                /* each CTA of the cluster finishes its share of the tokens */
                const uint32_t share = (((uint32_t)o.rows + a.split - 1) / a.split + 1u) & ~1u;
                const int32_t c0 = (int32_t)(rank * share);
                const int32_t c1 = min(o.rows, c0 + (int32_t)share);
                const uint32_t base = smem_addr(partial) + (uint32_t)(warp * 32 + lane) * 4u;
                for (int32_t c = c0; ok && c < c1; c += 16) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = 0.0f;
                    for (uint32_t r = 0; r < a.split; ++r) {
                        const uint32_t from = map_to(base, r);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float p = 0.0f;
                            if (c + j < c1)
                                asm volatile("ld.shared::cluster.f32 %0, [%1];"
                                             : "=f"(p)
                                             : "r"(from + (uint32_t)(c + j) * (kRows * 4u)));
                            v[j] += p;
                        }
                    }
                    finish<GATED>(a, v, o.row + c, c1 - c, col, in, bias, bias_up);
                }
                cluster_sync();
            }
        }
    }

    fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *(volatile int *)&s->dead) atomicMax(&g_status, 1);
    if (cluster) cluster_sync();
    if (warp == kIssuer) {
        if constexpr (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                         "r"(a.tmem_cols));
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                         "r"(a.tmem_cols));
    }
}

/* ---- host ---- */

struct Device {
    std::atomic<int> sms;          /* 0: not asked yet */
    std::atomic<int> clusters[2][9]; /* by gated and split: clusters that run at once, plus one */
    std::atomic<unsigned> ready;   /* kernels whose shared memory is granted */
};
constexpr int kMaxDevices = 64;
Device g_device[kMaxDevices];

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                             const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder()
{
    static std::atomic<void *> fn{nullptr};
    void *p = fn.load();
    if (!p) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000,
                                             cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        fn.store(p);
    }
    return reinterpret_cast<EncodeFn>(p);
}

bool encode(CUtensorMap *map, int f16, const void *base, int rank, const cuuint64_t *dim,
            const cuuint64_t *stride, const cuuint32_t *box)
{
    const cuuint32_t one[5] = {1, 1, 1, 1, 1};
    const EncodeFn fn = encoder();
    return fn && fn(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                    (cuuint32_t)rank, const_cast<void *>(base), dim, stride, box, one,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

const void *kernel_of(bool pair, bool gated)
{
    if (pair)
        return gated ? reinterpret_cast<const void *>(&cfa_matmul_kernel<true, true>)
                     : reinterpret_cast<const void *>(&cfa_matmul_kernel<true, false>);
    return gated ? reinterpret_cast<const void *>(&cfa_matmul_kernel<false, true>)
                 : reinterpret_cast<const void *>(&cfa_matmul_kernel<false, false>);
}

struct Config {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
};

void configure(Config *c, unsigned grid, unsigned cluster, bool early, cudaStream_t stream)
{
    c->cfg = {};
    c->cfg.gridDim = dim3(grid);
    c->cfg.blockDim = dim3(kThreads);
    c->cfg.dynamicSmemBytes = kSmem;
    c->cfg.stream = stream;
    c->cfg.attrs = c->attr;
    c->attr[0].id = cudaLaunchAttributeClusterDimension;
    c->attr[0].val.clusterDim.x = cluster;
    c->attr[0].val.clusterDim.y = c->attr[0].val.clusterDim.z = 1;
    c->cfg.numAttrs = 1;
    if (early) {
        c->attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        c->attr[1].val.programmaticStreamSerializationAllowed = 1;
        c->cfg.numAttrs = 2;
    }
}

/* Clusters of `size` CTAs that the device runs at once. */
cudaError_t clusters_of(Device &d, bool pair, bool gated, unsigned size, int *n)
{
    std::atomic<int> &known = d.clusters[gated][pair ? 0 : size];
    int v = known.load();
    if (!v) {
        Config c;
        configure(&c, size, size, false, nullptr);
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&v, kernel_of(pair, gated), &c.cfg);
        if (e) return e;
        known.store(++v);
    }
    *n = v - 1;
    return *n > 0 ? cudaSuccess : cudaErrorInvalidConfiguration;
}

} // namespace

cudaError_t cfa_launch_matmul(const cfa_matmul *m, int early, int release, cudaStream_t stream)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    Device &d = g_device[dev];
    int sms = d.sms.load();
    if (!sms) {
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e) return e;
        d.sms.store(sms);
    }
    const bool gated = m->gated;
    Args a = {};
    a.m = *m;
    a.outs = gated ? m->w_rows / 2 : m->w_rows;
    a.steps = (uint32_t)((m->cols + kDepth - 1) / kDepth);
    a.release = (uint32_t)release;

    /* rows of a group, as far as the host knows */
    const int64_t rows = (m->tokens + m->busy - 1) / m->busy;
    const bool pair = rows > 128;
    a.bn = 256;
    if (!pair)
        for (a.bn = 16; a.bn < rows; a.bn *= 2) {
        }
    const uint32_t features = (pair ? 2 : 1) * (gated ? kRows / 2 : kRows);
    a.f_tiles = (uint32_t)((a.outs + features - 1) / features);
    const int64_t likely = m->busy * ((rows + a.bn - 1) / a.bn) * a.f_tiles;
    const int64_t most = ((m->tokens + a.bn - 1) / a.bn + m->busy - 1) * a.f_tiles;
    a.split = 1;
    if (!pair && a.bn <= 64) {
        int64_t n = likely < sms ? sms / likely : 1;
        if (n > a.steps / 4) n = a.steps / 4;
        a.split = (uint32_t)(n < 1 ? 1 : n > 8 ? 8 : n);
    }
    const uint32_t x_rows = pair ? a.bn / 2 : a.bn;
    const uint32_t stage = (kRows + x_rows) * kRowBytes;
    const uint32_t left = kSmem - (uint32_t)sizeof(Shared) - 1024u -
                          (a.split > 1 ? a.bn * kRows * 4u : 0u);
    a.stages = left / stage < kMaxStages ? left / stage : kMaxStages;
    for (a.tmem_cols = 32; a.tmem_cols < 2 * a.bn; a.tmem_cols *= 2) {
    }

    const unsigned bit = 1u << ((pair ? 2 : 0) + (gated ? 1 : 0));
    const void *fn = kernel_of(pair, gated);
    if (!(d.ready.load() & bit)) {
        e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
        if (e) return e;
        d.ready.fetch_or(bit);
    }
    const unsigned size = pair ? 2 : a.split;
    int clusters = sms;
    if (size > 1) {
        e = clusters_of(d, pair, gated, size, &clusters);
        if (e) return e;
    }
    if (clusters > most) clusters = (int)most;

    const cuuint64_t k = (cuuint64_t)m->cols, whole = (k + 7) / 8 * 8;
    const cuuint64_t wld = (m->w_rows > 1 ? (cuuint64_t)m->w_stride : whole) * 2;
    const cuuint64_t xld = (m->tokens > 1 ? (cuuint64_t)m->x_stride : whole) * 2;
    bool fine;
    if (gated) {
        const cuuint64_t dim[4] = {k, (cuuint64_t)a.outs, 2, (cuuint64_t)m->n_groups};
        const cuuint64_t stride[3] = {wld, wld * a.outs, wld * a.outs * 2};
        const cuuint32_t box[4] = {kDepth, 16, 2, 1};
        fine = encode(&a.wmap, m->f16, m->w, 4, dim, stride, box);
    } else {
        const cuuint64_t dim[3] = {k, (cuuint64_t)m->w_rows, (cuuint64_t)m->n_groups};
        const cuuint64_t stride[2] = {wld, wld * m->w_rows};
        const cuuint32_t box[3] = {kDepth, kRows, 1};
        fine = encode(&a.wmap, m->f16, m->w, 3, dim, stride, box);
    }
    const cuuint64_t dim[2] = {k, (cuuint64_t)m->tokens}, stride[1] = {xld};
    const cuuint32_t box[2] = {kDepth, x_rows};
    if (!fine || !encode(&a.xmap, m->f16, m->x, 2, dim, stride, box))
        return cudaErrorInvalidValue;

    Config c;
    configure(&c, (unsigned)clusters * size, size, early != 0, stream);
    void *p[] = {&a};
    return cudaLaunchKernelExC(&c.cfg, fn, p);
}

cudaError_t cfa_matmul_status(int *word)
{
    const int zero = 0;
    const cudaError_t e = cudaMemcpyFromSymbol(word, g_status, sizeof *word);
    return e || !*word ? e : cudaMemcpyToSymbol(g_status, &zero, sizeof zero);
}
