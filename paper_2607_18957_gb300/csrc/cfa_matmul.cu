/*
 * y = act(x w^T + bias) + residual, for one weight or for a stack of them (cfa_matmul), on the
 * tensor cores (tcgen05).
 *
 * The weight's rows lie along the accumulator's lanes (M, 128 per SM) and the tokens along its
 * columns (N, 16 to 256).  So a few tokens cost a few columns while the weight streams through at
 * memory speed, ragged groups only shorten N, and a warp of the epilogue holds 32 neighbouring
 * output columns of one token, which it stores side by side.
 *
 * A CTA has ten warps: eight for the epilogue (two take turns at each 32 lanes of tensor memory), one
 * that asks the TMA for tiles of 64 columns of w and x, and one that issues the products.  Tiles come
 * in a ring of shared-memory stages; the accumulator is double buffered, so that the epilogue of one
 * output tile runs under the products of the next.  CTAs are persistent and take output tiles in turn.
 *
 * PAIR: two CTAs work on one tile of 256 weight rows (cta_group::2): each holds half of the rows and
 * half of the tokens, so each operand is loaded once per pair.
 * split: with few output tiles a cluster of CTAs shares one, each over its part of the columns of w;
 * the partial sums meet in shared memory and are added in the order of the CTAs.
 * Gated: the stage holds 8 gate rows, then the 8 up rows that belong to them, and so on, so both
 * values of an output lie in one warp, 8 lanes apart.
 * Of these, and of the heights of the tiles, `choose` takes those that a fit to timings puts first.
 *
 * What bounds it, and what it takes on one GB300 (bf16, weights from memory, not from L2):
 *   many tokens: the tensor cores.  2048 tokens, gated 28,672 x 4096: the tensor pipe is active in 95 %
 *     of the cycles, 4096 tokens take 475 us (2.0 PFLOP/s) in a burst and 550 (1.75) under the power
 *     limit, as cuBLAS does.
 *   few tokens: memory, 128 weight rows a stage and 150 to 200 KiB a CTA on their way.  One token,
 *     gated 28,672 x 4096 (235 MB): 38.8 us (6.1 TB/s); 57,344 x 4096: 72 us (6.5 TB/s); 128,256 x 4096
 *     (1.05 GB): 152 us (6.9 TB/s).
 *   few tokens and a small weight: start and end.  A launch of one block takes 3.1 us, 50 MB
 *     12.9 us (7.4 at the rate of memory), 117 MB 22.5 us (17).
 *   short rows: the epilogue.  2048 x 6400 x 64 takes 14.6 us, 2206 x 6360 x 392 with a residual 32, x
 *     6359 46 (results and residuals from memory).
 * What made the difference, in the order it was found, with the times of then: stores of pairs of
 * columns without a branch between them (1078 -> 562 us on 4096 x 28,672 x 4096); one elected lane for
 * loads and for products, which lets the compiler keep their operands in uniform registers (0.31 ->
 * 0.18 us a block), and a look at the next stage's barrier before the products of this one (0.25 ->
 * 0.21); one load for all blocks of a stage instead of one or, gated, four per block (627 -> 447 us on
 * the gate/up product); loads before the tensor memory is there and the epilogue's code warmed up under
 * them (4.0 -> 3.0 us for one block); eight epilogue warps instead of four (88 -> 65 us on 2247 tokens,
 * gated 16,384 x 1280 with SiLU); tiles turned round in shared memory and stored 16 bytes at a time, or
 * 4 where rows lie off that grid, by kernels that hold no other way to store (62 -> 56 there; 2206
 * tokens x 6359 x 392 with a residual 81 -> 37, x 6360 42 -> 27); rings of three stages or more beside
 * a cluster's sums (256 tokens x 4096 x 14,336 47 -> 37).
 *
 * exact: the tensor cores add in fp32, but cut each sum's last bits off where IEEE addition rounds, so
 * that an fp32 result is off by half a unit in the last place per addition in the same direction (1e-6
 * after 64 of them: 1024 columns).  For fp32 results the accumulator therefore takes parts of 256
 * columns, which the epilogue adds with rounding in a third place of tensor memory (2.3e-7 at 4096
 * columns, where a product in plain fp32 has 1.9e-7).  Results of 16 bits, whose own rounding is a
 * thousand times that, are summed in one go.
 *
 * Every wait on an mbarrier has a limit.  One that runs out is counted in what cfa_op_status reads; its
 * CTA then issues nothing more, lets its loads and products in flight end (again with a limit) and frees
 * its tensor memory.  (The longest sum that a call can ask for, 2^31 columns, takes 0.94 s and stays
 * inside the limit.)  The barriers of a cluster have none: they end because every thread goes through all
 * of its CTA's tiles and arrives at each one's barriers, whether or not a wait of its has run out.
 */
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <math.h>

#include <atomic>

#include "cfa_device.cuh"
#include "cfa_ops.h"
#include "cfa_tiles.h"

namespace {

using namespace cfa_tiles;

constexpr int kThreads = 320;
constexpr int kLoader = 8, kIssuer = 9;  /* warps; 0 to 7 are the epilogue's, two for each 32 lanes */
constexpr uint32_t kMaxStages = 32;      /* no more than a warp has lanes */
constexpr uint32_t kPart = 4;            /* blocks per part of a sum that is kept exact (m.exact) */
constexpr uint32_t kBand = 16;           /* token tiles that share a weight tile in turn */
constexpr uint32_t kBoxes = 4;           /* heights of the loads of x */
constexpr uint32_t kSpinLimit = 1u << 20;    /* polls of a wait */
constexpr uint32_t kDrainLimit = 1u << 16;   /* polls for loads in flight after one ran out */

/* What a kernel is made for.  An epilogue that holds what other products need (other ways to store,
 * functions that are not called) no longer fits the instruction caches: with all in one kernel, 2206
 * tokens x 6360 x 64 took 30 us where 18 do. */
enum : int {
    kPair = 1,
    kGated = 2,
    kF32 = 4,     /* y */
    kExact = 8,   /* see above; with kF32 */
    kWide = 16,   /* tiles are stored by way of shared memory, 16 bytes at a time .. */
    kNarrow = 32, /* .. or 4, y or the residual being off the 16-byte grid; neither: from registers */
    kCurves = 64, /* the activations with erf and tanh too */
};

struct Args {
    CUtensorMap wmap, xmap[kBoxes]; /* a stage's blocks of w and of x at once, whole blocks only */
    CUtensorMap wtail, xtail[kBoxes]; /* one block; columns behind the last read as zeros */
    cfa_matmul m;
    int64_t outs;        /* columns of y */
    uint32_t bn;         /* token tile */
    uint32_t x_box[kBoxes]; /* rows of x per load: all of the tile's, and less for ragged groups; 0:
                            no such map */
    uint32_t fr;         /* weight rows per CTA: a multiple of 8, gated of 16 */
    uint32_t stages;
    uint32_t deep;       /* blocks of kDepth columns per stage */
    uint32_t whole;      /* whole blocks; the last of steps may lack columns */
    int32_t f_whole;     /* gated, with a last group of fewer than 8 rows: the features before it, which
                            a tile at once has to stay inside; otherwise INT32_MAX */
    uint32_t steps;      /* blocks in all */
    uint32_t acc_on;     /* columns of tensor memory from one accumulator to the next */
    uint32_t f_tiles;    /* feature tiles per group */
    int32_t total;       /* output tiles, of one group */
    uint32_t split;      /* log2 of the CTAs per output tile along the columns */
    uint32_t tmem_cols;
    uint32_t release;
    uint32_t polls;      /* of a wait, before it gives up */
    uint32_t lose;       /* self-test, 1: the loader asks for nothing, but goes through its tiles; 2: an
                            accumulator is full only after one more arrival than the products' */
    uint32_t early_w;    /* w, and what tells the groups' rows, is there before the launch's wait */
    uint32_t pairs;      /* y and the residual can be read and written two columns at a time */
};

__device__ cfa_op_counts g_counts[2]; /* of waits that ran out; [1]: the self-test's */

/* What precedes the stages in shared memory. */
struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem;
    uint32_t polls;
    uint32_t loads;  /* stages that the loader has asked for */
    uint32_t sums;   /* accumulators that the issuer has committed */
    int dead;
    int32_t total;   /* output tiles */
    int32_t group[]; /* output tiles before each group's, and rows of x before each group's, in turn */
};

__host__ __device__ inline uint32_t shared_bytes(int32_t groups)
{
    return (uint32_t)sizeof(Shared) + ((uint32_t)groups + 1u) * 8u;
}

__device__ __forceinline__ uint32_t smem_addr(const void *p)
{
    return (uint32_t)__cvta_generic_to_shared(p);
}

/* Barriers go by their shared-memory address. */
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return done != 0;
}

/* Waits for phase `parity`; false if the limit ran out here or in another warp of the CTA. */
__device__ __noinline__ bool mbar_wait_long(uint32_t bar, uint32_t parity, Shared *s)
{
    const uint32_t polls = s->polls;
    for (uint32_t k = 0; k < polls; ++k) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((k & 1023u) == 1023u && *(volatile int *)&s->dead) return false;
    }
    *(volatile int *)&s->dead = 1;
    return false;
}

__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, Shared *s)
{
    return mbar_try_wait(bar, parity) || mbar_wait_long(bar, parity, s);
}

/* True for one lane of the warp; the compiler then knows that one lane alone issues what follows,
 * and keeps the operands of copies and products in uniform registers. */
__device__ __forceinline__ bool elect_one()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(one));
    return one != 0;
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

/* The same where nothing written has to be seen: the others have read what they need. */
__device__ __forceinline__ void cluster_done()
{
    asm volatile("barrier.cluster.arrive.relaxed;\n\tbarrier.cluster.wait;" ::: "memory");
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

/* Tiles of a tensor map of four or five dimensions into shared memory, counted on `bar` (of a pair, the
 * first CTA's). */
template <bool PAIR>
__device__ __forceinline__ void load4(uint32_t dst, const CUtensorMap *map, int32_t c0, int32_t c1,
                                      int32_t c2, int32_t c3, uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                     "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                     "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
                     : "memory");
}

template <bool PAIR>
__device__ __forceinline__ void load5(uint32_t dst, const CUtensorMap *map, int32_t c0, int32_t c1,
                                      int32_t c2, int32_t c3, int32_t c4, uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(
                         dst),
                     "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(
                         dst),
                     "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(bar)
                     : "memory");
}

template <bool PAIR>
__device__ __forceinline__ void load3(uint32_t dst, const CUtensorMap *map, int32_t c0, int32_t c1,
                                      int32_t c2, uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                     "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile"
                     ".mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                     "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
                     : "memory");
}

/* Descriptor of a shared-memory matrix of rows of 128 bytes, 128-byte swizzle, 8-row groups 1024
 * bytes apart: the word with the address, and the other. */
__device__ __forceinline__ uint32_t matrix_low(uint32_t addr)
{
    return ((addr & 0x3FFFFu) >> 4) | (1u << 16);
}
constexpr uint32_t kMatrixHigh = (1024u >> 4) | (1u << 14) | (2u << 29);

/* fp32 accumulator, both operands bf16 or both f16, rows of the contraction contiguous. */
__device__ __forceinline__ uint32_t instruction(int f16, uint32_t m, uint32_t n)
{
    const uint32_t type = f16 ? 0u : 1u;
    return (1u << 4) | (type << 7) | (type << 10) | ((n >> 3) << 17) | ((m >> 4) << 24);
}

/* Accumulator d (+)= a b^T, 16 columns of the contraction. */
template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint32_t b, uint32_t inst, uint32_t add)
{
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 ma, mb;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "mov.b64 ma, {%1, %5};\n\tmov.b64 mb, {%2, %5};\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], ma, mb, %3, p;\n\t}" ::"r"(d),
                     "r"(a), "r"(b), "r"(inst), "r"(add), "r"(kMatrixHigh)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 ma, mb;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "mov.b64 ma, {%1, %5};\n\tmov.b64 mb, {%2, %5};\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], ma, mb, %3, p;\n\t}" ::"r"(d),
                     "r"(a), "r"(b), "r"(inst), "r"(add), "r"(kMatrixHigh)
                     : "memory");
}

/* Arrives on the barrier (of both CTAs of a pair) once all products issued so far are done. */
template <bool PAIR> __device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster"
                     ".multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster"
                     ".b64 [%0];" ::"r"(bar)
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

__device__ __forceinline__ void tmem_store(uint32_t addr, const float (&v)[16])
{
    uint32_t r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(v[i]);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};\n\t"
                 "tcgen05.wait::st.sync.aligned;" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
                 : "memory");
}

/* Loads go past L1, which may hold what an older kernel read there: a launch can start before the one
 * before it has ended (cfa_launch_ctl), so that its start clears nothing written after it. */
__device__ __forceinline__ float value(const void *p, int64_t i, int f16)
{
    const unsigned short b = __ldcg(static_cast<const unsigned short *>(p) + i);
    return f16 ? __half2float(__ushort_as_half(b)) : __bfloat162float(__ushort_as_bfloat16(b));
}

__device__ __forceinline__ float value(const float *p, int64_t i) { return __ldcg(p + i); }

/* One switch for a batch of values, so that they run side by side. */
template <int KIND, int N> __device__ __forceinline__ void activate(float (&v)[N], int act)
{
    if (!(KIND & kCurves) && act != CFA_ACT_SILU) {
        if (act == CFA_ACT_RELU) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];
        }
        return;
    }
    switch (act) {
    case CFA_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];
        break;
    case CFA_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.5f * v[i] * (1.0f + erff(v[i] * 0.70710678118654752f));
        break;
    case CFA_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = 0.5f * v[i] *
                   (1.0f + tanhf(0.79788456080286536f * (v[i] + 0.044715f * v[i] * v[i] * v[i])));
        break;
    case CFA_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i)
        {
            /* Both fast forms are off by some units in the last place of fp32: the quotient by two,
             * which fp32 results may be, the exponential by |v|, which 16 bits do not show.  The fast
             * quotient is 0 for divisors above 2^126, which 1 + exp(-v) is from v = -87.4 on, with
             * the value at -9e-37; a quarter of both sides of it stays below to where exp(-v) leaves
             * fp32 (-88.7). */
            const float e = KIND & kExact ? expf(-v[i]) : __expf(-v[i]);
            v[i] = __fdividef(0.25f * v[i], fmaf(0.25f, e, 0.25f));
        }
        break;
    default: break;
    }
}

/* 16 columns of the accumulator, and with `more` the sums of the parts before. */
__device__ __forceinline__ void sum_load(uint32_t acc, uint32_t sum, bool more, float (&v)[16])
{
    tmem_load(acc, v);
    if (more) {
        float u[16];
        tmem_load(sum, u);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] += u[j];
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
    Tile o;
    int32_t rows = (int32_t)a.m.tokens, before = 0;
    uint32_t local = (uint32_t)t;
    o.group = 0;
    if (a.m.offs) {
        int32_t g = *group;
        while (t >= s->group[2 * g + 2]) ++g;
        *group = o.group = g;
        local = (uint32_t)(t - s->group[2 * g]);
        before = s->group[2 * g + 1];
        rows = s->group[2 * g + 3] - before;
    }
    uint32_t f = local, n = 0;
    if ((uint32_t)rows > a.bn) { /* more than one token tile */
        const uint32_t tiles = ((uint32_t)rows + a.bn - 1) / a.bn;
        const uint32_t band = tiles <= kBand ? 0 : local / (kBand * a.f_tiles);
        const uint32_t rest = local - band * kBand * a.f_tiles;
        const uint32_t left = tiles - band * kBand, width = left < kBand ? left : kBand;
        f = rest / width;
        n = band * kBand + rest - f * width;
    }
    o.feature = (int64_t)f * features;
    o.row = before + (int32_t)(n * a.bn);
    o.rows = min((int32_t)a.bn, rows - (int32_t)(n * a.bn));
    return o;
}

__device__ __forceinline__ uint32_t pack(float lo, float hi, int f16)
{
    if (f16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ float2 unpack(uint32_t v, int f16)
{
    if (f16) return __half22float2(*reinterpret_cast<const __half2 *>(&v));
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v));
}

/* What a lane stores of a batch of N tokens: token i of the batch stands at row + i * step, if i * step
 * + 1 <= n.  With a.pairs, neighbouring lanes trade every second value, so that an even lane stores
 * columns (c, c + 1) of the tokens 0, 2, .. of the batch and an odd lane (c - 1, c) of the tokens 1, 3,
 * ..; without (y or the residual off that grid, or a last column on its own) each lane stores its own
 * column of every token. */
struct Place {
    int64_t row, col;
    int step, n;
};

__device__ __forceinline__ bool by_pairs(const Args &a, const Place &p)
{
    return a.pairs && (p.col | 1) < a.outs;
}

/* The residual where the lane will store. */
struct Residual {
    uint32_t lo[16], hi[8]; /* pairs of fp32 take both, one of a pair at a time */
};

template <bool F32, int N>
__device__ __forceinline__ void fetch(const Args &a, const Place &p, Residual &r)
{
    const cfa_matmul &m = a.m;
    if (!m.residual) return;
    if (by_pairs(a, p)) {
        const int odd = threadIdx.x & 1, first = odd * p.step;
        const int64_t at = (p.row + first) * m.r_stride + p.col - odd;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if (first + 2 * i * p.step >= p.n) continue;
            const int64_t from = at + 2 * i * p.step * m.r_stride;
            if (F32) {
                const uint2 v = __ldcg(reinterpret_cast<const uint2 *>(
                    static_cast<const float *>(m.residual) + from));
                r.lo[i] = v.x;
                r.hi[i] = v.y;
            } else {
                r.lo[i] = __ldcg(reinterpret_cast<const uint32_t *>(
                    static_cast<const uint16_t *>(m.residual) + from));
            }
        }
    } else if (p.col < a.outs) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i * p.step >= p.n) continue;
            const int64_t from = (p.row + i * p.step) * m.r_stride + p.col;
            if (F32) r.lo[i] = __ldcg(static_cast<const uint32_t *>(m.residual) + from);
            else r.lo[i] = __ldcg(static_cast<const unsigned short *>(m.residual) + from);
        }
    }
}

template <bool F32, int N>
__device__ __forceinline__ void store(const Args &a, float (&v)[N], const Place &p, const Residual &r)
{
    const cfa_matmul &m = a.m;
    float2 o[N / 2];
    const int odd = threadIdx.x & 1, first = odd * p.step;
    if (a.pairs) { /* every lane trades */
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float got = __shfl_xor_sync(0xFFFFFFFFu, odd ? v[2 * i] : v[2 * i + 1], 1);
            o[i] = odd ? make_float2(got, v[2 * i + 1]) : make_float2(v[2 * i], got);
        }
    }
    if (by_pairs(a, p)) {
        if (m.residual) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float2 x = F32 ? make_float2(__uint_as_float(r.lo[i]),
                                                       __uint_as_float(r.hi[i]))
                                         : unpack(r.lo[i], m.f16);
                o[i].x += x.x;
                o[i].y += x.y;
            }
        }
        const int64_t at = (p.row + first) * m.y_stride + p.col - odd;
        if (F32) {
            float *to = static_cast<float *>(m.y) + at;
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                if (first + 2 * i * p.step < p.n)
                    *reinterpret_cast<float2 *>(to + 2 * i * p.step * m.y_stride) = o[i];
        } else {
            uint16_t *to = static_cast<uint16_t *>(m.y) + at;
#pragma unroll
            for (int i = 0; i < N / 2; ++i)
                if (first + 2 * i * p.step < p.n)
                    *reinterpret_cast<uint32_t *>(to + 2 * i * p.step * m.y_stride) =
                        pack(o[i].x, o[i].y, m.f16);
        }
    } else if (p.col < a.outs) {
        const int64_t at = p.row * m.y_stride + p.col;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i * p.step >= p.n) continue;
            float x = v[i];
            const int64_t to = at + i * p.step * m.y_stride;
            if (m.residual)
                x += F32 ? __uint_as_float(r.lo[i]) : unpack(r.lo[i], m.f16).x;
            if (F32) static_cast<float *>(m.y)[to] = x;
            else static_cast<uint16_t *>(m.y)[to] = (uint16_t)pack(x, 0.0f, m.f16);
        }
    }
}

/* N of 16 tokens' sums of the lane's weight row, of which n are in the tile: bias, activation, store.
 * Gated: of 16 lanes, 8 hold gate values and the next 8 the up values of the same columns; of two tokens
 * the gate's lanes finish the first and the others the second. */
template <bool GATED>
__device__ __forceinline__ Place place_of(int64_t row, int n, int64_t col)
{
    const int upper = GATED && (threadIdx.x & 8) ? 1 : 0;
    return {row + upper, col, GATED ? 2 : 1, n - upper};
}

template <int KIND, int N>
__device__ __forceinline__ void finish(const Args &a, float (&all)[16], const Place &p, float bias,
                                       const Residual &r)
{
    constexpr bool F32 = KIND & kF32;
    const cfa_matmul &m = a.m;
    float v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = m.bias ? all[j] + bias : all[j];
    if constexpr ((KIND & kGated) != 0) {
        const bool upper = threadIdx.x & 8;
        float gate[N / 2], up[N / 2];
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const float got = __shfl_xor_sync(0xFFFFFFFFu, upper ? v[2 * j] : v[2 * j + 1], 8);
            gate[j] = upper ? got : v[2 * j];
            up[j] = upper ? v[2 * j + 1] : got;
        }
        activate<KIND>(gate, m.act);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) gate[j] *= up[j];
        store<F32, N / 2>(a, gate, p, r);
    } else {
        activate<KIND>(v, m.act);
        store<F32, N>(a, v, p, r);
    }
}

/* A batch of 16 tokens by way of shared memory, in which token j's sums of the warp's 32 weight rows lie
 * side by side from word j * kStageRow on (four words more than they are, so that 16-byte reads of
 * neighbouring tokens meet different banks).  The registers hold 16 tokens of one column: stored from
 * there, each store writes 64 bytes of two tokens at most, after an exchange with the next lane.  Here a
 * lane takes 16 bytes of y at a time: 8 columns of 2 bytes or 4 of 4, of the tokens lane / CHUNKS + i *
 * STEP. */
template <bool GATED, bool F32> struct Wide {
    static constexpr int COLS = F32 ? 4 : 8, CHUNKS = (GATED ? 16 : 32) / COLS;
    static constexpr int ITEMS = kBatch * CHUNKS / 32, STEP = 32 / CHUNKS;
};

__device__ __forceinline__ uint4 pack16(const float (&v)[8], int f16)
{
    uint32_t o[4];
    if (f16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pack(v[2 * i], v[2 * i + 1], 1);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = pack(v[2 * i], v[2 * i + 1], 0);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}
__device__ __forceinline__ uint4 pack16(const float (&v)[4], int)
{
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                      __float_as_uint(v[3]));
}
__device__ __forceinline__ void add16(float (&v)[8], uint4 r, int f16)
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    if (f16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = unpack(w[i], 1);
            v[2 * i] += x.x;
            v[2 * i + 1] += x.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = unpack(w[i], 0);
            v[2 * i] += x.x;
            v[2 * i + 1] += x.y;
        }
    }
}
__device__ __forceinline__ void add16(float (&v)[4], uint4 r, int)
{
    v[0] += __uint_as_float(r.x);
    v[1] += __uint_as_float(r.y);
    v[2] += __uint_as_float(r.z);
    v[3] += __uint_as_float(r.w);
}

/* The residual of a batch of n tokens from `row` on, in columns [col, limit) of which the lane takes its
 * chunk. */
template <bool GATED, bool F32>
__device__ __forceinline__ void fetch_wide(const Args &a, int64_t row, int n, int64_t col, int64_t limit,
                                           uint4 (&r)[4])
{
    typedef Wide<GATED, F32> W;
    const int lane = threadIdx.x & 31, token = lane / W::CHUNKS;
    col += lane % W::CHUNKS * W::COLS;
    if (!a.m.residual || col + W::COLS > limit) return;
    const uint8_t *from = static_cast<const uint8_t *>(a.m.residual) +
                          ((row + token) * a.m.r_stride + col) * (16 / W::COLS);
#pragma unroll
    for (int i = 0; i < W::ITEMS; ++i)
        if (token + i * W::STEP < n)
            r[i] = __ldcg(reinterpret_cast<const uint4 *>(
                from + i * W::STEP * a.m.r_stride * (16 / W::COLS)));
}

template <int KIND>
__device__ __forceinline__ void finish_wide(const Args &a, const float *stage, int64_t row, int n,
                                            int64_t col, int64_t limit, const uint4 (&r)[4])
{
    constexpr bool GATED = KIND & kGated, F32 = KIND & kF32;
    typedef Wide<GATED, F32> W;
    const cfa_matmul &m = a.m;
    const int lane = threadIdx.x & 31, token = lane / W::CHUNKS, at = lane % W::CHUNKS * W::COLS;
    float v[W::ITEMS][W::COLS];
#pragma unroll
    for (int i = 0; i < W::ITEMS; ++i) {
        /* gated: 8 gate rows, then their 8 up rows */
        const float *from = stage + (token + i * W::STEP) * kStageRow +
                            (GATED ? at / 8 * 16 + at % 8 : at);
        float up[W::COLS];
#pragma unroll
        for (int j = 0; j < W::COLS; j += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(from + j);
            v[i][j] = x.x;
            v[i][j + 1] = x.y;
            v[i][j + 2] = x.z;
            v[i][j + 3] = x.w;
            if constexpr (GATED) {
                const float4 u = *reinterpret_cast<const float4 *>(from + j + 8);
                up[j] = u.x;
                up[j + 1] = u.y;
                up[j + 2] = u.z;
                up[j + 3] = u.w;
            }
        }
        activate<KIND>(v[i], m.act);
        if constexpr (GATED) {
#pragma unroll
            for (int j = 0; j < W::COLS; ++j) v[i][j] *= up[j];
        }
    }
    col += at;
    const int64_t first = (row + token) * m.y_stride + col;
    if (col + W::COLS <= limit) {
        uint8_t *to = static_cast<uint8_t *>(m.y) + first * (16 / W::COLS);
#pragma unroll
        for (int i = 0; i < W::ITEMS; ++i) {
            if (m.residual) add16(v[i], r[i], m.f16);
            const uint4 o = pack16(v[i], m.f16);
            if (token + i * W::STEP < n)
                *reinterpret_cast<uint4 *>(to + i * W::STEP * m.y_stride * (16 / W::COLS)) = o;
        }
    } else {
#pragma unroll
        for (int i = 0; i < W::ITEMS; ++i)
#pragma unroll
            for (int j = 0; j < W::COLS; ++j) {
                if (token + i * W::STEP >= n || col + j >= limit) continue;
                const int64_t to = first + i * W::STEP * m.y_stride + j;
                float x = v[i][j];
                if (m.residual) {
                    const int64_t from = (row + token + i * W::STEP) * m.r_stride + col + j;
                    x += F32 ? value(static_cast<const float *>(m.residual), from)
                             : value(m.residual, from, m.f16);
                }
                if (F32) static_cast<float *>(m.y)[to] = x;
                else static_cast<uint16_t *>(m.y)[to] = (uint16_t)pack(x, 0.0f, m.f16);
            }
    }
}

/* The same where y or the residual is off the 16-byte grid, for y of 2 bytes: a lane takes 4 bytes of y
 * of the tokens lane / WORDS + i * STEP.  Where a token's columns start between two words, its first
 * lane stores the first and the last of them by themselves. */
template <bool GATED> struct Narrow {
    static constexpr int COLS = GATED ? 16 : 32, WORDS = COLS / 2, STEP = 32 / WORDS;
    static constexpr int ITEMS = kBatch / STEP;
};

/* The two columns of the lane in row `row` of y, and in every second row from there: of them the first
 * lies at a word's address, unless they are the first lane's two of a row that starts between words. */
template <bool GATED>
__device__ __forceinline__ void narrow_columns(const Args &a, int64_t row, int64_t col, int &c0, int &c1)
{
    const int word = (int)(threadIdx.x & 31) % Narrow<GATED>::WORDS;
    const int odd = (int)(((uintptr_t)a.m.y >> 1) + row * a.m.y_stride + col) & 1;
    c1 = 2 * word + 1 - odd;
    c0 = c1 ? c1 - 1 : Narrow<GATED>::COLS - 1;
}

template <bool GATED>
__device__ __forceinline__ void fetch_narrow(const Args &a, int64_t row, int n, int64_t col,
                                             int64_t limit, uint32_t (&r)[16])
{
    typedef Narrow<GATED> W;
    if (!a.m.residual) return;
    const int token = (int)(threadIdx.x & 31) / W::WORDS;
    int c0, c1;
    narrow_columns<GATED>(a, row + token, col, c0, c1);
    const unsigned short *from = static_cast<const unsigned short *>(a.m.residual) +
                                 (row + token) * a.m.r_stride + col;
    const int in0 = col + c0 < limit ? n - token : 0, in1 = col + c1 < limit ? n - token : 0;
#pragma unroll
    for (int i = 0; i < W::ITEMS; ++i) {
        if (i * W::STEP < in0) r[2 * i] = __ldcg(from + c0);
        if (i * W::STEP < in1) r[2 * i + 1] = __ldcg(from + c1);
        from += W::STEP * a.m.r_stride;
    }
}

template <int KIND>
__device__ __forceinline__ void finish_narrow(const Args &a, const float *stage, int64_t row, int n,
                                              int64_t col, int64_t limit, const uint32_t (&r)[16])
{
    constexpr bool GATED = KIND & kGated;
    typedef Narrow<GATED> W;
    const cfa_matmul &m = a.m;
    const int token = (int)(threadIdx.x & 31) / W::WORDS;
    int c0, c1;
    narrow_columns<GATED>(a, row + token, col, c0, c1);
    float v[2 * W::ITEMS], up[GATED ? 2 * W::ITEMS : 1];
    /* gated: 8 gate rows, then their 8 up rows */
    const float *const from0 = stage + token * kStageRow + (GATED ? c0 + (c0 & 8) : c0);
    const float *const from1 = stage + token * kStageRow + (GATED ? c1 + (c1 & 8) : c1);
#pragma unroll
    for (int i = 0; i < W::ITEMS; ++i) {
        v[2 * i] = from0[i * W::STEP * kStageRow];
        v[2 * i + 1] = from1[i * W::STEP * kStageRow];
        if constexpr (GATED) {
            up[2 * i] = from0[i * W::STEP * kStageRow + 8];
            up[2 * i + 1] = from1[i * W::STEP * kStageRow + 8];
        }
    }
    activate<KIND>(v, m.act);
    if constexpr (GATED) {
#pragma unroll
        for (int i = 0; i < 2 * W::ITEMS; ++i) v[i] *= up[i];
    }
    if (m.residual) {
#pragma unroll
        for (int i = 0; i < 2 * W::ITEMS; ++i) v[i] += unpack(r[i], m.f16).x;
    }
    uint32_t o[W::ITEMS];
    if (m.f16) {
#pragma unroll
        for (int i = 0; i < W::ITEMS; ++i) o[i] = pack(v[2 * i], v[2 * i + 1], 1);
    } else {
#pragma unroll
        for (int i = 0; i < W::ITEMS; ++i) o[i] = pack(v[2 * i], v[2 * i + 1], 0);
    }
    uint16_t *to = static_cast<uint16_t *>(m.y) + (row + token) * m.y_stride + col;
    const int64_t step = W::STEP * m.y_stride;
    const int in0 = col + c0 < limit ? n - token : 0, in1 = col + c1 < limit ? n - token : 0;
    if (c0 < c1 && in0 == in1) {
        to += c0;
#pragma unroll
        for (int i = 0; i < W::ITEMS; ++i)
            if (i * W::STEP < in0) *reinterpret_cast<uint32_t *>(to + i * step) = o[i];
    } else {
#pragma unroll
        for (int i = 0; i < W::ITEMS; ++i) {
            if (i * W::STEP < in0) to[i * step + c0] = (uint16_t)o[i];
            if (i * W::STEP < in1) to[i * step + c1] = (uint16_t)(o[i] >> 16);
        }
    }
}

/* Waits, with a limit, until use `n` of a ring's barriers is over. */
__device__ __forceinline__ bool drained(const uint64_t *bars, uint32_t n, uint32_t ring)
{
    for (uint32_t k = 0; k < kDrainLimit; ++k)
        if (mbar_try_wait(smem_addr(bars + n % ring), (n / ring) & 1u)) return true;
    return false;
}

/* After a wait that ran out and with all warps out of their tiles, whichever of them gave up: lets the
 * loads and the products in flight end, as far as a limit allows.  One thread.  Of a pair, the first
 * CTA's barriers count the loads of both and it issues the products; the second only gives what it has
 * asked for some time. */
__device__ __noinline__ void drain(const Args &a, Shared *s, bool second)
{
    bool ended = true;
    if (second) {
        for (int k = 0; k < 100; ++k) __nanosleep(10000);
    } else {
        const uint32_t loads = s->loads, sums = s->sums;
        for (uint32_t n = loads < a.stages ? 0 : loads - a.stages; n < loads; ++n)
            ended = drained(s->full, n, a.stages) && ended;
        for (uint32_t n = sums < 2 ? 0 : sums - 2; n < sums; ++n) {
            if (a.lose == 2) /* the arrival that the epilogue was left waiting for */
                asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(
                                 smem_addr(s->acc_full + n % 2))
                             : "memory");
            ended = drained(s->acc_full, n, 2) && ended;
        }
    }
    cfa_op_counts &counts = g_counts[a.lose != 0];
    if (!ended) atomicAdd(&counts.in_flight, 1u);
    atomicAdd(&counts.ran_out, 1u);
}

/* A stage's blocks of w, from block k on. */
template <bool PAIR, bool GATED>
__device__ __forceinline__ void load_w(const Args &a, bool at_once, uint32_t dst, uint32_t blocks,
                                       uint32_t k, int32_t f, int32_t group, uint32_t bar)
{
    if (at_once) {
        if constexpr (GATED) load5<PAIR>(dst, &a.wmap, 0, 0, 2 * group, f / 8, (int32_t)k, bar);
        else load4<PAIR>(dst, &a.wmap, 0, f, (int32_t)k, group, bar);
        return;
    }
    for (uint32_t i = 0; i < blocks; ++i, dst += a.fr * kRowBytes) {
        const int32_t c = (int32_t)((k + i) * kDepth);
        if constexpr (GATED) {
            for (uint32_t q = 0; q < a.fr / 16; ++q)
                load4<PAIR>(dst + q * 16 * kRowBytes, &a.wtail, c, f + (int32_t)(8 * q), 0, group,
                            bar);
        } else {
            load3<PAIR>(dst, &a.wtail, c, f, group, bar);
        }
    }
}

__device__ __forceinline__ void launch_wait(const Args &a)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.release) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <int KIND>
__global__ void __launch_bounds__(kThreads, 1) cfa_matmul_kernel(const __grid_constant__ Args a)
{
    constexpr bool PAIR = KIND & kPair, GATED = KIND & kGated, F32 = KIND & kF32;
    constexpr bool EXACT = KIND & kExact, WIDE = KIND & kWide, NARROW = KIND & kNarrow;
    extern __shared__ uint8_t raw[];
    Shared *s = reinterpret_cast<Shared *>(raw);
    const uint32_t ring = (smem_addr(raw) + shared_bytes(a.m.n_groups) + 1023u) & ~1023u;
    const uint32_t x_rows = PAIR ? a.bn / 2 : a.bn;
    const uint32_t w_bytes = a.fr * kRowBytes, x_bytes = x_rows * kRowBytes;
    const uint32_t block = w_bytes + x_bytes, stage = block * a.deep;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t share = PAIR ? 1 : a.split; /* log2 of the CTAs that share a tile */
    const uint32_t rank = share ? cluster_rank() : 0;
    const uint32_t per_cta = GATED ? a.fr / 2 : a.fr, features = (PAIR ? 2 : 1) * per_cta;
    const cfa_matmul &m = a.m;
    const uint32_t full = smem_addr(s->full), empty = smem_addr(s->empty);
    const uint32_t acc_full = smem_addr(s->acc_full), acc_empty = smem_addr(s->acc_empty);

    /* The loader sets the barriers up and, where the host could count the tiles, goes on to its loads
     * while the others still wait for the tensor memory. */
    if (warp == kLoader) {
        if ((uint32_t)lane < a.stages) {
            mbar_init(full + 8 * lane, 1);
            mbar_init(empty + 8 * lane, 1);
        }
        if (lane < 2) {
            mbar_init(acc_full + 8 * lane, a.lose == 2 ? 2 : 1);
            mbar_init(acc_empty + 8 * lane, PAIR ? 16 : 8);
        }
        if (lane == 0) {
            s->dead = 0;
            s->loads = s->sums = 0;
            s->polls = a.polls;
            asm volatile("prefetch.tensormap [%0];" ::"l"(&a.wmap) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&a.xmap[0]) : "memory");
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
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
    if (!a.early_w) launch_wait(a);
    if (m.offs) { /* the groups' rows and tiles */
        if (m.ids) { /* counted from the pairs themselves */
            for (int32_t g = threadIdx.x; g < m.n_groups; g += kThreads) s->group[2 * g + 2] = 0;
            __syncthreads();
            for (int32_t i0 = threadIdx.x; i0 < m.n_ids; i0 += 8 * kThreads) {
                int64_t g[8]; /* eight loads under way at once */
#pragma unroll
                for (int32_t j = 0; j < 8; ++j) {
                    const int32_t i = i0 + j * kThreads;
                    g[j] = i < m.n_ids ? (int64_t)__ldcg(m.ids + i) - m.first : -1;
                }
#pragma unroll
                for (int32_t j = 0; j < 8; ++j)
                    if (g[j] >= 0 && g[j] < m.n_groups) atomicAdd(&s->group[2 * g[j] + 2], 1);
            }
            __syncthreads();
        }
        if (warp == 0) {
            int32_t tiles = 0, rows = 0;
            for (int32_t g0 = 0; g0 < m.n_groups; g0 += 32) {
                const int32_t g = g0 + lane;
                int32_t r = 0, n = 0;
                if (g < m.n_groups) {
                    r = m.ids ? s->group[2 * g + 2] : __ldcg(m.offs + g + 1) - __ldcg(m.offs + g);
                    n = (int32_t)(((uint32_t)r + a.bn - 1) / a.bn * a.f_tiles);
                }
                int32_t sum = n, row = r;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int32_t x = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                    const int32_t y = __shfl_up_sync(0xFFFFFFFFu, row, o);
                    if (lane >= o) {
                        sum += x;
                        row += y;
                    }
                }
                __syncwarp();
                if (g < m.n_groups) { /* what comes before the next group */
                    s->group[2 * g + 2] = tiles + sum;
                    s->group[2 * g + 3] = rows + row;
                }
                tiles += __shfl_sync(0xFFFFFFFFu, sum, 31);
                rows += __shfl_sync(0xFFFFFFFFu, row, 31);
            }
            if (lane == 0) {
                s->group[0] = s->group[1] = 0;
                s->total = tiles;
            }
        }
    }
    fence_before();
    if constexpr (PAIR) {
        __syncthreads();
        cluster_sync();
    } else if (warp == kLoader && !m.offs) {
        __syncwarp();
        asm volatile("barrier.cta.arrive 1, %0;" ::"n"(kThreads) : "memory");
    } else {
        asm volatile("barrier.cta.sync 1, %0;" ::"n"(kThreads) : "memory");
    }
    fence_after();
    const int32_t total = m.offs ? s->total : a.total;
    const int32_t stride = (int32_t)(gridDim.x >> share), begin = (int32_t)(blockIdx.x >> share);
    /* this CTA's part of the columns */
    const uint32_t k0 = PAIR ? 0 : rank * a.steps >> share;
    const uint32_t k1 = PAIR ? a.steps : (rank + 1) * a.steps >> share;
    const bool sync_tiles = !PAIR && share > 0;
    const uint32_t deep = a.deep, stages = a.stages, part = EXACT ? kPart : a.steps;
    bool ok = true;
    if (a.early_w && warp != kLoader) launch_wait(a);

    if (warp == kLoader) {
        if (elect_one()) {
            uint32_t at = 0, phase = 1; /* stage; an empty ring counts as released once */
            uint32_t issued = 0;
            int32_t group = 0;
            asm volatile("fence.proxy.async.global;" ::: "memory");
            bool waited = !a.early_w;
            const uint32_t load_to = a.lose == 1 ? k0 : k1;
            for (int32_t t = begin; t < total; t += stride) {
                const Tile o = tile_at(a, s, t, &group, features);
                /* rows of x for this CTA: of a pair, each holds half of the columns in use */
                uint32_t half = 0;
                if constexpr (PAIR) half = rank * (((uint32_t)o.rows + 31u) / 32u * 16u);
                const int32_t row = o.row + (int32_t)half;
                const int32_t f = (int32_t)o.feature + (PAIR ? (int32_t)(rank * per_cta) : 0);
                const uint32_t in_use = PAIR ? ((uint32_t)o.rows + 31u) / 32u * 16u
                                             : (uint32_t)o.rows;
                /* the lowest box of x that holds the rows in use */
                uint32_t box = 0;
                while (box + 1 < kBoxes && a.x_box[box + 1] >= in_use) ++box;
                const CUtensorMap *const xmap = a.xmap + box, *const xtail = a.xtail + box;
                const uint32_t x_one = a.x_box[box] * kRowBytes;
                const uint32_t w_loaded = deep * w_bytes, all = w_loaded + deep * x_one;
                /* blocks that a stage's loads can bring at once */
                const uint32_t at_once_to = f + (int32_t)per_cta <= a.f_whole ? a.whole : 0;
                /* Stages of the first tile get their w before the launch's wait, as many as there are,
                 * and then their x. */
                uint32_t ahead = 0;
                if (!waited) {
                    const uint32_t all_stages = (k1 - k0 + deep - 1) / deep;
                    ahead = all_stages < stages ? all_stages : stages;
                    for (uint32_t i = 0; i < ahead; ++i) {
                        const uint32_t k = k0 + i * deep, bar = full + 8 * i;
                        const uint32_t blocks = min(deep, k1 - k);
                        const bool at_once = k + blocks <= at_once_to;
                        mbar_expect_tx(bar, at_once ? all : blocks * (w_bytes + x_one));
                        load_w<PAIR, GATED>(a, at_once, ring + i * stage, blocks, k, f, o.group, bar);
                    }
                    waited = true;
                    launch_wait(a);
                    asm volatile("fence.proxy.async.global;" ::: "memory");
                }
                for (uint32_t k = k0; k < load_to; k += deep) {
                    const uint32_t blocks = min(deep, k1 - k);
                    const uint32_t dst = ring + at * stage;
                    /* all blocks of the stage at once, unless the one that lacks columns is among
                     * them */
                    const bool at_once = k + blocks <= at_once_to;
                    uint32_t bar = full + 8 * at;
                    if (ahead) {
                        --ahead;
                    } else {
                        ok = ok && mbar_wait(empty + 8 * at, phase, s);
                        if (!ok) break;
                        if (!PAIR || rank == 0) {
                            const uint32_t bytes = at_once ? all : blocks * (w_bytes + x_one);
                            mbar_expect_tx(bar, PAIR ? 2 * bytes : bytes);
                        }
                        if constexpr (PAIR) bar = map_to(bar, 0);
                        load_w<PAIR, GATED>(a, at_once, dst, blocks, k, f, o.group, bar);
                    }
                    if (at_once)
                        load3<PAIR>(dst + w_loaded, xmap, 0, row, (int32_t)k, bar);
                    else
                        for (uint32_t i = 0; i < blocks; ++i)
                            load3<PAIR>(dst + w_loaded + i * x_one, xtail,
                                        (int32_t)((k + i) * kDepth), row, 0, bar);
                    ++issued;
                    if (++at == stages) {
                        at = 0;
                        phase ^= 1;
                    }
                }
                if (sync_tiles) {
                    cluster_sync();
                    cluster_done();
                }
            }
            if (!waited) launch_wait(a);
            s->loads = issued;
        } else if (sync_tiles) {
            for (int32_t t = begin; t < total; t += stride) {
                cluster_sync();
                cluster_done();
            }
        }
        __syncwarp();
    } else if (warp == kIssuer) {
        if (elect_one()) {
            uint32_t at = 0, phase = 0, buf = 0, buf_phase = 1;
            uint32_t sums = 0;
            int32_t group = 0;
            const uint32_t tmem = s->tmem;
            /* descriptors count in 16 bytes */
            const uint32_t w_first = matrix_low(ring), x_first = w_first + (deep * w_bytes >> 4);
            const uint32_t stage_on = stage >> 4, w_on = w_bytes >> 4;
            for (int32_t t = begin; t < total; t += stride) {
                if (!PAIR || rank == 0) {
                    const Tile o = tile_at(a, s, t, &group, features);
                    const uint32_t unit = PAIR ? 32u : 16u;
                    const uint32_t inst = instruction(m.f16, PAIR ? 256u : 128u,
                                                      ((uint32_t)o.rows + unit - 1) / unit * unit);
                    const uint32_t in_use = PAIR ? ((uint32_t)o.rows + 31u) / 32u * 16u
                                                 : (uint32_t)o.rows;
                    uint32_t box = 0;
                    while (box + 1 < kBoxes && a.x_box[box + 1] >= in_use) ++box;
                    const uint32_t x_on = a.x_box[box] * kRowBytes >> 4;
                    /* each stage's barrier is looked at before the products of the one before are
                     * issued, so that the look costs no time of its own */
                    bool there = mbar_try_wait(full + 8 * at, phase);
                    for (uint32_t k = k0; k < k1;) {
                        const uint32_t d = tmem + buf * a.acc_on, stop = min(k1, k + part);
                        ok = ok && mbar_wait(acc_empty + 8 * buf, buf_phase, s);
                        fence_after();
                        uint32_t add = 0; /* the first product overwrites */
                        for (; k < stop; k += deep) {
                            ok = ok && (there || mbar_wait(full + 8 * at, phase, s));
                            if (!ok) break;
                            fence_after();
                            uint32_t blocks = min(deep, k1 - k);
                            uint32_t w = w_first + at * stage_on, x = x_first + at * stage_on;
                            const uint32_t done = empty + 8 * at;
                            if (++at == stages) {
                                at = 0;
                                phase ^= 1;
                            }
                            there = k + deep < k1 && mbar_try_wait(full + 8 * at, phase);
                            do {
#pragma unroll
                                for (uint32_t q = 0; q < kDepth / 16; ++q) { /* 32 bytes further */
                                    mma<PAIR>(d, w + q * 2, x + q * 2, inst, add);
                                    add = 1;
                                }
                                w += w_on;
                                x += x_on;
                            } while (--blocks);
                            commit<PAIR>(done);
                        }
                        if (!ok) break;
                        commit<PAIR>(acc_full + 8 * buf);
                        ++sums;
                        if (buf) buf_phase ^= 1;
                        buf ^= 1;
                    }
                }
                if (sync_tiles) {
                    cluster_sync();
                    cluster_done();
                }
            }
            if (!ok) { /* of a sum that was given up: its products count as one */
                commit<PAIR>(acc_full + 8 * buf);
                ++sums;
            }
            s->sums = sums;
        } else if (sync_tiles) {
            for (int32_t t = begin; t < total; t += stride) {
                cluster_sync();
                cluster_done();
            }
        }
        __syncwarp();
    } else {
        uint32_t buf = 0, buf_phase = 0;
        int32_t group = 0;
        /* Gives an accumulator back once its sums have been read.  Relaxed: the stores of y need not
         * have ended. */
        const auto acc_release = [&](uint32_t &b, uint32_t &ph) {
            fence_before();
            __syncwarp();
            if (lane == 0) {
                const uint32_t bar = acc_empty + 8 * b;
                asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                                 PAIR ? map_to(bar, 0) : bar)
                             : "memory");
            }
            if (b) ph ^= 1;
            b ^= 1;
        };
        const int quarter = warp & 3; /* of the lanes; the warp's batches start at `from` */
        const int32_t from = (warp >> 2) * kBatch;
        const uint32_t lanes = s->tmem + ((uint32_t)quarter * 32u << 16);
        float *partial = reinterpret_cast<float *>(
            raw + (ring - smem_addr(raw)) + a.stages * stage); /* [bn][128], split > 1 */
        /* The first tile is gone through twice: first without a wait, without rows and so without
         * stores, which brings the code into the instruction cache while the sums are under way. */
        bool dry = true;
        float *const staging = partial + warp * (kBatch * kStageRow); /* kWide, kNarrow */
        for (int32_t t = begin; t < total;) {
            const Tile o = tile_at(a, s, t, &group, features);
            int64_t col = o.feature + (GATED ? quarter * 16 + (lane >> 4) * 8 + (lane & 7)
                                             : quarter * 32 + lane);
            if constexpr (PAIR) col += rank * per_cta;
            if ((uint32_t)(quarter * 32 + lane) >= a.fr) col = a.outs; /* a lane without a row */
            float bias = 0.0f; /* of the lane's weight row */
            if (m.bias && col < a.outs) {
                const int64_t at = col + (GATED && (lane & 8) ? m.bias_up : 0);
                bias = m.bias_f32 ? value(static_cast<const float *>(m.bias), at)
                                  : value(m.bias, at, m.f16);
            }
            int32_t c0 = 0, c1 = o.rows; /* the tokens that this CTA finishes */
            if (sync_tiles) {            /* of a cluster, each its share */
                const int32_t even = (((o.rows - 1) >> share) + 2) & ~1;
                c0 = (int32_t)rank * even;
                c1 = min(o.rows, c0 + even);
            }
            /* the warp's columns of y, and the end of those that there are */
            const int64_t first = o.feature + (PAIR ? rank * per_cta : 0) + quarter * (GATED ? 16 : 32);
            const int32_t lanes_in = (int32_t)a.fr - quarter * 32;
            int64_t limit = first + (GATED ? lanes_in / 2 : lanes_in);
            if (limit > a.outs) limit = a.outs;
            /* the residual of the next batch, on its way since the one before */
            uint4 wide[4];
            uint32_t narrow[16];
            Residual next;
            if (!dry && c0 + from < c1) {
                const int64_t row = o.row + c0 + from;
                const int n = c1 - c0 - from;
                if constexpr (WIDE) fetch_wide<GATED, F32>(a, row, n, first, limit, wide);
                else if constexpr (NARROW) fetch_narrow<GATED>(a, row, n, first, limit, narrow);
                else fetch<F32, GATED ? 8 : 16>(a, place_of<GATED>(row, n, col), next);
            }
            /* the parts before the last are added up in tensor memory */
            bool more = false; /* a sum lies there */
            if (!dry) {
                for (uint32_t k = k0 + part; EXACT && k < k1; k += part) {
                    ok = ok && mbar_wait(acc_full + 8 * buf, buf_phase, s);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    fence_after();
                    for (int32_t c = from; ok && c < o.rows; c += kRound) {
                        float v[16], u[16];
                        tmem_load(lanes + buf * a.acc_on + c, v);
                        if (more) {
                            tmem_load(lanes + 2 * a.acc_on + c, u);
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] += u[j];
                        }
                        tmem_store(lanes + 2 * a.acc_on + c, v);
                    }
                    more = true;
                    acc_release(buf, buf_phase);
                }
                ok = ok && mbar_wait(acc_full + 8 * buf, buf_phase, s);
                ok = __all_sync(0xFFFFFFFFu, ok);
                fence_after();
            }
            const uint32_t src = lanes + buf * a.acc_on, sum = lanes + 2 * a.acc_on;
            uint32_t sharers = 0;
            float v[16];
            if (sync_tiles) {
                for (int32_t c = from; ok && c < o.rows; c += kRound) {
                    __syncwarp();
                    sum_load(src + c, sum + c, EXACT && more, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        partial[(c + j) * kRows + quarter * 32 + lane] = v[j];
                }
                if (!dry) cluster_sync();
                sharers = dry ? 1u : 1u << share;
            }
            const bool few = c1 - c0 <= 4;
            const uint32_t base = smem_addr(partial) + (uint32_t)(quarter * 32 + lane) * 4u;
            if (dry) c1 = min(c1, c0 + 1);
            if constexpr (WIDE || NARROW) {
                for (int32_t c = from; ok && c < c1; c += kRound) {
                    __syncwarp();
                    sum_load(src + c, sum + c, EXACT && more, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        staging[j * kStageRow + lane] = m.bias ? v[j] + bias : v[j];
                    __syncwarp();
                    const int64_t row = o.row + c;
                    const int n = dry ? 0 : c1 - c;
                    if constexpr (WIDE) {
                        uint4 r[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) r[j] = wide[j];
                        if (c + kRound < c1)
                            fetch_wide<GATED, F32>(a, row + kRound, n - kRound, first, limit, wide);
                        finish_wide<KIND>(a, staging, row, n, first, limit, r);
                    } else {
                        uint32_t r[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) r[j] = narrow[j];
                        if (c + kRound < c1)
                            fetch_narrow<GATED>(a, row + kRound, n - kRound, first, limit, narrow);
                        finish_narrow<KIND>(a, staging, row, n, first, limit, r);
                    }
                }
            } else {
                for (int32_t c = c0 + from; ok && c < c1; c += kRound) {
                    __syncwarp();
                    if (sharers == 0) {
                        sum_load(src + c, sum + c, EXACT && more, v);
                    } else {
                        float p[4][16]; /* all on their way before the first is added */
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint32_t from = map_to(base, dry ? rank : (uint32_t)r % sharers) +
                                                  (uint32_t)c * (kRows * 4u);
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                p[r][j] = 0.0f;
                                if (r < sharers && j < c1 - c)
                                    asm volatile("ld.shared::cluster.f32 %0, [%1];"
                                                 : "=f"(p[r][j])
                                                 : "r"(from + (uint32_t)j * (kRows * 4u)));
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            v[j] = ((p[0][j] + p[1][j]) + p[2][j]) + p[3][j];
                    }
                    const Place p = place_of<GATED>(o.row + c, dry ? 0 : c1 - c, col);
                    const Residual r = next;
                    if (c + kRound < c1)
                        fetch<F32, GATED ? 8 : 16>(
                            a, place_of<GATED>(o.row + c + kRound, c1 - c - kRound, col), next);
                    if (few) finish<KIND, 4>(a, v, p, bias, r);
                    else finish<KIND, 16>(a, v, p, bias, r);
                }
            }
            if (dry) {
                dry = false;
                continue;
            }
            acc_release(buf, buf_phase);
            if (sync_tiles) cluster_done();
            t += stride;
        }
    }

    fence_before();
    __syncthreads();
    if (*(volatile int *)&s->dead) {
        if (threadIdx.x == 0) drain(a, s, PAIR && rank);
        __syncthreads();
    }
    if constexpr (PAIR) cluster_sync();
    if (warp == kIssuer) {
        const uint32_t tmem = s->tmem;
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
    std::atomic<int> clusters[64][3]; /* by kernel and split: clusters that run at once, plus one */
    std::atomic<uint64_t> ready;   /* kernels whose shared memory is granted */
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

/* The kernels that there are.  The second product of the experts alone takes kF32 without kExact, with
 * y on the 16-byte grid and no activation. */
struct Kernel {
    int kind;
    const void *fn;
};
template <int KIND> Kernel kernel() { return {KIND, reinterpret_cast<const void *>(&cfa_matmul_kernel<KIND>)}; }
constexpr int kHalf = 0, kSingle = kF32 | kExact;
const Kernel g_kernel[] = {
    kernel<kWide>(),
    kernel<kWide | kCurves>(),
    kernel<kWide | kGated>(),
    kernel<kWide | kGated | kCurves>(),
    kernel<kWide | kPair>(),
    kernel<kWide | kPair | kCurves>(),
    kernel<kWide | kPair | kGated>(),
    kernel<kWide | kPair | kGated | kCurves>(),
    kernel<kWide | kF32>(),
    kernel<kWide | kF32 | kPair>(),
    kernel<kWide | kSingle>(),
    kernel<kWide | kSingle | kCurves>(),
    kernel<kWide | kSingle | kGated | kCurves>(),
    kernel<kWide | kSingle | kPair>(),
    kernel<kWide | kSingle | kPair | kCurves>(),
    kernel<kWide | kSingle | kPair | kGated | kCurves>(),
    kernel<kNarrow | kCurves>(),
    kernel<kNarrow | kCurves | kGated>(),
    kernel<kNarrow | kCurves | kPair>(),
    kernel<kNarrow | kCurves | kPair | kGated>(),
    kernel<kHalf>(),
    kernel<kCurves>(),
    kernel<kGated>(),
    kernel<kGated | kCurves>(),
    kernel<kF32>(),
    kernel<kSingle>(),
    kernel<kSingle | kCurves>(),
    kernel<kSingle | kGated | kCurves>(),
    kernel<kSingle | kPair>(),
    kernel<kSingle | kPair | kCurves>(),
    kernel<kSingle | kPair | kGated | kCurves>(),
};
constexpr int kKernels = sizeof g_kernel / sizeof g_kernel[0];
static_assert(kKernels <= 64, "a bit each in Device");

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
    c->cfg.numAttrs = 0;
    if (cluster > 1) {
        cudaLaunchAttribute &attr = c->attr[c->cfg.numAttrs++];
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = cluster;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    }
    if (early) {
        cudaLaunchAttribute &attr = c->attr[c->cfg.numAttrs++];
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
    }
}

/* Clusters of 2^log CTAs that the device runs at once. */
cudaError_t clusters_of(Device &d, const void *fn, unsigned kernel, unsigned log, int *n)
{
    std::atomic<int> &known = d.clusters[kernel][log];
    int v = known.load();
    if (!v) {
        Config c;
        configure(&c, 1u << log, 1u << log, false, nullptr);
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&v, fn, &c.cfg);
        if (e) return e;
        known.store(++v);
    }
    *n = v - 1;
    return *n > 0 ? cudaSuccess : cudaErrorInvalidConfiguration;
}

/* The cut of sizes seen lately on this thread is looked up: weighing them all takes as long as a
 * launch. */
Cut cut_of(const cfa_matmul *m, int sms)
{
    struct Known {
        int64_t likely, w_rows, cols;
        int32_t busy, gated, y_f32, exact, sms;
        Cut cut;
    };
    static thread_local Known known[64] = {};
    const uint64_t key = ((uint64_t)m->likely * 0x9E3779B97F4A7C15ull) ^
                         ((uint64_t)m->w_rows * 0xC2B2AE3D27D4EB4Full) ^
                         ((uint64_t)m->cols * 0x165667B19E3779F9ull) ^ (uint64_t)m->busy;
    Known &k = known[(key >> 40) & 63u];
    if (k.likely != m->likely || k.w_rows != m->w_rows || k.cols != m->cols || k.busy != m->busy ||
        k.gated != m->gated || k.y_f32 != m->y_f32 || k.exact != m->exact || k.sms != sms)
        k = {m->likely, m->w_rows, m->cols, m->busy, m->gated, m->y_f32, m->exact, sms,
             choose(m, m->gated ? m->w_rows / 2 : m->w_rows,
                    (uint32_t)((m->cols + kDepth - 1) / kDepth), sms)};
    return k.cut;
}

cudaError_t launch(const cfa_matmul *m, Device &d, int sms, const Cut &cut, int early, int release,
                   cudaStream_t stream)
{
    cudaError_t e;
    const bool gated = m->gated, pair = cut.pair;
    if (!cut.bn || !cut.fr) return cudaErrorInvalidValue;
    Args a = {};
    a.m = *m;
    a.outs = gated ? m->w_rows / 2 : m->w_rows;
    a.steps = (uint32_t)((m->cols + kDepth - 1) / kDepth);
    a.release = (uint32_t)release;
    a.polls = m->lose == 0 ? kSpinLimit : m->lose == 1 ? 4096 : 0;
    a.lose = m->lose;
    a.early_w = m->w_ready && !pair;
    a.bn = cut.bn;
    a.fr = cut.fr;
    a.split = cut.split;
    const uint32_t features = (pair ? 2 : 1) * (gated ? a.fr / 2 : a.fr);
    a.f_tiles = (uint32_t)((a.outs + features - 1) / features);
    const int64_t most = ((m->tokens + a.bn - 1) / a.bn + m->busy - 1) * a.f_tiles;
    a.total = (int32_t)most;
    const uint64_t two = m->y_f32 ? 8 : 4;
    a.pairs = (((uintptr_t)m->y | (uintptr_t)m->residual) % two) == 0 &&
              (m->tokens <= 1 || (m->y_stride % 2 == 0 && (!m->residual || m->r_stride % 2 == 0)));
    const uint32_t x_rows = pair ? a.bn / 2 : a.bn;
    a.x_box[0] = x_rows;
    if (m->offs) /* ragged groups: half as high, a quarter, an eighth */
        for (uint32_t i = 1; i < kBoxes && x_rows >> i >= 16; ++i) a.x_box[i] = (x_rows >> i) / 8 * 8;
    const uint32_t block = (a.fr + x_rows) * kRowBytes;
    a.deep = deep_of(cut);
    const uint32_t stage = block * a.deep;
    a.whole = (uint32_t)(m->cols / kDepth);
    a.f_whole = gated && a.outs % 8 ? (int32_t)(a.outs / 8 * 8) : INT32_MAX;
    /* the products read kRows rows of each block of w, whatever lies behind the a.fr of them */
    const uint32_t after = a.fr + a.deep * x_rows;
    const uint32_t behind = kRows > after ? (kRows - after) * kRowBytes : 0;
    const auto stages_beside = [&](uint32_t bytes) {
        const uint32_t left = kSmem - shared_bytes(m->n_groups) - 1024u - (bytes > behind ? bytes : behind);
        return left / stage < kMaxStages ? left / stage : kMaxStages;
    };
    /* Clusters have their sums in shared memory anyway, and a few tokens are stored as fast from the
     * registers.  So are those of low tiles where the staging would cost the ring a stage: they wait for
     * memory (64 tokens through all of 8 experts of 14,336 x 4096: 428 us, 414 from registers). */
    int kind = (pair ? kPair : 0) | (gated ? kGated : 0);
    if (m->exact) kind |= kSingle;
    else if (m->y_f32) kind |= kF32;
    a.stages = stages_beside(a.split ? a.bn * kRows * 4u : 0u);
    const uint32_t staged = stages_beside(kStageBytes);
    if (!a.split && m->tokens > 4 && (pair || a.bn > 128 || staged == a.stages || !a.pairs)) {
        if ((((uintptr_t)m->y | (uintptr_t)m->residual) & 15u) == 0 &&
            m->y_stride * (int64_t)(two / 2) % 16 == 0 &&
            (!m->residual || m->r_stride * (int64_t)(two / 2) % 16 == 0))
            kind |= kWide;
        else if (!m->y_f32)
            kind |= kNarrow | kCurves;
        if (kind & (kWide | kNarrow)) a.stages = staged;
    }
    if (m->act == CFA_ACT_GELU || m->act == CFA_ACT_GELU_TANH || (m->exact && gated)) kind |= kCurves;
    int kernel = 0;
    while (kernel < kKernels && g_kernel[kernel].kind != kind) ++kernel;
    if (kernel == kKernels) return cudaErrorInvalidValue;
    const void *fn = g_kernel[kernel].fn;
    for (a.acc_on = 16; a.acc_on < a.bn; a.acc_on *= 2) {
    }
    a.tmem_cols = m->exact ? 4 * a.acc_on : 2 * a.acc_on; /* a power of two */

    if (!(d.ready.load() & 1ull << kernel)) {
        e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
        if (e) return e;
        d.ready.fetch_or(1ull << kernel);
    }
    const unsigned log = pair ? 1 : a.split, size = 1u << log;
    int clusters = sms;
    if (log) {
        e = clusters_of(d, fn, (unsigned)kernel, log, &clusters);
        if (e) return e;
    }
    if (clusters > most) clusters = (int)most;

    const cuuint64_t k = (cuuint64_t)m->cols, whole = (k + 7) / 8 * 8;
    const cuuint64_t wld = (m->w_rows > 1 ? (cuuint64_t)m->w_stride : whole) * 2;
    const cuuint64_t xld = (m->tokens > 1 ? (cuuint64_t)m->x_stride : whole) * 2;
    /* The maps of whole blocks have the blocks as a dimension, so that one load brings several. */
    bool fine = true;
    const cuuint64_t on = kRowBytes, groups = (cuuint64_t)m->n_groups, blocks = a.whole;
    const cuuint64_t outs = (cuuint64_t)a.outs, rows = (cuuint64_t)m->w_rows;
    const cuuint64_t tokens = (cuuint64_t)m->tokens;
    if (blocks && a.f_whole) {
        if (gated) { /* 64 columns, 8 rows, gate or up of each group, the next 8 rows, block */
            const cuuint64_t dim[5] = {kDepth, 8, 2 * groups, outs / 8, blocks};
            const cuuint64_t stride[4] = {wld, wld * outs, wld * 8, on};
            const cuuint32_t box[5] = {kDepth, 8, 2, a.fr / 16, a.deep};
            fine = encode(&a.wmap, m->f16, m->w, 5, dim, stride, box);
        } else {
            const cuuint64_t dim[4] = {kDepth, rows, blocks, groups};
            const cuuint64_t stride[3] = {wld, on, wld * rows};
            const cuuint32_t box[4] = {kDepth, a.fr, a.deep, 1};
            fine = encode(&a.wmap, m->f16, m->w, 4, dim, stride, box);
        }
        const cuuint64_t dim[3] = {kDepth, tokens, blocks};
        const cuuint64_t stride[2] = {xld, on};
        for (uint32_t i = 0; fine && i < kBoxes && a.x_box[i]; ++i) {
            const cuuint32_t box[3] = {kDepth, a.x_box[i], a.deep};
            fine = encode(&a.xmap[i], m->f16, m->x, 3, dim, stride, box);
        }
    }
    if (fine && (a.f_whole != INT32_MAX || a.steps > a.whole)) {
        if (gated) {
            const cuuint64_t dim[4] = {k, outs, 2, groups};
            const cuuint64_t stride[3] = {wld, wld * outs, wld * outs * 2};
            const cuuint32_t box[4] = {kDepth, 8, 2, 1};
            fine = encode(&a.wtail, m->f16, m->w, 4, dim, stride, box);
        } else {
            const cuuint64_t dim[3] = {k, rows, groups};
            const cuuint64_t stride[2] = {wld, wld * rows};
            const cuuint32_t box[3] = {kDepth, a.fr, 1};
            fine = encode(&a.wtail, m->f16, m->w, 3, dim, stride, box);
        }
        const cuuint64_t dim[3] = {k, tokens, 1};
        const cuuint64_t stride[2] = {xld, xld * tokens};
        for (uint32_t i = 0; fine && i < kBoxes && a.x_box[i]; ++i) {
            const cuuint32_t box[3] = {kDepth, a.x_box[i], 1};
            fine = encode(&a.xtail[i], m->f16, m->x, 3, dim, stride, box);
        }
    }
    if (!fine) return cudaErrorInvalidValue;

    Config c;
    configure(&c, (unsigned)clusters * size, size, early != 0, stream);
    void *p[] = {&a};
    return cudaLaunchKernelExC(&c.cfg, fn, p);
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
    return launch(m, d, sms, cut_of(m, sms), early, release, stream);
}

/* Every thread has its own record of what it has been told: one that asks takes nothing from another,
 * and nothing that is counted between two of its calls is lost. */
cudaError_t cfa_matmul_status(int *word)
{
    static thread_local cfa_op_counts seen[kMaxDevices] = {};
    cfa_op_counts now;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (!e && (dev < 0 || dev >= kMaxDevices)) e = cudaErrorInvalidDevice;
    if (!e) e = cudaMemcpyFromSymbol(&now, g_counts, sizeof now);
    if (!e) *word = cfa_op_news(seen + dev, now);
    return e;
}

/* Products of 8 tokens on the default stream, by single CTAs, by clusters of two and four and by pairs:
 * first with loaders that ask for nothing, so that waits run out after 4096 polls each, then with
 * epilogues that give up at once, while all loads of the tile (four blocks, which the ring holds) are on
 * their way.  *word receives what this has been counted as, in counts of its own: 1, or the first that
 * was counted as something else. */
cudaError_t cfa_matmul_selftest(int *word)
{
    const Cut cuts[] = {{false, 16, 128, 0}, {false, 16, 128, 1}, {false, 16, 128, 2}, {true, 96, 128, 0}};
    const size_t w_bytes = 256 * 1024 * 2, x_bytes = 8 * 1024 * 2, y_bytes = 8 * 256 * 2;
    uint8_t *buf = nullptr;
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (!e && (dev < 0 || dev >= kMaxDevices)) e = cudaErrorInvalidDevice;
    if (!e) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (!e) e = cudaMalloc(reinterpret_cast<void **>(&buf), w_bytes + x_bytes + y_bytes);
    if (e) return e;
    e = cudaMemset(buf, 0, w_bytes + x_bytes + y_bytes);
    cfa_matmul m = {};
    m.w = buf;
    m.x = buf + w_bytes;
    m.y = buf + w_bytes + x_bytes;
    m.tokens = m.likely = 8;
    m.n_groups = m.busy = 1;
    m.w_rows = m.y_stride = 256;
    *word = 1;
    for (int i = 0; i < 8; ++i) {
        const Cut &cut = cuts[i / 2];
        cfa_op_counts before, after;
        m.lose = 1 + i % 2;
        m.cols = m.x_stride = m.w_stride = m.lose == 1 ? 1024 : (int64_t)256 << cut.split;
        if (!e) e = cudaMemcpyFromSymbol(&before, g_counts, sizeof before, sizeof before);
        if (!e) e = launch(&m, g_device[dev], sms, cut, 0, 0, nullptr);
        if (!e) e = cudaDeviceSynchronize();
        if (!e) e = cudaMemcpyFromSymbol(&after, g_counts, sizeof after, sizeof after);
        if (e) break;
        const int news = cfa_op_news(&before, after);
        if (*word == 1) *word = news;
    }
    const cudaError_t freed = cudaFree(buf);
    return e ? e : freed;
}
