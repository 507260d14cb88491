/*
 * How a product (cfa_matmul.cu) is cut into tiles: heights of the tiles, pairs or clusters of CTAs, and
 * blocks per stage, by an estimate of its time from its sizes.  Host code.
 */
#ifndef CFA_TILES_H
#define CFA_TILES_H

#include <math.h>

#include "cfa_ops.h"

namespace cfa_tiles {

constexpr uint32_t kRows = 128;          /* weight rows per CTA, at most */
constexpr uint32_t kDepth = 64;          /* columns of w and x per block: one 128-byte swizzle row */
constexpr uint32_t kDeepBytes = 65536;   /* a stage takes more than one block up to this (of a pair,
                                            whose products take longer: half of it) */
constexpr uint32_t kRowBytes = kDepth * 2;
constexpr uint32_t kSmem = 232448;       /* all that a CTA may have: one CTA per SM, so that the
                                            tensor memory is never asked for twice at once */
constexpr int32_t kBatch = 16, kRound = 32; /* columns that one of the two takes at a time, and both */
constexpr int kStageRow = 36;            /* words per token of a batch that is turned round in shared
                                            memory before it is stored: 32, and four more */
constexpr uint32_t kStageBytes = 8 * kBatch * kStageRow * 4;

/* How a product is cut. */
struct Cut {
    bool pair;
    uint32_t bn, fr, split; /* split: log2 */
};

/* Blocks of a stage: as many as kDeepBytes hold (of a pair, whose products take longer, half of it), if
 * the ring then has three stages or more (with two, 256 tokens x 4096 x 14,336 took 47 us where 37 do). */
inline uint32_t deep_of(const Cut &c)
{
    const uint32_t block = (c.fr + (c.pair ? c.bn / 2 : c.bn)) * kRowBytes;
    const uint32_t ring = kSmem - 4096u - (c.split ? c.bn * kRows * 4u : kStageBytes);
    uint32_t deep = 4;
    while (deep > 1 && (block * deep > (c.pair ? kDeepBytes / 2 : kDeepBytes) ||
                        block * deep * 3 > ring))
        deep /= 2;
    return deep;
}

/* Estimated microseconds of a product.  The CTAs take their tiles in turns.  A turn takes the longer
 * of a tile's blocks, at the pace of their products and their issue or of what one SM can take in, and
 * of the turn's bytes, at the rate of L2 and of memory; the epilogue of a tile runs under the next
 * tile's products, but for the last.  (Bytes by turns: a last turn of few CTAs cannot draw what memory
 * gives.)  Tiles whose rows of y do not fill lines of 128 bytes take longer to store.
 * The constants are a fit to 16,100 timings: 224 sizes (1 to 4096 tokens, 256 to 28,672 rows, 384 to
 * 14,336 columns), each cut in up to 130 ways.  The cut that this puts first takes 1.9 % longer than
 * the best of those on average, 20 % at the worst. */
inline double estimate(const cfa_matmul *m, int64_t outs, uint32_t steps, int sms, int64_t rows,
                       const Cut &c)
{
    const double kSplit[3] = {0.0, 1.67, 2.51}; /* one, two and four CTAs per tile */
    const uint32_t features = (c.pair ? 2 : 1) * (m->gated ? c.fr / 2 : c.fr);
    const int64_t n_tiles = (rows + c.bn - 1) / c.bn;
    const int64_t tiles = n_tiles * m->busy * ((outs + features - 1) / features);
    /* clusters of four leave some SMs out */
    const int64_t slots = c.pair || c.split == 1 ? sms / 2 : c.split == 2 ? sms * 9 / 38 : sms;
    const double blocks = (double)((steps + (1u << c.split) - 1) >> c.split);
    const double used = n_tiles == 1 ? (double)((rows + 15) / 16 * 16) : (double)c.bn;
    const double bytes = (double)(c.fr + (c.pair ? c.bn / 2 : c.bn)) * kRowBytes;
    const double mma = used * (c.pair ? 0.00075 : 0.00087);
    double step = (mma > 0.152 ? mma : 0.152) + 0.078 / deep_of(c);
    if (step < bytes / 166e3) step = bytes / 166e3;
    const double tokens = (double)(rows < c.bn ? rows : c.bn);
    const bool lines = (m->gated ? c.fr / 2 : c.fr) * (m->y_f32 ? 4 : 2) % 128 == 0;
    const double epilogue = (lines ? 0.0146 : 0.0194) * tokens / (1u << c.split), products = blocks * step;
    const double turn = (products > epilogue ? products : epilogue) + 0.6;
    const double l2 = steps * (c.pair ? 2 : 1) * bytes / 20e6; /* per tile */
    const double mem = 2.0 * m->cols * ((double)m->w_rows * m->busy + (double)m->likely) / 6.6e6 /
                       (double)tiles;
    const double share = l2 > mem ? l2 : mem;
    const int64_t full = tiles / slots, left = tiles - full * slots;
    double us = 2.8 + kSplit[c.split] + (c.split ? 0.006 * tokens : 0.0) + epilogue;
    us += (double)full * (turn > (double)slots * share ? turn : (double)slots * share);
    if (left) us += turn > (double)left * share ? turn : (double)left * share;
    return us;
}

/* The cut with the least estimate.  Groups are taken as equally full, their number of rows being all
 * that the host knows. */
inline Cut choose(const cfa_matmul *m, int64_t outs, uint32_t steps, int sms)
{
    const int64_t busy = m->busy, rows = (m->likely + busy - 1) / busy;
    /* columns of a tile: two accumulators fill the tensor memory's 512, exact sums take three (of four
     * places).  The loop below starts with the fewest tiles of that height and goes through these in any
     * case, so that there is a cut for every number of tokens */
    const uint32_t most = m->exact ? 128 : 256;
    const int64_t fewest = (rows + most - 1) / most, end = (rows + 255) / 256 + 64;
    Cut best = {};
    double least = 1e30;
    for (int pair = 0; pair < 2; ++pair) {
        const uint32_t unit = pair ? 32 : 16;
        uint32_t last = 0;
        for (int64_t parts = fewest; parts == fewest || parts < end; ++parts) {
            const int64_t even = (rows + parts - 1) / parts;
            /* uneven groups: room for two standard deviations of evenly drawn choices, so that most
             * have one tile */
            const int64_t room = busy > 1 && parts == 1 ? even + 2 + (int64_t)(2.0 * sqrt((double)even))
                                                        : even;
            uint32_t bn = (uint32_t)((room + unit - 1) / unit * unit);
            if (bn > most) bn = most;
            if (pair && bn < 96) break;
            if (bn == last) continue;
            last = bn;
            for (uint32_t fr = pair ? kRows : 32; fr <= kRows; fr += 16) {
                const uint32_t features = (pair ? 2 : 1) * (m->gated ? fr / 2 : fr);
                const int64_t tiles = (rows + bn - 1) / bn * busy * ((outs + features - 1) / features);
                for (uint32_t split = 0; split < 3; ++split) {
                    /* only while there is an SM for each: clusters go through their tiles one after the
                     * other, and with more turns took 175 us where single CTAs take 109 */
                    if (split && (pair || bn > 128 || steps < 4u << split || tiles << split > sms))
                        break;
                    const Cut c = {pair != 0, bn, fr, split};
                    const double us = estimate(m, outs, steps, sms, rows, c);
                    if (us < least * 0.995) {
                        least = us;
                        best = c;
                    }
                }
            }
        }
    }
    return best;
}

} // namespace cfa_tiles

#endif /* CFA_TILES_H */
