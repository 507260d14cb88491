// The cut of products (paper_2607_18957_gb300/csrc/cfa_tiles.h) over the whole range of sizes: there is
// one for every number of tokens, the launch can use it, and its tiles can be counted in 32 bits.
#include <cstdio>
#include <random>

#include "cfa_tiles.h"

using namespace cfa_tiles;

static int check(int64_t tokens, int64_t rows, int64_t cols, int gated, int f32, int exact,
                 int32_t groups, int sms)
{
    cfa_matmul m = {};
    m.tokens = m.likely = tokens;
    m.w_rows = gated ? 2 * rows : rows;
    m.cols = cols;
    m.gated = gated;
    m.y_f32 = f32;
    m.exact = exact;
    m.n_groups = groups;
    m.busy = (int32_t)(tokens < groups ? tokens : groups);
    const Cut c = choose(&m, rows, (uint32_t)((cols + kDepth - 1) / kDepth), sms);
    const uint32_t unit = c.pair ? 32 : 16;
    const bool ok = c.bn >= unit && c.bn % unit == 0 && c.bn <= (exact ? 128u : 256u) &&
                    c.fr >= 32 && c.fr <= kRows && c.fr % 16 == 0 && (!c.pair || c.fr == kRows) &&
                    c.split <= 2 && (!c.split || !c.pair) && deep_of(c) >= 1;
    if (!ok)
        std::printf("%lld tokens x %lld x %lld, gated %d f32 %d exact %d, %d groups, %d SMs: pair %d bn "
                    "%u fr %u split %u\n", (long long)tokens, (long long)rows, (long long)cols, gated,
                    f32, exact, groups, sms, c.pair, c.bn, c.fr, c.split);
    return !ok;
}

int main()
{
    const int64_t most = (1ll << 31) - 1;
    int bad = 0;
    for (int gated = 0; gated < 2; ++gated)
        for (int kind = 0; kind < 3; ++kind) { // results of 2 bytes, fp32, fp32 kept exact
            const int f32 = kind > 0, exact = kind == 2;
            for (int64_t t = 1; t <= 40000; t += t < 600 ? 1 : t > 16100 && t < 16500 ? 1 : 97)
                bad += check(t, 8, 4096, gated, f32, exact, 1, 152);
            for (int64_t t = 40000; t <= most; t = t * 5 / 4) {
                bad += check(t, 1, 64, gated, f32, exact, 1, 152);
                bad += check(t, 28672, 4096, gated, f32, exact, 1, 152);
            }
            bad += check(most, 1, 1, gated, f32, exact, 1, 152);
            if (!exact)
                for (int64_t t = 1; t <= most; t = t * 3 / 2 + 1)
                    for (int32_t g : {1, 2, 8, 60, 128, 1024})
                        bad += check(t, 768, 2048, gated, f32, exact, g, 152);
        }
    std::mt19937_64 rng(7);
    const auto size = [&](int bits) { return (int64_t)1 + (int64_t)(rng() >> (64 - 1 - rng() % bits)); };
    for (int i = 0; i < 4000; ++i) {
        const int exact = rng() % 2;
        bad += check(size(30), size(22), size(22), rng() % 2, exact || rng() % 2, exact,
                     exact ? 1 : (int32_t)size(9), rng() % 4 ? 152 : 8 + (int)(rng() % 200));
    }
    std::printf("%d without a cut\n", bad);
    return bad != 0;
}
