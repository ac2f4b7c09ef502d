// The order in which a product's tiles are walked through (csrc/rcd_walk.h): every tile once, whatever the bands; of symmetric products the blocks on
// and below the diagonal, those below it with their transposes.  And the shared memory that a block asks for.
#include <cmath>
#include <cstdio>
#include <set>
#include <utility>

#include "rcd_walk.h"

using namespace rcd;

static int fail(const char *what, int a, int b, int c)
{
    std::printf("%s: %d %d %d\n", what, a, b, c);
    return 1;
}

int main()
{
    for (int tm = 1; tm < 40; ++tm)
        for (int tn = 1; tn < 40; ++tn)
            for (int band : {1, 3, 8, tn}) {
                const Walk w{tm, tn, tm * tn, band < tn ? band : tn, 2, 0, 0};
                std::set<std::pair<int, int>> seen;
                for (int u = 0; u < 4 * w.tiles; ++u) {
                    const Unit t = unit_of(w, u);
                    if (t.batch != u / w.tiles / 2 || t.split != u / w.tiles % 2 || t.mirror || t.m < 0 || t.m >= tm || t.n < 0 || t.n >= tn) return fail("outside", tm, tn, u);
                    if (u < w.tiles && !seen.insert({t.m, t.n}).second) return fail("twice", tm, tn, u);
                }
            }
    for (int blocks = 1; blocks < 600; blocks += blocks < 80 ? 1 : 37)
        for (int subM : {1, 2})
            for (int subN : {1, 2, 4}) {
                const Walk w{blocks * subM, blocks * subN, blocks * (blocks + 1) / 2 * subM * subN, 1, 1, subM, subN};
                std::set<std::pair<int, int>> seen;
                for (int u = 0; u < w.tiles; ++u) {
                    const Unit t = unit_of(w, u);
                    const int i = t.m / subM, j = t.n / subN;
                    if (t.m < 0 || i >= blocks || t.n < 0 || j > i || t.mirror != (i != j) || t.batch || t.split) return fail("wrong", blocks, subM, u);
                    if (!seen.insert({t.m, t.n}).second) return fail("twice", blocks, subM, u);
                }
            }
    // Shared memory: what an instruction reads of A (128 rows) and of B lies inside, whatever lies behind the ring; and a block gets no more than there is.
    for (int rows = 1; rows <= 128; ++rows)
        for (int tn = 16; tn <= 256; tn += 16)
            for (int besides = 0; besides < 90 * 1024; besides += 1021) {
                const int aRows = (rows + 7) / 8 * 8;
                const OperandRing r = ring_of(aRows, tn, besides);
                const int last = (r.stages - 1) * r.stageBytes;
                if (r.stages < 2 || r.bytes > kBlockShared || r.stages * r.stageBytes + besides > r.bytes) return fail("shared memory", rows, tn, besides);
                if (last + 128 * kOperandSlab > r.bytes || last + (aRows + tn) * kOperandSlab > r.bytes) return fail("read outside", rows, tn, besides);
            }
    return 0;
}
