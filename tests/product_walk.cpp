// The order in which a product's tiles are walked through (csrc/rcd_walk.h): every tile once, whatever the bands; of symmetric products the blocks on
// and below the diagonal, those below it with their transposes.
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
    return 0;
}
