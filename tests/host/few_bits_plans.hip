// Plans of weight gradients: that the sizes the GPU tests take are of the forms they are taken for.
#include <cstdio>

#include "lowbits.h"

static int fails = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++fails; } \
    } while (0)

using namespace daq;

enum Form { kTiles, kFlat };
static bool is(const WgradPlan& w, Form form, bool big, bool several) { return !w.few && w.flat == (form == kFlat) && w.big == big && (w.splits > 1) == several; }

int main() {
    auto plan = [](int64_t M, int64_t N, int64_t K, int dtype) { return wgrad_plan(M, N, K, dtype, N, 0); };
    // large tiles: dY brought into tiles as its rows end, begin or (too many columns of X) are read too often otherwise, or read as it is
    EXPECT(is(plan(700, 4103, 4100, DAQ_BF16), kTiles, true, false) && is(plan(600, 4096, 8200, DAQ_BF16), kTiles, true, false));
    EXPECT(is(wgrad_plan(700, 4104, 4100, DAQ_BF16, 4112, 2), kTiles, true, false) && is(wgrad_plan(700, 4104, 4100, DAQ_BF16, 4112, 0), kFlat, true, false));
    EXPECT(is(plan(9000, 2049, 2100, DAQ_BF16), kTiles, true, true) && is(plan(6000, 1536, 1300, DAQ_BF16), kFlat, true, true));
    // small tiles
    EXPECT(is(plan(300, 1101, 1090, DAQ_BF16), kTiles, false, false) && is(plan(3001, 610, 1101, DAQ_BF16), kTiles, false, true));
    EXPECT(is(plan(1111, 3000, 900, DAQ_BF16), kFlat, false, false) && is(plan(2050, 1032, 1000, DAQ_BF16), kFlat, false, true));
    // three parts of dY: small tiles only, in one part of the tokens or several
    EXPECT(is(plan(300, 1101, 1090, DAQ_FP32), kTiles, false, false) && is(plan(700, 4103, 4100, DAQ_FP32), kTiles, false, false));
    const WgradPlan a = plan(1531, 607, 1100, DAQ_FP32), b = plan(3001, 610, 1101, DAQ_FP32);
    EXPECT(is(a, kTiles, false, true) && a.parts == 3 && a.splits == 4 && is(b, kTiles, false, true) && b.parts == 3 && b.splits == 5);
    if (!fails) std::printf("ok\n");
    return fails != 0;
}
