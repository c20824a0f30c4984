// Forms of the few-bit products at sizes where another one was measured slower, and plans of the weight gradient.
#include <cstdio>

#include "lowbits.h"

static int fails = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++fails; } \
    } while (0)

using namespace daq;

static void products() {
    auto form = [](int64_t M, int64_t N, int64_t K) { return matmul_form(ceil_div(M, 32), ceil_div(N, 32), ceil_div(K, 256)); };
    for (int64_t M : {1, 13, 32, 64, 128}) EXPECT(form(M, 2048, 2048) == MatmulForm::kFew && form(M, 512, 8192) == MatmulForm::kFew);
    EXPECT(form(512, 512, 8192) == MatmulForm::kFew && form(200, 64, 8192) == MatmulForm::kFew && form(128, 8192, 8192) == MatmulForm::kFew);
    EXPECT(form(512, 4096, 4096) == MatmulForm::kSmall && form(1777, 2080, 4096) == MatmulForm::kSmall && form(512, 8192, 8192) == MatmulForm::kSmall);
    EXPECT(form(2048, 4096, 4096) == MatmulForm::kSmall);
    EXPECT(form(16384, 8192, 8192) == MatmulForm::kBig && form(4096, 4096, 4096) == MatmulForm::kBig && form(3000, 4096, 8192) == MatmulForm::kBig);
    EXPECT(form(((int64_t)1 << 31) - 1, 32, 256) != MatmulForm::kFew);   // a grid's second axis ends at 65535
    EXPECT(raw_rows(1, 8192, DAQ_BF16, DAQ_ROUND_NEAREST) && raw_rows(16, 2048, DAQ_BF16, DAQ_ROUND_NEAREST) && raw_rows(2, 8192, DAQ_FP32, DAQ_ROUND_NEAREST));
    EXPECT(!raw_rows(1, 2048, DAQ_BF16, DAQ_ROUND_STOCHASTIC) && !raw_rows(32, 8192, DAQ_BF16, DAQ_ROUND_NEAREST) && !raw_rows(16, 2048, DAQ_FP32, DAQ_ROUND_NEAREST) &&
           !raw_rows(33, 32, DAQ_BF16, DAQ_ROUND_NEAREST));
}

static void weight_gradients() {
    auto plan = [](int64_t M, int64_t N, int64_t K, int dtype) { return wgrad_plan(M, N, K, dtype, N, 0); };
    const WgradPlan a = plan(16384, 8192, 4096, DAQ_BF16), b = plan(2048, 2048, 2048, DAQ_BF16), c = plan(16384, 256, 256, DAQ_FP32);
    EXPECT(a.big && a.splits == 1 && a.flat && a.off_x == 0);
    EXPECT(!b.big && b.splits == 1 && !b.flat);
    EXPECT(!c.big && c.splits > 8 && !c.flat && c.parts == 3);
    EXPECT(!plan(16384, 8191, 4096, DAQ_BF16).flat && !wgrad_plan(16384, 8192, 4096, DAQ_BF16, 8193, 0).flat && !wgrad_plan(16384, 8192, 4096, DAQ_BF16, 8192, 2).flat &&
           !plan(16384, 8192, 4096, DAQ_FP32).flat);
    EXPECT(c.few && !a.few && !b.few && plan(1, 2, 1, DAQ_FP32).few && !plan(1, 1, 1, DAQ_FP32).few && !plan(100, 4000, 4000, DAQ_BF16).few);
    // every stage (step, without tiles) belongs to a part, none of which is empty, and the workspace's pieces follow one another
    for (int64_t M : {1, 63, 64, 65, 1000, 16384, 100000})
        for (int64_t N : {1, 40, 607, 4096})
            for (int64_t K : {1, 33, 1100, 4096})
                for (int dtype : {DAQ_FP32, DAQ_BF16}) {
                    const WgradPlan w = plan(M, N, K, dtype);
                    if (w.few) {
                        const int64_t steps = (M + 15) / 16, tiles = ((N + 63) / 64) * ((K + 63) / 64);
                        EXPECT((int64_t)w.splits * w.per_split >= steps && (int64_t)(w.splits - 1) * w.per_split < steps && w.splits * tiles <= 256);
                        EXPECT(w.bytes >= (w.splits > 1 ? (int64_t)w.splits * N * w.pitch * 4 : 0) && w.pitch >= K && w.pitch % 4 == 0);
                        continue;
                    }
                    const int64_t stages = w.steps / 4;
                    EXPECT(w.steps % 4 == 0 && stages * 64 >= M && (int64_t)w.splits * w.per_split >= stages && (int64_t)(w.splits - 1) * w.per_split < stages);
                    EXPECT(w.off_x == (w.flat ? 0 : (int64_t)w.n_blocks * w.steps * w.parts * 1024) && w.off_part == w.off_x + (int64_t)w.k_blocks * w.steps * 1024);
                    EXPECT(w.bytes >= w.off_part + (w.splits > 1 ? (int64_t)w.splits * N * w.pitch * 4 : 0) && w.pitch >= K && w.pitch % 4 == 0);
                }
}

int main() {
    products();
    weight_gradients();
    if (!fails) std::printf("ok\n");
    return fails != 0;
}
