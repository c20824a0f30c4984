// Limits of what the few-bit products reach: choices at sizes whose operands no test can hold.
#include <cstdio>

#include "lowbits.h"

static int fails = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++fails; } \
    } while (0)

using namespace daq;

// A tile kernel reads a row block, 4 KiB a group, through one descriptor, which ends before 2^32 - 256 bytes.
static void reach_of_a_descriptor() {
    const int64_t most = (((int64_t)1 << 32) - 256) / 4096;   // groups
    for (int64_t blocks : {(int64_t)1, (int64_t)35, (int64_t)40, (int64_t)128}) {
        for (int64_t groups : {most + 1, (int64_t)1 << 20}) EXPECT(matmul_form(blocks, blocks, groups) == MatmulForm::kFew);
        EXPECT((matmul_form(blocks, blocks, most) == MatmulForm::kFew) == (blocks < 35));   // nothing else kept them from tiles
    }
}

// A launch takes fewer than 2^32 threads along an axis: 2^23 workgroups of 512 are too many, where tiles of 128 x 128 are not.
static void threads_of_a_launch() {
    const int64_t most = ((int64_t)1 << 23) - 1;   // column blocks
    EXPECT(matmul_form(1, most, 1) == MatmulForm::kFew && matmul_form(1, most + 1, 1) == MatmulForm::kSmall);
}

int main() {
    reach_of_a_descriptor();
    threads_of_a_launch();
    if (!fails) std::printf("ok\n");
    return fails != 0;
}
