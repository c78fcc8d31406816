// What the losses over the vocabulary plan (csrc/lm_loss_plan.h), at the limits of their sizes.  Built and run by tests/test_losses_host.py.
#include <stdio.h>

#include "lm_loss_plan.h"

static int wrong = 0;

#define CHECK(what, ...)                                                                  \
    do {                                                                                  \
        if (!(what)) {                                                                    \
            ++wrong;                                                                      \
            printf("%s:", #what);                                                         \
            for (unsigned long long v : {__VA_ARGS__}) printf(" %llu", v);                \
            printf("\n");                                                                 \
        }                                                                                 \
    } while (0)

// Laid out rows: every piece by one launch, whose threads fit 32 bits.
static void launches(uint64_t n, uint64_t dim, cnr_float_type type) {
    const uint64_t pieces = n * sizes_of(n, 1, dim, type).blocks * dense::kBlockBytes / 16;
    uint64_t done = 0;
    in_launches(pieces, [&](uint64_t first, unsigned groups) {
        CHECK(first == done && groups && (uint64_t)groups * kBlock < 1ull << 32, n, dim);
        done += (uint64_t)groups * kBlock;
    });
    CHECK(done >= pieces && done < pieces + kBlock, n, dim);
}

int main() {
    for (uint64_t n : {0ull, 1ull, 300ull, 1ull << 17, CNR_LOSS_MAX_ROWS + 0ull})
        for (uint64_t dim : {0ull, 1ull, 65ull, 16392ull, 1ull << 15, (1ull << 17) + 1, CNR_LOSS_MAX_DIM + 0ull})
            for (cnr_float_type type : {CNR_FLOAT_F32, CNR_FLOAT_BF16}) launches(n, dim, type);
    return wrong ? 1 : 0;
}
