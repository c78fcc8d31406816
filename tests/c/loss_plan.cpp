// What the losses over the vocabulary plan (csrc/lm_loss_plan.h), at the limits of their sizes.  Built and run by tests/test_losses_host.py.
#include <stdio.h>

#include <initializer_list>

#include "lm_loss_plan.h"

static int wrong = 0;

#define CHECK(what, ...)                                                                                       \
    do {                                                                                                       \
        if (!(what)) {                                                                                         \
            ++wrong;                                                                                           \
            printf("%s:", #what);                                                                              \
            for (unsigned long long v : std::initializer_list<unsigned long long>{__VA_ARGS__}) printf(" %llu", v); \
            printf("\n");                                                                                      \
        }                                                                                                      \
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

// A workspace serves its number of rows and fewer, and dz are held a piece of the vocabulary at a time.
static void workspaces(uint64_t n, uint64_t vocab, uint64_t dim, cnr_float_type type) {
    for (int wide = 0; wide < (type == CNR_FLOAT_F32 ? 1 : 2); ++wide) {
        const uint64_t forward = room_for(sizes_of(n, vocab, dim, type), false, false), training = room_for(sizes_of(n, vocab, dim, type), true, wide);
        for (uint64_t rows : {1ull, 16ull, 17ull, 32ull, 33ull, 64ull, 65ull, 128ull, 129ull, 256ull, 257ull, 5000ull, n + 0ull}) {
            if (rows > n) continue;
            const Sizes s = sizes_of(rows, vocab, dim, type);
            CHECK(forward_plan(nullptr, s).bytes <= forward, n, rows, vocab, dim, (uint64_t)type);
            for (int in_place = 0; in_place <= (type != CNR_FLOAT_F32); ++in_place) {
                const BackwardPlan b = backward_plan(nullptr, s, wide, in_place);
                CHECK(b.bytes <= training, n, rows, vocab, dim, (uint64_t)type);
                CHECK(b.piece && b.piece <= vocab && (b.piece == vocab || b.piece % 256 == 0), n, rows, vocab, dim, (uint64_t)type);
                const uint64_t dz = (b.narrow ? b.sum : b.hidden_at) - b.dz, tokens = rows * 256 * 2 * dz_parts(s, wide);
                CHECK(dz <= (512ull << 20) + tokens, n, rows, vocab, dim, (uint64_t)type);
            }
        }
    }
}

int main() {
    for (uint64_t n : {1ull, 16ull, 33ull, 64ull, 129ull, 300ull, 8192ull, CNR_LOSS_MAX_ROWS + 0ull})
        for (uint64_t vocab : {1ull, 257ull, 50257ull, (1ull << 21) + 1, (1ull << 24) + 0, CNR_LOSS_MAX_VOCABULARY + 0ull})
            for (uint64_t dim : {0ull, 1ull, 64ull, 1000ull, 4096ull, 1ull << 17, CNR_LOSS_MAX_DIM + 0ull})
                for (cnr_float_type type : {CNR_FLOAT_F32, CNR_FLOAT_BF16}) workspaces(n, vocab, dim, type);
    for (uint64_t n : {0ull, 1ull, 300ull, 1ull << 17, CNR_LOSS_MAX_ROWS + 0ull})
        for (uint64_t dim : {0ull, 1ull, 65ull, 16392ull, 1ull << 15, (1ull << 17) + 1, CNR_LOSS_MAX_DIM + 0ull})
            for (cnr_float_type type : {CNR_FLOAT_F32, CNR_FLOAT_BF16}) launches(n, dim, type);
    return wrong ? 1 : 0;
}
