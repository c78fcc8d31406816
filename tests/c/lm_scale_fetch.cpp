// Every lane's fetches of a tile's scales (csrc/lm_scale_fetch.h), of every block and tile of products of many sizes: they stay within the array of scales
// and hold the scales of the lane's rows.  Built and run by tests/test_language_kernels_host.py.
#include <algorithm>
#include <cstdio>

#include "lm_scale_fetch.h"

static long fetches = 0;

template <uint32_t SIZE>
static bool check(uint32_t rows, uint32_t blocks, bool tiles, uint32_t n, uint32_t first_block) {
    const uint64_t whole = (rows + 127) / 128, stride = tiles ? whole : whole * 128, count = blocks * stride;
    const char *at = reinterpret_cast<const char *>(uintptr_t(1) << 20);  // never read
    for (uint32_t row0 = 0; row0 < rows; row0 += n)
        for (uint32_t lane = 0; lane < 64; ++lane) {
            ScaleFetch<SIZE> f(at, stride, blocks, tiles ? 7 : 0, row0, n, lane, first_block);
            for (uint32_t kb = first_block; kb < blocks; ++kb) {
                const uint64_t from = f.base + f.offset(), begin = from - uint64_t(uintptr_t(at));
                // a load of several words takes those that lie within the records, one of a byte or a word only what does so whole
                const uint64_t left = f.base + f.records - from, taken = f.records == 0xffffffffu ? f.bytes() : std::min<uint64_t>(f.bytes(), left / std::min(f.bytes(), 4u) * std::min(f.bytes(), 4u));
                if (from % std::min(f.bytes(), 4u) || begin + taken > count * SIZE) return std::printf("out of bounds: "), false;
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t row = row0 + 4 * std::min(lane, n / 4 - 1) + i;
                    if (row >= rows) continue;
                    const uint64_t scale = (kb * stride + (tiles ? row / 128 : row)) * SIZE;
                    if (scale < begin || scale + SIZE > begin + taken) return std::printf("not held: "), false;
                    // where the kernel looks for it: a row's own in order, a shared byte as the only one, a shared float by its number
                    if (tiles ? (SIZE == 1 ? scale != begin : (scale - begin) / SIZE != scale / SIZE % 4) : scale - begin != i * SIZE) return std::printf("misplaced: "), false;
                }
                ++fetches;
                f.advance(kb + 1 < blocks);
            }
        }
    return true;
}

int main() {
    for (uint32_t rows : {1u, 5u, 127u, 128u, 129u, 300u, 513u, 640u, 900u, 1111u})
        for (uint32_t blocks : {1u, 2u, 3u, 5u, 7u, 8u, 13u})
            for (uint32_t n : {64u, 128u, 256u})
                for (int tiles = 0; tiles < 2; ++tiles)
                    for (uint32_t first : {0u, blocks / 2})
                        if (!check<1>(rows, blocks, tiles, n, first) || !check<4>(rows, blocks, tiles, n, first)) {
                            std::printf("rows %u blocks %u n %u tiles %d first %u\n", rows, blocks, n, tiles, first);
                            return 1;
                        }
    std::printf("scale fetches ok: %ld\n", fetches);
    return 0;
}
