// Where the scales of a tile of a product lie in memory: what each lane asks for, block by block.  Without the GPU's headers.
//
// The tile's rows go by fours, four to a lane.  Where rows have scales of their own a lane asks for its four; where 128 rows share one, for that
// one: a byte, or the aligned four floats that it lies in, of which `records` leaves out those beyond the array.
#ifndef CNR_LM_SCALE_FETCH_H
#define CNR_LM_SCALE_FETCH_H

#include <stdint.h>

#ifdef __HIPCC__
#define CNR_BOTH __host__ __device__ __forceinline__
#else
#define CNR_BOTH inline
#endif

// SIZE: bytes of a scale, 1 or 4.
template <uint32_t SIZE>
struct ScaleFetch {
    uint64_t base, step;           // address that offsets of the block to fetch next count from, bytes to the next block's
    uint32_t block, block_step;    // the same within an array of tiles' scales, whose fours are not aligned with its blocks
    uint32_t in_block;
    uint32_t records;              // bytes from `base` that there are
    uint32_t tiles;                // not 0: 128 rows share a scale
    // Scales at `p` of `blocks` blocks, `stride` to a block; `row0`: first of the tile's `n` rows.  Rows beyond the matrix take the last scales that there are.
    CNR_BOTH ScaleFetch(const void *p, uint64_t stride, uint32_t blocks, uint32_t shift, uint32_t row0, uint32_t n, uint32_t lane, uint32_t kb) {
        tiles = shift;
        const uint32_t row = row0 + 4 * (lane < n / 4 ? lane : n / 4 - 1);
        const uint32_t last = (uint32_t)stride - (tiles ? 1 : 4), entry = tiles ? row >> shift : row;
        const uint32_t low = tiles ? 0 : row0;  // goes into the base, so that offsets stay small
        in_block = ((entry < last ? entry : last) - low) * SIZE;
        base = (uint64_t)(uintptr_t)p + (tiles ? 0 : ((uint64_t)kb * stride + low) * SIZE);
        step = tiles ? 0 : stride * SIZE;
        block = tiles ? (uint32_t)(kb * stride) * SIZE : 0;
        block_step = tiles ? (uint32_t)stride * SIZE : 0;
        const uint64_t all = blocks * stride * SIZE;
        records = tiles && all < 0xffffffffull ? (uint32_t)all : 0xffffffffu;
    }
    // Rows' scales are four side by side at a multiple of four from the base anyway.
    CNR_BOTH uint32_t offset() const { return SIZE == 1 ? block + in_block : (block + in_block) & ~(4 * SIZE - 1); }
    CNR_BOTH uint32_t bytes() const { return SIZE == 1 && tiles ? 1 : 4 * SIZE; }
    // `on`: the block is not the last one; there it stays.
    CNR_BOTH void advance(bool on) {
        base += on ? step : 0;
        block += on ? block_step : 0;
    }
};
#endif
