// Products of plain matrices, out[row][column] = sum over k of down[row][k] across[column][k], for kernels that do something of their own with the outputs.
//
// Elements have 16 bits and go through the matrix instructions of their type: exact products, added up in fp32.  Each operand lies either along k (a row or
// column of the output in a row of its own, in whole pieces of eight elements) or across it ([k][row or column], read through the LDS's transposing
// loads; columns in whole pieces of eight).  An operand may be held in several parts, side by side in its rows, that add up to it (a float in three bfloat16): the sum then goes over
// pairs of parts ("terms") of each block.
#pragma once

#include "lm_common.h"

#include <math.h>
#include <type_traits>

namespace dense {

constexpr uint32_t kBlockBytes = 128, kBlockElements = 64;
constexpr uint32_t kNoIndex = 0xffffffffu;

struct Operand {
    const void *at;       // 16-byte aligned
    uint64_t stride;      // bytes from row to row, a multiple of 16; below 2^23 where rows lie along k
    uint32_t row_bytes;   // of a row with all its parts, a multiple of 16; the last row ends with them
    uint32_t part_bytes;  // from one part to the next in a row
    uint32_t parts;       // which part each term takes, four bits a term, the first term lowest
    uint32_t last;        // pieces of 16 bytes in the last block of a row that lies along k, from 1 to 8; zeros are taken for the others
};
struct Args {
    Operand across, down;
    uint32_t columns, rows;  // of the output
    uint32_t blocks;         // along k, >= 1
    uint32_t k;              // rows of operands that lie across k; behind them zeros are read
    uint32_t terms;          // >= 1
    uint32_t splits;         // parts of the sum, each in its own workgroups
};

#ifdef __HIPCC__
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <int I>
struct Index {
    static constexpr int value = I;
};
template <int N, int I = 0, typename Body>
__device__ __forceinline__ void unrolled(const Body &body) {
    if constexpr (I < N) {
        body(Index<I>());
        unrolled<N, I + 1>(body);
    }
}

// Half h of the products of 16 rows by 16, 32 bytes of each: lane l holds bytes of row l % 16, which ones does not matter as long as both operands agree.
// Sum i of a lane belongs to row 4 (l / 16) + i of x and row l % 16 of y.
template <int TYPE, int H>
__device__ __forceinline__ f32x4 multiply(const i32x8 &x, const i32x8 &y, const f32x4 &sum) {
    i32x4 a, b;
    if constexpr (H == 0) {
        a = __builtin_shufflevector(x, x, 0, 1, 2, 3);
        b = __builtin_shufflevector(y, y, 0, 1, 2, 3);
    } else {
        a = __builtin_shufflevector(x, x, 4, 5, 6, 7);
        b = __builtin_shufflevector(y, y, 4, 5, 6, 7);
    }
    if constexpr (TYPE == CNR_FLOAT_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), sum, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), sum, 0, 0, 0);
}

constexpr uint32_t kNowhere = 0xf0000000u;  // beyond every buffer, whatever is added: zeros arrive

// Base and size are the same for all lanes.
__device__ __forceinline__ i32x4 buffer_of(uint64_t base, uint64_t bytes) {
    i32x4 r;
    r[0] = (int)(uint32_t)base;
    r[1] = (int)((uint32_t)(base >> 32) & 0xffffu);
    r[2] = (int)(uint32_t)(bytes < 0xffffffffull ? bytes : 0xffffffffull);
    r[3] = 0x00027000;
    return r;
}
// 64 pieces of 16 bytes, one for each lane, from memory to `lds` and on in lane order; waited for by wait_for_loads.  Written as an instruction since
// the compiler, which cannot tell the stages of the LDS apart, would wait for it before every read of another.  It sets M0 for itself.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const i32x4 &buffer, uint32_t lds, uint32_t offset, uint32_t all) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(all) : "m0");
}
#pragma clang diagnostic pop
template <int LEFT>  // loads that need not have arrived
__device__ __forceinline__ void wait_for_loads() {
    static_assert(LEFT < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What a workgroup's outputs are to its epilogue.  A lane holds MF / 2 times eight columns side by side, 32 apart, of NF rows: value(acc, i, g) is that of
// column column_of(i) and row row(g).  The four lanes of a row thus write 64 bytes of 16-bit outputs side by side at a time.
template <int MF, int NF, bool DOWN, uint32_t THREADS, uint32_t LDS>
struct Place {
    static constexpr uint32_t kThreads = THREADS, kLdsBytes = LDS;
    uint32_t row0, column0;  // first output of the workgroup
    uint32_t lane_row;       // the lane's first row within the workgroup's
    uint32_t column;         // the lane's first
    uint32_t split, tile_column;
    uint32_t wave_column;    // which of the WM parts of the workgroup's columns is the wave's
    uint8_t *lds;            // kLdsBytes, free
    // (rows from an operand across k: chunks of odd lanes change places by pairs, see Across)
    __device__ __forceinline__ uint32_t row_within(uint32_t g) const { return lane_row + g / 2 * 32 + (DOWN ? (g ^ tid_x() / 4) % 2 : g % 2) * 4; }
    __device__ __forceinline__ uint32_t row(uint32_t g) const { return row0 + row_within(g); }
    __device__ __forceinline__ uint32_t column_of(uint32_t i) const { return column + i / 8 * 32 + i % 8; }
    // The i with column_of(i) = column + from, kNoIndex where that is none of the lane's.
    static __device__ __forceinline__ uint32_t index_of(uint64_t from) { return from < 16 * MF && from % 32 < 8 ? (uint32_t)from / 32 * 8 + (uint32_t)from % 8 : kNoIndex; }
    static __device__ __forceinline__ float value(const f32x4 (&acc)[MF][NF], int i, int g) { return acc[i / 4][g][i % 4]; }
};

// One operand's way from memory through LDS into fragments of 16 of its F * 16 * waves rows (T), a block of k at a time.  Lane r = lane % 16 of fragment f has
// row 32 (f / 2) + 8 (r / 4) + 4 (f % 2) + r % 4 of the wave's section: the four sums of a lane of the product, and those of the next fragment, lie side
// by side.
//
// Along k: LDS holds two rows of 128 bytes to a line of 256, its sixteen pieces of 16 bytes permuted by r / 2: sixteen lanes that read the same piece of
// their rows find it in sixteen different places, all banks in use.  Memory is read straight into LDS, where a wave's 64 pieces lie in
// order, so the permutation is in which piece a lane asks for.
template <int F, int T, int LOADS>
struct Along {
    i32x4 buffer;
    uint32_t from[LOADS];
    uint32_t beyond;     // bit j: load j's piece is beyond the end of the row, where the block is its last
    uint32_t piece[2];   // of the first fragment's row, by half of the block
    // Rows beyond the matrix read its last one again.
    __device__ __forceinline__ Along(const Operand &o, uint32_t first, uint32_t count, uint32_t, uint32_t wave, uint32_t section, uint32_t region) {
        const uint32_t lane = tid_x() % kWave, r = lane % 16, quarter = lane / 16, rows = count - first < T ? count - first : T;
        buffer = buffer_of(reinterpret_cast<uint64_t>(o.at) + (uint64_t)first * o.stride, (uint64_t)(rows - 1) * o.stride + o.row_bytes);
        beyond = 0;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const uint32_t line = (wave * LOADS + j) * 4 + quarter, logical = r ^ (line / 4 % 4 * 2 + line % 2);
            const uint32_t row = 2 * line + logical / 8;
            from[j] = (row < rows ? row : rows - 1) * (uint32_t)o.stride + logical % 8 * 16;
            beyond |= logical % 8 >= o.last ? 1u << j : 0u;
        }
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) piece[h] = region + section * kBlockBytes + (r / 4 * 4 + r % 4 / 2) * 256 + ((r % 2 * 8 + quarter + 4 * h) ^ r / 2) * 16;
    }
    template <int J>
    __device__ __forceinline__ void fetch(const Operand &, uint32_t lds, uint32_t part, uint32_t block) const {
        load_to_lds(buffer, lds, from[J], part + block * kBlockBytes);
    }
    // From here on the last block is read.  (Where rows end within it there is one term: an operand of several parts is laid out in whole blocks.)
    __device__ __forceinline__ void end() {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) from[j] = beyond >> j & 1u ? kNowhere : from[j];
    }
    __device__ __forceinline__ void move(uint32_t by) {
        piece[0] += by;
        piece[1] += by;
    }
    __device__ __forceinline__ i32x8 fragment(const uint8_t *lds, uint32_t f) const {
        i32x4 part[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) part[h] = *reinterpret_cast<const i32x4 *>(lds + piece[h] + f / 2 * 4096 + f % 2 * 512);
        return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Across k: LDS holds 64 rows of k with T columns each.  The transposing load gives a lane four rows of one column, sixteen lanes four rows of sixteen columns
// that are four chunks of four from anywhere: chunk c = r / 4 of fragment f holds columns 32 (f / 2) + 8 c + 4 (f % 2 ^ c % 2).  Sixteen lanes thus read four
// chunks of 8 bytes in each of four rows; that these sixteen lie in different banks takes the other half of a piece of 16 bytes for odd chunks, and pieces
// permuted by the row (`turned`), on the way in as in the layout along k.
template <int F, int T, int LOADS>
struct Across {
    static constexpr uint32_t kRow = T * 2, kPieces = T / 8;
    uint64_t at, left;  // of the first row's first column in bytes, to the end
    uint32_t from[LOADS];
    uint32_t chunk;
    static __device__ __forceinline__ uint32_t turned(uint32_t piece, uint32_t row) { return piece ^ row % 2 ^ row / 2 % 2 * 4; }
    __device__ __forceinline__ Across(const Operand &o, uint32_t first, uint32_t, uint32_t k, uint32_t wave, uint32_t section, uint32_t region) {
        static_assert(T >= 64, "places in LDS");
        const uint32_t lane = tid_x() % kWave, quarter = lane / 16, c = lane % 4, row = lane % 16 / 4;
        at = reinterpret_cast<uint64_t>(o.at) + first * 2;
        left = (uint64_t)(k - 1) * o.stride + o.row_bytes - first * 2;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const uint32_t i = (wave * LOADS + j) * kWave + lane;
            from[j] = i / kPieces * (uint32_t)o.stride + turned(i % kPieces, i / kPieces) * 16;
        }
        chunk = region + (quarter * 8 + row) * kRow + turned(section / 8 + c, row) * 16 + c % 2 * 8;
    }
    // Beyond the end nothing is read, and zeros arrive.
    template <int J>
    __device__ __forceinline__ void fetch(const Operand &o, uint32_t lds, uint32_t part, uint32_t block) const {
        const uint64_t on = part + (uint64_t)block * kBlockElements * o.stride;
        load_to_lds(buffer_of(at + on, on < left ? left - on : 0), lds, from[J], 0);
    }
    __device__ __forceinline__ void end() {}
    __device__ __forceinline__ void move(uint32_t by) { chunk += by; }
    __device__ __forceinline__ i32x8 fragment(const uint8_t *lds, uint32_t f) const {
        typedef __attribute__((address_space(3))) s16x4 *Lds;
        i32x2 part[4];
        const uint8_t *from = lds + (chunk ^ (f / 2 * 64 + f % 2 * 8));  // (these bits of the section's place are 0)
#pragma unroll
        for (int h = 0; h < 4; ++h) part[h] = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(from + (h / 2 * 32 + h % 2 * 4) * kRow)));
        const i32x4 lo = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3), hi = __builtin_shufflevector(part[2], part[3], 0, 1, 2, 3);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// A workgroup of WM x WN waves has 16 WM MF columns by 16 WN NF rows, a wave 16 MF by 16 NF of them, and walks along k a block at a time; the next
// STAGES - 1 blocks travel from memory into LDS while this one's are multiplied.
//
// A block's products go by quarters, each half of the wave's columns with each half of its rows, so that half of the operands are in registers while
// the other half, or the next block's first, are on their way from LDS; loads go between matrix instructions.  The last quarter needs nothing more
// from this stage: before it all waves meet, in it the stage is filled again.
//
// Bound by the matrix units: 4096 x 131072 x 4096 in bfloat16, both operands along k, 3.18 ms, 1.38 PFLOP/s (on the same card the installed library's plain product
// of 8192^3 1.14); one or both across k 1.29 to 1.32 (16384 x 16384 x 4096 1.67 to 1.70 ms).  Transposing copies in memory instead took 40 us more for each
// 134 MB, and dz in both directions.
template <int TYPE, bool ACROSS, bool DOWN, int WM, int WN, int MF, int NF, int STAGES, typename Epilogue>
__global__ void __launch_bounds__(WM * WN * kWave, 2) tile_kernel(const Args p, const Epilogue epilogue) {
    constexpr uint32_t TM = WM * 16 * MF, TN = WN * 16 * NF;
    constexpr int LA = 2 * MF / WN, LB = 2 * NF / WM;  // loads of 1 KB that each wave sends for a block of each operand
    static_assert(LA * WN == 2 * MF && LB * WM == 2 * NF, "whole loads");
    constexpr uint32_t kB = TM * kBlockBytes, kStage = kB + TN * kBlockBytes;
    constexpr int kLoads = LA + LB;
    __shared__ __align__(256) uint8_t lds[STAGES * kStage];
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint32_t r = lane % 16, quarter = lane / 16;
    const uint32_t wave_m = wave / WN * 16 * MF, wave_n = wave % WN * 16 * NF;

    // Workgroups go to the eight XCDs in turn: each XCD gets tiles that lie together, in bands of kBand rows of tiles, for its L2.
    constexpr uint32_t kBand = 4;
    const uint32_t down = (p.rows + TN - 1) / TN, across = (p.columns + TM - 1) / TM, tiles = down * across, all = tiles * p.splits;
    const uint32_t xcd = wg_x() % 8, each = all / 8, more = all % 8;
    const uint32_t id = xcd * each + (xcd < more ? xcd : more) + wg_x() / 8;
    const uint32_t split = id / tiles, at = id % tiles;
    const uint32_t band = at / (kBand * across), band_rows = down - band * kBand < kBand ? down - band * kBand : kBand;
    const uint32_t in_band = at - band * kBand * across;
    const uint32_t tile_column = in_band / band_rows, row0 = (band * kBand + in_band % band_rows) * TN, column0 = tile_column * TM;
    // Blocks of this part of the sum, over all terms; the host sees to it that there are some.
    const uint32_t whole = p.blocks * p.terms;
    const uint32_t begin = (uint32_t)((uint64_t)whole * split / p.splits), end = (uint32_t)((uint64_t)whole * (split + 1) / p.splits);

    typename std::conditional<ACROSS, Across<MF, TM, LA>, Along<MF, TM, LA>>::type a(p.across, column0, p.columns, p.k, wave, wave_m, 0);
    typename std::conditional<DOWN, Across<NF, TN, LB>, Along<NF, TN, LB>>::type b(p.down, row0, p.rows, p.k, wave, wave_n, kB);
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // The block to be fetched next; behind the last one it stays there, and nobody reads what arrives: the count of loads stays the same without a branch.
    uint32_t ahead = begin, block = begin / p.terms, term = begin % p.terms;
    auto end_of_rows = [&]() {
        if (block + 1 == p.blocks) {
            a.end();
            b.end();
        }
    };
    end_of_rows();
    auto fetch = [&](uint32_t to, auto index) {
        constexpr int J = decltype(index)::value;
        if constexpr (J < LA)
            a.template fetch<J>(p.across, lds_at + to + (wave * LA + J) * 1024, (p.across.parts >> 4 * term & 15u) * p.across.part_bytes, block);
        else
            b.template fetch<J - LA>(p.down, lds_at + to + kB + (wave * LB + J - LA) * 1024, (p.down.parts >> 4 * term & 15u) * p.down.part_bytes, block);
    };
    auto go_on = [&]() {
        if (ahead + 1 < end) {
            ++ahead;
            const bool over = term + 1 == p.terms;
            term = over ? 0 : term + 1;
            block += over ? 1 : 0;
            end_of_rows();
        }
    };

    f32x4 acc[MF][NF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // The i-th of `of` even shares of N things to do.
    auto share = [](auto i, auto of, auto n, const auto &act) {
        constexpr int I = decltype(i)::value, OF = decltype(of)::value, N = decltype(n)::value, from = I * N / OF, to = (I + 1) * N / OF;
        unrolled<to - from>([&](auto j) { act(Index<from + decltype(j)::value>()); });
    };

    constexpr int HM = MF / 2, HN = NF / 2, kPairs = HM * HN, kSteps = kPairs * 2;
    unrolled<STAGES>([&](auto i) {
        unrolled<kLoads>([&](auto j) { fetch(decltype(i)::value * kStage, j); });
        go_on();
    });
    wait_for_loads<(STAGES - 1) * kLoads>();
    barrier();
    i32x8 x[2][HM], y[2][HN];
#pragma unroll
    for (int f = 0; f < HM; ++f) x[0][f] = a.fragment(lds, f);
#pragma unroll
    for (int g = 0; g < HN; ++g) y[0][g] = b.fragment(lds, g);
    // One quarter; with its i-th matrix instruction goes beside(i).  Sums take turns, so that none waits for the one before.
    auto quarter_of = [&](auto half_a, auto half_b, const auto &beside) {
        constexpr int A = decltype(half_a)::value, B = decltype(half_b)::value;
        unrolled<kSteps>([&](auto step) {
            constexpr int H = decltype(step)::value / kPairs, PAIR = decltype(step)::value % kPairs, F = PAIR % HM, G = PAIR / HM, MA = A * HM + F, NB = B * HN + G;
            acc[MA][NB] = multiply<TYPE, H>(x[A][F], y[B][G], acc[MA][NB]);
            beside(step);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    uint32_t stage = 0;  // where it begins in LDS
    for (uint32_t kb = begin; kb < end; ++kb) {
        const uint32_t next = stage + kStage < STAGES * kStage ? stage + kStage : 0;
        quarter_of(Index<0>(), Index<0>(), [&](auto step) {
            share(step, Index<kSteps>(), Index<HN>(), [&](auto g) { y[1][decltype(g)::value] = b.fragment(lds, HN + decltype(g)::value); });
        });
        quarter_of(Index<0>(), Index<1>(), [&](auto step) {
            share(step, Index<kSteps>(), Index<HM>(), [&](auto f) { x[1][decltype(f)::value] = a.fragment(lds, HM + decltype(f)::value); });
        });
        quarter_of(Index<1>(), Index<0>(), [&](auto) {});
        wait_for_loads<(STAGES - 2) * kLoads>();
        barrier();
        a.move(next - stage);
        b.move(next - stage);
        quarter_of(Index<1>(), Index<1>(), [&](auto step) {
            share(step, Index<kSteps>(), Index<HM + HN>(), [&](auto j) {
                constexpr int J = decltype(j)::value;
                if constexpr (J < HM)
                    x[0][J] = a.fragment(lds, J);
                else
                    y[0][J - HM] = b.fragment(lds, J - HM);
            });
            share(step, Index<kSteps>(), Index<kLoads>(), [&](auto j) { fetch(stage, j); });
        });
        go_on();
        stage = next;
    }
    wait_for_loads<0>();
    if constexpr (Epilogue::kUsesLds) __syncthreads();
    if constexpr (ACROSS) {
        // chunks of odd quarters back in order
#pragma unroll
        for (int f = 0; f < MF; f += 2)
#pragma unroll
            for (int g = 0; g < NF; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = acc[f][g][i], w = acc[f + 1][g][i];
                    acc[f][g][i] = quarter % 2 ? w : v;
                    acc[f + 1][g][i] = quarter % 2 ? v : w;
                }
    }
    Place<MF, NF, DOWN, WM * WN * kWave, STAGES * kStage> place;
    place.row0 = row0;
    place.column0 = column0;
    place.lane_row = wave_n + r / 4 * 8 + r % 4;
    place.column = column0 + wave_m + quarter * 8;
    place.split = split;
    place.tile_column = tile_column;
    place.wave_column = wave / WN;
    place.lds = lds;
    epilogue.template finish<TM, TN, WM>(p, place, acc);
}
#endif

// ---- which tiles ----------------------------------------------------------------------------------------------
//
// A workgroup's time for a block by how many share a compute unit, in us, and what it takes besides: until the first block is there, and for its outputs,
// which a unit writes at its share of what memory takes and which only another workgroup's products hide.
struct Tiles {
    uint32_t columns, rows, threads, resident;
    float block[2];
};
constexpr Tiles kTiles[] = {
    {256, 256, 512, 1, {1.65f, 0.0f}},  // eight waves of 128 x 64, two stages
    {128, 128, 512, 1, {0.54f, 0.0f}},  // eight waves of 64 x 32, four stages
    {128, 128, 256, 2, {0.65f, 1.0f}},  // four waves of 64 x 64, two stages
    {256, 64, 512, 1, {0.6f, 0.0f}},    // eight waves of 64 x 32, three stages
    {64, 64, 256, 2, {0.28f, 0.42f}},   // four waves of 32 x 32, four stages
};
constexpr int kKinds = (int)(sizeof(kTiles) / sizeof(kTiles[0]));
constexpr uint32_t kMaxSplits = 32, kMinBlocks = 4;  // parts of a sum, blocks of a part

struct Plan {
    int kind;  // of kTiles
    uint32_t splits;
    float time;  // estimated, us
};
// The tiles and parts of the shortest estimated time; parts of up to part_bytes in all, of rows of a multiple of four floats.
static inline Plan plan_of(const cnr_ctx *ctx, uint64_t columns, uint64_t rows, uint64_t blocks, float out_bytes, uint64_t part_bytes) {
    const float units = ctx ? (float)ctx->n_cu : 256.0f;
    const float outputs = (float)columns * (float)rows;
    const float memory = (((float)columns + (float)rows) * (float)blocks * (float)kBlockBytes + outputs * out_bytes) / 4.7e6f;
    Plan best = {0, 1, 3e38f};
    for (int i = 0; i < kKinds; ++i) {
        const Tiles &t = kTiles[i];
        const float tiles = (float)cnr_ceil_div(columns, t.columns) * (float)cnr_ceil_div(rows, t.rows);
        if (tiles * (float)t.threads >= 4.2e9f) continue;  // grids count threads in 32 bits
        for (uint32_t s = 1; s == 1 || (s <= kMaxSplits && blocks >= (uint64_t)s * kMinBlocks && tiles * (float)s <= 4.0f * units &&
                                        s * rows * cnr_ceil_div(columns, 4) * 16 <= part_bytes); ++s) {
            const float groups = tiles * (float)s, round = units * (float)t.resident, rounds = floorf(groups / round);
            const float rest = ceilf((groups - rounds * round) / units);  // workgroups on a unit in the last round
            const float each = 2.5f + (float)(t.columns * t.rows) * (s > 1 ? 4.0f : out_bytes) * units / 4.7e6f;
            const float some = ceilf((float)blocks / (float)s);
            float time = rounds * (some * t.block[t.resident - 1] + each) + (rest > 0.0f ? some * t.block[(int)rest - 1] + each : 0.0f);
            time = (time > memory ? time : memory) + 0.25f * (time < memory ? time : memory);  // one does not quite hide the other
            if (s > 1) time += 3.5f + (float)(s + 1) * outputs * 4.0f / 3e6f;  // joining the parts
            if (time < best.time) best = {i, s, time};
        }
    }
    return best;
}
// Rows [0, first_rows) by one plan and the others by another: whole rounds of workgroups, and what is left in smaller tiles or parts of its sums.
struct Plans {
    Plan first, rest;
    uint64_t first_rows;
};
static inline Plans plans_of(const cnr_ctx *ctx, uint64_t columns, uint64_t rows, uint64_t blocks, float out_bytes, uint64_t part_bytes) {
    Plans best = {plan_of(ctx, columns, rows, blocks, out_bytes, part_bytes), {0, 1, 0.0f}, rows};
    const Tiles &t = kTiles[0];
    const uint64_t units = ctx ? (uint64_t)ctx->n_cu : 256, across = cnr_ceil_div(columns, t.columns), rounds = cnr_ceil_div(rows, t.rows) * across / units;
    const uint64_t first_rows = rounds * units / across * t.rows;
    if (first_rows == 0 || first_rows >= rows) return best;
    const Plan first = plan_of(ctx, columns, first_rows, blocks, out_bytes, 0), rest = plan_of(ctx, columns, rows - first_rows, blocks, out_bytes, part_bytes);
    if (first.time + rest.time + 3.0f < best.first.time) best = {first, rest, first_rows};
    return best;
}

#ifdef __HIPCC__
template <int TYPE, bool ACROSS, bool DOWN, typename Epilogue>
void launch(const Args &p, int kind, const Epilogue &e, hipStream_t s) {
    const Tiles &t = kTiles[kind];
    const dim3 grid((unsigned)(cnr_ceil_div(p.columns, t.columns) * cnr_ceil_div(p.rows, t.rows) * p.splits)), threads(t.threads);
    switch (kind) {
        case 0: hipLaunchKernelGGL((tile_kernel<TYPE, ACROSS, DOWN, 2, 4, 8, 4, 2, Epilogue>), grid, threads, 0, s, p, e); break;
        case 1: hipLaunchKernelGGL((tile_kernel<TYPE, ACROSS, DOWN, 2, 4, 4, 2, 4, Epilogue>), grid, threads, 0, s, p, e); break;
        case 2: hipLaunchKernelGGL((tile_kernel<TYPE, ACROSS, DOWN, 2, 2, 4, 4, 2, Epilogue>), grid, threads, 0, s, p, e); break;
        case 3: hipLaunchKernelGGL((tile_kernel<TYPE, ACROSS, DOWN, 4, 2, 4, 2, 3, Epilogue>), grid, threads, 0, s, p, e); break;
        default: hipLaunchKernelGGL((tile_kernel<TYPE, ACROSS, DOWN, 2, 2, 2, 2, 4, Epilogue>), grid, threads, 0, s, p, e); break;
    }
}
#endif

}  // namespace dense
