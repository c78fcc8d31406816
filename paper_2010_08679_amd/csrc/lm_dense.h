// Products of plain matrices, out[m][n] = sum over k of A[m][k] B[n][k], for kernels that do something of their own with the outputs.
//
// Both operands have k along their rows, as multiples of 128 bytes ("blocks"), rows a multiple of 16 bytes apart.  16-bit elements go through the
// matrix instructions of their type, floats through the fp32 ones: products and sums are fp32's for all three.
#pragma once

#include "lm_common.h"

#include <math.h>

namespace dense {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kBlockBytes = 128;

struct Args {
    const void *a, *b;
    uint64_t a_bytes, b_bytes;  // from one row to the next, below 2^23
    uint32_t m, n, blocks;      // blocks >= 1
    uint32_t splits;            // parts of the sum, each in its own workgroups
};

#ifdef __HIPCC__
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

// Part h of kParts of the product of 16 rows of A by 16 of B, 32 bytes of each row: lane l holds bytes of row l % 16, which ones does not matter as
// long as both operands agree.  Sum i of a lane belongs to A's row 4 (l / 16) + i and B's row l % 16.
template <int TYPE>
struct Multiply {
    static constexpr int kParts = TYPE == CNR_FLOAT_F32 ? 8 : 2;
    template <int H>
    static __device__ __forceinline__ f32x4 part(const i32x8 &x, const i32x8 &y, const f32x4 &sum) {
        if constexpr (TYPE == CNR_FLOAT_F32) {
            return __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(x[H]), __int_as_float(y[H]), sum, 0, 0, 0);
        } else {
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
    }
};

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

// What a workgroup's outputs are to its epilogue.  A lane holds 4 MF consecutive rows from `m` on by NF consecutive columns from `n` on: row i and
// column g in acc[i % MF][g][i / MF].
struct Place {
    uint32_t m0, n0;        // first output of the workgroup
    uint32_t m, n;          // of the lane
    uint32_t row, column;   // the lane's first row and column within the workgroup's
    uint32_t split, tile_n;
    uint8_t *lds;           // free, as large as the stages were
};

// A workgroup of WM x WN waves has 16 WM MF x 16 WN NF outputs, a wave 16 MF x 16 NF of them, and walks along k a block at a time; the next
// STAGES - 1 blocks travel from memory into LDS while this one's are multiplied.
//
// Fragment f of a wave holds rows MF r + f of its part of A (r = lane % 16), and likewise of B, so that a lane's outputs lie side by side.  LDS
// holds two rows of 128 bytes to a line of 256, its sixteen pieces of 16 bytes permuted by r: sixteen lanes that read the same piece of their rows
// find it in sixteen different places, all banks in use.  Memory is read straight into LDS, where a wave's 64 pieces lie in
// order, so the permutation is in which piece a lane asks for.
//
// A block's products go by quarters, each half of the wave's rows of A with each half of those of B, so that half of the operands are in registers while
// the other half, or the next block's first, are on their way from LDS; loads go between matrix instructions.  The last quarter needs nothing more
// from this stage: before it all waves meet, in it the stage is filled again.
template <int TYPE, int WM, int WN, int MF, int NF, int STAGES, typename Epilogue>
__global__ void __launch_bounds__(WM * WN * kWave, 2) tile_kernel(const Args p, const Epilogue epilogue) {
    constexpr uint32_t TM = WM * 16 * MF, TN = WN * 16 * NF;
    constexpr int LA = 2 * MF / WN, LB = 2 * NF / WM;  // loads of 1 KB that each wave sends for a block of A and of B
    static_assert(LA * WN == 2 * MF && LB * WM == 2 * NF, "whole loads");
    constexpr uint32_t kB = TM * kBlockBytes, kStage = kB + TN * kBlockBytes;
    constexpr int kLoads = LA + LB;
    __shared__ __align__(256) uint8_t lds[STAGES * kStage];
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint32_t r = lane % 16, quarter = lane / 16;
    const uint32_t wave_m = wave / WN * 16 * MF, wave_n = wave % WN * 16 * NF;

    // Workgroups go to the eight XCDs in turn: each XCD gets tiles that lie together, in bands of kBand rows of tiles, for its L2.
    constexpr uint32_t kBand = 4;
    const uint32_t tiles_m = (p.m + TM - 1) / TM, tiles_n = (p.n + TN - 1) / TN, tiles = tiles_m * tiles_n, all = tiles * p.splits;
    const uint32_t xcd = wg_x() % 8, each = all / 8, more = all % 8;
    const uint32_t id = xcd * each + (xcd < more ? xcd : more) + wg_x() / 8;
    const uint32_t split = id / tiles, at = id % tiles;
    const uint32_t band = at / (kBand * tiles_n), band_rows = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
    const uint32_t in_band = at - band * kBand * tiles_n;
    const uint32_t tile_n = in_band / band_rows, m0 = (band * kBand + in_band % band_rows) * TM, n0 = tile_n * TN;
    // Blocks of this part of the sum; the host sees to it that there are some.
    const uint32_t begin = (uint32_t)((uint64_t)p.blocks * split / p.splits), end = (uint32_t)((uint64_t)p.blocks * (split + 1) / p.splits);

    // Rows beyond the matrix read its last one again.
    const uint32_t rows_a = p.m - m0 < TM ? p.m - m0 : TM, rows_b = p.n - n0 < TN ? p.n - n0 : TN;
    const uint32_t row_bytes = p.blocks * kBlockBytes;
    const i32x4 buffer_a = buffer_of(reinterpret_cast<uint64_t>(p.a) + (uint64_t)m0 * p.a_bytes, (uint64_t)(rows_a - 1) * p.a_bytes + row_bytes);
    const i32x4 buffer_b = buffer_of(reinterpret_cast<uint64_t>(p.b) + (uint64_t)n0 * p.b_bytes, (uint64_t)(rows_b - 1) * p.b_bytes + row_bytes);
    uint32_t from_a[LA], from_b[LB];
#pragma unroll
    for (int j = 0; j < LA; ++j) {
        const uint32_t line = (wave * LA + j) * 4 + quarter, logical = (lane % 16) ^ (2 * line / MF % 16);
        const uint32_t row = 2 * line + logical / 8;
        from_a[j] = (row < rows_a ? row : rows_a - 1) * (uint32_t)p.a_bytes + logical % 8 * 16;
    }
#pragma unroll
    for (int j = 0; j < LB; ++j) {
        const uint32_t line = (wave * LB + j) * 4 + quarter, logical = (lane % 16) ^ (2 * line / NF % 16);
        const uint32_t row = 2 * line + logical / 8;
        from_b[j] = (row < rows_b ? row : rows_b - 1) * (uint32_t)p.b_bytes + logical % 8 * 16;
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // Load j of the wave's kLoads for block kb of this part of the sum into the stage at `to`; beyond its end the last block once more, which
    // nobody reads: the count of loads stays the same without a branch.
    auto fetch = [&](uint32_t kb, uint32_t to, auto index) {
        constexpr int J = decltype(index)::value;
        const uint32_t along = (kb < end - 1 ? kb : end - 1) * kBlockBytes;
        if constexpr (J < LA)
            load_to_lds(buffer_a, lds_at + to + (wave * LA + J) * 1024, from_a[J], along);
        else
            load_to_lds(buffer_b, lds_at + to + kB + (wave * LB + J - LA) * 1024, from_b[J - LA], along);
    };

    f32x4 acc[MF][NF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Where a lane's row of fragment f lies: lines of 256 bytes for each pair of fragments, in them the piece h at one of two places that
    // depend on the lane alone, in the other half of the line for an odd f.  These addresses move from stage to stage.
    uint32_t piece_a[2][2], piece_b[2][2];  // [odd][h]
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t place = ((quarter + 4 * (i % 2)) ^ r) * 16 ^ i / 2 * 128;
        piece_a[i / 2][i % 2] = (wave_m + r * MF) * kBlockBytes + place;
        piece_b[i / 2][i % 2] = kB + (wave_n + r * NF) * kBlockBytes + place;
    }
    auto move_pieces = [&](uint32_t by) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            piece_a[i / 2][i % 2] += by;
            piece_b[i / 2][i % 2] += by;
        }
    };
    auto fragment = [&](const uint32_t (&piece)[2][2], uint32_t f) {
        i32x4 part[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) part[h] = *reinterpret_cast<const i32x4 *>(lds + piece[f % 2][h] + f / 2 * 256);
        return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // The i-th of `of` even shares of N things to do.
    auto share = [](auto i, auto of, auto n, const auto &act) {
        constexpr int I = decltype(i)::value, OF = decltype(of)::value, N = decltype(n)::value, from = I * N / OF, to = (I + 1) * N / OF;
        unrolled<to - from>([&](auto j) { act(Index<from + decltype(j)::value>()); });
    };

    typedef Multiply<TYPE> Product;
    constexpr int HM = MF / 2, HN = NF / 2, kPairs = HM * HN, kSteps = kPairs * Product::kParts;
    unrolled<STAGES>([&](auto i) { unrolled<kLoads>([&](auto j) { fetch(begin + decltype(i)::value, decltype(i)::value * kStage, j); }); });
    wait_for_loads<(STAGES - 1) * kLoads>();
    barrier();
    i32x8 x[2][HM], y[2][HN];
#pragma unroll
    for (int f = 0; f < HM; ++f) x[0][f] = fragment(piece_a, f);
#pragma unroll
    for (int g = 0; g < HN; ++g) y[0][g] = fragment(piece_b, g);
    // One quarter; with its i-th matrix instruction goes beside(i).  Sums take turns, so that none waits for the one before.
    auto quarter_of = [&](auto half_a, auto half_b, const auto &beside) {
        constexpr int A = decltype(half_a)::value, B = decltype(half_b)::value;
        unrolled<kSteps>([&](auto step) {
            constexpr int H = decltype(step)::value / kPairs, PAIR = decltype(step)::value % kPairs, F = PAIR % HM, G = PAIR / HM, MA = A * HM + F, NB = B * HN + G;
            acc[MA][NB] = Product::template part<H>(x[A][F], y[B][G], acc[MA][NB]);
            beside(step);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    uint32_t stage = 0;  // where it begins in LDS
    for (uint32_t kb = begin; kb < end; ++kb) {
        const uint32_t next = stage + kStage < STAGES * kStage ? stage + kStage : 0;
        quarter_of(Index<0>(), Index<0>(), [&](auto step) {
            share(step, Index<kSteps>(), Index<HN>(), [&](auto g) { y[1][decltype(g)::value] = fragment(piece_b, HN + decltype(g)::value); });
        });
        quarter_of(Index<0>(), Index<1>(), [&](auto step) {
            share(step, Index<kSteps>(), Index<HM>(), [&](auto f) { x[1][decltype(f)::value] = fragment(piece_a, HM + decltype(f)::value); });
        });
        quarter_of(Index<1>(), Index<0>(), [&](auto) {});
        wait_for_loads<(STAGES - 2) * kLoads>();
        barrier();
        move_pieces(next - stage);
        quarter_of(Index<1>(), Index<1>(), [&](auto step) {
            share(step, Index<kSteps>(), Index<HM + HN>(), [&](auto j) {
                constexpr int J = decltype(j)::value;
                if constexpr (J < HM)
                    x[0][J] = fragment(piece_a, J);
                else
                    y[0][J - HM] = fragment(piece_b, J - HM);
            });
            share(step, Index<kSteps>(), Index<kLoads>(), [&](auto j) { fetch(kb + STAGES, stage, j); });
        });
        stage = next;
    }
    wait_for_loads<0>();
    if constexpr (Epilogue::kUsesLds) __syncthreads();
    Place place;
    place.m0 = m0;
    place.n0 = n0;
    place.row = wave_m + quarter * 4 * MF;
    place.column = wave_n + r * NF;
    place.m = m0 + place.row;
    place.n = n0 + place.column;
    place.split = split;
    place.tile_n = tile_n;
    place.lds = lds;
    epilogue.template finish<TM, TN, WN, MF, NF>(p, place, acc);
}
#endif

// ---- which tiles ----------------------------------------------------------------------------------------------
//
// A workgroup's time for a block by how many share a compute unit, in us, with 16-bit elements; the fp32 instructions take kSlow32 times as long.
struct Tiles {
    uint32_t rows, columns, resident;
    float block[2];
};
constexpr Tiles kTiles[] = {
    {256, 256, 1, {1.65f, 0.0f}},   // eight waves of 128 x 64, two stages
    {128, 128, 1, {0.54f, 0.0f}},   // eight waves of 64 x 32, four stages
    {64, 64, 2, {0.28f, 0.42f}},    // four waves of 32 x 32, four stages
};
constexpr int kKinds = (int)(sizeof(kTiles) / sizeof(kTiles[0]));
constexpr float kSlow32 = 8.0f;
constexpr uint32_t kMaxSplits = 16, kMinBlocks = 4;  // parts of a sum, blocks of a part

struct Plan {
    int kind;  // of kTiles
    uint32_t splits;
};
// The tiles and parts of the shortest estimated time; parts of up to part_bytes in all, of rows of a multiple of four floats.
static inline Plan plan_of(const cnr_ctx *ctx, cnr_float_type type, uint64_t m, uint64_t n, uint64_t blocks, uint64_t part_bytes) {
    const float units = ctx ? (float)ctx->n_cu : 256.0f, slow = type == CNR_FLOAT_F32 ? kSlow32 : 1.0f;
    const float memory = ((float)m + (float)n) * (float)blocks * (float)kBlockBytes / 4.7e6f;
    Plan best = {0, 1};
    float least = 3e38f;
    for (int i = 0; i < kKinds; ++i) {
        const Tiles &t = kTiles[i];
        const float tiles = (float)cnr_ceil_div(m, t.rows) * (float)cnr_ceil_div(n, t.columns);
        for (uint32_t s = 1; s == 1 || (s <= kMaxSplits && blocks >= (uint64_t)s * kMinBlocks && s * m * cnr_ceil_div(n, 4) * 16 <= part_bytes); s *= 2) {
            const float groups = tiles * (float)s, round = units * (float)t.resident, rounds = floorf(groups / round);
            if (groups * (i < 2 ? 512.0f : 256.0f) >= 4.2e9f) continue;  // grids count threads in 32 bits
            const float rest = ceilf((groups - rounds * round) / units);  // workgroups on a unit in the last round
            float time = ceilf((float)blocks / (float)s) * slow * (rounds * t.block[t.resident - 1] + (rest > 0.0f ? t.block[(int)rest - 1] : 0.0f));
            time += 1.5f * (rounds + (rest > 0.0f ? 1.0f : 0.0f));
            time = (time > memory ? time : memory) + 0.25f * (time < memory ? time : memory);  // one does not quite hide the other
            if (s > 1) time += 3.5f + (float)(s + 1) * (float)m * (float)n * 4.0f / 3e6f;        // writing the parts, and joining them
            if (time < least) {
                least = time;
                best = {i, s};
            }
        }
    }
    return best;
}

#ifdef __HIPCC__
template <int TYPE, typename Epilogue>
void launch(const Args &p, int kind, const Epilogue &e, hipStream_t s) {
    const Tiles &t = kTiles[kind];
    const dim3 grid((unsigned)(cnr_ceil_div(p.m, t.rows) * cnr_ceil_div(p.n, t.columns) * p.splits));
    switch (kind) {
        case 0: hipLaunchKernelGGL((tile_kernel<TYPE, 2, 4, 8, 4, 2, Epilogue>), grid, dim3(512), 0, s, p, e); break;
        case 1: hipLaunchKernelGGL((tile_kernel<TYPE, 2, 4, 4, 2, 4, Epilogue>), grid, dim3(512), 0, s, p, e); break;
        default: hipLaunchKernelGGL((tile_kernel<TYPE, 2, 2, 2, 2, 4, Epilogue>), grid, dim3(256), 0, s, p, e); break;
    }
}
#endif

}  // namespace dense
