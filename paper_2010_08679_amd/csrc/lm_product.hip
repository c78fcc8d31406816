// Products of blocked matrices: out[m][n] = sum over blocks of scale_a scale_b (codes_a . codes_b).
//
// Both operands have k along their rows, so a matrix instruction's operand is 32 bytes in a row of codes for each lane,
// whichever way a block is held.  Which of the block's 128 columns a lane's bytes are does not matter as long as
// both operands agree: a lane takes the 32 bytes from 32 * (lane / 16) of row lane % 16.
//
// Two ways to add up a block's 16 x 16 x 128 products:
//   8-bit instructions, scales of powers of two applied by them.  Exact products; of each eight that are added in one
//     step what lies 2^-14 or more below the largest is dropped (measured: normal codes 1.5e-5 of the result, codes
//     of uniformly spread exponents 7e-5), a small part of a bfloat16's (2^-9) or a half's (2^-12) rounding;
//   bfloat16 instructions on the codes converted in registers, exact as well (4 of 8 bits of mantissa), their scales
//     of powers of two applied by the conversion, added up in fp32 (measured 1e-8 to 6e-8): float outputs.
// Scales of any value multiply each block's sum before it is added to the total.
#include "lm_common.h"

#include <type_traits>

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
    const uint8_t *a, *b;           // codes
    const void *a_scale, *b_scale;
    uint64_t row_bytes;             // of both
    uint64_t a_stride, b_stride;    // scales of one block of columns
    uint32_t m, n, blocks;
    uint32_t a_shift, b_shift;      // rows that share a scale: 2^shift
    void *out;
    uint64_t out_stride;
    int out_type, accumulate;
};

template <int SCALE>
struct ScaleOf;
template <>
struct ScaleOf<CNR_SCALE_E8M0> {
    typedef uint8_t type;
};
template <>
struct ScaleOf<CNR_SCALE_F32> {
    typedef float type;
};

// A lane's 32 codes as bfloat16, times 2^(scale - 127).
struct Wide {
    bf16x8 part[4];
};
__device__ __forceinline__ Wide widen(const i32x8 &codes, uint32_t scale) {
    Wide w;
    const float s = __uint_as_float(scale << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[i], s, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[i], s, true);
        w.part[i / 2][4 * (i % 2)] = lo[0];
        w.part[i / 2][4 * (i % 2) + 1] = lo[1];
        w.part[i / 2][4 * (i % 2) + 2] = hi[0];
        w.part[i / 2][4 * (i % 2) + 3] = hi[1];
    }
    return w;
}

__device__ __forceinline__ i32x8 load_codes(const uint8_t *p) {
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(p), hi = *reinterpret_cast<const i32x4 *>(p + 16);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ void store_out(const ProductArgs &p, uint32_t m, uint32_t n, float v) {
    const uint64_t at = (uint64_t)m * p.out_stride + n;
    if (p.out_type == CNR_FLOAT_F32) {
        float *o = reinterpret_cast<float *>(p.out) + at;
        *o = p.accumulate ? *o + v : v;
    } else if (p.out_type == CNR_FLOAT_BF16) {
        __bf16 *o = reinterpret_cast<__bf16 *>(p.out) + at;
        *o = (__bf16)(p.accumulate ? (float)*o + v : v);
    } else {
        _Float16 *o = reinterpret_cast<_Float16 *>(p.out) + at;
        *o = (_Float16)(p.accumulate ? (float)*o + v : v);
    }
}

// Few rows of A: the codes of B are read once, straight into the matrix instructions' registers.  A workgroup has 16 MF x 16 NF
// outputs; its waves take every fourth block of columns and add up their sums in LDS at the end.
template <int SCALE, bool FULL, int MF, int NF>
__global__ void __launch_bounds__(kBlock) narrow_kernel(const ProductArgs p) {
    typedef typename ScaleOf<SCALE>::type S;
    __shared__ f32x4 sums[kWavesPerBlock][MF * NF][kWave];
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint32_t m0 = wg_y() * 16 * MF, n0 = wg_x() * 16 * NF;
    const uint8_t *a[MF], *b[NF];
    const S *sa[MF], *sb[NF];
    uint32_t sa_at[MF][4];  // scales of the rows of A that a lane's four sums belong to
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        uint32_t r = m0 + 16 * f + lane % 16;
        r = r < p.m ? r : p.m - 1;
        a[f] = p.a + (uint64_t)r * p.row_bytes + lane / 16 * 32;
        sa[f] = reinterpret_cast<const S *>(p.a_scale) + (r >> p.a_shift);
        if (SCALE == CNR_SCALE_F32) {
            sa[f] = reinterpret_cast<const S *>(p.a_scale);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t q = m0 + 16 * f + lane / 16 * 4 + i;
                sa_at[f][i] = (q < p.m ? q : p.m - 1) >> p.a_shift;
            }
        }
    }
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        uint32_t r = n0 + 16 * f + lane % 16;
        r = r < p.n ? r : p.n - 1;
        b[f] = p.b + (uint64_t)r * p.row_bytes + lane / 16 * 32;
        sb[f] = reinterpret_cast<const S *>(p.b_scale) + (r >> p.b_shift);
    }
    f32x4 acc[MF][NF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (uint32_t kb = wave; kb < p.blocks; kb += kWavesPerBlock) {
        i32x8 x[MF], y[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) y[f] = load_codes(b[f] + (uint64_t)kb * CNR_BLOCK);
#pragma unroll
        for (int f = 0; f < MF; ++f) x[f] = load_codes(a[f] + (uint64_t)kb * CNR_BLOCK);
        S t[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) t[f] = sb[f][kb * p.b_stride];
        if (SCALE == CNR_SCALE_E8M0) {
            uint32_t s[MF];
#pragma unroll
            for (int f = 0; f < MF; ++f) s[f] = (uint32_t)sa[f][kb * p.a_stride];
            if (FULL) {
                Wide wx[MF];
#pragma unroll
                for (int f = 0; f < MF; ++f) wx[f] = widen(x[f], s[f]);
#pragma unroll
                for (int g = 0; g < NF; ++g) {
                    const Wide wy = widen(y[g], (uint32_t)t[g]);
#pragma unroll
                    for (int f = 0; f < MF; ++f)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[f][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wx[f].part[i], wy.part[i], acc[f][g], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int f = 0; f < MF; ++f)
#pragma unroll
                    for (int g = 0; g < NF; ++g)
                        acc[f][g] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[f], y[g], acc[f][g], 0, 0, 0, (int)s[f], 0, (int)t[g]);
            }
        } else {
            const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                const S *from = sa[f] + kb * p.a_stride;
                const f32x4 s = {(float)from[sa_at[f][0]], (float)from[sa_at[f][1]], (float)from[sa_at[f][2]], (float)from[sa_at[f][3]]};
                Wide wx;
                if (FULL) wx = widen(x[f], 127);
#pragma unroll
                for (int g = 0; g < NF; ++g) {
                    f32x4 d = zero;
                    if (FULL) {
                        const Wide wy = widen(y[g], 127);
#pragma unroll
                        for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wx.part[i], wy.part[i], d, 0, 0, 0);
                    } else {
                        d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[f], y[g], zero, 0, 0, 0, 127, 0, 127);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[f][g][i] = __builtin_fmaf(d[i] * s[i], (float)t[g], acc[f][g][i]);
                }
            }
        }
    }
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) sums[wave][f * NF + g][lane] = acc[f][g];
    __syncthreads();
    for (uint32_t e = tid_x(); e < 16 * MF * 16 * NF; e += kBlock) {
        const uint32_t m = e / (16 * NF), n = e % (16 * NF);
        if (m0 + m >= p.m || n0 + n >= p.n) continue;
        const uint32_t from = m % 16 / 4 * 16 + n % 16;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) v += sums[w][m / 16 * NF + n / 16][from][m % 4];
        store_out(p, m0 + m, n0 + n, v);
    }
}

template <int MF, int NF>
void narrow(const ProductArgs &p, cnr_scale_type scale, hipStream_t s) {
    const dim3 grid((unsigned)cnr_ceil_div(p.n, 16 * NF), (unsigned)cnr_ceil_div(p.m, 16 * MF));
    const bool full = p.out_type == CNR_FLOAT_F32;
    if (scale == CNR_SCALE_E8M0) {
        if (full)
            hipLaunchKernelGGL((narrow_kernel<CNR_SCALE_E8M0, true, MF, NF>), grid, dim3(kBlock), 0, s, p);
        else
            hipLaunchKernelGGL((narrow_kernel<CNR_SCALE_E8M0, false, MF, NF>), grid, dim3(kBlock), 0, s, p);
    } else {
        if (full)
            hipLaunchKernelGGL((narrow_kernel<CNR_SCALE_F32, true, MF, NF>), grid, dim3(kBlock), 0, s, p);
        else
            hipLaunchKernelGGL((narrow_kernel<CNR_SCALE_F32, false, MF, NF>), grid, dim3(kBlock), 0, s, p);
    }
}

// ---- many rows: tiles staged in LDS -----------------------------------------------------------------------------
//
// A workgroup of four waves has 32 MF x 32 NF outputs, each wave 16 MF x 16 NF, and walks along k a block of 128 at a time; the next
// block's codes travel from memory into LDS while this one's are multiplied.
//
// Fragment f of a wave holds rows MF * r + f of its part of A (r = lane % 16), and likewise of B: a lane's fragments are rows side by
// side, so that it reads their scales in one load (a byte of which each matrix instruction picks), and holds
// NF outputs side by side, which it stores in one go.
//
// LDS holds two rows of 128 codes to a line of 256 bytes, its sixteen pieces of 16 bytes permuted by r: sixteen lanes that
// read the same piece of their rows find it in sixteen different places, all banks in use.  Memory is read straight
// into LDS, where a wave's 64 pieces lie in order, so the permutation is in which piece a lane asks for.

__device__ __forceinline__ i32x4 buffer_of(const void *base, uint64_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    i32x4 r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)p);
    r[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xffffu));
    r[2] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(bytes < 0xffffffffull ? bytes : 0xffffffffull));
    r[3] = 0x00027000;
    return r;
}

// 64 pieces of 16 bytes, one for each lane, from memory to `lds` and on in lane order.  Written as an instruction because the
// compiler, which cannot tell the halves of the LDS apart, would wait for it before every read of the other half;
// wait_for_loads() below does, once a block.  (Nothing else here uses M0.)
__device__ __forceinline__ void load_to_lds(const i32x4 &buffer, uint32_t lds, uint32_t offset, uint32_t all) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(all));
}
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Scales of the F rows that a lane's fragments have, as exponents (a byte each) and, where they are of any value, as fractions.
template <int SCALE, int F>
struct Scales {
    uint32_t exponent[(F + 3) / 4];
    float fraction[SCALE == CNR_SCALE_F32 ? F : 1];
};
// A scale's exponent goes into the matrix instruction and its fraction, from 1 to 2, multiplies the sum: neither leaves fp32's range
// unless the result does.  (A scale below 2^-126 counts as 0.)
__device__ __forceinline__ float fraction_of(float s) {
    const uint32_t b = __float_as_uint(s);
    return b & 0x7f800000u ? __uint_as_float((b & 0x807fffffu) | 0x3f800000u) : 0.0f;
}
__device__ __forceinline__ uint32_t exponent_of(float s) { return __float_as_uint(s) >> 23 & 255u; }

// In two parts, so that the loads are waited for where they are used.  Without a branch, which would end the compiler's sight of the
// block: a tile's one scale is taken from the aligned word (or four) that it lies in, of which rows' scales fill one and the next.
template <int SCALE, int F>
struct LoadedScales {
    typedef typename std::conditional<SCALE == CNR_SCALE_E8M0, uint32_t, f32x4>::type Word;
    static_assert(F % 4 == 0, "whole words of scales");
    Word word[F / 4];
    uint32_t pick;
    bool tile;
    __device__ __forceinline__ void load(const typename ScaleOf<SCALE>::type *p, bool of_tile) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        const Word *from = reinterpret_cast<const Word *>(at & ~(uintptr_t)(sizeof(Word) - 1));
#pragma unroll
        for (int i = 0; i < F / 4; ++i) word[i] = from[of_tile ? 0 : i];
        tile = of_tile;
        pick = SCALE == CNR_SCALE_F32 ? (uint32_t)at / 4 % 4 : of_tile ? ((uint32_t)at & 3u) * 0x01010101u : 0x03020100u;
    }
    __device__ __forceinline__ Scales<SCALE, F> scales() const {
        Scales<SCALE, F> s;
#pragma unroll
        for (int i = 0; i < F / 4; ++i) {
            if constexpr (SCALE == CNR_SCALE_E8M0) {
                s.exponent[i] = __builtin_amdgcn_perm(0u, word[i], pick);
            } else {
                const f32x4 w = word[i];
                const float one = pick & 2 ? (pick & 1 ? w[3] : w[2]) : (pick & 1 ? w[1] : w[0]);
                s.exponent[i] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = tile ? one : w[j];
                    s.exponent[i] |= exponent_of(v) << (8 * j);
                    s.fraction[4 * i + j] = fraction_of(v);
                }
            }
        }
        return s;
    }
};
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

// acc += A B, written as instructions for the sake of their registers: 128 x 128 sums fill all accumulation registers of a lane
// and the operands lie in the others, which the compiler does not find by itself (it moves sums to and fro and
// spills).  The idle states in front are what an operand needs that an ordinary instruction has just written.  Sums are not touched in any other way between settle() before the first and settle() after the last of these.
template <int BYTE_A, int BYTE_B>
__device__ __forceinline__ void multiply_add(f32x4 &acc, const i32x8 &x, const i32x8 &y, uint32_t sx, uint32_t sy) {
    asm("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]"
        : "+a"(acc)
        : "v"(x), "v"(y), "v"(sx), "v"(sy), "n"(BYTE_A % 2), "n"(BYTE_B % 2), "n"(BYTE_A / 2), "n"(BYTE_B / 2));
}
__device__ __forceinline__ void multiply_add(f32x4 &acc, const bf16x8 &x, const bf16x8 &y) {
    asm("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(x), "v"(y));
}
// Longer than any matrix instruction takes to write its sums, or a move to become visible to one.
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory"); }

template <typename T, int NF>
__device__ __forceinline__ void store_row(const ProductArgs &p, uint32_t m, uint32_t n, const float *v) {
    T *o = reinterpret_cast<T *>(p.out) + (uint64_t)m * p.out_stride + n;
    if (n + NF <= p.n) {
        Pack<T, NF> w;
        if (p.accumulate) {
            const Pack<T, NF> old = *reinterpret_cast<const Pack<T, NF> *>(o);
#pragma unroll
            for (int j = 0; j < NF; ++j) w.v[j] = (T)((float)old.v[j] + v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < NF; ++j) w.v[j] = (T)v[j];
        }
        *reinterpret_cast<Pack<T, NF> *>(o) = w;
    } else {
#pragma unroll
        for (int j = 0; j < NF; ++j)
            if (n + j < p.n) o[j] = (T)(p.accumulate ? (float)o[j] + v[j] : v[j]);
    }
}

template <int SCALE, bool FULL, int MF, int NF>
__global__ void __launch_bounds__(kBlock, 1) tile_kernel(const ProductArgs p) {
    typedef typename ScaleOf<SCALE>::type S;
    constexpr uint32_t TM = 32 * MF, TN = 32 * NF, kStage = (TM + TN) * CNR_BLOCK;
    __shared__ __align__(256) uint8_t lds[2 * kStage];
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint32_t r = lane % 16, quarter = lane / 16;
    const uint32_t wave_m = wave / 2 * 16 * MF, wave_n = wave % 2 * 16 * NF;

    // Workgroups go to the eight XCDs in turn: each XCD gets tiles that lie together, in bands of kBand rows of tiles, for its L2.
    constexpr uint32_t kBand = 4;
    const uint32_t tiles_m = (p.m + TM - 1) / TM, tiles_n = (p.n + TN - 1) / TN, tiles = tiles_m * tiles_n;
    const uint32_t xcd = wg_x() % 8, each = tiles / 8, more = tiles % 8;
    const uint32_t at = xcd * each + (xcd < more ? xcd : more) + wg_x() / 8;
    const uint32_t band = at / (kBand * tiles_n), band_rows = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
    const uint32_t in_band = at - band * kBand * tiles_n;
    const uint32_t m0 = (band * kBand + in_band % band_rows) * TM, n0 = in_band / band_rows * TN;

    // Rows beyond the matrix read its last one again.
    const uint32_t rows_a = p.m - m0 < TM ? p.m - m0 : TM, rows_b = p.n - n0 < TN ? p.n - n0 : TN;
    const i32x4 buffer_a = buffer_of(p.a + (uint64_t)m0 * p.row_bytes, (uint64_t)rows_a * p.row_bytes);
    const i32x4 buffer_b = buffer_of(p.b + (uint64_t)n0 * p.row_bytes, (uint64_t)rows_b * p.row_bytes);
    uint32_t from_a[MF], from_b[NF];
#pragma unroll
    for (int j = 0; j < MF; ++j) {
        const uint32_t line = (wave * MF + j) * 4 + quarter, logical = (lane % 16) ^ (2 * line / MF % 16);
        const uint32_t row = 2 * line + logical / 8;
        from_a[j] = (row < rows_a ? row : rows_a - 1) * (uint32_t)p.row_bytes + logical % 8 * 16;
    }
#pragma unroll
    for (int j = 0; j < NF; ++j) {
        const uint32_t line = (wave * NF + j) * 4 + quarter, logical = (lane % 16) ^ (2 * line / NF % 16);
        const uint32_t row = 2 * line + logical / 8;
        from_b[j] = (row < rows_b ? row : rows_b - 1) * (uint32_t)p.row_bytes + logical % 8 * 16;
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    auto fetch = [&](uint32_t kb, uint32_t stage) {
#pragma unroll
        for (int j = 0; j < MF; ++j) load_to_lds(buffer_a, lds_at + stage * kStage + (wave * MF + j) * 1024, from_a[j], kb * CNR_BLOCK);
#pragma unroll
        for (int j = 0; j < NF; ++j) load_to_lds(buffer_b, lds_at + stage * kStage + TM * CNR_BLOCK + (wave * NF + j) * 1024, from_b[j], kb * CNR_BLOCK);
    };
    // Row of each kind's scales that a lane starts at; rows beyond the matrix take ones that are there.
    const bool tile_a = p.a_shift != 0, tile_b = p.b_shift != 0;
    auto scale_row = [&](uint32_t row, uint64_t stride, bool tile, uint32_t per) {
        const uint64_t at = tile ? row / CNR_BLOCK : row, last = stride - (tile ? 1 : per);
        return at < last ? at : last;
    };
    const S *scale_a = reinterpret_cast<const S *>(p.a_scale) + scale_row(m0 + wave_m + r * MF, p.a_stride, tile_a, MF);
    const S *scale_b = reinterpret_cast<const S *>(p.b_scale) + scale_row(n0 + wave_n + r * NF, p.b_stride, tile_b, NF);

    f32x4 acc[MF][NF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Where a lane's row of fragment f lies: lines of 256 bytes for each pair of fragments, in them the piece h at one of two places that
    // depend on the lane alone, in the other half of the line for an odd f.
    uint32_t piece_a[2], piece_b[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        piece_a[h] = (wave_m + r * MF) * CNR_BLOCK + ((2 * quarter + h) ^ r) * 16;
        piece_b[h] = TM * CNR_BLOCK + (wave_n + r * NF) * CNR_BLOCK + ((2 * quarter + h) ^ r) * 16;
    }
    auto fragment = [&](const uint32_t (&piece)[2], uint32_t f) {
        i32x4 part[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) part[h] = *reinterpret_cast<const i32x4 *>(lds + (piece[h] ^ (f % 2 * 128)) + f / 2 * 256);
        return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    fetch(0, 0);
    LoadedScales<SCALE, MF> next_a;
    LoadedScales<SCALE, NF> next_b;
    next_a.load(scale_a, tile_a);
    next_b.load(scale_b, tile_b);
    wait_for_loads();
    barrier();
    Scales<SCALE, MF> sa = next_a.scales();
    Scales<SCALE, NF> sb = next_b.scales();
    settle();
    for (uint32_t kb = 0; kb < p.blocks; ++kb) {
        const uint32_t next = kb + 1 < p.blocks ? kb + 1 : kb;  // at the end once more what nobody reads
        fetch(next, (kb + 1) % 2);
        next_a.load(scale_a + (uint64_t)next * p.a_stride, tile_a);
        next_b.load(scale_b + (uint64_t)next * p.b_stride, tile_b);
        float rows[SCALE == CNR_SCALE_F32 ? MF : 1][4];  // fractions of the rows of the lane's sums
        if (SCALE == CNR_SCALE_F32) {
#pragma unroll
            for (int f = 0; f < MF; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) rows[f][i] = __shfl(sa.fraction[f], (int)(quarter * 4 + i));
        }
        typename std::conditional<FULL, Wide, i32x8>::type x[MF];
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            if constexpr (FULL)
                x[f] = widen(fragment(piece_a, f), sa.exponent[f / 4] >> (8 * (f % 4)) & 255u);
            else
                x[f] = fragment(piece_a, f);
        }
        i32x8 ahead = fragment(piece_b, 0);
        unrolled<NF>([&](auto g) {
            constexpr int G = decltype(g)::value;
            const i32x8 y = ahead;
            if constexpr (G + 1 < NF) ahead = fragment(piece_b, G + 1);
            Wide wy;
            if constexpr (FULL) wy = widen(y, sb.exponent[G / 4] >> (8 * (G % 4)) & 255u);
            if constexpr (SCALE == CNR_SCALE_E8M0 && FULL) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int f = 0; f < MF; ++f) multiply_add(acc[f][G], x[f].part[i], wy.part[i]);
            } else {
                unrolled<MF>([&](auto f) {
                    constexpr int F = decltype(f)::value;
                    if constexpr (SCALE == CNR_SCALE_E8M0) {
                        multiply_add<F % 4, G % 4>(acc[F][G], x[F], y, sa.exponent[F / 4], sb.exponent[G / 4]);
                    } else {
                        f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
                        if constexpr (FULL) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[F].part[i], wy.part[i], d, 0, 0, 0);
                        } else {
                            d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[F], y, d, 0, 0, F % 4, (int)sa.exponent[F / 4], G % 4, (int)sb.exponent[G / 4]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[F][G][i] = __builtin_fmaf(d[i], rows[F][i] * sb.fraction[G], acc[F][G][i]);
                    }
                });
            }
            __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t other = kb % 2 ? 0u - kStage : kStage;
            piece_a[h] += other;
            piece_b[h] += other;
        }
        wait_for_loads();
        barrier();
        sa = next_a.scales();
        sb = next_b.scales();
    }
    settle();

#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t m = m0 + wave_m + (quarter * 4 + i) * MF + f, n = n0 + wave_n + r * NF;
            if (m >= p.m || n >= p.n) continue;
            float v[NF];
#pragma unroll
            for (int g = 0; g < NF; ++g) v[g] = acc[f][g][i];
            if (FULL)
                store_row<float, NF>(p, m, n, v);
            else if (p.out_type == CNR_FLOAT_BF16)
                store_row<__bf16, NF>(p, m, n, v);
            else
                store_row<_Float16, NF>(p, m, n, v);
        }
}

template <int MF, int NF>
void tiled(const ProductArgs &p, cnr_scale_type scale, hipStream_t s) {
    const dim3 grid((unsigned)(cnr_ceil_div(p.m, 32 * MF) * cnr_ceil_div(p.n, 32 * NF)));
    const bool full = p.out_type == CNR_FLOAT_F32;
    if constexpr (MF * NF > 32) {
        if (full)
            hipLaunchKernelGGL((tile_kernel<CNR_SCALE_E8M0, true, MF, NF>), grid, dim3(kBlock), 0, s, p);
        else
            hipLaunchKernelGGL((tile_kernel<CNR_SCALE_E8M0, false, MF, NF>), grid, dim3(kBlock), 0, s, p);
    } else {
        if (full)
            hipLaunchKernelGGL((tile_kernel<CNR_SCALE_F32, true, MF, NF>), grid, dim3(kBlock), 0, s, p);
        else
            hipLaunchKernelGGL((tile_kernel<CNR_SCALE_F32, false, MF, NF>), grid, dim3(kBlock), 0, s, p);
    }
}

}  // namespace

extern "C" {

size_t cnr_block_product_workspace_bytes(const cnr_ctx *, uint64_t, uint64_t, uint64_t) { return 0; }

cnr_status cnr_block_product(cnr_ctx *ctx, const uint8_t *a_codes, const void *a_scale, cnr_block_kind a_kind,
                             uint64_t m, const uint8_t *b_codes, const void *b_scale, cnr_block_kind b_kind,
                             uint64_t n, uint64_t k, cnr_scale_type scale_type, void *out, cnr_float_type out_type,
                             uint64_t out_stride, int accumulate, void *workspace, void *stream) {
    if (!ctx || !cnr_valid_float_type(out_type) || (a_kind != CNR_BLOCK_ROW && a_kind != CNR_BLOCK_TILE) ||
        (b_kind != CNR_BLOCK_ROW && b_kind != CNR_BLOCK_TILE) || (scale_type != CNR_SCALE_E8M0 && scale_type != CNR_SCALE_F32) || out_stride < n)
        return CNR_E_INVALID;
    if (m > CNR_LM_MAX_SIZE || n > CNR_LM_MAX_SIZE || k > CNR_LM_MAX_SIZE) return CNR_E_TOO_LARGE;
    if (m == 0 || n == 0 || (k == 0 && accumulate)) return CNR_OK;
    // more outputs than a GPU holds; grids count threads in 32 bits
    if (cnr_ceil_div(m, 128) * cnr_ceil_div(n, 128) >= 1u << 24 || (m > 64 && k >= (1u << 24) - CNR_BLOCK && m > 1u << 19)) return CNR_E_TOO_LARGE;
    if (!out || (k && (!a_codes || !a_scale || !b_codes || !b_scale))) return CNR_E_INVALID;
    if (!cnr_aligned(a_codes, 16) || !cnr_aligned(a_scale, 16) || !cnr_aligned(b_codes, 16) || !cnr_aligned(b_scale, 16) ||
        !cnr_aligned(out, cnr_float_bytes(out_type)) || !cnr_aligned(workspace, 16))
        return CNR_E_ALIGN;
    cnr_status st = cnr_enter(ctx);
    if (st != CNR_OK) return st;
    ProductArgs p;
    p.a = a_codes;
    p.b = b_codes;
    p.a_scale = a_scale;
    p.b_scale = b_scale;
    p.row_bytes = cnr_block_row_bytes(k);
    p.a_stride = cnr_block_scale_stride(m, a_kind);
    p.b_stride = cnr_block_scale_stride(n, b_kind);
    p.m = (uint32_t)m;
    p.n = (uint32_t)n;
    p.blocks = (uint32_t)cnr_ceil_div(k, CNR_BLOCK);
    p.a_shift = a_kind == CNR_BLOCK_TILE ? 7 : 0;
    p.b_shift = b_kind == CNR_BLOCK_TILE ? 7 : 0;
    p.out = out;
    p.out_stride = out_stride;
    p.out_type = out_type;
    p.accumulate = accumulate ? 1 : 0;
    // A tile's offsets are 32 bits: 256 rows of less than 2^24 codes.
    if (m > 64 && p.row_bytes < 1u << 24)
        scale_type == CNR_SCALE_E8M0 ? tiled<8, 8>(p, scale_type, as_stream(stream)) : tiled<4, 8>(p, scale_type, as_stream(stream));
    else
        narrow<1, 1>(p, scale_type, as_stream(stream));
    return cnr_launch_status(ctx);
}

}  // extern "C"
