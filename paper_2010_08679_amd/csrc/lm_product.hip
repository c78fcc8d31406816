// Products of blocked matrices: out[m][n] = sum over blocks of scale_a scale_b (codes_a . codes_b).
//
// Both operands have k along their rows, so a matrix instruction's operand is 32 bytes in a row of codes for each lane,
// whichever way a block is held.  Which of the block's 128 columns a lane's bytes are does not matter as long as
// both operands agree: a lane takes 16 bytes from 16 * (lane / 16) of row lane % 16 and 16 from 64 bytes further on, so
// that a load of all lanes reads 64 bytes in a row.
//
// Two ways to add up a block's 16 x 16 x 128 products:
//   8-bit instructions, scales of powers of two applied by them: the 16-bit outputs.  Exact products; of each eight that are added in
//     one step what lies 2^-14 or more below the largest is dropped.  Of the sum of the products' magnitudes that is (measured) 1e-5 with
//     normal codes, 1.4e-4 with codes of evenly spread exponents, 4.3e-4 where one of each eight is 2^14 times the others: less than the
//     half step of a bfloat16 (2^-8) or a half (2^-11), but not of a result that is small since products cancel.  Chosen for twice the rate;
//   bfloat16 instructions on the codes converted in registers, exact as well (4 of 8 bits of mantissa), their scales
//     of powers of two applied by the conversion, added up in fp32 (measured 1e-8 to 6e-8): float outputs.  Scales that would
//     take a code out of bfloat16's range multiply the block's sum instead (sum_any_range).
// Scales of any value multiply each block's sum before it is added to the total.
#include "lm_common.h"
#include "lm_scale_fetch.h"

#include <math.h>
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
    uint32_t splits;                // parts of the sum, each in its own workgroups
    float *partial;                 // [splits][m][partial_stride]
    uint64_t partial_stride;
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
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(p), hi = *reinterpret_cast<const i32x4 *>(p + 64);
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

// A scale's exponent goes into the 8-bit matrix instruction, or into the conversion to bfloat16 (see sum_any_range), and its fraction, from 1 to
// 2, multiplies the sum: neither leaves fp32's range unless the result does.  (A scale below 2^-126 counts as 0.)
__device__ __forceinline__ float fraction_of(float s) {
    const uint32_t b = __float_as_uint(s);
    return b & 0x7f800000u ? __uint_as_float((b & 0x807fffffu) | 0x3f800000u) : 0.0f;
}
__device__ __forceinline__ uint32_t exponent_of(float s) { return __float_as_uint(s) >> 23 & 255u; }

// Whether a sum that belongs to the matrix is infinite or NaN, for the whole wave.  A code that its scale takes out of bfloat16's range
// (2^128 and more) becomes infinite, and every sum that it enters infinite or NaN: nothing in the loop has to look for such
// scales.  Of the lane's rows i * MF + f and columns g the first `rows` and `columns` belong.
template <int MF, int NF>
__device__ __forceinline__ bool not_finite(const f32x4 (&acc)[MF][NF], uint32_t rows, uint32_t columns) {
    float none = 0.0f;
    if (__all((rows >= 4 * MF) & (columns >= NF))) {
#pragma unroll
        for (int f = 0; f < MF; ++f)
#pragma unroll
            for (int g = 0; g < NF; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) none = __builtin_fmaf(acc[f][g][i], 0.0f, none);
    } else {
#pragma unroll
        for (int f = 0; f < MF; ++f)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float row = 0.0f;
#pragma unroll
                for (uint32_t g = 0; g < NF; ++g) row = __builtin_fmaf(g < columns ? acc[f][g][i] : 0.0f, 0.0f, row);
                none += (uint32_t)(i * MF + f) < rows ? row : 0.0f;
            }
    }
    return __any(!(none == 0.0f));
}

// acc[f][g] = the sums over blocks [begin, end) of A's row_a[f] and B's row_b[g] (of each lane), with scales of any range: a block's codes are
// multiplied as they are and its sum takes fractions and exponents.  Operands come straight from memory, one fragment at a time.
template <int SCALE, int MF, int NF>
__device__ __forceinline__ void sum_any_range(const ProductArgs &p, const uint32_t (&row_a)[MF], const uint32_t (&row_b)[NF], uint32_t begin, uint32_t end,
                                              f32x4 (&acc)[MF][NF]) {
    typedef typename ScaleOf<SCALE>::type S;
    const uint32_t quarter = tid_x() % kWave / 16;
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (uint32_t kb = begin; kb < end; ++kb) {
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            const i32x8 x = load_codes(p.a + (uint64_t)row_a[f] * p.row_bytes + (uint64_t)kb * CNR_BLOCK + quarter * 16);
            const S sa = reinterpret_cast<const S *>(p.a_scale)[kb * p.a_stride + (row_a[f] >> p.a_shift)];
            float fraction[4];  // of the rows of the lane's sums
            int exponent[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const S s = __shfl(sa, (int)(quarter * 4 + i));
                if constexpr (SCALE == CNR_SCALE_E8M0) {
                    exponent[i] = (int)s - 254;
                } else {
                    exponent[i] = (int)exponent_of(s) - 254;
                    fraction[i] = fraction_of(s);
                }
            }
#pragma unroll
            for (int g = 0; g < NF; ++g) {
                const i32x8 y = load_codes(p.b + (uint64_t)row_b[g] * p.row_bytes + (uint64_t)kb * CNR_BLOCK + quarter * 16);
                const S sb = reinterpret_cast<const S *>(p.b_scale)[kb * p.b_stride + (row_b[g] >> p.b_shift)];
                f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(x, 127).part[i], widen(y, 127).part[i], d, 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);  // no more registers than the caller's own loop
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (SCALE == CNR_SCALE_E8M0)
                        acc[f][g][i] += __builtin_ldexpf(d[i], exponent[i] + (int)sb);
                    else
                        acc[f][g][i] += __builtin_ldexpf(d[i] * (fraction[i] * fraction_of(sb)), exponent[i] + (int)exponent_of(sb));
                }
                __builtin_amdgcn_sched_barrier(0);  // no more registers than the caller's own loop
            }
        }
    }
}

// ---- few rows or few tiles: operands straight from memory ---------------------------------------------------------
//
// A workgroup has 16 MF x 16 NF outputs; each of its waves takes a quarter of the columns, U blocks at a time so that enough loads are
// under way, straight into the matrix instructions' registers; they add up their sums in LDS at the end.  Bound by reading B: 1 x 131072 x 4096
// 86 us (6.2 TB/s), 1 x 32000 x 4096 22.4; with every fourth block to a wave a tenth more.
// (Waves on a SIMD: as many as the loop leaves room for, which sum_any_range would take from them.)
template <int SCALE, bool FULL, int MF, int NF, int U>
__global__ void __launch_bounds__(kBlock, U == 1 ? 6 : 4) narrow_kernel(const ProductArgs p) {
    typedef typename ScaleOf<SCALE>::type S;
    __shared__ f32x4 sums[kWavesPerBlock][MF * NF][kWave];
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint32_t quarter = lane / 16, m0 = wg_y() * 16 * MF, n0 = wg_x() * 16 * NF;
    // Rows beyond the matrix read its last one again.
    const uint8_t *a[MF], *b[NF];
    const S *sa[MF], *sb[NF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        uint32_t r = m0 + 16 * f + lane % 16;
        r = r < p.m ? r : p.m - 1;
        a[f] = p.a + (uint64_t)r * p.row_bytes + quarter * 16;
        sa[f] = reinterpret_cast<const S *>(p.a_scale) + (r >> p.a_shift);
    }
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        uint32_t r = n0 + 16 * f + lane % 16;
        r = r < p.n ? r : p.n - 1;
        b[f] = p.b + (uint64_t)r * p.row_bytes + quarter * 16;
        sb[f] = reinterpret_cast<const S *>(p.b_scale) + (r >> p.b_shift);
    }
    f32x4 acc[MF][NF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const uint32_t each = (p.blocks + kWavesPerBlock - 1) / kWavesPerBlock, begin = wave * each;
    const uint32_t end = begin + each < p.blocks ? begin + each : p.blocks;
    for (uint32_t first = begin; first < end; first += U) {
        i32x8 x[U][MF], y[U][NF];
        S s[U][MF], t[U][NF];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t kb = first + u;
            if (u && kb >= end) break;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                y[u][f] = load_codes(b[f] + (uint64_t)kb * CNR_BLOCK);
                t[u][f] = sb[f][kb * p.b_stride];
            }
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                x[u][f] = load_codes(a[f] + (uint64_t)kb * CNR_BLOCK);
                s[u][f] = sa[f][kb * p.a_stride];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u && first + u >= end) break;
            uint32_t ex[MF], ey[NF];
            float fy[NF], rows[MF][4];  // fractions; of A's those of the rows of the lane's sums
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                if constexpr (SCALE == CNR_SCALE_E8M0) {
                    ex[f] = s[u][f];
                } else {
                    ex[f] = exponent_of(s[u][f]);
                    const float fx = fraction_of(s[u][f]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) rows[f][i] = __shfl(fx, (int)(quarter * 4 + i));
                }
            }
#pragma unroll
            for (int g = 0; g < NF; ++g) {
                if constexpr (SCALE == CNR_SCALE_E8M0) {
                    ey[g] = t[u][g];
                } else {
                    ey[g] = exponent_of(t[u][g]);
                    fy[g] = fraction_of(t[u][g]);
                }
            }
            Wide wx[MF];
            if constexpr (FULL)
#pragma unroll
                for (int f = 0; f < MF; ++f) wx[f] = widen(x[u][f], ex[f]);
#pragma unroll
            for (int g = 0; g < NF; ++g) {
                Wide wy;
                if constexpr (FULL) wy = widen(y[u][g], ey[g]);
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    f32x4 d = SCALE == CNR_SCALE_F32 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[f][g];
                    if constexpr (FULL) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wx[f].part[i], wy.part[i], d, 0, 0, 0);
                    } else {
                        d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[u][f], y[u][g], d, 0, 0, 0, (int)ex[f], 0, (int)ey[g]);
                    }
                    if constexpr (SCALE == CNR_SCALE_F32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[f][g][i] = __builtin_fmaf(d[i], rows[f][i] * fy[g], acc[f][g][i]);
                    } else {
                        acc[f][g] = d;
                    }
                }
            }
        }
    }
    if constexpr (FULL) {
        if (not_finite(acc, 4 * MF, NF)) {
            uint32_t row_a[MF], row_b[NF];
#pragma unroll
            for (int f = 0; f < MF; ++f) row_a[f] = m0 + 16 * f + lane % 16 < p.m ? m0 + 16 * f + lane % 16 : p.m - 1;
#pragma unroll
            for (int f = 0; f < NF; ++f) row_b[f] = n0 + 16 * f + lane % 16 < p.n ? n0 + 16 * f + lane % 16 : p.n - 1;
            sum_any_range<SCALE, MF, NF>(p, row_a, row_b, begin, end, acc);
        }
    }
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) sums[wave][f * NF + g][lane] = acc[f][g];
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < MF * NF; ++i) {
        const uint32_t e = i * kBlock + tid_x(), m = e / (16 * NF), n = e % (16 * NF);
        if (m0 + m >= p.m || n0 + n >= p.n) continue;
        const uint32_t from = m % 16 / 4 * 16 + n % 16;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) v += sums[w][m / 16 * NF + n / 16][from][m % 4];
        store_out(p, m0 + m, n0 + n, v);
    }
}

template <bool FULL, int SCALE, int MF, int NF, int U>
void narrow(const ProductArgs &p, hipStream_t s) {
    const dim3 grid((unsigned)cnr_ceil_div(p.n, 16 * NF), (unsigned)cnr_ceil_div(p.m, 16 * MF));
    hipLaunchKernelGGL((narrow_kernel<SCALE, FULL, MF, NF, U>), grid, dim3(kBlock), 0, s, p);
}

// ---- many rows: tiles staged in LDS -----------------------------------------------------------------------------
//
// A workgroup of four waves has 32 MF x 32 NF outputs, each wave 16 MF x 16 NF, and walks along k a block of 128 at a time; the codes
// and scales of the next STAGES - 1 blocks travel from memory into LDS while this one's are multiplied.
//
// Fragment f of a wave holds rows MF * r + f of its part of A (r = lane % 16), and likewise of B: a lane's fragments are rows side by
// side, so that it finds their scales in one or two words (a byte of which each matrix instruction picks), and holds
// NF outputs side by side, which it stores in one go.
//
// LDS holds two rows of 128 codes to a line of 256 bytes, its sixteen pieces of 16 bytes permuted by r: sixteen lanes that
// read the same piece of their rows find it in sixteen different places, all banks in use.  Memory is read straight
// into LDS, where a wave's 64 pieces lie in order, so the permutation is in which piece a lane asks for.

// Base and size are the same for all lanes.
__device__ __forceinline__ i32x4 buffer_of(uint64_t base, uint64_t bytes) {
    i32x4 r;
    r[0] = (int)(uint32_t)base;
    r[1] = (int)((uint32_t)(base >> 32) & 0xffffu);
    r[2] = (int)(uint32_t)(bytes < 0xffffffffull ? bytes : 0xffffffffull);
    r[3] = 0x00027000;
    return r;
}

// 64 pieces of 16 (or 4) bytes, one for each lane, from memory to `lds` and on in lane order.  Written as instructions because the
// compiler, which cannot tell the stages of the LDS apart, would wait for them before every read of another;
// wait_for_loads() below does, once a block.  Each sets the place in LDS, M0, for itself.  (The compiler warns that it does not save
// a reserved register that a statement changes; what counts is that it does not take M0 for unchanged.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const i32x4 &buffer, uint32_t lds, uint32_t offset, uint32_t all) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(all) : "m0");
}
// The same of four bytes, or of `one`, which becomes the lowest of four.
__device__ __forceinline__ void load_bytes_to_lds(const i32x4 &buffer, uint32_t lds, uint32_t offset, uint32_t one) {
    asm volatile("s_mov_b32 m0, %0\n\ts_cmp_lg_u32 %3, 0\n\ts_cbranch_scc1 .Lone_byte_%=\n\t"
                 "buffer_load_dword %1, %2, 0 offen lds\n\ts_branch .Lloaded_%=\n"
                 ".Lone_byte_%=:\n\tbuffer_load_ubyte %1, %2, 0 offen lds\n.Lloaded_%=:" ::"s"(lds), "v"(offset), "s"(buffer), "s"(one)
                 : "m0", "scc");
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

// Scales of the F rows that a lane's fragments have, as exponents (a byte each) and, where they are of any value, as fractions.
template <int SCALE, int F>
struct Scales {
    uint32_t exponent[(F + 3) / 4];
    float fraction[SCALE == CNR_SCALE_F32 ? F : 1];
};

// One operand's scales on their way through LDS: for each four rows of the tile a word (E8M0) or four (F32), which rows' own scales fill.  A
// scale that 128 rows share is the lowest byte of each word, or one of the aligned four floats that it lies in.
template <int SCALE>
struct ScaleStream : ScaleFetch<SCALE == CNR_SCALE_E8M0 ? 1 : 4> {
    typedef ScaleFetch<SCALE == CNR_SCALE_E8M0 ? 1 : 4> Fetch;
    static constexpr uint32_t kBytes = kWave * 4 * (SCALE == CNR_SCALE_E8M0 ? 1 : 4);  // in LDS
    using Fetch::Fetch;
    __device__ __forceinline__ void fetch(uint32_t lds, bool on) {
        const i32x4 buffer = buffer_of(this->base, this->records);
        if constexpr (SCALE == CNR_SCALE_E8M0)
            load_bytes_to_lds(buffer, lds, this->offset(), this->tiles);
        else
            load_to_lds(buffer, lds, this->offset(), 0);
        this->advance(on);
    }
};
// The scales of rows [row, row + F) of the tile, in two parts: the words from where they were put, and what they say.  `pick`: which of
// its word's four all rows share (the wave's rows lie within one 128); 4: rows have their own.
template <int SCALE, int F>
struct ScaleWords {
    typedef typename std::conditional<SCALE == CNR_SCALE_E8M0, uint32_t, f32x4>::type Word;
    Word word[(F + 3) / 4];
    uint32_t within;  // first row of the word's four: 0, or 2 where F is 2
    __device__ __forceinline__ ScaleWords(const uint8_t *lds, uint32_t row) : within(row % 4) {
#pragma unroll
        for (int i = 0; i < (F + 3) / 4; ++i) word[i] = *reinterpret_cast<const Word *>(lds + (row / 4 + i) * sizeof(Word));
    }
    __device__ __forceinline__ Scales<SCALE, F> scales(uint32_t pick) const {
        Scales<SCALE, F> s;
#pragma unroll
        for (int i = 0; i < (F + 3) / 4; ++i) {
            if constexpr (SCALE == CNR_SCALE_E8M0) {
                const uint32_t own = 0u - pick / 4;
                const uint32_t order = (pick * 0x01010101u & ~own) | (0x03020100u + (F == 2 ? within * 0x0101u : 0u) & own);
                s.exponent[i] = __builtin_amdgcn_perm(0u, word[i], order);
            } else {
                const f32x4 w = word[i];
                const float one = pick & 2 ? (pick & 1 ? w[3] : w[2]) : (pick & 1 ? w[1] : w[0]);
                s.exponent[i] = 0;
#pragma unroll
                for (int j = 0; j < 4 && 4 * i + j < F; ++j) {
                    const float v = pick != 4 ? one : F == 2 && within ? w[(j + 2) % 4] : w[j];
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

template <typename T, int NF>
__device__ __forceinline__ void store_row(T *o, uint32_t n, uint32_t n_end, const float *v, bool accumulate) {
    if (n + NF <= n_end) {
        Pack<T, NF> w;
        if (accumulate) {
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
            if (n + j < n_end) o[j] = (T)(accumulate ? (float)o[j] + v[j] : v[j]);
    }
}

template <int SCALE, bool FULL, int WM, int WN, int MF, int NF, int STAGES>
__global__ void __launch_bounds__(WM * WN * kWave, 2) tile_kernel(const ProductArgs p) {
    constexpr uint32_t TM = WM * 16 * MF, TN = WN * 16 * NF;
    constexpr int LA = 2 * MF / WN, LB = 2 * NF / WM;  // loads of 1 KB that each wave sends for a block of A and of B
    static_assert(LA * WN == 2 * MF && LB * WM == 2 * NF, "whole loads");
    typedef ScaleStream<SCALE> Stream;
    constexpr uint32_t kB = TM * CNR_BLOCK, kScaleA = kB + TN * CNR_BLOCK, kScaleB = kScaleA + Stream::kBytes, kStage = kScaleB + Stream::kBytes;
    constexpr int kLoads = LA + LB + 1;
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
    const uint32_t m0 = (band * kBand + in_band % band_rows) * TM, n0 = in_band / band_rows * TN;
    // Blocks of this part of the sum.
    const uint32_t begin = (uint32_t)((uint64_t)p.blocks * split / p.splits), end = (uint32_t)((uint64_t)p.blocks * (split + 1) / p.splits);

    // Rows beyond the matrix read its last one again.
    const uint32_t rows_a = p.m - m0 < TM ? p.m - m0 : TM, rows_b = p.n - n0 < TN ? p.n - n0 : TN;
    const i32x4 buffer_a = buffer_of(reinterpret_cast<uint64_t>(p.a) + (uint64_t)m0 * p.row_bytes, (uint64_t)rows_a * p.row_bytes);
    const i32x4 buffer_b = buffer_of(reinterpret_cast<uint64_t>(p.b) + (uint64_t)n0 * p.row_bytes, (uint64_t)rows_b * p.row_bytes);
    uint32_t from_a[LA], from_b[LB];
#pragma unroll
    for (int j = 0; j < LA; ++j) {
        const uint32_t line = (wave * LA + j) * 4 + quarter, logical = (lane % 16) ^ (2 * line / MF % 16);
        const uint32_t row = 2 * line + logical / 8;
        from_a[j] = (row < rows_a ? row : rows_a - 1) * (uint32_t)p.row_bytes + logical % 8 * 16;
    }
#pragma unroll
    for (int j = 0; j < LB; ++j) {
        const uint32_t line = (wave * LB + j) * 4 + quarter, logical = (lane % 16) ^ (2 * line / NF % 16);
        const uint32_t row = 2 * line + logical / 8;
        from_b[j] = (row < rows_b ? row : rows_b - 1) * (uint32_t)p.row_bytes + logical % 8 * 16;
    }
    // Half of the waves bring the scales of A, half those of B: the same ones, so that all have as many loads under way.
    const bool brings_a = wave % 2 == 0;
    ScaleStream<SCALE> stream(brings_a ? p.a_scale : p.b_scale, brings_a ? p.a_stride : p.b_stride, p.blocks, brings_a ? p.a_shift : p.b_shift,
                              brings_a ? m0 : n0, brings_a ? TM : TN, lane, begin);
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // Load j of the wave's kLoads for block kb of this part of the sum into the stage at `to`; beyond its end the last block once more, which
    // nobody reads: the count of loads stays the same without a branch, which would end the compiler's sight of the loop.
    auto fetch = [&](uint32_t kb, uint32_t to, auto index) {
        constexpr int J = decltype(index)::value;
        const uint32_t at = (kb < end - 1 ? kb : end - 1) * CNR_BLOCK;
        if constexpr (J < LA)
            load_to_lds(buffer_a, lds_at + to + (wave * LA + J) * 1024, from_a[J], at);
        else if constexpr (J < LA + LB)
            load_to_lds(buffer_b, lds_at + to + kB + (wave * LB + J - LA) * 1024, from_b[J - LA], at);
        else
            stream.fetch(lds_at + to + (brings_a ? kScaleA : kScaleB), kb < end - 1);
    };
    // Which of its word's four a shared scale is, block by block (see ScaleWords), or 4 where rows have their own.
    struct Pick {
        uint32_t now, step, own;
        __device__ __forceinline__ Pick(uint32_t kb, uint32_t shift, uint64_t stride, uint32_t row) {
            const uint32_t at = row >> 7, last = (uint32_t)stride - 1;
            own = shift ? 0 : 4;
            step = shift && SCALE == CNR_SCALE_F32 ? (uint32_t)stride : 0;
            now = step ? kb * step + (at < last ? at : last) : 0;
        }
        __device__ __forceinline__ uint32_t operator()() const { return (now & 3) | own; }
        __device__ __forceinline__ void advance() { now += step; }
    };
    Pick pick_a(begin, p.a_shift, p.a_stride, m0 + wave_m), pick_b(begin, p.b_shift, p.b_stride, n0 + wave_n);
    auto words_a = [&](uint32_t at) { return ScaleWords<SCALE, MF>(lds + at + kScaleA, wave_m + r * MF); };
    auto words_b = [&](uint32_t at) { return ScaleWords<SCALE, NF>(lds + at + kScaleB, wave_n + r * NF); };

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
        const uint32_t at = ((quarter + 4 * (i % 2)) ^ r) * 16 ^ i / 2 * 128;
        piece_a[i / 2][i % 2] = (wave_m + r * MF) * CNR_BLOCK + at;
        piece_b[i / 2][i % 2] = kB + (wave_n + r * NF) * CNR_BLOCK + at;
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
    if constexpr (SCALE == CNR_SCALE_E8M0 && !FULL) {
        // A block's products go by quarters, each half of the wave's rows of A with each half of those of B, so that half of the
        // operands are in registers while the other half, or the next block's first, are on their way from LDS; a wave alone on its SIMD can
        // issue about four other instructions for each matrix instruction without holding it up, so loads go between
        // them.  The last quarter needs nothing more from this stage: before it all waves meet, in it the stage is filled
        // again.
        constexpr int HM = MF / 2, HN = NF / 2, kQuarter = HM * HN;
        unrolled<STAGES>([&](auto i) { unrolled<kLoads>([&](auto j) { fetch(begin + decltype(i)::value, decltype(i)::value * kStage, j); }); });
        wait_for_loads<(STAGES - 1) * kLoads>();
        barrier();
        Scales<SCALE, MF> sa = words_a(0).scales(pick_a());
        Scales<SCALE, NF> sb = words_b(0).scales(pick_b());
        i32x8 x[2][HM], y[2][HN];
#pragma unroll
        for (int f = 0; f < HM; ++f) x[0][f] = fragment(piece_a, f);
#pragma unroll
        for (int g = 0; g < HN; ++g) y[0][g] = fragment(piece_b, g);
        // One quarter; with its i-th product goes beside(i).
        auto quarter_of = [&](auto half_a, auto half_b, const auto &beside) {
            constexpr int A = decltype(half_a)::value, B = decltype(half_b)::value;
            unrolled<kQuarter>([&](auto at) {
                constexpr int F = decltype(at)::value % HM, G = decltype(at)::value / HM, MA = A * HM + F, NB = B * HN + G;
                acc[MA][NB] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[A][F], y[B][G], acc[MA][NB], 0, 0, MA % 4, (int)sa.exponent[MA / 4],
                                                                               NB % 4, (int)sb.exponent[NB / 4]);
                beside(at);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        uint32_t stage = 0;  // where it begins in LDS
        for (uint32_t kb = begin; kb < end; ++kb) {
            const uint32_t next = stage + kStage < STAGES * kStage ? stage + kStage : 0;
            quarter_of(Index<0>(), Index<0>(), [&](auto at) {
                share(at, Index<kQuarter>(), Index<HN>(), [&](auto g) { y[1][decltype(g)::value] = fragment(piece_b, HN + decltype(g)::value); });
            });
            quarter_of(Index<0>(), Index<1>(), [&](auto at) {
                share(at, Index<kQuarter>(), Index<HM>(), [&](auto f) { x[1][decltype(f)::value] = fragment(piece_a, HM + decltype(f)::value); });
            });
            quarter_of(Index<1>(), Index<0>(), [&](auto) {});
            wait_for_loads<(STAGES - 2) * kLoads>();
            barrier();
            move_pieces(next - stage);
            const ScaleWords<SCALE, MF> next_a = words_a(next);
            const ScaleWords<SCALE, NF> next_b = words_b(next);
            quarter_of(Index<1>(), Index<1>(), [&](auto at) {
                share(at, Index<kQuarter>(), Index<HM + HN>(), [&](auto j) {
                    constexpr int J = decltype(j)::value;
                    if constexpr (J < HM)
                        x[0][J] = fragment(piece_a, J);
                    else
                        y[0][J - HM] = fragment(piece_b, J - HM);
                });
                share(at, Index<kQuarter>(), Index<kLoads>(), [&](auto j) { fetch(kb + STAGES, stage, j); });
            });
            pick_a.advance();
            pick_b.advance();
            sa = next_a.scales(pick_a());
            sb = next_b.scales(pick_b());
            stage = next;
        }
    } else {
        // Operands that are converted, or sums that are scaled, keep the ordinary units busy next to the matrix units: a plain order, all of
        // A's fragments, then B's one ahead.
        unrolled<STAGES - 1>([&](auto i) { unrolled<kLoads>([&](auto j) { fetch(begin + decltype(i)::value, decltype(i)::value * kStage, j); }); });
        wait_for_loads<(STAGES - 2) * kLoads>();
        barrier();
        uint32_t stage = 0;
        for (uint32_t kb = begin; kb < end; ++kb) {
            unrolled<kLoads>([&](auto j) { fetch(kb + STAGES - 1, stage ? stage - kStage : (STAGES - 1) * kStage, j); });
            const Scales<SCALE, MF> sa = words_a(stage).scales(pick_a());
            const Scales<SCALE, NF> sb = words_b(stage).scales(pick_b());
            float rows[SCALE == CNR_SCALE_F32 ? MF : 1][4];  // fractions of the rows of the lane's sums
            if constexpr (SCALE == CNR_SCALE_F32) {
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
                f32x4 d[MF];
#pragma unroll
                for (int f = 0; f < MF; ++f) d[f] = SCALE == CNR_SCALE_F32 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[f][G];
                if constexpr (FULL) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int f = 0; f < MF; ++f) d[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[f].part[i], wy.part[i], d[f], 0, 0, 0);
                } else {
                    unrolled<MF>([&](auto f) {
                        constexpr int F = decltype(f)::value;
                        d[F] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[F], y, d[F], 0, 0, F % 4, (int)sa.exponent[F / 4], G % 4, (int)sb.exponent[G / 4]);
                    });
                }
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    if constexpr (SCALE == CNR_SCALE_F32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[f][G][i] = __builtin_fmaf(d[f][i], rows[f][i] * sb.fraction[G], acc[f][G][i]);
                    } else {
                        acc[f][G] = d[f];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            const uint32_t next = stage + kStage < STAGES * kStage ? stage + kStage : 0;
            move_pieces(next - stage);
            stage = next;
            pick_a.advance();
            pick_b.advance();
            wait_for_loads<(STAGES - 2) * kLoads>();
            barrier();
        }
        if constexpr (FULL) {
            const uint32_t first_m = m0 + wave_m + quarter * 4 * MF, first_n = n0 + wave_n + r * NF;
            if (not_finite(acc, first_m < p.m ? p.m - first_m : 0, first_n < p.n ? p.n - first_n : 0)) {
                uint32_t row_a[MF], row_b[NF];
#pragma unroll
                for (int f = 0; f < MF; ++f) row_a[f] = m0 + wave_m + r * MF + f < p.m ? m0 + wave_m + r * MF + f : p.m - 1;
#pragma unroll
                for (int f = 0; f < NF; ++f) row_b[f] = n0 + wave_n + r * NF + f < p.n ? n0 + wave_n + r * NF + f : p.n - 1;
                sum_any_range<SCALE, MF, NF>(p, row_a, row_b, begin, end, acc);
            }
        }
    }
    wait_for_loads<0>();

    const uint32_t m = m0 + wave_m + quarter * 4 * MF, n = n0 + wave_n + r * NF;
    auto write = [&](auto *out, uint64_t stride, bool accumulate) {
        typedef typename std::remove_pointer<decltype(out)>::type T;
        T *o = out + (uint64_t)m * stride + n;
        if (m0 + wave_m + 16 * MF <= p.m && n0 + wave_n + 16 * NF <= p.n && !accumulate) {
#pragma unroll
            for (int i = 0; i < 4 * MF; ++i) {
                Pack<T, NF> w;
#pragma unroll
                for (int g = 0; g < NF; ++g) w.v[g] = (T)acc[i % MF][g][i / MF];
                *reinterpret_cast<Pack<T, NF> *>(o) = w;
                o += stride;
            }
        } else {
            // What is added to is read for eight rows at once: one row after the other would wait for memory each time
            // (1000 x 1111 x 1100 onto half 11.6 -> 9.1 us).  Rows and columns beyond the matrix read its last ones.
            const uint32_t rows_left = m < p.m ? p.m - m : 0;
            const bool whole = n + NF <= p.n;
#pragma unroll
            for (int first = 0; first < 4 * MF; first += 8) {
                Pack<T, NF> old[8];
                if (accumulate && rows_left && n < p.n) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const uint32_t down = (uint32_t)(first + u) < rows_left ? (uint32_t)(first + u) : rows_left - 1;
                        const T *from = o + (uint64_t)down * stride;
                        if (whole) {
                            old[u] = *reinterpret_cast<const Pack<T, NF> *>(from);
                        } else {
#pragma unroll
                            for (int g = 0; g < NF; ++g) old[u].v[g] = from[n + g < p.n ? g : p.n - 1 - n];
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int i = first + u;
                    if ((uint32_t)i >= rows_left) continue;
                    float v[NF];
#pragma unroll
                    for (int g = 0; g < NF; ++g) v[g] = accumulate ? (float)old[u].v[g] + acc[i % MF][g][i / MF] : acc[i % MF][g][i / MF];
                    store_row<T, NF>(o + (uint64_t)i * stride, n, p.n, v, false);
                }
            }
        }
    };
    if (p.splits > 1)
        write(p.partial + (uint64_t)split * p.m * p.partial_stride, p.partial_stride, false);
    else if constexpr (FULL)
        write(reinterpret_cast<float *>(p.out), p.out_stride, p.accumulate);
    else if (p.out_type == CNR_FLOAT_BF16)
        write(reinterpret_cast<__bf16 *>(p.out), p.out_stride, p.accumulate);
    else
        write(reinterpret_cast<_Float16 *>(p.out), p.out_stride, p.accumulate);
}

// The parts of sums that were split, added up in order: four outputs of a row to a thread.
template <typename T>
__global__ void __launch_bounds__(kBlock) join_kernel(const ProductArgs p) {
    const uint32_t across = (uint32_t)(p.partial_stride / 4);
    const uint64_t at = (uint64_t)wg_x() * kBlock + tid_x();
    if (at >= (uint64_t)p.m * across) return;
    const uint32_t m = (uint32_t)(at / across), n = (uint32_t)(at % across) * 4;
    const float *from = p.partial + (uint64_t)m * p.partial_stride + n;
    f32x4 sum = *reinterpret_cast<const f32x4 *>(from);
    for (uint32_t s = 1; s < p.splits; ++s) sum += *reinterpret_cast<const f32x4 *>(from + (uint64_t)s * p.m * p.partial_stride);
    const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    store_row<T, 4>(reinterpret_cast<T *>(p.out) + m * p.out_stride + n, n, p.n, v, p.accumulate);
}

template <bool FULL, int SCALE, int WM, int WN, int MF, int NF, int STAGES>
void tiled(const ProductArgs &p, hipStream_t s) {
    const dim3 grid((unsigned)(cnr_ceil_div(p.m, 16 * WM * MF) * cnr_ceil_div(p.n, 16 * WN * NF) * p.splits));
    hipLaunchKernelGGL((tile_kernel<SCALE, FULL, WM, WN, MF, NF, STAGES>), grid, dim3(WM * WN * kWave), 0, s, p);
    if (p.splits > 1) {
        const dim3 join((unsigned)cnr_ceil_div((uint64_t)p.m * (p.partial_stride / 4), kBlock));
        if (FULL)
            hipLaunchKernelGGL((join_kernel<float>), join, dim3(kBlock), 0, s, p);
        else if (p.out_type == CNR_FLOAT_BF16)
            hipLaunchKernelGGL((join_kernel<__bf16>), join, dim3(kBlock), 0, s, p);
        else
            hipLaunchKernelGGL((join_kernel<_Float16>), join, dim3(kBlock), 0, s, p);
    }
}

// ---- which kernel ---------------------------------------------------------------------------------------------------
//
// Each kernel's time for a product is estimated and the shortest taken.  A workgroup's time for a block of 128 columns, by how
// many share a compute unit, in us; measured with 8-bit instructions; conversion or scaled sums take 1.7 times as long (1.5 to 1.85).
// 8192^3 with each (bfloat16, powers of two): 401, 593, 492, 627 and 837 us; 2048^3 25.8, 13.4, 13.4, 15.4 and 19.0; 512 x 4096 x 4096
// 42.9, 19.2, 23.1, 21.6 and 17.0; 64 x 8192 x 8192 82.6, 31.4, 41.7, 38.1 and 18.4 (15.5 in two parts), the narrow kernel 59.9.
struct Tiles {
    uint32_t rows, columns, resident;  // outputs of a workgroup; workgroups on a compute unit
    float block[3];
};
constexpr Tiles kTiles[] = {
    {256, 256, 1, {1.65f, 0.0f, 0.0f}},   // eight waves of 128 x 64, 8-bit instructions only
    {128, 128, 1, {0.54f, 0.0f, 0.0f}},   // eight waves of 64 x 32, four stages: one tile for each compute unit
    {128, 128, 2, {0.65f, 1.0f, 0.0f}},   // four waves of 64 x 64
    {64, 128, 3, {0.55f, 0.68f, 0.96f}},  // four waves of 32 x 64
    {64, 64, 2, {0.28f, 0.42f, 0.0f}},    // four waves of 32 x 32, four stages
};
constexpr int kNarrow = (int)(sizeof(kTiles) / sizeof(kTiles[0]));
constexpr uint32_t kMaxSplits = 8, kMinBlocks = 4;  // parts of a sum, blocks of a part

struct Plan {
    int kernel;  // of kTiles, or kNarrow
    uint32_t splits;
};
Plan plan_of(const cnr_ctx *ctx, uint64_t m, uint64_t n, uint64_t k, bool plain, bool may_split) {
    const float units = ctx ? (float)ctx->n_cu : 256.0f, blocks = (float)cnr_ceil_div(k, CNR_BLOCK), outputs = (float)m * (float)n;
    const float memory = 3.5f + ((float)m * k + (float)n * k + 2.0f * outputs) / 4.7e6f;  // us at what codes are read at
    // The narrow kernel reads B once for each sixteen rows of A; a lone workgroup takes 0.115 us a block.
    Plan best = {kNarrow, 1};
    const float passes = (float)cnr_ceil_div(m, 16);
    const float read = passes * (float)(n < 16 ? 16 : n) * k / 4.2e6f, alone = 0.115f * blocks;
    float least = 3.5f + (read > alone ? read : alone);
    if (k == 0 || cnr_block_row_bytes(k) >= 1u << 24) return best;  // tiles have a block at least; a tile's offsets are 32 bits: 256 rows of less than 2^24 codes
    for (int i = 0; i < kNarrow; ++i) {
        if (i == 0 && !plain) continue;
        const Tiles &t = kTiles[i];
        const float tiles = (float)cnr_ceil_div(m, t.rows) * (float)cnr_ceil_div(n, t.columns), slow = plain ? 1.0f : 1.7f;
        for (uint32_t s = 1; s == 1 || (may_split && s <= kMaxSplits && blocks >= (float)(s * kMinBlocks)); s *= 2) {
            const float groups = tiles * (float)s;
            if (groups * (float)(i < 2 ? 512 : 256) >= 4.2e9f) continue;  // grids count threads in 32 bits
            const float round = units * (float)t.resident, rounds = floorf(groups / round);
            const float rest = ceilf((groups - rounds * round) / units);  // workgroups on a unit in the last round
            float time = ceilf(blocks / (float)s) * slow * (rounds * t.block[t.resident - 1] + (rest > 0.0f ? t.block[(int)rest - 1] : 0.0f));
            time += 3.5f + 1.5f * (rounds + (rest > 0.0f ? 1.0f : 0.0f));
            time = (time > memory ? time : memory) + 0.25f * (time < memory ? time : memory);  // one does not quite hide the other
            if (s > 1) time += 3.5f + (float)(s + 1) * outputs * 4.0f / 3e6f;  // writing the parts, and joining them
            if (time < least) {
                least = time;
                best = {i, s};
            }
        }
    }
    return best;
}
uint64_t partial_bytes(uint64_t m, uint64_t n, uint32_t splits) {
    return splits > 1 ? (uint64_t)splits * m * (cnr_ceil_div(n, 4) * 4) * sizeof(float) : 0;
}

constexpr uint64_t kNarrowRows = 1u << 19, kNarrowColumns = 1u << 27;

template <bool FULL, int SCALE>
void narrow_part(const ProductArgs &p, hipStream_t s) {
    // Two fragments of B to a wave where that still gives every SIMD a wave: A's codes are read half as often (16 x 32000 x 4096 to bfloat16 37 -> 30 us
    // when it was chosen, 24.6 now).
    if (p.m > 1 && p.n >= 16384)
        narrow<FULL, SCALE, 1, 2, 1>(p, s);
    else
        narrow<FULL, SCALE, 1, 1, 4>(p, s);
}

template <bool FULL, int SCALE>
void launch(const ProductArgs &p, const Plan &plan, hipStream_t s) {
    if constexpr (!FULL && SCALE == CNR_SCALE_E8M0) {
        if (plan.kernel == 0) return tiled<FULL, SCALE, 2, 4, 8, 4, 2>(p, s);
    }
    switch (plan.kernel) {
        case 1: return tiled<FULL, SCALE, 2, 4, 4, 2, 4>(p, s);
        case 2: return tiled<FULL, SCALE, 2, 2, 4, 4, 2>(p, s);
        case 3: return tiled<FULL, SCALE, 2, 2, 2, 4, 2>(p, s);
        case 4: return tiled<FULL, SCALE, 2, 2, 2, 2, 4>(p, s);
    }
    // A grid has fewer than 2^16 workgroups one below the other and 2^32 threads side by side: larger products go by parts, each from a whole tile's scale on.
    for (uint64_t n0 = 0; n0 < p.n; n0 += kNarrowColumns) {
        for (uint64_t m0 = 0; m0 < p.m; m0 += kNarrowRows) {
            ProductArgs q = p;
            q.m = (uint32_t)(p.m - m0 < kNarrowRows ? p.m - m0 : kNarrowRows);
            q.n = (uint32_t)(p.n - n0 < kNarrowColumns ? p.n - n0 : kNarrowColumns);
            q.a += m0 * p.row_bytes;
            q.b += n0 * p.row_bytes;
            q.a_scale = reinterpret_cast<const typename ScaleOf<SCALE>::type *>(p.a_scale) + (m0 >> p.a_shift);
            q.b_scale = reinterpret_cast<const typename ScaleOf<SCALE>::type *>(p.b_scale) + (n0 >> p.b_shift);
            q.out = reinterpret_cast<uint8_t *>(p.out) + (m0 * p.out_stride + n0) * cnr_float_bytes((cnr_float_type)p.out_type);
            narrow_part<FULL, SCALE>(q, s);
        }
    }
}

}  // namespace

extern "C" {

size_t cnr_block_product_workspace_bytes(const cnr_ctx *ctx, uint64_t m, uint64_t n, uint64_t k) {
    if (m > CNR_LM_MAX_SIZE || n > CNR_LM_MAX_SIZE || k > CNR_LM_MAX_SIZE) return 0;
    const uint64_t a = partial_bytes(m, n, plan_of(ctx, m, n, k, true, true).splits), b = partial_bytes(m, n, plan_of(ctx, m, n, k, false, true).splits);
    return (size_t)(a > b ? a : b);
}

cnr_status cnr_block_product(cnr_ctx *ctx, const uint8_t *a_codes, const void *a_scale, cnr_block_kind a_kind,
                             uint64_t m, const uint8_t *b_codes, const void *b_scale, cnr_block_kind b_kind,
                             uint64_t n, uint64_t k, cnr_scale_type scale_type, void *out, cnr_float_type out_type,
                             uint64_t out_stride, int accumulate, void *workspace, void *stream) {
    if (!ctx || !cnr_valid_float_type(out_type) || (a_kind != CNR_BLOCK_ROW && a_kind != CNR_BLOCK_TILE) ||
        (b_kind != CNR_BLOCK_ROW && b_kind != CNR_BLOCK_TILE) || (scale_type != CNR_SCALE_E8M0 && scale_type != CNR_SCALE_F32) || out_stride < n)
        return CNR_E_INVALID;
    if (m > CNR_LM_MAX_SIZE || n > CNR_LM_MAX_SIZE || k > CNR_LM_MAX_SIZE) return CNR_E_TOO_LARGE;
    if (m == 0 || n == 0 || (k == 0 && accumulate)) return CNR_OK;
    // more outputs or codes than a GPU holds
    if (cnr_ceil_div(m, 128) * cnr_ceil_div(n, 128) >= 1u << 24 || (k >= (1u << 24) - CNR_BLOCK && m > 1u << 19)) return CNR_E_TOO_LARGE;
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
    const bool full = out_type == CNR_FLOAT_F32, powers = scale_type == CNR_SCALE_E8M0;
    const Plan plan = plan_of(ctx, m, n, k, powers && !full, workspace != nullptr);
    p.splits = plan.splits;
    p.partial = reinterpret_cast<float *>(workspace);
    p.partial_stride = cnr_ceil_div(n, 4) * 4;
    hipStream_t to = as_stream(stream);
    if (full)
        powers ? launch<true, CNR_SCALE_E8M0>(p, plan, to) : launch<true, CNR_SCALE_F32>(p, plan, to);
    else
        powers ? launch<false, CNR_SCALE_E8M0>(p, plan, to) : launch<false, CNR_SCALE_F32>(p, plan, to);
    return cnr_launch_status(ctx);
}

}  // extern "C"
