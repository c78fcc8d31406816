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
    narrow<1, 1>(p, scale_type, as_stream(stream));
    return cnr_launch_status(ctx);
}

}  // extern "C"
