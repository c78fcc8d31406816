// Block quantization: a matrix, and its transpose, to e4m3 codes with a scale for each block of 128.
//
// Bound by memory: x is read once, codes written once for each direction.  A workgroup takes 128 x 128 elements, so that both
// directions' blocks lie within it: each thread holds 8 rows x 8 columns in registers (16 lanes across the
// tile, so that a wave reads four rows' 128 columns in one instruction), the maxima of a row's blocks are
// combined across those 16 lanes by DPP, those of a column's across the 4 rows of lanes and the 4 waves.  Codes
// of the transpose pass through LDS, so that whole lines of 128 bytes are stored in both directions.  8192 x 4096 bfloat16 both ways 23 us
// (5.9 TB/s), 1 M x 128 floats 117 (5.5); a few tiles take 3.5, a load's and a store's latency.
#include "lm_common.h"

namespace {

constexpr int kTile = (int)CNR_BLOCK;
constexpr int kPer = 8;                 // rows and columns of the tile that a thread holds
constexpr int kAcross = kTile / kPer;   // lanes across a row of the tile
constexpr int kPitch = kTile + 16;      // bytes from one column's codes to the next in LDS: 16-byte reads start in different banks

struct QuantizeArgs {
    const void *x;
    uint64_t stride;
    uint32_t n_rows, dim;
    uint32_t tiles_across;
    uint8_t *codes, *codes_t;
    void *scale, *scale_t;
    uint64_t row_bytes, row_bytes_t;        // of codes and codes_t
    uint64_t scale_stride, scale_stride_t;
};

// Magnitudes of elements by their bits, which order like the values: a word holds two of a 16-bit type or one float.
template <int TYPE>
struct Magnitude {
    static constexpr int kIn = TYPE == CNR_FLOAT_F32 ? 1 : 2;  // elements in a word
    static constexpr uint32_t kInfinite = TYPE == CNR_FLOAT_F32 ? 0x7f800000u : TYPE == CNR_FLOAT_BF16 ? 0x7f80u : 0x7c00u;
    static __device__ __forceinline__ uint32_t of(uint32_t w) { return w & (kIn == 1 ? 0x7fffffffu : 0x7fff7fffu); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        if constexpr (kIn == 1) return a > b ? a : b;
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    static __device__ __forceinline__ uint32_t largest(uint32_t w) { return kIn == 1 ? w : (w & 0xffffu) > (w >> 16) ? w & 0xffffu : w >> 16; }
    static __device__ __forceinline__ uint32_t part(uint32_t w, int i) { return kIn == 1 ? w : i ? w >> 16 : w & 0xffffu; }
    static __device__ __forceinline__ bool odd(uint32_t w) { return largest(w) >= kInfinite; }  // one that is infinite or NaN
    static __device__ __forceinline__ uint32_t without_odd(uint32_t w) {
        if constexpr (kIn == 1) return w < kInfinite ? w : 0u;
        return ((w & 0xffffu) < kInfinite ? w & 0xffffu : 0u) | ((w >> 16) < kInfinite ? w & 0xffff0000u : 0u);
    }
    static __device__ __forceinline__ uint32_t as_float(uint32_t m) {  // bits
        if constexpr (TYPE == CNR_FLOAT_F32) return m;
        if constexpr (TYPE == CNR_FLOAT_BF16) return m << 16;
        return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)m));
    }
};

template <typename M>
__device__ __forceinline__ uint32_t max_across(uint32_t m) {  // of the 16 lanes that hold a row
    m = M::larger(m, (uint32_t)dpp_i<0xB1>((int)m));
    m = M::larger(m, (uint32_t)dpp_i<0x4E>((int)m));
    m = M::larger(m, (uint32_t)dpp_i<0x141>((int)m));
    return M::larger(m, (uint32_t)dpp_i<0x140>((int)m));
}
template <typename M>
__device__ __forceinline__ uint32_t max_down(uint32_t m) {  // of the wave's lanes that hold the same columns
    m = M::larger(m, (uint32_t)__shfl_xor((int)m, 16));
    return M::larger(m, (uint32_t)__shfl_xor((int)m, 32));
}

// A block's scale from the bits of its largest magnitude.  Powers of two: 448 = 1.75 * 2^8, so the exponent is the magnitude's less
// 8, one more where its fraction is above 1.75.  They divide exactly, a transposed tile's codes are the tile's, and
// the matrix instructions take them as they are.
struct Scale {
    float value;              // the scale
    uint8_t byte;             // as e8m0
    float up, divisor, inv;   // for scales of any value: 1 or 2^64, that times the scale, and one divided by that
    float below, above;       // factors a little below and above 1 / scale
};
template <int SCALE>
__device__ __forceinline__ Scale scale_of(uint32_t amax) {
    Scale s;
    if (SCALE == CNR_SCALE_E8M0) {
        int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
        e = e < 1 ? 1 : e;
        e = amax ? e : 127;
        s.byte = (uint8_t)e;
        s.value = __uint_as_float((uint32_t)e << 23);
    } else {
        // Small blocks are scaled up by 2^64, so that no remainder leaves fp32's range.  amax / 448 correctly rounded is amax / 7 by its
        // rounded reciprocal and one correction with the exact remainder, times a power of two.
        s.up = amax < 0x21000000u ? 0x1p64f : 1.0f;  // amax below 2^-61
        const float m = __uint_as_float(amax) * s.up, seventh = 1.0f / 7.0f, near = m * seventh;
        const float v = __builtin_fmaf(__builtin_fmaf(-near, 7.0f, m), seventh, near) * 0x1p-6f;
        const float least = 0x1p-126f * s.up;
        s.divisor = amax ? (v < least ? least : v) : s.up;
        s.value = s.divisor * (s.up == 1.0f ? 1.0f : 0x1p-64f);
        s.inv = __builtin_amdgcn_rcpf(s.divisor);  // within 2^-23; the quotient is corrected
        s.below = s.inv * s.up * (1.0f - 0x1p-21f);  // the divisor is 2^-62 at least, so that nothing leaves fp32's range
        s.above = s.inv * s.up * (1.0f + 0x1p-21f);
    }
    return s;
}

// The quotient whose e4m3 rounding is that of x / scale exactly, for scales of any value: the rounded quotient could fall on the
// middle between two codes where the true one lies beside it, so a quotient that is not exact gets its last bit set after rounding towards zero (a
// middle has that bit clear).  The remainder decides both.
__device__ __forceinline__ float quotient(float x, const Scale &s) {
    const float d = s.divisor, inv = s.inv;
    x *= s.up;
    float q = x * inv;
    q = __builtin_fmaf(__builtin_fmaf(-q, d, x), inv, q);
    const float rest = __builtin_fmaf(-q, d, x);
    uint32_t b = __float_as_uint(q);
    b -= (__float_as_uint(rest) ^ b) >> 31;  // |q| was rounded up: the remainder's sign is not q's
    return __builtin_copysignf(__uint_as_float(rest != 0.0f ? b | 1u : __float_as_uint(q)), x);  // -0 became 0
}

// The codes of two elements, in the half HIGH of a word.  Scales of powers of two divide in the conversion itself: its results are the
// definition's for every 16-bit input, and floats, at scales from 2^-126 to 2^120.
typedef short s16x2 __attribute__((ext_vector_type(2)));
template <int TYPE, bool HIGH>
__device__ __forceinline__ s16x2 encode_pair(s16x2 word, uint32_t pair, float scale) {
    if constexpr (TYPE == CNR_FLOAT_BF16) {
        typedef __bf16 pair_of __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(word, __builtin_bit_cast(pair_of, pair), scale, HIGH);
    } else {
        typedef _Float16 pair_of __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(word, __builtin_bit_cast(pair_of, pair), scale, HIGH);
    }
}
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// The codes of eight elements, given as words of them.
//
// Floats and scales of any value: products with a factor below 1 / scale and with one above it have the quotient between them, so that codes on which
// both agree are its; only where they do not, a middle lying within 2^-20 of a quotient (one wave in a hundred), and where there are
// infinities (`odd`) are quotients computed.  8192 x 4096 both ways 40.6 -> 35.5 us, 5760 x 760 11.9 -> 10.0.  The 16-bit types always compute
// them: their few values lie near a middle so often that most waves would do both (bfloat16 38.2 and 45.6 us, half 43.2 and 42.9).
template <int TYPE, int SCALE>
__device__ __forceinline__ u32x2 encode8(const uint32_t *w, const Scale &s, bool odd) {
    u32x2 codes;
    if constexpr (SCALE == CNR_SCALE_F32) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (TYPE == CNR_FLOAT_F32)
                x[e] = __uint_as_float(w[e]);
            else
                x[e] = Element<TYPE>::wide(__builtin_bit_cast(typename Element<TYPE>::type, (uint16_t)(w[e / 2] >> (16 * (e % 2)))));
        }
        if constexpr (TYPE == CNR_FLOAT_F32) {
            u32x2 other;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                codes[i] = four_codes(x[4 * i] * s.below, x[4 * i + 1] * s.below, x[4 * i + 2] * s.below, x[4 * i + 3] * s.below);
                other[i] = four_codes(x[4 * i] * s.above, x[4 * i + 1] * s.above, x[4 * i + 2] * s.above, x[4 * i + 3] * s.above);
            }
            if (!__any(odd || ((codes[0] ^ other[0]) | (codes[1] ^ other[1])) != 0u)) return codes;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) codes[i] = four_codes(quotient(x[4 * i], s), quotient(x[4 * i + 1], s), quotient(x[4 * i + 2], s), quotient(x[4 * i + 3], s));
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2 word = {0, 0};
            if constexpr (TYPE == CNR_FLOAT_F32) {
                word = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(word, __uint_as_float(w[4 * i]), __uint_as_float(w[4 * i + 1]), s.value, false);
                word = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(word, __uint_as_float(w[4 * i + 2]), __uint_as_float(w[4 * i + 3]), s.value, true);
            } else {
                word = encode_pair<TYPE, false>(word, w[2 * i], s.value);
                word = encode_pair<TYPE, true>(word, w[2 * i + 1], s.value);
            }
            codes[i] = __builtin_bit_cast(uint32_t, word);
        }
    }
    return codes;
}
template <int SCALE>
__device__ __forceinline__ void store_scale(void *to, uint64_t at, const Scale &s) {
    if (SCALE == CNR_SCALE_E8M0)
        reinterpret_cast<uint8_t *>(to)[at] = s.byte;
    else
        reinterpret_cast<float *>(to)[at] = s.value;
}

// grid.x: tiles, those of one row of tiles side by side.
template <int TYPE, int KIND, int SCALE, bool BOTH>
__global__ void __launch_bounds__(kBlock) quantize_kernel(const QuantizeArgs a) {
    typedef typename Element<TYPE>::type T;
    typedef Magnitude<TYPE> M;
    constexpr int kWords = kPer / M::kIn;  // of a thread's part of a row
    __shared__ __align__(16) uint8_t turned[BOTH ? kTile * kPitch : 16];
    __shared__ __align__(16) uint32_t largest[kWavesPerBlock][kTile / M::kIn];
    const uint32_t tile_row = wg_x() / a.tiles_across, tile_col = wg_x() % a.tiles_across;
    const uint32_t t = tid_x(), wave = t / kWave;
    const uint32_t r0 = tile_row * kTile + t / kAcross * kPer, c0 = tile_col * kTile + t % kAcross * kPer;
    const T *x = reinterpret_cast<const T *>(a.x);

    // Rows beyond the matrix read its last one, and count as zeros.
    uint32_t w[kPer][kWords];
    const uint32_t last = a.n_rows - 1;
    if (c0 + kPer <= a.dim) {
#pragma unroll
        for (int r = 0; r < kPer; ++r)
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const u32x4 got = load16(x + (uint64_t)(r0 + r < last ? r0 + r : last) * a.stride + c0 + i * (16 / sizeof(T)));
#pragma unroll
                for (int j = 0; j < 4; ++j) w[r][4 * i + j] = got[j];
            }
    } else {
#pragma unroll
        for (int r = 0; r < kPer; ++r) {
            T part[kPer];
            const T *from = x + (uint64_t)(r0 + r < last ? r0 + r : last) * a.stride;
#pragma unroll
            for (int c = 0; c < kPer; ++c) part[c] = c0 + c < a.dim ? from[c0 + c] : (T)0.0f;
            __builtin_memcpy(w[r], part, sizeof(part));
        }
    }
    if (tile_row * kTile + kTile > a.n_rows) {
#pragma unroll
        for (int r = 0; r < kPer; ++r)
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[r][i] = r0 + r <= last ? w[r][i] : 0u;
    }

    // Magnitudes, and the largest of each column; infinities and NaN, which do not count, are rare.
    uint32_t mag[kPer][kWords], down[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        down[i] = mag[0][i] = M::of(w[0][i]);
#pragma unroll
        for (int r = 1; r < kPer; ++r) {
            mag[r][i] = M::of(w[r][i]);
            down[i] = M::larger(down[i], mag[r][i]);
        }
    }
    uint32_t all = down[0];
#pragma unroll
    for (int i = 1; i < kWords; ++i) all = M::larger(all, down[i]);
    const bool odd = __any(M::odd(all));
    if (odd) {
        all = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            down[i] = 0;
#pragma unroll
            for (int r = 0; r < kPer; ++r) {
                mag[r][i] = M::without_odd(mag[r][i]);
                down[i] = M::larger(down[i], mag[r][i]);
            }
            all = M::larger(all, down[i]);
        }
    }

    if constexpr (KIND == CNR_BLOCK_TILE) {
        all = max_down<M>(max_across<M>(all));
        if (t % kWave == 0) largest[wave][0] = all;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWavesPerBlock; ++i) all = M::larger(all, largest[i][0]);
        const Scale s = scale_of<SCALE>(M::as_float(M::largest(all)));
        if (t == 0) {
            if (a.codes) store_scale<SCALE>(a.scale, tile_col * a.scale_stride + tile_row, s);
            if (BOTH) store_scale<SCALE>(a.scale_t, tile_row * a.scale_stride_t + tile_col, s);
        }
        u32x2 codes[kPer];
#pragma unroll
        for (int r = 0; r < kPer; ++r) codes[r] = encode8<TYPE, SCALE>(w[r], s, odd);
        if (a.codes) {
#pragma unroll
            for (int r = 0; r < kPer; ++r)
                if (r0 + r < a.n_rows) *reinterpret_cast<u32x2 *>(a.codes + (uint64_t)(r0 + r) * a.row_bytes + c0) = codes[r];
        }
        if constexpr (BOTH) {
            // eight rows of eight codes, transposed by bytes: pairs of rows, then pairs of pairs
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t pair[kPer / 2][2];
#pragma unroll
                for (int r = 0; r < kPer / 2; ++r) {
                    pair[r][0] = __builtin_amdgcn_perm(codes[2 * r + 1][h], codes[2 * r][h], 0x05010400u);  // columns 0 and 1 of rows 2 r, 2 r + 1
                    pair[r][1] = __builtin_amdgcn_perm(codes[2 * r + 1][h], codes[2 * r][h], 0x07030602u);
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t pick = c % 2 ? 0x07060302u : 0x05040100u;
                    const u32x2 column = {__builtin_amdgcn_perm(pair[1][c / 2], pair[0][c / 2], pick), __builtin_amdgcn_perm(pair[3][c / 2], pair[2][c / 2], pick)};
                    *reinterpret_cast<u32x2 *>(turned + (t % kAcross * kPer + 4 * h + c) * kPitch + t / kAcross * kPer) = column;
                }
            }
        }
    } else {
        if (a.codes) {
#pragma unroll
            for (int r = 0; r < kPer; ++r) {
                uint32_t m = mag[r][0];
#pragma unroll
                for (int i = 1; i < kWords; ++i) m = M::larger(m, mag[r][i]);
                const Scale s = scale_of<SCALE>(M::as_float(M::largest(max_across<M>(m))));
                if (r0 + r < a.n_rows) {
                    *reinterpret_cast<u32x2 *>(a.codes + (uint64_t)(r0 + r) * a.row_bytes + c0) = encode8<TYPE, SCALE>(w[r], s, odd);
                    if (t % kAcross == 0) store_scale<SCALE>(a.scale, tile_col * a.scale_stride + r0 + r, s);
                }
            }
        }
        if constexpr (BOTH) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                down[i] = max_down<M>(down[i]);
                if (t % kWave < kAcross) largest[wave][t % kAcross * kWords + i] = down[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWords; ++i)
#pragma unroll
                for (int v = 0; v < kWavesPerBlock; ++v) down[i] = M::larger(down[i], largest[v][t % kAcross * kWords + i]);
#pragma unroll
            for (int c = 0; c < kPer; ++c) {
                const Scale s = scale_of<SCALE>(M::as_float(M::part(down[c / M::kIn], c % M::kIn)));
                uint32_t column[kWords];  // the thread's eight rows of column c, side by side
#pragma unroll
                for (int i = 0; i < kWords; ++i) {
                    if constexpr (M::kIn == 1)
                        column[i] = w[i][c];
                    else
                        column[i] = __builtin_amdgcn_perm(w[2 * i + 1][c / 2], w[2 * i][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
                }
                *reinterpret_cast<u32x2 *>(turned + (t % kAcross * kPer + c) * kPitch + t / kAcross * kPer) =
                    encode8<TYPE, SCALE>(column, s, odd);
                if (t < kAcross && c0 + c < a.dim) store_scale<SCALE>(a.scale_t, tile_row * a.scale_stride_t + c0 + c, s);
            }
        }
    }
    if constexpr (BOTH) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kTile * kTile / 16 / kBlock; ++i) {
            const uint32_t at = i * kBlock + t, c = at / (kTile / 16), part = at % (kTile / 16);
            if (tile_col * kTile + c < a.dim)
                *reinterpret_cast<u32x4 *>(a.codes_t + (uint64_t)(tile_col * kTile + c) * a.row_bytes_t + (uint64_t)tile_row * kTile + part * 16) =
                    *reinterpret_cast<const u32x4 *>(turned + c * kPitch + part * 16);
        }
    }
}

template <int TYPE, int KIND, int SCALE>
void launch(const QuantizeArgs &a, unsigned tiles, hipStream_t s) {
    if (a.codes_t)
        hipLaunchKernelGGL((quantize_kernel<TYPE, KIND, SCALE, true>), dim3(tiles), dim3(kBlock), 0, s, a);
    else
        hipLaunchKernelGGL((quantize_kernel<TYPE, KIND, SCALE, false>), dim3(tiles), dim3(kBlock), 0, s, a);
}
template <int TYPE>
void launch(const QuantizeArgs &a, cnr_block_kind kind, cnr_scale_type scale, unsigned tiles, hipStream_t s) {
    if (kind == CNR_BLOCK_ROW)
        scale == CNR_SCALE_E8M0 ? launch<TYPE, CNR_BLOCK_ROW, CNR_SCALE_E8M0>(a, tiles, s) : launch<TYPE, CNR_BLOCK_ROW, CNR_SCALE_F32>(a, tiles, s);
    else
        scale == CNR_SCALE_E8M0 ? launch<TYPE, CNR_BLOCK_TILE, CNR_SCALE_E8M0>(a, tiles, s) : launch<TYPE, CNR_BLOCK_TILE, CNR_SCALE_F32>(a, tiles, s);
}

}  // namespace

extern "C" {

size_t cnr_block_row_bytes(uint64_t dim) { return (size_t)(cnr_ceil_div(dim, CNR_BLOCK) * CNR_BLOCK); }

size_t cnr_block_scale_stride(uint64_t n_rows, cnr_block_kind kind) {
    const uint64_t tiles = cnr_ceil_div(n_rows, CNR_BLOCK);
    return (size_t)(kind == CNR_BLOCK_TILE ? tiles : tiles * CNR_BLOCK);
}

size_t cnr_block_scale_count(uint64_t n_rows, uint64_t dim, cnr_block_kind kind) {
    return (size_t)(cnr_ceil_div(dim, CNR_BLOCK) * cnr_block_scale_stride(n_rows, kind));
}

cnr_status cnr_quantize_blocks(cnr_ctx *ctx, const void *x, cnr_float_type type, uint64_t n_rows, uint64_t dim,
                               uint64_t stride, cnr_block_kind kind, cnr_scale_type scale_type, uint8_t *codes,
                               void *scale, uint8_t *codes_t, void *scale_t, void *stream) {
    if (!ctx || !cnr_valid_float_type(type) || (kind != CNR_BLOCK_ROW && kind != CNR_BLOCK_TILE) ||
        (scale_type != CNR_SCALE_E8M0 && scale_type != CNR_SCALE_F32) || stride < dim)
        return CNR_E_INVALID;
    if ((codes == nullptr) != (scale == nullptr) || (codes_t == nullptr) != (scale_t == nullptr)) return CNR_E_INVALID;
    if (n_rows > CNR_LM_MAX_SIZE || dim > CNR_LM_MAX_SIZE) return CNR_E_TOO_LARGE;
    const uint64_t across = cnr_ceil_div(dim, CNR_BLOCK), tiles = cnr_ceil_div(n_rows, CNR_BLOCK) * across;
    if (tiles == 0) return CNR_OK;
    if (tiles >= 1u << 24) return CNR_E_TOO_LARGE;  // threads of a grid are counted in 32 bits
    if (!x || (!codes && !codes_t)) return CNR_E_INVALID;
    if (!cnr_aligned(x, cnr_float_bytes(type)) || !cnr_aligned(codes, 16) || !cnr_aligned(scale, 16) || !cnr_aligned(codes_t, 16) ||
        !cnr_aligned(scale_t, 16))
        return CNR_E_ALIGN;
    cnr_status st = cnr_enter(ctx);
    if (st != CNR_OK) return st;
    QuantizeArgs a;
    a.x = x;
    a.stride = stride;
    a.n_rows = (uint32_t)n_rows;
    a.dim = (uint32_t)dim;
    a.tiles_across = (uint32_t)across;
    a.codes = codes;
    a.scale = scale;
    a.codes_t = codes_t;
    a.scale_t = scale_t;
    a.row_bytes = cnr_block_row_bytes(dim);
    a.row_bytes_t = cnr_block_row_bytes(n_rows);
    a.scale_stride = cnr_block_scale_stride(n_rows, kind);
    a.scale_stride_t = cnr_block_scale_stride(dim, kind);
    if (type == CNR_FLOAT_F32)
        launch<CNR_FLOAT_F32>(a, kind, scale_type, (unsigned)tiles, as_stream(stream));
    else if (type == CNR_FLOAT_BF16)
        launch<CNR_FLOAT_BF16>(a, kind, scale_type, (unsigned)tiles, as_stream(stream));
    else
        launch<CNR_FLOAT_F16>(a, kind, scale_type, (unsigned)tiles, as_stream(stream));
    return cnr_launch_status(ctx);
}

}  // extern "C"
