// Block quantization: a matrix, and its transpose, to e4m3 codes with a scale for each block of 128.
//
// Bound by memory: x is read once, codes written once for each direction.  A workgroup takes 128 x 128 elements, so that both
// directions' blocks lie within it: each thread holds 8 rows x 8 columns in registers (16 lanes across the
// tile, so that a wave reads four rows' 128 columns in one instruction), the maxima of a row's blocks are
// combined across those 16 lanes by DPP, those of a column's across the 4 rows of lanes and the 4 waves.  Codes
// of the transpose pass through LDS, so that whole lines of 128 bytes are stored in both directions.
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

// Largest absolute value by its bits (they order like the values); infinities and NaN have none.
__device__ __forceinline__ uint32_t magnitude(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint32_t max_across(uint32_t m) {  // of the 16 lanes that hold a row
    m = umax(m, (uint32_t)dpp_i<0xB1>((int)m));
    m = umax(m, (uint32_t)dpp_i<0x4E>((int)m));
    m = umax(m, (uint32_t)dpp_i<0x141>((int)m));
    return umax(m, (uint32_t)dpp_i<0x140>((int)m));
}
__device__ __forceinline__ uint32_t max_down(uint32_t m) {  // of the wave's lanes that hold the same columns
    m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
    return umax(m, (uint32_t)__shfl_xor((int)m, 32));
}

// A block's scale from the bits of its largest magnitude.  Powers of two: 448 = 1.75 * 2^8, so the exponent is the magnitude's less
// 8, one more where its fraction is above 1.75.  They divide exactly, a transposed tile's codes are the tile's, and
// the matrix instructions take them as they are.  code = e4m3(x / scale): `inv` is 1 / scale.
struct Scale {
    float value, inv;
    uint8_t byte;
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
        s.inv = __uint_as_float((uint32_t)(254 - e) << 23);
    } else {
        const float v = __uint_as_float(amax) / 448.0f;
        s.value = amax ? (v < 0x1p-126f ? 0x1p-126f : v) : 1.0f;
        s.inv = 1.0f / s.value;
        s.byte = 0;
    }
    return s;
}

// The quotient whose e4m3 rounding is that of x / scale exactly.  With powers of two that is the quotient itself.
// Else the rounded quotient could fall on the middle between two codes where the true one lies beside it: a
// quotient that is not exact gets its last bit set after rounding towards zero, and a middle has that bit clear.
// The remainder decides both; scaled up by 2^64 where it could leave fp32's range.
template <int SCALE>
__device__ __forceinline__ float quotient(float x, const Scale &s, bool tiny) {
    if (SCALE == CNR_SCALE_E8M0) return x * s.inv;
    float d = s.value, inv = s.inv;
    if (tiny) {
        const float up = d < 0x1p-60f ? 0x1p64f : 1.0f, down = d < 0x1p-60f ? 0x1p-64f : 1.0f;
        x *= up;
        d *= up;
        inv *= down;
    }
    float q = x * inv;
    q = __builtin_fmaf(__builtin_fmaf(-q, d, x), inv, q);
    const float rest = __builtin_fmaf(-q, d, x);
    uint32_t b = __float_as_uint(q);
    b -= (__float_as_uint(rest) ^ b) >> 31;  // |q| was rounded up: the remainder's sign is not q's
    return __builtin_copysignf(__uint_as_float(rest != 0.0f ? b | 1u : __float_as_uint(q)), x);  // -0 became 0
}

template <int SCALE>
__device__ __forceinline__ u32x2 encode8(const float *v, const Scale &s, bool tiny) {
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(quotient<SCALE>(v[4 * i], s, tiny), quotient<SCALE>(v[4 * i + 1], s, tiny), 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(quotient<SCALE>(v[4 * i + 2], s, tiny), quotient<SCALE>(v[4 * i + 3], s, tiny), r, true);
    }
    return w;
}
template <int SCALE>
__device__ __forceinline__ bool any_tiny(const Scale &s) {
    return SCALE == CNR_SCALE_F32 && __any(s.value < 0x1p-60f);
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
    __shared__ __align__(16) uint8_t turned[BOTH ? kTile * kPitch : 16];
    __shared__ uint32_t largest[kWavesPerBlock][kTile];
    const uint32_t tile_row = wg_x() / a.tiles_across, tile_col = wg_x() % a.tiles_across;
    const uint32_t t = tid_x(), wave = t / kWave;
    const uint32_t r0 = tile_row * kTile + t / kAcross * kPer, c0 = tile_col * kTile + t % kAcross * kPer;
    const T *x = reinterpret_cast<const T *>(a.x);

    float v[kPer][kPer];
    Pack<T, kPer> got[kPer];
    const bool whole = tile_row * kTile + kTile <= a.n_rows && tile_col * kTile + kTile <= a.dim;
    if (whole) {
#pragma unroll
        for (int r = 0; r < kPer; ++r) got[r] = *reinterpret_cast<const Pack<T, kPer> *>(x + (uint64_t)(r0 + r) * a.stride + c0);
    } else {
#pragma unroll
        for (int r = 0; r < kPer; ++r)
#pragma unroll
            for (int c = 0; c < kPer; ++c)
                got[r].v[c] = r0 + r < a.n_rows && c0 + c < a.dim ? x[(uint64_t)(r0 + r) * a.stride + c0 + c] : (T)0.0f;
    }
#pragma unroll
    for (int r = 0; r < kPer; ++r)
#pragma unroll
        for (int c = 0; c < kPer; ++c) v[r][c] = Element<TYPE>::wide(got[r].v[c]);

    if (KIND == CNR_BLOCK_TILE) {
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < kPer; ++r)
#pragma unroll
            for (int c = 0; c < kPer; ++c) m = umax(m, magnitude(v[r][c]));
        m = max_down(max_across(m));
        if (t % kWave == 0) largest[wave][0] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) m = umax(m, largest[w][0]);
        const Scale s = scale_of<SCALE>(m);
        const bool tiny = any_tiny<SCALE>(s);
        if (t == 0) {
            if (a.codes) store_scale<SCALE>(a.scale, tile_col * a.scale_stride + tile_row, s);
            if (BOTH) store_scale<SCALE>(a.scale_t, tile_row * a.scale_stride_t + tile_col, s);
        }
        u32x2 w[kPer];
#pragma unroll
        for (int r = 0; r < kPer; ++r) w[r] = encode8<SCALE>(v[r], s, tiny);
        if (a.codes) {
#pragma unroll
            for (int r = 0; r < kPer; ++r)
                if (r0 + r < a.n_rows) *reinterpret_cast<u32x2 *>(a.codes + (uint64_t)(r0 + r) * a.row_bytes + c0) = w[r];
        }
        if (BOTH) {
#pragma unroll
            for (int c = 0; c < kPer; ++c) {
                u32x2 o;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    o[h] = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[h] |= ((w[4 * h + i][c / 4] >> (8 * (c % 4))) & 255u) << (8 * i);
                }
                *reinterpret_cast<u32x2 *>(turned + (t % kAcross * kPer + c) * kPitch + t / kAcross * kPer) = o;
            }
        }
    } else {
        if (a.codes) {
#pragma unroll
            for (int r = 0; r < kPer; ++r) {
                uint32_t m = 0;
#pragma unroll
                for (int c = 0; c < kPer; ++c) m = umax(m, magnitude(v[r][c]));
                const Scale s = scale_of<SCALE>(max_across(m));
                if (r0 + r < a.n_rows) {
                    *reinterpret_cast<u32x2 *>(a.codes + (uint64_t)(r0 + r) * a.row_bytes + c0) = encode8<SCALE>(v[r], s, any_tiny<SCALE>(s));
                    if (t % kAcross == 0) store_scale<SCALE>(a.scale, tile_col * a.scale_stride + r0 + r, s);
                }
            }
        }
        if (BOTH) {
#pragma unroll
            for (int c = 0; c < kPer; ++c) {
                uint32_t m = 0;
#pragma unroll
                for (int r = 0; r < kPer; ++r) m = umax(m, magnitude(v[r][c]));
                m = max_down(m);
                if (t % kWave < kAcross) largest[wave][t % kAcross * kPer + c] = m;
            }
            __syncthreads();
#pragma unroll
            for (int c = 0; c < kPer; ++c) {
                uint32_t m = 0;
#pragma unroll
                for (int w = 0; w < kWavesPerBlock; ++w) m = umax(m, largest[w][t % kAcross * kPer + c]);
                const Scale s = scale_of<SCALE>(m);
                float down[kPer];
#pragma unroll
                for (int r = 0; r < kPer; ++r) down[r] = v[r][c];
                *reinterpret_cast<u32x2 *>(turned + (t % kAcross * kPer + c) * kPitch + t / kAcross * kPer) =
                    encode8<SCALE>(down, s, any_tiny<SCALE>(s));
                if (t < kAcross && c0 + c < a.dim) store_scale<SCALE>(a.scale_t, tile_row * a.scale_stride_t + c0 + c, s);
            }
        }
    }
    if (BOTH) {
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
