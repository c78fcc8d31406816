// Losses of the matrix that gives the logits, z = hidden weight^T, and their gradients, without all logits in memory.
//
// The softmax cross entropy of a target is the distillation from a teacher that is certain: both are
//   loss = sum_j q_j (log q_j - z'[token_j] + lse),  z' = z / T,  lse = log sum_v exp z'_v
//   dz_v = dloss / T (exp(z'_v - lse) - sum of q_j with token_j = v)
// with a few (token, share) entries a row, so one machine serves them.  The entries of a teacher are sorted by token first, and those of one token put together.
//   forward   a product whose tiles leave, for each row, the largest logit and the sum of exponentials relative to it (kept to base 2: exp2 is one
//             instruction), and the logits of its target or, by way of LDS, of its entries; one workgroup a row then joins them and writes the loss;
//   backward  for a piece of the vocabulary at a time, the logits once more, turned into dz in the epilogue; the entries' own dz, a few a row, are put in
//             by a kernel of its own; then dhidden += dz weight and dweight = dz^T hidden, products that read the weight, the hidden states and dz along
//             whichever side their sum goes, so nothing is transposed in memory.
// Rows that are left out, and rows whose dloss is 0, have dz = 0 and are zeros in the copy of the hidden states that the backward pass makes: whatever they
// hold reaches no gradient.
//
// The matrix instructions take 16-bit elements.  A float is the sum of three bfloat16, its bits cut in three; of the nine products of two floats' parts
// six are added up, the rest is below 2^-21 of the product in the worst case (2^-24 on average).  All parts have the float's sign, and a part that is zero of a float that is
// not, or of an infinite one, is +-2^-133 instead, bfloat16's smallest, which the matrix instructions keep: so an infinity times a float is the infinity that it ought to be
// in every term.  A float is thus off by 2^-131 at most, which is more than 2^-21 of it below 2^-110 only.
#include "lm_loss_plan.h"

#include <type_traits>

namespace {

using dense::i32x4;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ Stats join(const Stats &a, const Stats &b) {
    const float top = __builtin_fmaxf(a.top, b.top), at = top == -__builtin_inff() ? 0.0f : top;
    return {top, a.sum * exp2_of(a.top - at) + b.sum * exp2_of(b.top - at)};
}
// The same over the sixteen lanes of a row, in all of them.
__device__ __forceinline__ float max16(float v) {
    v = __builtin_fmaxf(v, dpp_f<0xB1>(v));
    v = __builtin_fmaxf(v, dpp_f<0x4E>(v));
    v = __builtin_fmaxf(v, dpp_f<0x141>(v));
    return __builtin_fmaxf(v, dpp_f<0x140>(v));
}
__device__ __forceinline__ float sum16(float v) {
    v += dpp_f<0xB1>(v);
    v += dpp_f<0x4E>(v);
    v += dpp_f<0x141>(v);
    return v + dpp_f<0x140>(v);
}
__device__ __forceinline__ float wave_max(float v) {
    v = max16(v);
    v = __builtin_fmaxf(v, __shfl_xor(v, 16));
    return __builtin_fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float wave_sum(float v) {
    v = sum16(v);
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}
// Stats of N logits of one row in each of sixteen lanes, of those with a set bit in `valid`; c = log2(e) / T.
template <int N>
__device__ __forceinline__ Stats stats16(const float (&z)[N], float c, uint32_t valid) {
    float top = -__builtin_inff();
#pragma unroll
    for (int g = 0; g < N; ++g) top = __builtin_fmaxf(top, valid >> g & 1u ? z[g] : -__builtin_inff());
    top = max16(top) * c;
    const float at = top == -__builtin_inff() ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int g = 0; g < N; ++g) sum += valid >> g & 1u ? exp2_of(__builtin_fmaf(z[g], c, -at)) : 0.0f;
    return {top, sum16(sum)};
}

// ---- what the products' tiles do with their outputs ----------------------------------------------------------------

struct TargetArgs {
    const void *tokens, *logits;
    uint64_t token_stride, logit_stride;
    uint32_t top;
    int token_type, logit_type;
    float temperature;
};
__device__ __forceinline__ int64_t token_of(const TargetArgs &t, uint64_t row, uint32_t j) {
    const uint64_t at = row * t.token_stride + j;
    return t.token_type == CNR_IDX_I64 ? reinterpret_cast<const int64_t *>(t.tokens)[at] : reinterpret_cast<const int32_t *>(t.tokens)[at];
}

// A teacher's entries, [n][top], in the order of their tokens; kNoToken behind the last.
constexpr int32_t kNoToken = 0x7fffffff;
struct Entries {
    int32_t *tokens;
    float *share;   // all of a token's at its first entry
    float *picked;  // its logit
    uint32_t top;
};

// Stats of each row over the tile's columns, and the logits there of the row's target or, SOFT, of its entries: the same sums that the stats are of, so that of
// a certain token's loss nothing but the other tokens is left.
template <bool SOFT>
struct KeepStats {
    static constexpr bool kUsesLds = true;
    Stats *parts;      // [rows][n_parts], from the piece's first part on
    uint32_t n_parts;
    float c;
    uint32_t first;          // token of the first column
    TargetArgs targets;      // not SOFT
    uint64_t row0;           // the first row
    float *picked;           // [rows]: its target's logit
    const uint16_t *begins;  // SOFT: [rows][n_parts + 1], as parts: a tile's first entry in a row
    Entries entries;         // from the first row on
    template <uint32_t TM, uint32_t TN, int WM, typename Place, int MF, int NF>
    __device__ __forceinline__ void finish(const dense::Args &p, const Place &at, const f32x4 (&acc)[MF][NF]) const {
        if (at.column0 + TM <= p.columns)
            reduce<TM, TN, WM, true>(p, at, acc);
        else
            reduce<TM, TN, WM, false>(p, at, acc);
    }
    template <uint32_t TM, uint32_t TN, int WM, bool WHOLE, typename Place, int MF, int NF>
    __device__ __forceinline__ void reduce(const dense::Args &p, const Place &at, const f32x4 (&acc)[MF][NF]) const {
        Stats *lds = reinterpret_cast<Stats *>(at.lds);  // [WM][TN]
        uint32_t target[NF];  // which of the lane's columns
#pragma unroll
        for (int g = 0; g < NF; ++g) {
            target[g] = kNoTarget;
            // (tokens that are none are below or behind all columns that count)
            if constexpr (!SOFT)
                if (at.row(g) < p.rows) target[g] = at.index_of((uint64_t)token_of(targets, row0 + at.row(g), 0) - first - at.column);
        }
#pragma unroll
        for (int g = 0; g < NF; ++g) {
            float top = -__builtin_inff();
#pragma unroll
            for (uint32_t i = 0; i < 4 * MF; ++i) top = __builtin_fmaxf(top, WHOLE || at.column_of(i) < p.columns ? at.value(acc, i, g) : -__builtin_inff());
            top = __builtin_fmaxf(top, __shfl_xor(top, 16));
            top = __builtin_fmaxf(top, __shfl_xor(top, 32)) * c;
            const float from = top == -__builtin_inff() ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 4 * MF; ++i) sum += WHOLE || at.column_of(i) < p.columns ? exp2_of(__builtin_fmaf(at.value(acc, i, g), c, -from)) : 0.0f;
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (tid_x() % kWave < 16) lds[at.wave_column * TN + at.row_within(g)] = {top, sum};
            if (!SOFT && __any(target[g] != kNoTarget)) {
                float z = 0.0f;
#pragma unroll
                for (uint32_t i = 0; i < 4 * MF; ++i) z = target[g] == i ? at.value(acc, i, g) : z;
                if (target[g] != kNoTarget) picked[at.row(g)] = z;
            }
        }
        __syncthreads();
        const uint32_t row = tid_x();
        if (row < TN && at.row0 + row < p.rows) {
            Stats s = lds[row];
#pragma unroll
            for (int w = 1; w < WM; ++w) s = join(s, lds[w * TN + row]);
            parts[(uint64_t)(at.row0 + row) * n_parts + at.tile_column] = s;
        }
        if constexpr (SOFT) pick<TM, TN>(p, at, acc);
    }
    // The tile goes into LDS, as many rows at a time as there is room for, and each entry looks its logit up: what it costs does not depend on where the entries
    // are (8192 x 32000 x 4096 with 64 entries a row 1640 -> 1680 us; as dot products of rows from memory they took 680).  Pieces of four columns are permuted by the
    // row, so that rows that are written together take different banks.
    template <uint32_t TM, uint32_t TN, typename Place, int MF, int NF>
    __device__ __forceinline__ void pick(const dense::Args &p, const Place &at, const f32x4 (&acc)[MF][NF]) const {
        constexpr uint32_t kRoom = Place::kLdsBytes / (TM * 4), kRows = kRoom < TN ? kRoom : TN, kEach = Place::kThreads / kRows;
        static_assert(TN % kRows == 0 && Place::kThreads % kRows == 0, "whole phases");
        float *lds = reinterpret_cast<float *>(at.lds);
        const uint32_t column0 = at.column - at.column0, sub = tid_x() / kRows, own = tid_x() % kRows;
#pragma unroll
        for (uint32_t phase = 0; phase < TN / kRows; ++phase) {
            const uint32_t row = at.row0 + phase * kRows + own;
            uint32_t begin = 0, end = 0;
            if (row < p.rows) {
                const uint16_t *b = begins + (uint64_t)row * (n_parts + 1) + at.tile_column;
                begin = b[0];
                end = b[1];
            }
            __syncthreads();
#pragma unroll
            for (int g = 0; g < NF; ++g) {
                const uint32_t within = at.row_within(g) - phase * kRows;
                if (within >= kRows) continue;
#pragma unroll
                for (int i = 0; i < 4 * MF; i += 4) {
                    const f32x4 v = {at.value(acc, i, g), at.value(acc, i + 1, g), at.value(acc, i + 2, g), at.value(acc, i + 3, g)};
                    const uint32_t piece = (column0 + i / 8 * 32 + i % 8) / 4;
                    *reinterpret_cast<f32x4 *>(lds + within * TM + (piece ^ within % 16) * 4) = v;
                }
            }
            __syncthreads();
            for (uint32_t e = begin + sub; e < end; e += kEach) {
                const uint64_t entry = (uint64_t)row * entries.top + e;
                const uint32_t column = (uint32_t)entries.tokens[entry] - first - at.column0;
                if (column < TM) entries.picked[entry] = lds[own * TM + ((column / 4) ^ own % 16) * 4 + column % 4];
            }
        }
    }
};

// v as PARTS numbers of 16 bits that add up to it.
template <int TYPE, int PARTS>
__device__ __forceinline__ void apart(float v, typename Element<TYPE>::type (&part)[PARTS]) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        part[i] = Element<TYPE>::narrow(v);
        v -= Element<TYPE>::wide(part[i]);
    }
}

// dz of the tile's rows and columns, with zeros up to the next whole block of columns, in PARTS parts side by side.  Its stores are not hidden: 8192 x 25344 x 2048
// 715 us, with the stats alone 646.
template <int TYPE, int PARTS>
struct KeepGradient {
    static constexpr bool kUsesLds = false;
    typedef typename Element<TYPE>::type T;
    T *dz;
    uint64_t width, stride;    // of a part, of a row: PARTS * width, whole blocks
    const RowGradient *rows;   // up to a multiple of 256
    uint32_t first;            // token of the first column
    float c;
    template <int MF, int NF, bool TARGET, typename Place>
    __device__ __forceinline__ void write(const dense::Args &p, const Place &at, const f32x4 (&acc)[MF][NF], int g, const RowGradient &r, uint32_t target, T *to) const {
#pragma unroll
        for (int from = 0; from < 4 * MF; from += 8) {
            const uint32_t column = at.column_of(from);
            if (column >= width) continue;
            Pack<T, 8> w[PARTS];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = exp2_of(__builtin_fmaf(at.value(acc, from + j, g), c, -r.lse2));
                if (TARGET && target == (uint32_t)(from + j)) v -= 1.0f;
                T part[PARTS];
                apart<TYPE, PARTS>(r.gradient == 0.0f || column + j >= p.columns ? 0.0f : r.gradient * v, part);
#pragma unroll
                for (int i = 0; i < PARTS; ++i) w[i].v[j] = part[i];
            }
#pragma unroll
            for (int i = 0; i < PARTS; ++i) *reinterpret_cast<Pack<T, 8> *>(to + i * width + column) = w[i];
        }
    }
    template <uint32_t TM, uint32_t TN, int WM, typename Place, int MF, int NF>
    __device__ __forceinline__ void finish(const dense::Args &p, const Place &at, const f32x4 (&acc)[MF][NF]) const {
#pragma unroll
        for (int g = 0; g < NF; ++g) {
            const uint32_t row = at.row(g);
            const RowGradient r = rows[row];
            if (row >= p.rows) continue;
            T *to = dz + row * stride;
            const uint32_t target = at.index_of(r.target - first - at.column);  // which of the lane's
            if (__any(target != kNoTarget))
                write<MF, NF, true>(p, at, acc, g, r, target, to);
            else
                write<MF, NF, false>(p, at, acc, g, r, target, to);
        }
    }
};

// out = there + scale * product, rounded once; either may be float or TYPE.
struct Target {
    void *out;
    uint64_t stride;
    int type;
};
__device__ __forceinline__ float read(const Target &t, uint64_t m, uint32_t n) {
    const uint64_t at = m * t.stride + n;
    if (t.type == CNR_FLOAT_F32) return reinterpret_cast<const float *>(t.out)[at];
    if (t.type == CNR_FLOAT_BF16) return (float)reinterpret_cast<const __bf16 *>(t.out)[at];
    return (float)reinterpret_cast<const _Float16 *>(t.out)[at];
}
template <int N>
__device__ __forceinline__ void read_row(const Target &t, uint64_t m, uint32_t n, uint32_t n_end, float (&v)[N]) {
    if (n + N <= n_end) {
        const uint64_t at = m * t.stride + n;
        if (t.type == CNR_FLOAT_F32) {
            const Pack<float, N> w = *reinterpret_cast<const Pack<float, N> *>(reinterpret_cast<const float *>(t.out) + at);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = w.v[j];
        } else if (t.type == CNR_FLOAT_BF16) {
            const Pack<__bf16, N> w = *reinterpret_cast<const Pack<__bf16, N> *>(reinterpret_cast<const __bf16 *>(t.out) + at);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (float)w.v[j];
        } else {
            const Pack<_Float16, N> w = *reinterpret_cast<const Pack<_Float16, N> *>(reinterpret_cast<const _Float16 *>(t.out) + at);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = (float)w.v[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = n + j < n_end ? read(t, m, n + j) : 0.0f;
    }
}
template <typename T, int N>
__device__ __forceinline__ void write_as(T *to, uint32_t n, uint32_t n_end, const float (&v)[N]) {
    if (n + N <= n_end) {
        Pack<T, N> w;
#pragma unroll
        for (int j = 0; j < N; ++j) w.v[j] = (T)v[j];
        *reinterpret_cast<Pack<T, N> *>(to) = w;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (n + j < n_end) to[j] = (T)v[j];
    }
}
template <int N>
__device__ __forceinline__ void write_row(const Target &t, uint64_t m, uint32_t n, uint32_t n_end, const float (&v)[N]) {
    const uint64_t at = m * t.stride + n;
    if (t.type == CNR_FLOAT_F32)
        write_as(reinterpret_cast<float *>(t.out) + at, n, n_end, v);
    else if (t.type == CNR_FLOAT_BF16)
        write_as(reinterpret_cast<__bf16 *>(t.out) + at, n, n_end, v);
    else
        write_as(reinterpret_cast<_Float16 *>(t.out) + at, n, n_end, v);
}

struct KeepSum {
    static constexpr bool kUsesLds = false;
    Target out, there;      // there.out NULL: nothing is added
    const float *scale;     // NULL: 1
    float *partial;         // [splits][m][partial_stride] where sums are split
    uint64_t partial_stride;
    const RowGradient *rows; // NULL: all count.  The others' outputs are 0, also where the weight holds infinities or NaN
    __device__ __forceinline__ bool counts(uint32_t row) const { return !rows || rows[row].gradient != 0.0f; }
    template <uint32_t TM, uint32_t TN, int WM, typename Place, int MF, int NF>
    __device__ __forceinline__ void finish(const dense::Args &p, const Place &at, const f32x4 (&acc)[MF][NF]) const {
        const float by = scale ? *scale : 1.0f;
#pragma unroll
        for (int g = 0; g < NF; ++g) {
            const uint32_t row = at.row(g);
            if (row >= p.rows) continue;
            if (p.splits > 1) {
                float *to = partial + ((uint64_t)at.split * p.rows + row) * partial_stride;
#pragma unroll
                for (int first = 0; first < 4 * MF; first += 4) {
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = at.value(acc, first + j, g);
                    write_as(to + at.column_of(first), at.column_of(first), p.columns, v);
                }
                continue;
            }
            const bool all = counts(row);
            // What is added to is read for the whole row at once: one piece after the other would wait for memory each time.
            float old[4 * MF / 8][8];
#pragma unroll
            for (int u = 0; u < 4 * MF / 8; ++u) {
#pragma unroll
                for (int j = 0; j < 8; ++j) old[u][j] = 0.0f;
                if (there.out) read_row(there, row, at.column_of(8 * u), p.columns, old[u]);
            }
#pragma unroll
            for (int u = 0; u < 4 * MF / 8; ++u) {
#pragma unroll
                for (int j = 0; j < 8; ++j) old[u][j] = all ? __builtin_fmaf(at.value(acc, 8 * u + j, g), by, old[u][j]) : 0.0f;
                write_row(out, row, at.column_of(8 * u), p.columns, old[u]);
            }
        }
    }
};

// The parts of sums that were split, added up in order: four outputs of a row to a thread, or to LANES threads, each with every LANES-th part.
template <uint32_t LANES>
__global__ void __launch_bounds__(kBlock) join_sums_kernel(const KeepSum k, uint32_t m, uint32_t n, uint32_t splits) {
    const uint32_t across = (uint32_t)(k.partial_stride / 4), lane = tid_x() / (kBlock / LANES);
    const uint64_t at = (uint64_t)wg_x() * (kBlock / LANES) + tid_x() % (kBlock / LANES);
    const bool there = at < (uint64_t)m * across;
    const uint32_t row = (uint32_t)(at / across), column = (uint32_t)(at % across) * 4;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (there) {
        const float *from = k.partial + (uint64_t)row * k.partial_stride + column;
        for (uint32_t s = lane; s < splits; s += 8 * LANES) {
            f32x4 part[8];
#pragma unroll
            for (uint32_t u = 0; u < 8; ++u) {
                part[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (s + u * LANES < splits) part[u] = *reinterpret_cast<const f32x4 *>(from + (uint64_t)(s + u * LANES) * m * k.partial_stride);
            }
#pragma unroll
            for (uint32_t u = 0; u < 8; ++u) sum += part[u];
        }
    }
    if constexpr (LANES > 1) {
        __shared__ f32x4 lds[LANES][kBlock / LANES];
        lds[lane][tid_x() % (kBlock / LANES)] = sum;
        __syncthreads();
        if (lane) return;
#pragma unroll
        for (uint32_t l = 1; l < LANES; ++l) sum += lds[l][tid_x()];
    }
    if (!there) return;
    const float by = k.scale ? *k.scale : 1.0f;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (k.there.out) read_row(k.there, row, column, n, v);
    const bool all = k.counts(row);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = all ? __builtin_fmaf(sum[j], by, v[j]) : 0.0f;
    write_row(k.out, row, column, n, v);
}

// ---- operands laid out for the products -----------------------------------------------------------------------

// One of the parts of a float (see above).
__device__ __forceinline__ __bf16 float_part(float v, int part) {
    const uint32_t sign = __float_as_uint(v) & 0x80000000u;
    float rest = v;
    for (int i = 0; i < part; ++i) rest -= __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
    uint32_t bits = __float_as_uint(rest) & 0xffff0000u;
    if (part) {
        if (!(__builtin_fabsf(v) < __builtin_inff())) bits = 0;
    } else if (v != v) {
        bits = 0x7fc00000u;
    }
    if ((bits & 0x7fffffffu) == 0 && v != 0.0f) bits = sign | 0x00010000u;
    return __builtin_bit_cast(__bf16, (unsigned short)(bits >> 16));
}
// dst[rows][parts][whole blocks] = src, zeros behind it; rows that add nothing to a gradient are zeros.
struct Layout {
    const void *src;
    uint64_t stride;
    uint64_t rows;
    const float *lse2, *dloss;  // NULL: every row counts
    u32x4 *dst;
};
// Two matrices (either may have no rows), 16 bytes of each part to a thread.  Bound by memory: 34000 rows of 1024 floats 53.5 us, 6.5 TB/s.
template <typename T>
__global__ void __launch_bounds__(kBlock) lay_out_kernel(const Layout a, const Layout b, uint32_t dim, uint32_t pieces /* of a part */, uint64_t first) {
    constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    uint64_t at = first + (uint64_t)wg_x() * kBlock + tid_x();
    const bool second = at >= a.rows * pieces;
    const Layout &m = second ? b : a;
    at -= second ? a.rows * pieces : 0;
    if (at >= m.rows * pieces) return;
    const uint64_t row = at / pieces;
    const uint32_t piece = (uint32_t)(at % pieces), column = piece * 8;
    const T *from = reinterpret_cast<const T *>(m.src) + row * m.stride + column;
    Pack<T, 8> w;
    if (m.lse2 && (m.lse2[row] == __builtin_inff() || m.dloss[row] == 0.0f)) {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) w.v[j] = (T)0.0f;
    } else if (column + 8 <= dim) {
        w = *reinterpret_cast<const Pack<T, 8> *>(from);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) w.v[j] = column + j < dim ? from[j] : (T)0.0f;
    }
    u32x4 *to = m.dst + row * pieces * kParts + piece;
    if constexpr (kParts == 1) {
        *to = __builtin_bit_cast(u32x4, w);
    } else {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            Pack<__bf16, 8> part;
#pragma unroll
            for (int j = 0; j < 8; ++j) part.v[j] = float_part(w.v[j], i);
            to[(uint64_t)i * pieces] = __builtin_bit_cast(u32x4, part);
        }
    }
}

// ---- few rows: operands straight from memory -------------------------------------------------------------------
//
// Logits: a workgroup has 16 G rows by 16 NF columns; each of its waves takes a quarter of the sum, U blocks at a time so that enough loads are under way,
// straight into the matrix instructions' registers (floats into the fp32 ones); they add up their sums in LDS.  Bound by reading the weight: 1 x 32000 x
// 4096 in bfloat16 40.8 us, 6.4 TB/s.
//
// The gradients' products go through the fp32 matrix instructions too, with dz in fp32: sixteen rows of dz by four tokens (or sixteen tokens by sixteen rows) by
// sixteen columns at a time, a lane with four columns side by side of each row of the weight, or of its gradient.
struct NarrowArgs {
    const void *hidden, *weight;
    uint64_t hidden_stride, weight_stride;  // elements
    uint32_t n, vocab, dim;
    float c;
    // forward:
    Stats *parts;
    uint32_t n_parts;
    bool soft;
    TargetArgs targets;        // not soft
    float *picked;
    Entries entries;           // soft
    // backward, of a piece of the vocabulary:
    const RowGradient *rows;
    uint32_t first;            // its first token
    float *dz;                 // [vocab][16 G], zeros in rows from n on
};
template <int TYPE>
__device__ __forceinline__ f32x4 multiply(const dense::i32x8 &x, const dense::i32x8 &y, f32x4 sum) {
    if constexpr (TYPE == CNR_FLOAT_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(x[i]), __int_as_float(y[i]), sum, 0, 0, 0);
        return sum;
    } else {
        return dense::multiply<TYPE, 1>(x, y, dense::multiply<TYPE, 0>(x, y, sum));
    }
}
template <typename T>
__device__ __forceinline__ dense::i32x8 load_fragment(const T *row, uint32_t at, uint32_t dim) {
    constexpr uint32_t kPer = 16 / sizeof(T);
    i32x4 part[2];
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
        const uint32_t from = at + h * 4 * kPer;
        if (from + kPer <= dim) {
            part[h] = __builtin_bit_cast(i32x4, load16(row + from));
        } else {
            Pack<T, kPer> w;
#pragma unroll
            for (uint32_t j = 0; j < kPer; ++j) w.v[j] = from + j < dim ? row[from + j] : (T)0.0f;
            part[h] = __builtin_bit_cast(i32x4, w);
        }
    }
    return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int TYPE, int G, int NF, int U, bool GRADIENT>
__global__ void __launch_bounds__(kBlock, G > 2 ? 3 : 4) narrow_kernel(const NarrowArgs p) {
    typedef typename Element<TYPE>::type T;
    constexpr uint32_t kPer = 16 / sizeof(T), kColumns = dense::kBlockBytes / sizeof(T);
    __shared__ f32x4 sums[kWavesPerBlock][G * NF][kWave];
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint32_t quarter = lane / 16, n0 = wg_x() * 16 * NF;
    // Rows beyond the matrix read its last one again.
    const T *a[G], *b[NF];
#pragma unroll
    for (int f = 0; f < G; ++f) {
        const uint32_t row = 16 * f + lane % 16;
        a[f] = reinterpret_cast<const T *>(p.hidden) + (row < p.n ? row : p.n - 1) * p.hidden_stride;
    }
#pragma unroll
    for (int g = 0; g < NF; ++g) {
        const uint32_t v = n0 + 16 * g + lane % 16;
        b[g] = reinterpret_cast<const T *>(p.weight) + (uint64_t)(v < p.vocab ? v : p.vocab - 1) * p.weight_stride;
    }
    f32x4 acc[G][NF];
#pragma unroll
    for (int f = 0; f < G; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t blocks = (p.dim + kColumns - 1) / kColumns, each = (blocks + kWavesPerBlock - 1) / kWavesPerBlock, begin = wave * each;
    const uint32_t end = begin + each < blocks ? begin + each : blocks;
    for (uint32_t first = begin; first < end; first += U) {
        dense::i32x8 x[U][G], y[U][NF];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u && first + u >= end) break;
            const uint32_t at = (first + u) * kColumns + quarter * kPer;
#pragma unroll
            for (int g = 0; g < NF; ++g) y[u][g] = load_fragment(b[g], at, p.dim);
#pragma unroll
            for (int f = 0; f < G; ++f) x[u][f] = load_fragment(a[f], at, p.dim);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u && first + u >= end) break;
#pragma unroll
            for (int f = 0; f < G; ++f)
#pragma unroll
                for (int g = 0; g < NF; ++g) acc[f][g] = multiply<TYPE>(x[u][f], y[u][g], acc[f][g]);
        }
    }
#pragma unroll
    for (int f = 0; f < G; ++f)
#pragma unroll
        for (int g = 0; g < NF; ++g) sums[wave][f * NF + g][lane] = acc[f][g];
    __syncthreads();
    // Sixteen threads to a row, each with one column of each sixteen.
    const uint32_t m = tid_x() / 16, n = tid_x() % 16;
#pragma unroll
    for (uint32_t f = 0; f < G; ++f) {
        const uint32_t row = 16 * f + m;
        float z[NF];
        uint32_t valid = 0;
#pragma unroll
        for (uint32_t g = 0; g < NF; ++g) {
            z[g] = 0.0f;
#pragma unroll
            for (int w = 0; w < kWavesPerBlock; ++w) z[g] += sums[w][f * NF + g][m / 4 * 16 + n][m % 4];
            valid |= n0 + 16 * g + n < p.vocab ? 1u << g : 0u;
        }
        if constexpr (GRADIENT) {
            const RowGradient r = p.rows[row];  // (padded with rows that add nothing)
#pragma unroll
            for (uint32_t g = 0; g < NF; ++g) {
                const uint32_t v = n0 + 16 * g + n;
                const float e = exp2_of(__builtin_fmaf(z[g], p.c, -r.lse2));
                if (valid >> g & 1u) p.dz[(uint64_t)v * (16 * G) + row] = r.gradient == 0.0f ? 0.0f : r.gradient * (p.first + v == r.target ? e - 1.0f : e);
            }
        } else {
            const Stats s = stats16(z, p.c, valid);
            if (n == 0 && row < p.n) p.parts[(uint64_t)row * p.n_parts + wg_x()] = s;
            if (p.soft) {
#pragma unroll
                for (uint32_t g = 0; g < NF; ++g) sums[0][f * NF + g][m / 4 * 16 + n][m % 4] = z[g];  // (nobody else has read this one)
            } else if (row < p.n) {
                const int64_t t = token_of(p.targets, row, 0);
#pragma unroll
                for (uint32_t g = 0; g < NF; ++g)
                    if (t == (int64_t)(n0 + 16 * g + n)) p.picked[row] = z[g];
            }
        }
    }
    if constexpr (!GRADIENT) {
        if (!p.soft) return;
        __syncthreads();
        // A row's threads look at every sixteenth part of its entries, which are in order, then go on from the last that begins below these columns.  (With a
        // list of where each workgroup's entries begin, as tiles have one, a loss of 1 x 262144 x 64 took 33 us instead of 29: one workgroup writes it.)
        const uint32_t top = p.entries.top, part = (top + 15) / 16;
#pragma unroll
        for (uint32_t f = 0; f < G; ++f) {
            const uint32_t row = 16 * f + m;
            if (row >= p.n) continue;
            const uint64_t entry = (uint64_t)row * top;
            auto among_row = [&](bool is) { return (uint32_t)(__ballot(is) >> lane / 16 * 16) & 0xffffu; };
            const uint32_t below = (uint32_t)__popc(among_row(n * part < top && (uint32_t)p.entries.tokens[entry + n * part] < n0));
            for (uint32_t e = (below ? below - 1 : 0) * part + n;; e += 16) {
                const uint32_t token = e < top ? (uint32_t)p.entries.tokens[entry + e] : (uint32_t)kNoToken, column = token - n0;
                if (column < 16 * NF && e < top) p.entries.picked[entry + e] = sums[0][f * NF + column / 16][m / 4 * 16 + column % 16][m % 4];
                if (among_row(token >= n0 + 16 * NF)) break;
            }
        }
    }
}

// Four elements from `column` on, 0 beyond the row.
template <typename T>
__device__ __forceinline__ f32x4 load_four(const T *row, uint32_t column, uint32_t dim) {
    f32x4 v;
    if (column + 4 <= dim) {
        const Pack<T, 4> w = *reinterpret_cast<const Pack<T, 4> *>(row + column);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)w.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = column + j < dim ? (float)row[column + j] : 0.0f;
    }
    return v;
}
struct SlabArgs {
    const void *matrix;        // the weight, or the hidden states
    uint64_t stride;
    const float *dz;           // [vocab][16 G]
    uint32_t vocab, dim, n;
    uint32_t groups, slabs;    // of 64 columns, of the vocabulary: a wave has one of each
    float *partial;            // [slabs][n][partial_stride]
    uint64_t partial_stride;
    const float *lse2, *dloss; // which hidden states count
    Target out, there;
};
// partial[slab][i][column] = sum over the slab's tokens of dz[v][i] * weight[v][column].  13 x 213243 x 1536 in fp32 254 us, 5.2 TB/s (by the ordinary units,
// dz as scalars, 850 for 16 x 131072 x 4096 in bfloat16, 444 so).
template <int TYPE, int G>
__global__ void __launch_bounds__(kBlock) narrow_hidden_kernel(const SlabArgs p) {
    typedef typename Element<TYPE>::type T;
    const uint32_t wave = wave_in_grid(), group = wave % p.groups, slab = wave / p.groups, lane = tid_x() % kWave, quarter = lane / 16, r = lane % 16;
    if (slab >= p.slabs) return;
    const uint32_t column = group * 64 + r * 4;
    const uint32_t begin = (uint32_t)((uint64_t)p.vocab * slab / p.slabs), end = (uint32_t)((uint64_t)p.vocab * (slab + 1) / p.slabs);
    const T *matrix = reinterpret_cast<const T *>(p.matrix);
    f32x4 acc[G][4];  // [sixteen rows][column]
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[g][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr uint32_t kAtOnce = 8;
    for (uint32_t v0 = begin; v0 < end; v0 += 4 * kAtOnce) {
        f32x4 w[kAtOnce];
        float d[kAtOnce][G];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            const uint32_t v = v0 + 4 * u + quarter, at = v < end ? v : end - 1;
            w[u] = load_four(matrix + (uint64_t)at * p.stride, column, p.dim);
#pragma unroll
            for (uint32_t g = 0; g < G; ++g) {
                d[u][g] = p.dz[(uint64_t)at * (16 * G) + 16 * g + r];
                d[u][g] = v < end ? d[u][g] : 0.0f;
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[g][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(d[u][g], w[u][j], acc[g][j], 0, 0, 0);
    }
    // sum i of a lane: row 4 quarter + i of its sixteen, column r of each of the four sixteens
#pragma unroll
    for (uint32_t g = 0; g < G; ++g)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const float v[4] = {acc[g][0][i], acc[g][1][i], acc[g][2][i], acc[g][3][i]};
            const uint32_t row = 16 * g + 4 * quarter + i;
            if (row < p.n) write_as(p.partial + ((uint64_t)slab * p.n + row) * p.partial_stride + column, column, p.dim, v);
        }
}
// out[v][column] = there + sum over i of dz[v][i] * hidden[i][column].  13 x 213243 x 1536 onto an fp32 gradient 650 us, 4.0 TB/s read and written.
template <int TYPE, int G>
__global__ void __launch_bounds__(kBlock) narrow_weight_kernel(const SlabArgs p) {
    typedef typename Element<TYPE>::type T;
    const uint32_t wave = wave_in_grid(), group = wave % p.groups, slab = wave / p.groups, lane = tid_x() % kWave, quarter = lane / 16, r = lane % 16;
    if (slab >= p.slabs) return;
    const uint32_t begin = (uint32_t)((uint64_t)p.vocab * slab / p.slabs), end = (uint32_t)((uint64_t)p.vocab * (slab + 1) / p.slabs);
    const T *matrix = reinterpret_cast<const T *>(p.matrix);
    // Sixteen columns f are 32 (f / 2) + 8 (r / 4) + 4 (f % 2) + r % 4: a lane has eight outputs side by side, and the four lanes of a token 32.
    float x[4][4 * G];  // [f][row of hidden states 16 (s / 4) + 4 quarter + s % 4]
#pragma unroll
    for (uint32_t s = 0; s < 4 * G; ++s) {
        const uint32_t row = s / 4 * 16 + 4 * quarter + s % 4;
        const bool counts = row < p.n && p.lse2[row] != __builtin_inff() && p.dloss[row] != 0.0f;
#pragma unroll
        for (uint32_t f = 0; f < 4; ++f) {
            const uint32_t column = group * 64 + f / 2 * 32 + r / 4 * 8 + f % 2 * 4 + r % 4;
            x[f][s] = counts && column < p.dim ? (float)matrix[row * p.stride + column] : 0.0f;
        }
    }
    constexpr uint32_t kAtOnce = 2;
    for (uint32_t v0 = begin; v0 < end; v0 += 16 * kAtOnce) {
        f32x4 d[kAtOnce][G];
        float old[kAtOnce][2][8];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            const uint32_t v = v0 + 16 * u + r, at = v < end ? v : end - 1;
#pragma unroll
            for (uint32_t g = 0; g < G; ++g) d[u][g] = *reinterpret_cast<const f32x4 *>(p.dz + (uint64_t)at * (16 * G) + 16 * g + 4 * quarter);
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
#pragma unroll
                for (int j = 0; j < 8; ++j) old[u][h][j] = 0.0f;
                if (p.there.out) read_row(p.there, at, group * 64 + h * 32 + quarter * 8, p.dim, old[u][h]);
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            const uint32_t v = v0 + 16 * u + r;
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
#pragma unroll
                for (uint32_t f = 0; f < 2; ++f) {
                    // (sum i of a lane: column i of its four, token r)
                    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int s = 0; s < 4 * G; ++s) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(x[2 * h + f][s], d[u][s / 4][s % 4], sum, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) old[u][h][4 * f + i] += sum[i];
                }
                if (v < end) write_row(p.out, v, group * 64 + h * 32 + quarter * 8, p.dim, old[u][h]);
            }
        }
    }
}
// dz of a teacher's entries.
__global__ void __launch_bounds__(kBlock) narrow_entries_kernel(const NarrowArgs p, const Entries entries, uint32_t padded) {
    const uint32_t at = wg_x() * kBlock + tid_x();
    if (at >= p.n * entries.top) return;
    const float q = entries.share[at];
    const uint32_t row = at / entries.top, t = (uint32_t)entries.tokens[at] - p.first;
    const RowGradient r = p.rows[row];
    if (q == 0.0f || r.gradient == 0.0f || t >= p.vocab) return;
    p.dz[(uint64_t)t * padded + row] = r.gradient * (exp2_of(__builtin_fmaf(entries.picked[at], p.c, -r.lse2)) - q);
}

// ---- forward: a row's loss -------------------------------------------------------------------------------------

__device__ __forceinline__ float logit_of(const TargetArgs &t, uint64_t row, uint32_t j) {
    return read({const_cast<void *>(t.logits), t.logit_stride, t.logit_type}, row, j);
}
constexpr uint32_t kMaxTop = CNR_LOSS_MAX_TOP;
__device__ __forceinline__ float max_of_block(float v, float (&parts)[kWavesPerBlock]) {
    v = wave_max(v);
    __syncthreads();
    if (tid_x() % kWave == 0) parts[tid_x() / kWave] = v;
    __syncthreads();
    return __builtin_fmaxf(__builtin_fmaxf(parts[0], parts[1]), __builtin_fmaxf(parts[2], parts[3]));
}
__device__ __forceinline__ float sum_of_block(float v, float (&parts)[kWavesPerBlock]) {
    v = wave_sum(v);
    __syncthreads();
    if (tid_x() % kWave == 0) parts[tid_x() / kWave] = v;
    __syncthreads();
    return (parts[0] + parts[1]) + (parts[2] + parts[3]);
}

// A row's teacher: the shares of its entries, sorted; loss[row] = sum of share * log(share), lse2[row] = 0, or infinity where the row is left out;
// begins (NULL: not wanted) for tiles of `columns`.  A workgroup to a row; each entry counts those before it: 8192 rows of 64 30 us.
struct TeacherArgs {
    TargetArgs targets;
    uint64_t vocab, row0;
    Entries entries;
    float *loss, *lse2;
    uint16_t *begins;  // of the launch's first row
    uint32_t n_parts, columns;
    cnr_dev_errors *err;
};
__global__ void __launch_bounds__(kBlock) teacher_kernel(const TeacherArgs p) {
    __shared__ int32_t token[kMaxTop], sorted[kMaxTop];
    __shared__ float share[kMaxTop], in_order[kMaxTop];
    __shared__ float parts[kWavesPerBlock];
    const uint64_t row = p.row0 + wg_x();
    const uint32_t top = p.targets.top;
    float largest = -__builtin_inff();
    for (uint32_t j = tid_x(); j < top; j += kBlock) {
        const int64_t t = token_of(p.targets, row, j);
        const bool there = t >= 0 && (uint64_t)t < p.vocab;
        if (t >= 0 && !there) atomicAdd(&p.err->n_bad_indices, 1ull);
        token[j] = there ? (int32_t)t : kNoToken;
        const float v = there ? logit_of(p.targets, row, j) / p.targets.temperature : -__builtin_inff();
        share[j] = v;
        largest = v != v ? __builtin_inff() : __builtin_fmaxf(largest, v);  // NaN, as infinity does, makes the shares NaN
    }
    largest = max_of_block(largest, parts);
    const bool counts = largest != -__builtin_inff();  // else nothing is left of the row
    float sum = 0.0f;
    for (uint32_t j = tid_x(); j < top; j += kBlock) sum += token[j] != kNoToken && counts ? expf(share[j] - largest) : 0.0f;
    sum = sum_of_block(sum, parts);
    const float log_sum = logf(sum);
    float negative_entropy = 0.0f;
    for (uint32_t j = tid_x(); j < top; j += kBlock) {
        const float v = share[j] - largest, q = token[j] != kNoToken && counts ? expf(v) / sum : 0.0f;
        if (q != 0.0f) negative_entropy += q * (v - log_sum);
        share[j] = q;
    }
    negative_entropy = sum_of_block(negative_entropy, parts);
    for (uint32_t j = tid_x(); j < top; j += kBlock) {
        const int32_t t = token[j];
        uint32_t place = 0;
        for (uint32_t i = 0; i < top; ++i) place += token[i] < t || (token[i] == t && i < j) ? 1u : 0u;
        sorted[place] = t;
        in_order[place] = share[j];
    }
    __syncthreads();
    for (uint32_t j = tid_x(); j < top; j += kBlock) {
        const int32_t t = sorted[j];
        float all = 0.0f;
        if (t != kNoToken && (j == 0 || sorted[j - 1] != t))
            for (uint32_t i = j; i < top && sorted[i] == t; ++i) all += in_order[i];
        p.entries.tokens[row * top + j] = t;
        p.entries.share[row * top + j] = all;
        p.entries.picked[row * top + j] = 0.0f;
    }
    if (tid_x() == 0) {
        p.loss[row] = counts ? negative_entropy : 0.0f;
        p.lse2[row] = counts ? 0.0f : __builtin_inff();
    }
    if (!p.begins) return;
    for (uint64_t tile = tid_x(); tile <= p.n_parts; tile += kBlock) {
        uint32_t lo = 0, hi = top;  // the first entry whose token is not below
        while (lo < hi) {
            const uint32_t middle = (lo + hi) / 2;
            if ((uint64_t)(uint32_t)sorted[middle] < tile * p.columns)
                lo = middle + 1;
            else
                hi = middle;
        }
        // (behind the last tile lie those without a token)
        p.begins[(uint64_t)wg_x() * (p.n_parts + 1) + tile] = (uint16_t)lo;
    }
}

struct LossArgs {
    uint64_t vocab;
    TargetArgs targets;
    Entries entries;
    const float *picked;  // of the launch's first row on; without a teacher
    const Stats *parts;
    uint32_t n_parts;
    uint64_t row0;      // of this launch
    float *loss, *lse2; // lse2: NULL where there is no state
    float c;
    cnr_dev_errors *err;
};
template <bool SOFT>
__global__ void __launch_bounds__(kBlock) loss_kernel(const LossArgs p) {
    __shared__ Stats joined[kWavesPerBlock];
    __shared__ float sums[kWavesPerBlock];
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint64_t row = p.row0 + wg_x();
    // eight of the row's parts to a thread at a time, so that their loads and exponentials do not wait for each other
    Stats s = {-__builtin_inff(), 0.0f};
    for (uint32_t first = tid_x(); first < p.n_parts; first += 8 * kBlock) {
        Stats part[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            part[i] = {-__builtin_inff(), 0.0f};
            if (first + i * kBlock < p.n_parts) part[i] = p.parts[(uint64_t)wg_x() * p.n_parts + first + i * kBlock];
        }
        float top = s.top;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) top = __builtin_fmaxf(top, part[i].top);
        const float at = top == -__builtin_inff() ? 0.0f : top;
        float sum = s.sum * exp2_of(s.top - at);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) sum = __builtin_fmaf(part[i].sum, exp2_of(part[i].top - at), sum);
        s = {top, sum};
    }
    {
        const float top = wave_max(s.top), at = top == -__builtin_inff() ? 0.0f : top;
        s = {top, wave_sum(s.sum * exp2_of(s.top - at))};
    }
    if (lane == 0) joined[wave] = s;
    __syncthreads();
    s = joined[0];
#pragma unroll
    for (int w = 1; w < kWavesPerBlock; ++w) s = join(s, joined[w]);
    // How far the expected logit, the target's or that of the teacher, is below the largest.  The sum is of powers of exact differences from the largest, which
    // was rounded: so are these (with the products rounded first, a certain token of |z| = 4000 had a loss of 1.6e-4 below 0).
    float below = 0.0f;
    bool counts;
    if constexpr (SOFT) {
        counts = p.lse2[row] != __builtin_inff();
        for (uint32_t j = tid_x(); j < p.entries.top; j += kBlock) {
            const float q = p.entries.share[row * p.entries.top + j];
            if (q != 0.0f) below = __builtin_fmaf(q, __builtin_fmaf(-p.entries.picked[row * p.entries.top + j], p.c, s.top), below);
        }
        below = sum_of_block(below, sums);
        if (tid_x() != 0) return;
    } else {
        if (tid_x() != 0) return;
        const int64_t t = token_of(p.targets, row, 0);
        counts = t >= 0 && (uint64_t)t < p.vocab;
        if (t >= 0 && !counts) atomicAdd(&p.err->n_bad_indices, 1ull);
        if (counts) below = __builtin_fmaf(-p.picked[wg_x()], p.c, s.top);
    }
    const float log_sum = __builtin_amdgcn_logf(s.sum);  // to base 2
    float loss = (below + log_sum) * kLn2;
    if constexpr (SOFT)
        loss += p.loss[row];
    else
        loss = loss < 0.0f ? 0.0f : loss;  // what roundings leave of a certain token's: a few 2^-24
    p.loss[row] = counts ? loss : 0.0f;
    if (p.lse2) p.lse2[row] = counts ? s.top + log_sum : __builtin_inff();
}

// ---- backward: rows and entries ---------------------------------------------------------------------------------

// rows[i] up to a multiple of 256; scale = {by what dz is multiplied, its inverse}: for halves, whose range is small, the power of two that takes the
// largest |dloss / T| to 2^13 to 2^14; 1 for the others.  Each workgroup looks for the largest itself.
constexpr uint32_t kRowThreads = 1024, kRowGroups = 16;
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const float *lse2, const float *dloss, uint64_t n, const TargetArgs targets, uint64_t vocab, int half, RowGradient *rows,
                                                           float *scale) {
    __shared__ float largest[kRowThreads / kWave];
    float up = 1.0f, down = 1.0f;
    if (half) {
        float most = 0.0f;
        for (uint64_t i = tid_x(); i < n; i += kRowThreads) {
            const float g = fabsf(dloss[i] / targets.temperature);
            if (lse2[i] < __builtin_inff() && g < __builtin_inff()) most = __builtin_fmaxf(most, g);
        }
        most = wave_max(most);
        if (tid_x() % kWave == 0) largest[tid_x() / kWave] = most;
        __syncthreads();
        most = largest[0];
        for (uint32_t w = 1; w < kRowThreads / kWave; ++w) most = __builtin_fmaxf(most, largest[w]);
        if (most > 0.0f) {
            int e;
            (void)frexpf(most, &e);  // most = fraction 2^e, fraction from 1/2 to 1
            e = 14 - e;
            e = e > 120 ? 120 : e < -120 ? -120 : e;
            up = ldexpf(1.0f, e);
            down = ldexpf(1.0f, -e);
        }
    }
    if (wg_x() == 0 && tid_x() == 0) {
        scale[0] = up;
        scale[1] = down;
    }
    const uint64_t padded = (n + 255) / 256 * 256;
    for (uint64_t i = wg_x() * kRowThreads + tid_x(); i < padded; i += kRowGroups * kRowThreads) {
        RowGradient r = {__builtin_inff(), 0.0f, kNoTarget, 0};
        if (i < n && lse2[i] != __builtin_inff()) {
            r.lse2 = lse2[i];
            r.gradient = dloss[i] / targets.temperature * up;
            const int64_t t = targets.logits ? -1 : token_of(targets, i, 0);
            if (t >= 0 && (uint64_t)t < vocab) r.target = (uint32_t)t;
        }
        rows[i] = r;
    }
}

// dz of the entries whose tokens lie in [first, first + columns): a thread for each entry.
template <int TYPE, int PARTS>
__global__ void __launch_bounds__(kBlock) entries_kernel(const KeepGradient<TYPE, PARTS> k, const Entries entries, uint64_t n, uint32_t columns) {
    typedef typename Element<TYPE>::type T;
    const uint64_t at = (uint64_t)wg_x() * kBlock + tid_x();
    if (at >= n * entries.top) return;
    const float q = entries.share[at];
    const uint64_t row = at / entries.top;
    const RowGradient r = k.rows[row];
    const uint32_t column = (uint32_t)entries.tokens[at] - k.first;
    if (q == 0.0f || r.gradient == 0.0f || column >= columns) return;
    T part[PARTS];
    apart<TYPE, PARTS>(r.gradient * (exp2_of(__builtin_fmaf(entries.picked[at], k.c, -r.lse2)) - q), part);
#pragma unroll
    for (int i = 0; i < PARTS; ++i) k.dz[row * k.stride + i * k.width + column] = part[i];
}

// Zeros: what a sum over nothing is.
constexpr uint32_t kZeroGroups = 8192;
__global__ void __launch_bounds__(kBlock) zero_kernel(const Target out, uint64_t rows, uint32_t columns) {
    const float none[1] = {0.0f};
    for (uint64_t at = (uint64_t)wg_x() * kBlock + tid_x(); at < rows * columns; at += (uint64_t)kZeroGroups * kBlock) write_row(out, at / columns, (uint32_t)(at % columns), columns, none);
}

// ---- the host's side ------------------------------------------------------------------------------------------

// Rows as a product can read them: where they are, or, where `layout` has rows, laid out in `space` by lay_out.
dense::Operand operand_of(const Sizes &s, const void *src, uint64_t stride, uint64_t rows, bool in_place, void *space, Layout &layout) {
    const uint32_t part = s.blocks * dense::kBlockBytes;
    layout = {src, stride, in_place ? 0 : rows, nullptr, nullptr, reinterpret_cast<u32x4 *>(space)};
    if (in_place) return {src, (rows > 1 ? stride : s.dim) * 2, (uint32_t)s.dim * 2, 0, 0, (uint32_t)((s.dim - 1) % dense::kBlockElements / 8 + 1)};
    return {space, s.row, (uint32_t)s.row, part, 0, 8};
}
template <typename T>
void lay_out(const Sizes &s, const Layout &a, const Layout &b, hipStream_t to) {
    const uint32_t pieces = s.blocks * dense::kBlockBytes / 16;
    in_launches((a.rows + b.rows) * pieces,
                [&](uint64_t first, unsigned groups) { hipLaunchKernelGGL((lay_out_kernel<T>), dim3(groups), dim3(kBlock), 0, to, a, b, (uint32_t)s.dim, pieces, first); });
}
dense::Operand in_terms(dense::Operand o, uint32_t parts) {
    o.parts = parts;
    return o;
}

TargetArgs targets_of(const cnr_targets &t) {
    TargetArgs a;
    a.tokens = t.tokens;
    a.logits = t.logits;
    a.token_stride = t.token_stride;
    a.logit_stride = t.logit_stride;
    a.top = (uint32_t)t.top;
    a.token_type = t.token_type;
    a.logit_type = t.logit_type;
    a.temperature = t.logits ? t.temperature : 1.0f;
    return a;
}

// Where a state holds a teacher's entries, behind a number for each row.
Entries entries_of(const float *state, uint64_t n, uint64_t top) {
    float *at = const_cast<float *>(state ? state + n : nullptr);
    return {reinterpret_cast<int32_t *>(at), at + n * top, at + 2 * n * top, (uint32_t)top};
}

// The type of the elements that products of a type are made of.
template <int TYPE>
constexpr int kOf = TYPE == CNR_FLOAT_F16 ? CNR_FLOAT_F16 : CNR_FLOAT_BF16;

template <int TYPE, bool GRADIENT>
void narrow(const NarrowArgs &a, uint32_t fragments, hipStream_t to) {
    const dim3 grid((unsigned)cnr_ceil_div(a.vocab, 16 * fragments)), threads(kBlock);
    if (a.n <= 16) {
        if (fragments == 2)
            hipLaunchKernelGGL((narrow_kernel<TYPE, 1, 2, 2, GRADIENT>), grid, threads, 0, to, a);
        else
            hipLaunchKernelGGL((narrow_kernel<TYPE, 1, 1, 4, GRADIENT>), grid, threads, 0, to, a);
    } else if constexpr (TYPE == CNR_FLOAT_F32) {
        if (a.n <= 32) {
            if (fragments == 2)
                hipLaunchKernelGGL((narrow_kernel<TYPE, 2, 2, 1, GRADIENT>), grid, threads, 0, to, a);
            else
                hipLaunchKernelGGL((narrow_kernel<TYPE, 2, 1, 2, GRADIENT>), grid, threads, 0, to, a);
        } else {
            if (fragments == 2)
                hipLaunchKernelGGL((narrow_kernel<TYPE, 4, 2, 1, GRADIENT>), grid, threads, 0, to, a);
            else
                hipLaunchKernelGGL((narrow_kernel<TYPE, 4, 1, 1, GRADIENT>), grid, threads, 0, to, a);
        }
    }
}

template <int TYPE>
void forward(cnr_ctx *ctx, const cnr_vocabulary &v, const cnr_targets &t, float *loss, float *state, void *workspace, hipStream_t to) {
    typedef typename Element<TYPE>::type T;
    const Sizes s = sizes_of(v.n, v.vocab, v.dim, v.type);
    const bool in_place = whole_rows(v.type, v.weight, v.weight_stride, v.dim, v.vocab);
    const ForwardPlan f = forward_plan(ctx, s);
    uint8_t *space = reinterpret_cast<uint8_t *>(workspace);
    const T *hidden = reinterpret_cast<const T *>(v.hidden), *weight = reinterpret_cast<const T *>(v.weight);
    LossArgs l;
    l.targets = targets_of(t);
    l.vocab = v.vocab;
    l.picked = reinterpret_cast<const float *>(space + f.picked);
    l.parts = reinterpret_cast<const Stats *>(space + f.parts);
    l.n_parts = f.n_parts;
    l.loss = loss;
    l.lse2 = state;
    l.entries = entries_of(state, v.n, t.top);
    l.err = ctx->dev_err;
    const float c = l.c = kLog2e / l.targets.temperature;
    const uint32_t columns = f.narrow ? 16 * f.fragments : dense::kTiles[f.tiles.kind].columns;
    TeacherArgs teacher = {l.targets, v.vocab, 0, l.entries, loss, state, f.narrow || !v.vocab ? nullptr : reinterpret_cast<uint16_t *>(space + f.begins), f.n_parts, columns,
                           ctx->dev_err};
    for (uint64_t row0 = 0; row0 < v.n; row0 += f.rows) {
        const uint64_t rows = v.n - row0 < f.rows ? v.n - row0 : f.rows;
        Stats *parts = reinterpret_cast<Stats *>(space + f.parts);
        float *picked = reinterpret_cast<float *>(space + f.picked);
        const T *x = hidden + row0 * v.hidden_stride;
        teacher.row0 = row0;
        Entries entries = l.entries;
        entries.tokens += row0 * t.top;
        entries.picked += row0 * t.top;
        if (t.logits) hipLaunchKernelGGL(teacher_kernel, dim3((unsigned)rows), dim3(kBlock), 0, to, teacher);
        if (f.n_parts == 0) {
        } else if (f.narrow) {
            const NarrowArgs a = {x, weight, v.hidden_stride, v.weight_stride, (uint32_t)rows, (uint32_t)v.vocab, (uint32_t)v.dim, c, parts, f.n_parts, t.logits != nullptr,
                                  l.targets, picked, entries, nullptr, 0, nullptr};
            narrow<TYPE, false>(a, f.fragments, to);
        } else {
            const Terms terms = s.parts == 3 ? kOfFloats : kOne;
            Layout of_x, of_w;
            const dense::Operand x_at = in_terms(operand_of(s, x, v.hidden_stride, rows, whole_rows(v.type, x, v.hidden_stride, v.dim, rows), space + f.hidden, of_x), terms.down);
            const uint64_t most = in_place ? rounded((1ull << 22) / cnr_ceil_div(rows, 64) * 64, 256) : f.piece;
            for (uint64_t v0 = 0; v0 < v.vocab; v0 += most) {
                const uint64_t width = v.vocab - v0 < most ? v.vocab - v0 : most;
                const dense::Operand w_at = in_terms(operand_of(s, weight + v0 * v.weight_stride, v.weight_stride, width, in_place, space + f.weight, of_w), terms.across);
                lay_out<T>(s, of_w, of_x, to);
                of_x.rows = 0;
                const dense::Args args = {w_at, x_at, (uint32_t)width, (uint32_t)rows, s.blocks, 0, terms.number, 1};
                Stats *of_piece = parts + v0 / columns;
                if (t.logits)
                    dense::launch<kOf<TYPE>, false, false>(args, f.tiles.kind,
                                                           KeepStats<true>{of_piece, f.n_parts, c, (uint32_t)v0, l.targets, row0, nullptr, teacher.begins + v0 / columns, entries}, to);
                else
                    dense::launch<kOf<TYPE>, false, false>(args, f.tiles.kind, KeepStats<false>{of_piece, f.n_parts, c, (uint32_t)v0, l.targets, row0, picked, nullptr, entries}, to);
            }
        }
        l.row0 = row0;
        if (t.logits)
            hipLaunchKernelGGL(loss_kernel<true>, dim3((unsigned)rows), dim3(kBlock), 0, to, l);
        else
            hipLaunchKernelGGL(loss_kernel<false>, dim3((unsigned)rows), dim3(kBlock), 0, to, l);
    }
}

template <int TYPE, bool DOWN>
void product(const dense::Args &args, const dense::Plan &plan, const KeepSum &k, hipStream_t to) {
    dense::Args a = args;
    a.splits = plan.splits;
    dense::launch<kOf<TYPE>, true, DOWN>(a, plan.kind, k, to);
    if (a.splits > 1)
        hipLaunchKernelGGL((join_sums_kernel<1>), dim3((unsigned)cnr_ceil_div((uint64_t)a.rows * (k.partial_stride / 4), kBlock)), dim3(kBlock), 0, to, k, a.rows, a.columns, a.splits);
}
Target from_row(Target t, uint64_t row) {
    if (t.out) t.out = reinterpret_cast<uint8_t *>(t.out) + row * t.stride * cnr_float_bytes((cnr_float_type)t.type);
    return t;
}
template <int TYPE, bool DOWN>
void product(cnr_ctx *ctx, const dense::Args &args, const KeepSum &k, hipStream_t to) {
    const dense::Plans plans = dense::plans_of(ctx, args.columns, args.rows, (uint64_t)args.blocks * args.terms, (float)cnr_float_bytes((cnr_float_type)k.out.type) * (k.there.out ? 2.0f : 1.0f),
                                               kPartBytes);
    dense::Args a = args;
    a.rows = (uint32_t)plans.first_rows;
    product<TYPE, DOWN>(a, plans.first, k, to);
    if (plans.first_rows == args.rows) return;
    KeepSum rest = k;
    rest.out = from_row(k.out, plans.first_rows);
    rest.there = from_row(k.there, plans.first_rows);
    if (rest.rows) rest.rows += plans.first_rows;
    a.rows = args.rows - a.rows;
    const uint64_t skipped = plans.first_rows * (DOWN ? 2 : a.down.stride);
    a.down.at = reinterpret_cast<const uint8_t *>(a.down.at) + skipped;
    if (DOWN) a.down.row_bytes -= (uint32_t)skipped;
    product<TYPE, DOWN>(a, plans.rest, rest, to);
}

// The backward pass of few rows.
template <int TYPE>
void narrow_backward(cnr_ctx *ctx, const cnr_vocabulary &v, const cnr_targets &t, const float *state, const float *dloss, const Target &dhidden, const Target &dweight, bool accumulate,
                     const BackwardPlan &b, uint8_t *space, hipStream_t to) {
    const TargetArgs targets = targets_of(t);
    RowGradient *rows = reinterpret_cast<RowGradient *>(space + b.rows);
    hipLaunchKernelGGL(rows_kernel, dim3(1), dim3(kRowThreads), 0, to, state, dloss, v.n, targets, v.vocab, 0, rows, reinterpret_cast<float *>(space + b.scale));
    const uint32_t n = (uint32_t)v.n, dim = (uint32_t)v.dim;
    const auto by_rows = [&](const auto &launch) {
        if (n <= 16) return launch(std::integral_constant<int, 1>());
        if constexpr (TYPE == CNR_FLOAT_F32) return n <= 32 ? launch(std::integral_constant<int, 2>()) : launch(std::integral_constant<int, 4>());
    };
    const uint64_t stride = rounded(v.dim, 4), by_room = kPartBytes / 4 / (v.n * stride * sizeof(float));
    const Target between = {space + b.sum, v.dim, CNR_FLOAT_F32}, none = {nullptr, 0, CNR_FLOAT_F32};
    SlabArgs s = {};
    s.dz = reinterpret_cast<float *>(space + b.dz);
    s.dim = dim;
    s.n = n;
    s.groups = (uint32_t)cnr_ceil_div(v.dim, 64);
    for (uint64_t v0 = 0; v0 < v.vocab; v0 += b.piece) {
        const uint64_t width = least(v.vocab - v0, b.piece);
        const void *weight = reinterpret_cast<const typename Element<TYPE>::type *>(v.weight) + v0 * v.weight_stride;
        const NarrowArgs a = {v.hidden, weight, v.hidden_stride, v.weight_stride, n, (uint32_t)width, dim, kLog2e / targets.temperature, nullptr, 0, false, targets, nullptr, {},
                              rows, (uint32_t)v0, reinterpret_cast<float *>(space + b.dz)};
        narrow<TYPE, true>(a, narrow_fragments(v.n, width), to);
        if (t.logits && t.top)
            hipLaunchKernelGGL(narrow_entries_kernel, dim3((unsigned)cnr_ceil_div(v.n * t.top, kBlock)), dim3(kBlock), 0, to, a, entries_of(state, v.n, t.top), (uint32_t)padded_rows(v.n));
        // Sixteen waves to a compute unit, slabs of 64 tokens at least, parts of sums of up to a quarter of the room for them (they are read again).
        const uint64_t wanted = least(cnr_ceil_div(16ull * ctx->n_cu, s.groups), cnr_ceil_div(width, 64));
        s.vocab = (uint32_t)width;
        if (dhidden.out) {
            s.slabs = (uint32_t)least(wanted, by_room ? by_room : 1);
            s.matrix = weight;
            s.stride = v.weight_stride;
            s.partial = reinterpret_cast<float *>(space + b.partial);
            s.partial_stride = stride;
            by_rows([&](auto g) {
                hipLaunchKernelGGL((narrow_hidden_kernel<TYPE, decltype(g)::value>), dim3((unsigned)cnr_ceil_div((uint64_t)s.groups * s.slabs, kWavesPerBlock)), dim3(kBlock), 0, to, s);
            });
            const KeepSum sum = {v0 + width == v.vocab ? dhidden : between, v0 ? between : none, nullptr, s.partial, stride, rows};
            hipLaunchKernelGGL((join_sums_kernel<16>), dim3((unsigned)cnr_ceil_div(v.n * (stride / 4), kBlock / 16)), dim3(kBlock), 0, to, sum, n, dim, s.slabs);
        }
        if (dweight.out) {
            s.slabs = (uint32_t)wanted;
            s.matrix = v.hidden;
            s.stride = v.hidden_stride;
            s.lse2 = state;
            s.dloss = dloss;
            s.out = from_row(dweight, v0);
            s.there = accumulate ? s.out : none;
            by_rows([&](auto g) {
                hipLaunchKernelGGL((narrow_weight_kernel<TYPE, decltype(g)::value>), dim3((unsigned)cnr_ceil_div((uint64_t)s.groups * s.slabs, kWavesPerBlock)), dim3(kBlock), 0, to, s);
            });
        }
    }
}

template <int TYPE, int PARTS>
void backward(cnr_ctx *ctx, const cnr_vocabulary &v, const cnr_targets &t, const float *state, const float *dloss, void *dhidden, uint64_t dhidden_stride, void *dweight,
              cnr_float_type dweight_type, uint64_t dweight_stride, bool accumulate, void *workspace, hipStream_t to) {
    typedef typename Element<TYPE>::type T;
    typedef typename Element<kOf<TYPE>>::type Part;
    const Sizes s = sizes_of(v.n, v.vocab, v.dim, v.type);
    const bool in_place = whole_rows(v.type, v.weight, v.weight_stride, v.dim, v.vocab);
    const bool wide = TYPE != CNR_FLOAT_F32 && dweight && dweight_type == CNR_FLOAT_F32;
    const BackwardPlan b = backward_plan(ctx, s, wide, in_place);
    uint8_t *space = reinterpret_cast<uint8_t *>(workspace);
    if (b.narrow)
        return narrow_backward<TYPE>(ctx, v, t, state, dloss, {dhidden, dhidden_stride, v.type}, {dweight, dweight_stride, dweight_type}, accumulate, b, space, to);
    const T *weight = reinterpret_cast<const T *>(v.weight);
    const TargetArgs targets = targets_of(t);
    const Entries entries = entries_of(state, v.n, t.top);
    RowGradient *rows = reinterpret_cast<RowGradient *>(space + b.rows);
    float *scale = reinterpret_cast<float *>(space + b.scale);
    hipLaunchKernelGGL(rows_kernel, dim3((unsigned)least(cnr_ceil_div(v.n, kRowThreads), kRowGroups)), dim3(kRowThreads), 0, to, state, dloss, v.n, targets, v.vocab, TYPE == CNR_FLOAT_F16,
                       rows, scale);
    Layout of_x, of_w;
    const dense::Operand x = operand_of(s, v.hidden, v.hidden_stride, v.n, false, space + b.hidden_at, of_x);
    of_x.lse2 = state;
    of_x.dloss = dloss;
    KeepGradient<kOf<TYPE>, PARTS> k;
    k.dz = reinterpret_cast<Part *>(space + b.dz);
    k.rows = rows;
    k.c = kLog2e / targets.temperature;
    KeepSum sum;
    sum.scale = TYPE == CNR_FLOAT_F16 ? scale + 1 : nullptr;
    sum.partial = reinterpret_cast<float *>(space + b.partial);
    sum.partial_stride = rounded(v.dim, 4);
    const Target between = {space + b.sum, v.dim, CNR_FLOAT_F32}, none = {nullptr, 0, CNR_FLOAT_F32};
    // (two parts for the hidden states too where rows are few)
    const Terms logits = TYPE == CNR_FLOAT_F32 ? kOfFloats : kOne, to_hidden = TYPE != CNR_FLOAT_F32 && v.n <= kTwoPartRows ? kOfTwoParts : logits;
    const Terms to_weight = TYPE == CNR_FLOAT_F32 ? kOfFloats : PARTS == 3 ? kOfThreeParts : PARTS == 2 ? kOfTwoParts : kOne;
    const uint32_t n = (uint32_t)v.n, dim = (uint32_t)v.dim;
    for (uint64_t v0 = 0; v0 < v.vocab; v0 += b.piece) {
        const uint32_t width = (uint32_t)(v.vocab - v0 < b.piece ? v.vocab - v0 : b.piece), blocks = (uint32_t)cnr_ceil_div(width, dense::kBlockElements);
        k.width = (uint64_t)blocks * dense::kBlockElements;
        k.stride = PARTS * k.width;
        k.first = (uint32_t)v0;
        const dense::Operand w = operand_of(s, weight + v0 * v.weight_stride, v.weight_stride, width, in_place, space + b.weight_at, of_w);
        lay_out<T>(s, of_w, of_x, to);
        of_x.rows = 0;
        const dense::Plan tiles = dense::plan_of(ctx, width, v.n, s.blocks * logits.number, 2.0f * PARTS, 0);
        dense::launch<kOf<TYPE>, false, false>(dense::Args{in_terms(w, logits.across), in_terms(x, logits.down), width, n, s.blocks, 0, logits.number, 1}, tiles.kind, k, to);
        if (t.logits && t.top)
            hipLaunchKernelGGL((entries_kernel<kOf<TYPE>, PARTS>), dim3((unsigned)cnr_ceil_div(v.n * t.top, kBlock)), dim3(kBlock), 0, to, k, entries, v.n, width);
        const dense::Operand dz = {k.dz, k.stride * 2, (uint32_t)(k.stride * 2), (uint32_t)(k.width * 2), 0, 8};
        if (dhidden) {
            sum.rows = rows;
            sum.there = v0 == 0 ? none : between;
            sum.out = v0 + width == v.vocab ? Target{dhidden, dhidden_stride, v.type} : between;
            product<TYPE, false>(ctx, dense::Args{in_terms(w, to_hidden.across), in_terms(dz, to_hidden.down), dim, n, blocks, width, to_hidden.number, 1}, sum, to);
        }
        if (dweight) {
            sum.out = {reinterpret_cast<uint8_t *>(dweight) + v0 * dweight_stride * cnr_float_bytes(dweight_type), dweight_stride, dweight_type};
            sum.rows = nullptr;
            sum.there = accumulate ? sum.out : none;
            product<TYPE, true>(ctx, dense::Args{in_terms(x, to_weight.across), in_terms(dz, to_weight.down), dim, width, (uint32_t)cnr_ceil_div(v.n, dense::kBlockElements), n,
                                            to_weight.number, 1}, sum, to);
        }
    }
}

void zeros(const Target &out, uint64_t rows, uint64_t columns, hipStream_t to) {
    if (rows && columns) hipLaunchKernelGGL(zero_kernel, dim3(kZeroGroups), dim3(kBlock), 0, to, out, rows, (uint32_t)columns);
}

constexpr float kMinTemperature = 0x1p-126f;  // log2(e) / T stays finite: 0 / T is 0
cnr_status checked(const cnr_vocabulary *v, const cnr_targets *t) {
    if (!v || !t || !cnr_valid_float_type(v->type) || (t->token_type != CNR_IDX_I32 && t->token_type != CNR_IDX_I64)) return CNR_E_INVALID;
    if (v->hidden_stride < v->dim || v->weight_stride < v->dim || t->token_stride < t->top) return CNR_E_INVALID;
    if (t->logits ? !cnr_valid_float_type(t->logit_type) || t->logit_stride < t->top || !(t->temperature >= kMinTemperature) || t->temperature > 3e38f : t->top != 1) return CNR_E_INVALID;
    if (v->n > kMaxRows || v->vocab > kMaxVocabulary || v->dim > kMaxDim || t->top > kMaxTop) return CNR_E_TOO_LARGE;
    if (v->n && ((!t->tokens && t->top) || (v->dim && (!v->hidden || (v->vocab && !v->weight))))) return CNR_E_INVALID;
    const size_t e = cnr_float_bytes(v->type);
    if (!cnr_aligned(v->hidden, e) || !cnr_aligned(v->weight, e) || !cnr_aligned(t->tokens, t->token_type == CNR_IDX_I64 ? 8 : 4) ||
        (t->logits && !cnr_aligned(t->logits, cnr_float_bytes(t->logit_type))))
        return CNR_E_ALIGN;
    return CNR_OK;
}

}  // namespace

extern "C" {

size_t cnr_loss_state_floats(uint64_t n, uint64_t top) { return n > kMaxRows || top > kMaxTop ? 0 : (size_t)(n * (1 + 3 * top)); }

size_t cnr_loss_workspace_bytes(uint64_t n, uint64_t vocab, uint64_t dim, cnr_float_type type, int training, cnr_float_type dweight_type) {
    if (n == 0 || vocab == 0 || n > kMaxRows || vocab > kMaxVocabulary || dim > kMaxDim || !cnr_valid_float_type(type)) return 0;
    return (size_t)room_for(sizes_of(n, vocab, dim, type), training != 0, type != CNR_FLOAT_F32 && dweight_type == CNR_FLOAT_F32);
}

cnr_status cnr_vocabulary_loss(cnr_ctx *ctx, const cnr_vocabulary *vocabulary, const cnr_targets *targets, float *loss, float *state, void *workspace, size_t workspace_bytes,
                               void *stream) {
    if (!ctx) return CNR_E_INVALID;
    cnr_status st = checked(vocabulary, targets);
    if (st != CNR_OK) return st;
    const cnr_vocabulary &v = *vocabulary;
    if (v.n == 0) return CNR_OK;
    if (targets->logits && !state) return CNR_E_INVALID;
    if (!loss || workspace_bytes < cnr_loss_workspace_bytes(v.n, v.vocab, v.dim, v.type, 0, v.type) || (workspace_bytes && !workspace)) return CNR_E_INVALID;
    if (!cnr_aligned(loss, 4) || !cnr_aligned(state, 4) || !cnr_aligned(workspace, 256)) return CNR_E_ALIGN;
    if (forward_plan(ctx, sizes_of(v.n, v.vocab, v.dim, v.type)).bytes > workspace_bytes) return CNR_E_INVALID;
    st = cnr_enter(ctx);
    if (st != CNR_OK) return st;
    if (v.type == CNR_FLOAT_F32)
        forward<CNR_FLOAT_F32>(ctx, v, *targets, loss, state, workspace, as_stream(stream));
    else if (v.type == CNR_FLOAT_BF16)
        forward<CNR_FLOAT_BF16>(ctx, v, *targets, loss, state, workspace, as_stream(stream));
    else
        forward<CNR_FLOAT_F16>(ctx, v, *targets, loss, state, workspace, as_stream(stream));
    return cnr_launch_status(ctx);
}

cnr_status cnr_vocabulary_loss_backward(cnr_ctx *ctx, const cnr_vocabulary *vocabulary, const cnr_targets *targets, const float *state, const float *dloss, void *dhidden,
                                        uint64_t dhidden_stride, void *dweight, cnr_float_type dweight_type, uint64_t dweight_stride, int accumulate, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    if (!ctx) return CNR_E_INVALID;
    cnr_status st = checked(vocabulary, targets);
    if (st != CNR_OK) return st;
    const cnr_vocabulary &v = *vocabulary;
    if (dhidden && dhidden_stride < v.dim) return CNR_E_INVALID;
    if (dweight && (dweight_stride < v.dim || (dweight_type != v.type && dweight_type != CNR_FLOAT_F32))) return CNR_E_INVALID;
    if (v.n && (!state || !dloss)) return CNR_E_INVALID;
    const size_t needed = cnr_loss_workspace_bytes(v.n, v.vocab, v.dim, v.type, 1, dweight ? dweight_type : v.type);
    if (workspace_bytes < needed || (needed && !workspace)) return CNR_E_INVALID;
    if (!cnr_aligned(state, 4) || !cnr_aligned(dloss, 4) || !cnr_aligned(dhidden, cnr_float_bytes(v.type)) ||
        (dweight && !cnr_aligned(dweight, cnr_float_bytes(dweight_type))) || !cnr_aligned(workspace, 256))
        return CNR_E_ALIGN;
    if (v.dim == 0 || (!dhidden && !dweight)) return CNR_OK;
    st = cnr_enter(ctx);
    if (st != CNR_OK) return st;
    hipStream_t to = as_stream(stream);
    if (v.n == 0 || v.vocab == 0) {  // sums over nothing
        if (dhidden) zeros({dhidden, dhidden_stride, v.type}, v.n, v.dim, to);
        if (dweight && !accumulate) zeros({dweight, dweight_stride, dweight_type}, v.vocab, v.dim, to);
        return cnr_launch_status(ctx);
    }
    const bool wide = v.type != CNR_FLOAT_F32 && dweight && dweight_type == CNR_FLOAT_F32;
    const Sizes sizes = sizes_of(v.n, v.vocab, v.dim, v.type);
    const uint32_t parts = dz_parts(sizes, wide);
    if (backward_plan(ctx, sizes, wide, whole_rows(v.type, v.weight, v.weight_stride, v.dim, v.vocab)).bytes > workspace_bytes)
        return CNR_E_INVALID;
    auto call = [&](auto kind, auto part) {
        backward<decltype(kind)::value, decltype(part)::value>(ctx, v, *targets, state, dloss, dhidden, dhidden_stride, dweight, dweight_type, dweight_stride, accumulate != 0,
                                                               workspace, to);
    };
    if (v.type == CNR_FLOAT_F32)
        call(std::integral_constant<int, CNR_FLOAT_F32>(), std::integral_constant<int, 3>());
    else if (v.type == CNR_FLOAT_BF16)
        parts == 3   ? call(std::integral_constant<int, CNR_FLOAT_BF16>(), std::integral_constant<int, 3>())
        : parts == 2 ? call(std::integral_constant<int, CNR_FLOAT_BF16>(), std::integral_constant<int, 2>())
                     : call(std::integral_constant<int, CNR_FLOAT_BF16>(), std::integral_constant<int, 1>());
    else
        parts == 2 ? call(std::integral_constant<int, CNR_FLOAT_F16>(), std::integral_constant<int, 2>())
                   : call(std::integral_constant<int, CNR_FLOAT_F16>(), std::integral_constant<int, 1>());
    return cnr_launch_status(ctx);
}

}  // extern "C"
