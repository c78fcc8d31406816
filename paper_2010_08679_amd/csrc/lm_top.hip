// The largest logits of each row with their tokens, and the logarithm of the sum of all exponentials.
//
// One workgroup a row, which it reads once.  The sum of exponentials is taken along, and the largest of every sixteen bytes (of several such vectors, in long
// rows) stays in a register.  The top-th largest of the threads' own largest is at most the top-th largest of all, and hardly more elements reach it than
// are wanted: the vectors whose largest does are read again, all at once, and their elements that reach it are collected in LDS, in any order; each finds
// its place by counting those before it.  Keys (the value, then the lower token) are all different, so the order they were collected in does not matter.
// Where too many reach the bound, they are equal values, of which the first are taken in order, or the largest are all in a few threads' shares, and the bound is raised
// digit by digit.
//
// 64 of 8192 x 32000 bfloat16 101 us, 5.2 TB/s, of 512 x 131072 34 us, 3.9 TB/s (177 and 60 with rows held in registers, so that fewer of them share a compute unit; 312
// and 70 read twice), 94 where all are equal; 50 of 1 x 50257 floats 12 us, one workgroup's latency.
#include "cnr_loss.h"
#include "lm_common.h"

namespace {


struct TopArgs {
    const void *logits;
    uint64_t stride;
    uint32_t vocab, top;
    uint64_t n;
    int32_t *tokens;
    void *values;
    float *lse;
};

constexpr uint32_t kNan = 0xffffffffu, kZero = 0x80000000u;
// In the order of the values, NaN last.
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t u = __float_as_uint(v);
    if (v != v) return kNan;
    if (v == 0.0f) return kZero;
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
constexpr float kLog2e = 1.44269504088896340736f;
constexpr uint32_t kInfinity = 0xff800000u, kMinusInfinity = 0x007fffffu;
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key ^ (key >> 31 ? 0x80000000u : 0xffffffffu)); }
// All of a row's keys are different, and larger ones come first.
__device__ __forceinline__ uint64_t place_of(uint32_t key, uint32_t token) { return (uint64_t)key << 32 | (uint32_t)~token; }

struct Exponentials {
    float top, sum;
};
// The same of a wave's, in all lanes.
__device__ __forceinline__ float max_of(float v, float w) { return __builtin_fmaxf(v, w); }
__device__ __forceinline__ Exponentials over_wave(Exponentials e) {
    float top = e.top;
    top = max_of(top, dpp_f<0xB1>(top));
    top = max_of(top, dpp_f<0x4E>(top));
    top = max_of(top, dpp_f<0x141>(top));
    top = max_of(top, dpp_f<0x140>(top));
    top = max_of(top, __shfl_xor(top, 16));
    top = max_of(top, __shfl_xor(top, 32));
    float sum = e.sum * __expf(e.top - (top == -__builtin_inff() ? 0.0f : top));
    sum += dpp_f<0xB1>(sum);
    sum += dpp_f<0x4E>(sum);
    sum += dpp_f<0x141>(sum);
    sum += dpp_f<0x140>(sum);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    return {top, sum};
}

// each(element's value, token) for all of a row's elements, sixteen bytes to a thread at a time.
template <int TYPE, uint32_t THREADS, typename Each>
__device__ __forceinline__ void for_row(const typename Element<TYPE>::type *row, uint32_t vocab, const Each &each) {
    typedef typename Element<TYPE>::type T;
    constexpr uint32_t kPer = 16 / sizeof(T);
    for (uint32_t at = tid_x() * kPer; at < vocab; at += THREADS * kPer) {
        if (at + kPer <= vocab) {
            const Pack<T, kPer> w = *reinterpret_cast<const Pack<T, kPer> *>(row + at);
#pragma unroll
            for (uint32_t j = 0; j < kPer; ++j) each(Element<TYPE>::wide(w.v[j]), at + j);
        } else {
            for (uint32_t j = at; j < vocab; ++j) each(Element<TYPE>::wide(row[j]), j);
        }
    }
}

template <uint32_t THREADS>
struct Lds {
    static constexpr uint32_t kRoom = 4 * THREADS;
    uint64_t found[kRoom];
    uint32_t hits[2 * THREADS];
    uint32_t largest[THREADS];
    uint32_t bins[256];
    Exponentials parts[THREADS / kWave];
    uint32_t n_found, n_hits, digit, above;
    uint32_t bound;
};

// GROUPS groups of EACH vectors to a thread, 0: of as many as the row takes.  Rows with a NaN or an infinity are looked through again by their keys.
template <int TYPE, uint32_t THREADS, uint32_t GROUPS, uint32_t EACH>
__global__ void __launch_bounds__(THREADS, EACH == 2 ? 8 : 1) top_kernel(const TopArgs p) {
    typedef typename Element<TYPE>::type T;
    constexpr uint32_t kPer = 16 / sizeof(T);
    typedef Pack<T, kPer> Vector;
    constexpr uint32_t kWaves = THREADS / kWave, kRoom = Lds<THREADS>::kRoom;
    __shared__ Lds<THREADS> lds;
    const uint32_t lane = tid_x() % kWave, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid_x() / kWave));
    const uint64_t row_at = wg_x();
    const T *row = reinterpret_cast<const T *>(p.logits) + row_at * p.stride;
    const uint32_t top = p.top < p.vocab ? p.top : p.vocab;

    // Whole vectors, thread by thread, and an element of what is left for each of the first threads; -infinity beyond the row's end.
    const uint32_t whole = p.vocab / kPer, left = p.vocab % kPer, each = EACH ? EACH : (whole + GROUPS * THREADS - 1) / (GROUPS * THREADS);
    float most[GROUPS];  // of each group of `each` vectors
    const float last = tid_x() < left ? Element<TYPE>::wide(row[whole * kPer + tid_x()]) : -__builtin_inff();
    Exponentials e = {last, last == -__builtin_inff() ? 0.0f : __expf(last - last)};
    auto load = [&](uint32_t i) {  // the thread's i-th vector
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : TYPE == CNR_FLOAT_BF16 ? 0xff80ff80u : 0xfc00fc00u;
        u32x4 w = {kNone, kNone, kNone, kNone};
        if (i * THREADS + tid_x() < whole) w = load16(row + (uint64_t)(i * THREADS + tid_x()) * kPer);
        return w;
    };
    auto add = [&](u32x4 words) {
        // (the compiler would have the elements of many as floats at once)
        asm volatile("" : "+v"(words), "+v"(e.sum));
        const Vector w = __builtin_bit_cast(Vector, words);
        float largest = Element<TYPE>::wide(w.v[0]);
#pragma unroll
        for (uint32_t j = 1; j < kPer; ++j) largest = __builtin_fmaxf(largest, Element<TYPE>::wide(w.v[j]));
        const float now = __builtin_fmaxf(e.top, largest), from = now == -__builtin_inff() ? 0.0f : now;  // (differences first: the type's lowest value times log2(e) is infinite)
        float sum = 0.0f;
#pragma unroll
        for (uint32_t j = 0; j < kPer; ++j) sum += __builtin_amdgcn_exp2f((Element<TYPE>::wide(w.v[j]) - from) * kLog2e);
        e.sum = __builtin_fmaf(e.sum, __builtin_amdgcn_exp2f((e.top - from) * kLog2e), sum);
        e.top = now;
        return largest;
    };
    if constexpr (EACH == 0) {
#pragma unroll
        for (uint32_t q = 0; q < GROUPS; ++q) {
            most[q] = -__builtin_inff();
            for (uint32_t i = q * each; i < (q + 1) * each; i += 4) {
                u32x4 w[4];
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) w[j] = i + j < (q + 1) * each ? load(i + j) : load(0xffffffffu / THREADS);
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) most[q] = __builtin_fmaxf(most[q], add(w[j]));
            }
        }
    } else {
        constexpr uint32_t kAtOnce = 4;
#pragma unroll
        for (uint32_t first = 0; first < GROUPS * EACH; first += kAtOnce) {
            u32x4 w[kAtOnce];
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j) w[j] = load(first + j);
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j) {
                const float largest = add(w[j]);
                float &of = most[(first + j) / EACH];
                of = (first + j) % EACH ? __builtin_fmaxf(of, largest) : largest;
            }
        }
    }
    lds.largest[tid_x()] = key_of(e.top);
    if (tid_x() == 0) lds.n_found = lds.n_hits = 0;
    e = over_wave(e);
    if (lane == 0) lds.parts[wave] = e;
    __syncthreads();
    e = {lds.parts[0].top, 0.0f};
#pragma unroll
    for (uint32_t w = 1; w < kWaves; ++w) e.top = __builtin_fmaxf(e.top, lds.parts[w].top);
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) e.sum = __builtin_fmaf(lds.parts[w].sum, __expf(lds.parts[w].top - (e.top == -__builtin_inff() ? 0.0f : e.top)), e.sum);
    // (a NaN, or the difference of two infinities, stays in the sum)
    const bool odd = e.sum != e.sum;
    if (odd) {
        uint32_t largest = 0;
        for_row<TYPE, THREADS>(row, p.vocab, [&](float v, uint32_t) {
            const uint32_t key = key_of(v);
            largest = key > largest ? key : largest;
        });
        lds.largest[tid_x()] = largest;
        __syncthreads();
    }
    if (wave == 0 && top) {
        // The largest bound that at least `top` of the threads' largest reach, to 16 bits.
        uint32_t own[THREADS / kWave], bound = 0;
#pragma unroll
        for (uint32_t i = 0; i < THREADS / kWave; ++i) own[i] = lds.largest[i * kWave + lane];
        for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
            uint32_t reach = 0;
#pragma unroll
            for (uint32_t i = 0; i < THREADS / kWave; ++i) reach += (uint32_t)__popcll(__ballot(own[i] >= (bound | bit)));
            if (reach >= top) bound |= bit;
        }
        if (lane == 0) lds.bound = bound;
    } else if (wave == 1 && p.lse) {
        uint32_t largest = 0;
        if (odd)
            for (uint32_t i = lane; i < THREADS; i += kWave) largest = lds.largest[i] > largest ? lds.largest[i] : largest;
#pragma unroll
        for (int by = 1; by < kWave; by *= 2) {
            const uint32_t other = (uint32_t)__shfl_xor((int)largest, by);
            largest = other > largest ? other : largest;
        }
        if (lane == 0) p.lse[row_at] = !odd ? e.top + __logf(e.sum) : largest > kInfinity ? __builtin_nanf("") : __builtin_inff();
    }
    if (!p.tokens && !p.values) return;
    __syncthreads();
    bool again = odd;  // the whole row is looked through
    auto collect = [&](uint64_t from) {
        auto take = [&](float v, uint32_t token) {
            const uint64_t place = place_of(key_of(v), token);
            // (once there are too many, there is no need to count on)
            if (place >= from && token < p.vocab && *reinterpret_cast<volatile uint32_t *>(&lds.n_found) <= kRoom) {
                const uint32_t at = atomicAdd(&lds.n_found, 1u);
                if (at < kRoom) lds.found[at] = place;
            }
        };
        if (again) {
            for_row<TYPE, THREADS>(row, p.vocab, take);
        } else {
            const uint32_t hits = lds.n_hits;
            for (uint32_t i = tid_x(); i < hits * each; i += THREADS) {
                const uint32_t hit = lds.hits[i / each], at = (hit / THREADS * each + i % each) * THREADS + hit % THREADS;
                if (at >= whole) continue;
                const Vector w = __builtin_bit_cast(Vector, load16(row + (uint64_t)at * kPer));
#pragma unroll
                for (uint32_t j = 0; j < kPer; ++j) take(Element<TYPE>::wide(w.v[j]), at * kPer + j);
            }
            if (tid_x() < left) take(last, whole * kPer + tid_x());
        }
        __syncthreads();
    };
    const uint32_t bound = lds.bound;
    if (top && !odd) {
        const float least = bound <= kMinusInfinity ? -__builtin_inff() : value_of(bound);
#pragma unroll
        for (uint32_t q = 0; q < GROUPS; ++q) {
            if (!(most[q] >= least)) continue;
            const uint32_t at = atomicAdd(&lds.n_hits, 1u);
            if (at < 2 * THREADS) lds.hits[at] = q * THREADS + tid_x();
        }
        __syncthreads();
        again = lds.n_hits > 2 * THREADS;  // far too many elements
    }
    if (top) collect((uint64_t)bound << 32);  // places from there on
    if (top && lds.n_found > kRoom) {
        // Most often that is since many are equal: where fewer than `top` exceed the threads' top-th largest, the others are the first that equal it.
        __syncthreads();
        if (wave == 0) {
            uint32_t own[THREADS / kWave], exact = lds.bound;
#pragma unroll
            for (uint32_t i = 0; i < THREADS / kWave; ++i) own[i] = lds.largest[i * kWave + lane];
            for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
                uint32_t reach = 0;
#pragma unroll
                for (uint32_t i = 0; i < THREADS / kWave; ++i) reach += (uint32_t)__popcll(__ballot(own[i] >= (exact | bit)));
                if (reach >= top) exact |= bit;
            }
            if (lane == 0) {
                lds.bound = exact;
                lds.n_found = 0;
            }
        }
        __syncthreads();
        const uint32_t exact = lds.bound;
        again = true;
        if (exact != 0xffffffffu) collect((uint64_t)(exact + 1) << 32);
        const uint32_t larger = lds.n_found;
        __syncthreads();
        if (larger < top) {
            const uint32_t wanted = top - larger;
            for (uint32_t base = 0, got = 0; got < wanted && base < p.vocab; base += THREADS) {
                const uint32_t token = base + tid_x();
                const bool equal = token < p.vocab && key_of(Element<TYPE>::wide(row[token])) == exact;
                const uint64_t mask = __ballot(equal);
                if (lane == 0) lds.bins[wave] = (uint32_t)__popcll(mask);
                __syncthreads();
                uint32_t before = got + (uint32_t)__popcll(mask & ((1ull << lane) - 1));
#pragma unroll
                for (uint32_t w = 0; w < kWaves; ++w) {
                    before += w < wave ? lds.bins[w] : 0u;
                    got += lds.bins[w];
                }
                if (equal && before < wanted) lds.found[larger + before] = place_of(exact, token);
                __syncthreads();
            }
            if (tid_x() == 0) lds.n_found = top;
            __syncthreads();
        } else {
            // Eight bits of the place at a time: how many have each digit behind those that are settled; the digit that the top-th place has.
            uint64_t settled = 0;
            uint32_t above = 0;  // places that are larger than any with these digits
            for (int shift = 56; shift >= 0; shift -= 8) {
                for (uint32_t i = tid_x(); i < 256; i += THREADS) lds.bins[i] = 0;
                __syncthreads();
                for_row<TYPE, THREADS>(row, p.vocab, [&](float v, uint32_t token) {
                    const uint64_t place = place_of(key_of(v), token);
                    if (shift == 56 || place >> (shift + 8) == settled >> (shift + 8)) {
                        // what has the first lane's digit is added at once: this way is for rows with many equal ones
                        const uint32_t digit = (uint32_t)(place >> shift) & 255u, common = (uint32_t)__builtin_amdgcn_readfirstlane((int)digit);
                        const uint64_t same = __ballot(digit == common);
                        if (digit != common)
                            atomicAdd(&lds.bins[digit], 1u);
                        else if (lane == (uint32_t)__builtin_ctzll(same))
                            atomicAdd(&lds.bins[common], (uint32_t)__popcll(same));
                    }
                });
                __syncthreads();
                if (tid_x() == 0) {
                    uint32_t more = above;
                    int digit = 255;
                    while (more + lds.bins[digit] < top) more += lds.bins[digit--];
                    lds.digit = (uint32_t)digit;
                    lds.above = more;
                    lds.n_found = 0;
                }
                __syncthreads();
                const uint32_t with = lds.bins[lds.digit];
                settled |= (uint64_t)lds.digit << shift;
                above = lds.above;
                __syncthreads();
                if (above + with <= kRoom) break;
            }
            again = true;
            collect(settled);
        }
    }
    const uint32_t found = top ? lds.n_found : 0;
    T *values = p.values ? reinterpret_cast<T *>(p.values) + row_at * p.top : nullptr;
    int32_t *tokens = p.tokens ? p.tokens + row_at * p.top : nullptr;
    for (uint32_t i = tid_x(); i < found; i += THREADS) {
        const uint64_t place = lds.found[i];
        uint32_t before = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < found; ++j) before += lds.found[j] > place ? 1u : 0u;
        if (before >= top) continue;
        const uint32_t token = ~(uint32_t)place, key = (uint32_t)(place >> 32);
        if (tokens) tokens[before] = (int32_t)token;
        // exactly what it was: a key has neither a zero's sign nor a NaN's bits
        if (values) values[before] = key == kZero || key == kNan ? row[token] : Element<TYPE>::narrow(value_of(key));
    }
    for (uint32_t i = top + tid_x(); i < p.top; i += THREADS) {
        if (tokens) tokens[i] = -1;
        if (values) values[i] = (T)(-__builtin_inff());
    }
}

template <int TYPE, uint32_t THREADS>
void launch(const TopArgs &a, uint64_t vectors, hipStream_t s) {
    const dim3 grid((unsigned)a.n), threads(THREADS);
    if (vectors <= 4)
        hipLaunchKernelGGL((top_kernel<TYPE, THREADS, 4, 1>), grid, threads, 0, s, a);
    else if (vectors <= 8)
        hipLaunchKernelGGL((top_kernel<TYPE, THREADS, 8, 1>), grid, threads, 0, s, a);
    else if (vectors <= 16)
        hipLaunchKernelGGL((top_kernel<TYPE, THREADS, THREADS == 1024 ? 8 : 16, THREADS == 1024 ? 2 : 1>), grid, threads, 0, s, a);
    else
        hipLaunchKernelGGL((top_kernel<TYPE, THREADS, 16, 0>), grid, threads, 0, s, a);
}
// The fewer threads have a row, the more rows share a compute unit and hide each other's steps that have little to do; few rows want many threads (512 x 131072 by 512
// threads 46.6 us, by 1024 34.4).  A bound
// is of use where clearly more threads than are asked for have elements.
template <int TYPE>
void top_of(const TopArgs &a, const cnr_ctx *ctx, hipStream_t s) {
    const uint64_t vectors = (uint64_t)a.vocab * sizeof(typename Element<TYPE>::type) / 16, per_unit = cnr_ceil_div(a.n, ctx->n_cu);
    if (per_unit > 4 && a.top <= 192)
        launch<TYPE, 256>(a, cnr_ceil_div(vectors, 256), s);
    else if (per_unit > 2 && a.top <= 384)
        launch<TYPE, 512>(a, cnr_ceil_div(vectors, 512), s);
    else
        launch<TYPE, 1024>(a, cnr_ceil_div(vectors, 1024), s);
}

}  // namespace

extern "C" {

cnr_status cnr_top_logits(cnr_ctx *ctx, const void *logits, uint64_t stride, cnr_float_type type, uint64_t n, uint64_t vocab, uint64_t top, int32_t *tokens, void *values,
                          float *lse, void *stream) {
    if (!ctx || !cnr_valid_float_type(type) || stride < vocab) return CNR_E_INVALID;
    if (n > CNR_LM_MAX_SIZE || vocab > CNR_LM_MAX_SIZE || top > CNR_LOSS_MAX_TOP || n * 1024 >= 1ull << 32) return CNR_E_TOO_LARGE;
    if (n == 0 || ((top == 0 || (!tokens && !values)) && !lse)) return CNR_OK;
    if (vocab && !logits) return CNR_E_INVALID;
    const size_t element = cnr_float_bytes(type);
    if (!cnr_aligned(logits, element) || !cnr_aligned(values, element) || !cnr_aligned(tokens, 4) || !cnr_aligned(lse, 4)) return CNR_E_ALIGN;
    cnr_status st = cnr_enter(ctx);
    if (st != CNR_OK) return st;
    const TopArgs a = {logits, stride, (uint32_t)vocab, (uint32_t)top, n, tokens, values, lse};
    hipStream_t s = as_stream(stream);
    if (type == CNR_FLOAT_F32)
        top_of<CNR_FLOAT_F32>(a, ctx, s);
    else if (type == CNR_FLOAT_BF16)
        top_of<CNR_FLOAT_BF16>(a, ctx, s);
    else
        top_of<CNR_FLOAT_F16>(a, ctx, s);
    return cnr_launch_status(ctx);
}

}  // extern "C"
