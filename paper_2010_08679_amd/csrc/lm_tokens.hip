// Tokens that sequences hold, and what follows from them for their logits.
//
// A sequence's state is a slot: a bitmap of the vocabulary (laid out as a table's tracking bitmap) and a counter for each token.
// The bitmap is what makes the adjustment cheap: of a row's 4 bytes a token of counters only those of seen
// tokens are read, so that beside the logits a row costs its two bitmaps, 1/16 byte a token each way.
#include "lm_common.h"

namespace {

// ---- counts ---------------------------------------------------------------------------------------------------

struct CountArgs {
    uint32_t *seen, *counts;
    uint64_t n_slots, vocab, words;
    const void *tokens;
    uint64_t n_tokens;
    const uint64_t *offsets;
    const int32_t *slots;
    uint64_t n;
    cnr_dev_errors *err;
};

// Slot of sequence i, or n_slots where it has none.
__device__ __forceinline__ uint64_t slot_of(const int32_t *slots, uint64_t n_slots, uint64_t i) {
    const int64_t s = slots ? (int64_t)slots[i] : (int64_t)i;
    return s >= 0 && (uint64_t)s < n_slots ? (uint64_t)s : n_slots;
}

// Empties the slots of the call: grid.y a sequence, grid.x shares of its state.
__global__ void __launch_bounds__(kBlock) restart_kernel(const CountArgs a, uint32_t shares) {
    for (uint64_t i = wg_y(); i < a.n; i += 32768) {
        const uint64_t slot = slot_of(a.slots, a.n_slots, i);
        if (slot == a.n_slots) continue;
        uint32_t *seen = a.seen + slot * a.words;
        for (uint64_t at = (uint64_t)wg_x() * kBlock + tid_x(); at < a.words; at += (uint64_t)shares * kBlock) seen[at] = 0u;
        if (!a.counts) continue;
        uint32_t *counts = a.counts + slot * a.vocab;
        for (uint64_t at = (uint64_t)wg_x() * kBlock + tid_x(); at < a.vocab; at += (uint64_t)shares * kBlock) counts[at] = 0u;
    }
}

// The sequence that token p belongs to: the last one that begins at or before p; n where p lies in none.
__device__ __forceinline__ uint64_t sequence_of(const uint64_t *offsets, uint64_t n, uint64_t p) {
    uint64_t lo = 0, hi = n;  // offsets[lo] <= p, if any is
    while (hi - lo > 1) {
        const uint64_t mid = (lo + hi) / 2;
        if (offsets[mid] <= p)
            lo = mid;
        else
            hi = mid;
    }
    return offsets[lo] <= p && p < offsets[lo + 1] ? lo : n;
}

// A thread for each token.
template <typename Index>
__global__ void __launch_bounds__(kBlock) count_kernel(const CountArgs a) {
    const uint64_t p = (uint64_t)wg_x() * kBlock + tid_x();
    if (p >= a.n_tokens) return;
    const int64_t token = (int64_t)reinterpret_cast<const Index *>(a.tokens)[p];
    const uint64_t i = a.offsets ? sequence_of(a.offsets, a.n, p) : p;
    if (i >= a.n) return;
    const uint64_t slot = slot_of(a.slots, a.n_slots, i);
    if (slot == a.n_slots) {
        raise_flag(a.err, CNR_FLAG_ROW_ID);
        return;
    }
    if (token < 0 || (uint64_t)token >= a.vocab) {
        atomicAdd(&a.err->n_bad_indices, 1ull);
        return;
    }
    uint32_t *word = a.seen + slot * a.words + ((uint64_t)token >> 5);
    const uint32_t bit = 1u << ((uint32_t)token & 31u);
    if (!(*word & bit)) atomicOr(word, bit);
    if (a.counts) atomicAdd(a.counts + slot * a.vocab + (uint64_t)token, 1u);
}

// ---- counts of prompts ------------------------------------------------------------------------------------------

// A workgroup for each slice of the vocabulary of each sequence: it counts the sequence's tokens of its slice in LDS.  A sequence that
// begins has its slice of the state written whole, without its old contents or atomics in memory, which is bound by the stores; to one that goes on the
// counters that are not 0 are added.  The sequence's tokens are read once for each slice, from L2 but for the first.
// 64 prompts of up to 8192 tokens, 131072 in the vocabulary: 10.2 us, of which the state's 34 MB take 7 at the rate of a copy (with an
// atomic in memory for each token after the state is emptied 21.5).
constexpr uint32_t kSlice = 16384;   // tokens: 64 KiB of counters, so that a CU holds two workgroups (16384 with 1024 threads 13.4 us, 8192 with 512 12.5)
constexpr uint32_t kCounting = 512;  // threads
constexpr uint32_t kAtOnce = 8;      // tokens that a thread loads before it counts them
// Which kernels a call takes depends on its average number of tokens a sequence, all that the host knows of them without waiting, and on
// how many sequences there are.  Lengths of one order are meant: a long sequence among short ones goes the short ones' way or is counted by
// one workgroup a slice (131072 tokens that go on alone 9.6 us, among 63 of one 91; that begin 15 and 33; 2^20 tokens that begin alone 62, among
// 63 of a hundred 217).
constexpr uint64_t kAddFrom = 8192;       // from here on tokens are added slice by slice: 8192 x 8 9.2 us, by count_kernel 9.0; 131072 x 1 10.8 and 91; 2048 x 1 7.8 and 4.4
constexpr uint64_t kBeginUpTo = 65536;    // up to here a state that begins is written whole: 65536 x 1 17 us, emptied and added to 17; 131072 x 1 27 and 17; 32768 x 1 11 and 12
constexpr uint64_t kLookedThrough = 4096; // sequences with slots up to which a state that begins is written whole: each workgroup looks through all slots for its own
constexpr uint64_t kPart = 8192;          // tokens of a sequence's part where they are added

// Tokens of sequence i.
struct Range {
    uint64_t lo, hi;
};
__device__ __forceinline__ Range tokens_of(const CountArgs &a, uint64_t i) {
    Range r = {i, i + 1};
    if (a.offsets) r = {a.offsets[i], a.offsets[i + 1]};
    if (r.hi > a.n_tokens) r.hi = a.n_tokens;
    return r;
}

// Enters tokens [r.lo, r.hi) that lie in the slice from `begin`; returns how many of the thread's lie outside the vocabulary.
template <typename Index>
__device__ __forceinline__ uint32_t count_range(const CountArgs &a, uint32_t *counters, Range r, uint32_t begin) {
    const Index *tokens = reinterpret_cast<const Index *>(a.tokens);
    uint32_t bad = 0;
    for (uint64_t p = r.lo + tid_x(); p < r.hi; p += kAtOnce * kCounting) {
        int64_t token[kAtOnce];
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) {
            const uint64_t at = p + i * kCounting;
            token[i] = (int64_t)tokens[at < r.hi ? at : p];
        }
#pragma unroll
        for (uint32_t i = 0; i < kAtOnce; ++i) {
            if (p + i * kCounting >= r.hi) continue;
            if ((uint64_t)token[i] >= a.vocab)  // negative ones too
                ++bad;
            else if ((uint32_t)token[i] - begin < kSlice)
                atomicAdd(counters + ((uint32_t)token[i] - begin), 1u);
        }
    }
    return bad;
}

// Bits of `v` of eight lanes side by side, in each of them.
__device__ __forceinline__ uint32_t or_of_eight(uint32_t v) {
    v |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true);   // quads' lanes 1 0 3 2
    v |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true);   // quads' lanes 2 3 0 1
    v |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true);  // eights mirrored
    return v;
}

// grid.x: slices, grid.y: sequences, grid.z: parts of a sequence that goes on.
template <typename Index, bool BEGIN>
__global__ void __launch_bounds__(kCounting) slice_kernel(const CountArgs a, bool prompt, uint32_t parts) {
    __shared__ uint32_t counters[kSlice];
    __shared__ uint32_t before, after;  // sequences of the same slot on either side of this one
    const uint32_t t = tid_x(), begin = wg_x() * kSlice, vocab = (uint32_t)a.vocab;
    for (uint64_t i = wg_y(); i < a.n; i += 32768) {
        const uint64_t slot = slot_of(a.slots, a.n_slots, i);
        Range own = tokens_of(a, i);
        if (!BEGIN && own.lo < own.hi) {
            const uint64_t part = (own.hi - own.lo + parts - 1) / parts;
            own.lo += part * __builtin_amdgcn_workgroup_id_z();
            own.hi = own.hi < own.lo + part ? own.hi : own.lo + part;
        }
        if (slot == a.n_slots || (!BEGIN && own.lo >= own.hi)) {
            if (t == 0 && begin == 0 && own.lo < own.hi) raise_flag(a.err, CNR_FLAG_ROW_ID);
            continue;
        }
        if (BEGIN && t == 0) before = after = 0;
        for (uint32_t at = t * 4; at < kSlice; at += kCounting * 4) *reinterpret_cast<u32x4 *>(counters + at) = u32x4{0, 0, 0, 0};
        __syncthreads();
        bool first = true, alone = true;
        if constexpr (BEGIN) {
            if (a.slots)
                for (uint64_t j = t; j < a.n; j += kCounting)
                    if (j != i && slot_of(a.slots, a.n_slots, j) == slot) atomicAdd(j < i ? &before : &after, 1u);
            __syncthreads();
            first = before == 0, alone = after == 0;
        }
        if (first) {  // the slot's first sequence enters those that share it too
            uint32_t bad = count_range<Index>(a, counters, own, begin);
            if (!alone)
                for (uint64_t j = i + 1; j < a.n; ++j)
                    if (slot_of(a.slots, a.n_slots, j) == slot) bad += count_range<Index>(a, counters, tokens_of(a, j), begin);
            if (begin == 0 && bad) atomicAdd(&a.err->n_bad_indices, (unsigned long long)bad);
            __syncthreads();
            uint32_t *counts = a.counts ? a.counts + slot * a.vocab + begin : nullptr, *seen = a.seen + slot * a.words + begin / 32;
            const uint32_t left = vocab - begin < kSlice ? vocab - begin : kSlice;
            for (uint32_t at = t * 4; at < kSlice; at += kCounting * 4) {
                const u32x4 c = *reinterpret_cast<const u32x4 *>(counters + at);
                const uint32_t bits = (c[0] != 0) | (uint32_t)(c[1] != 0) << 1 | (uint32_t)(c[2] != 0) << 2 | (uint32_t)(c[3] != 0) << 3;
                const uint32_t word = or_of_eight(bits << (t % 8 * 4));
                if constexpr (BEGIN) {
                    if (t % 8 == 0 && at < left) seen[at / 32] = word;
                    const u32x4 kept = prompt ? u32x4{0, 0, 0, 0} : c;
                    if (!counts) continue;
                    if (at + 4 <= left) {
                        store16(counts + at, kept);
                    } else {
#pragma unroll
                        for (uint32_t e = 0; e < 4; ++e)
                            if (at + e < left) counts[at + e] = kept[e];
                    }
                } else {
                    if (t % 8 == 0 && word && (seen[at / 32] & word) != word) atomicOr(seen + at / 32, word);
                    if (!counts || prompt) continue;
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e)
                        if (c[e]) atomicAdd(counts + at + e, c[e]);
                }
            }
        }
        __syncthreads();
    }
}

// ---- logits -----------------------------------------------------------------------------------------------------

// Bound by memory: a logit is read and written once, a bit of each bitmap beside it.  A thread holds kSegments times 16 bytes of a
// row, those of a wave side by side each time: four where rows are long and many, for enough under way; one where the tokens
// that a thread looks after would make it the last (see adjust()).  Seen and biased tokens are few and far between: a row's logits are stored as the
// masks leave them, and then each thread sees to its own special tokens, one after the other.  (Its neighbours' and its own counters
// share sectors, so that the first brings the others; all counters at once and the arithmetic for every token would keep the vector
// units busy for longer than memory.)
constexpr uint32_t kScannedBiases = 4 * kBlock;  // lists up to this are looked through, each workgroup all of it; longer ones searched

struct AdjustArgs {
    const void *logits;
    void *out;
    uint64_t stride, out_stride;
    uint64_t n, vocab, words;
    cnr_adjustments with;
    // the rows' lists, or words that are there in their place
    const int32_t *slots, *mask_of;
    const float *repetition, *frequency, *presence;
    bool has_slots, has_mask_of, has_repetition, has_frequency, has_presence;
    cnr_dev_errors *err;
};

// First entry of bias_tokens[lo, hi) that is not below `token`.
__device__ __forceinline__ uint64_t bias_from(const int32_t *tokens, uint64_t lo, uint64_t hi, int64_t token) {
    while (lo < hi) {
        const uint64_t mid = (lo + hi) / 2;
        if ((int64_t)tokens[mid] < token)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// Biases of a chunk of N tokens: which have one, and which entry of the row's list it is, from the first that was looked at.
template <uint32_t N>
struct Biases {
    uint16_t entry[N];
    uint32_t there[N / 32];
};
template <>
struct Biases<0> {};

// Words whose elements bits of `allowed` (from bit 0) leave as they are; the others become -infinity.
template <int TYPE>
__device__ __forceinline__ u32x4 masked_words(u32x4 w, uint32_t allowed) {
    constexpr uint32_t kNever = TYPE == CNR_FLOAT_F32 ? 0xff800000u : TYPE == CNR_FLOAT_BF16 ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t keep;
        if constexpr (TYPE == CNR_FLOAT_F32) {
            keep = (uint32_t)((int32_t)(allowed << (31 - i)) >> 31);
        } else {
            const uint32_t lo = (uint32_t)((int32_t)(allowed << (31 - 2 * i)) >> 31), hi = (uint32_t)((int32_t)(allowed << (30 - 2 * i)) >> 31);
            keep = (lo & 0xffffu) | (hi & 0xffff0000u);
        }
        w[i] = (w[i] & keep) | (kNever & ~keep);
    }
    return w;
}

// The thread's share of one row of a chunk.  WHOLE: all of the chunk is in the vocabulary.
template <int TYPE, bool BIASED, uint32_t kSegments, bool WHOLE, typename Lds>
__device__ __forceinline__ void adjust_row(const AdjustArgs &a, Lds &lds, uint64_t row, uint32_t begin) {
    typedef typename Element<TYPE>::type T;
    constexpr uint32_t kPer = 16 / sizeof(T), kSegment = kBlock * kPer, kChunk = kSegments * kSegment, kBits = (1u << kPer) - 1u;
    static_assert(kSegments * kPer <= 32 && kChunk <= 65536 && kScannedBiases <= 65536, "bits of a word, entries of 16 bits");
    const cnr_adjustments &w = a.with;
    const uint32_t t = tid_x(), own = t * kPer, vocab = (uint32_t)a.vocab;
    const T *from = reinterpret_cast<const T *>(a.logits) + row * a.stride + begin;
    T *to = reinterpret_cast<T *>(a.out) + row * a.out_stride + begin;
    u32x4 v[kSegments];
    if constexpr (WHOLE) {
#pragma unroll
        for (uint32_t i = 0; i < kSegments; ++i) v[i] = load16(from + i * kSegment + own);
    }
    // What the row has, all asked for at once: lists that are not given are replaced by words that are there.
    const int32_t mask = a.mask_of[a.has_mask_of ? row : 0], id = a.slots[a.has_slots ? row : 0];
    const int64_t m = a.has_mask_of ? (int64_t)mask : (int64_t)row, s = a.has_slots ? (int64_t)id : (int64_t)row;
    const bool masked = w.masks && m >= 0 && (uint64_t)m < w.n_masks, counted = w.seen && s >= 0 && (uint64_t)s < w.n_slots;
    if (begin + own == 0 && ((w.masks && m >= 0 && !masked) || (w.seen && s >= 0 && !counted))) raise_flag(a.err, CNR_FLAG_ROW_ID);
    // The bits of kPer tokens lie in one word of a bitmap, since they begin at a multiple of their number.
    uint32_t allowed = 0xffffffffu, seen = 0, valid = 0xffffffffu;
    if (masked) {
        const uint32_t *words = w.masks + (uint64_t)m * a.words;
        allowed = 0;
#pragma unroll
        for (uint32_t i = 0; i < kSegments; ++i) {
            const uint32_t first = begin + i * kSegment + own;
            if (WHOLE || first < vocab) allowed |= (words[first / 32] >> (first % 32) & kBits) << (i * kPer);
        }
    }
    if (counted) {
        const uint32_t *words = w.seen + (uint64_t)s * a.words;
#pragma unroll
        for (uint32_t i = 0; i < kSegments; ++i) {
            const uint32_t first = begin + i * kSegment + own;
            if (WHOLE || first < vocab) seen |= (words[first / 32] >> (first % 32) & kBits) << (i * kPer);
        }
    }
    if constexpr (!WHOLE) {
        valid = 0;
#pragma unroll
        for (uint32_t i = 0; i < kSegments; ++i) {
            const uint32_t first = begin + i * kSegment + own;
            if (first < vocab) valid |= (first + kPer <= vocab ? kBits : (1u << (vocab - first)) - 1u) << (i * kPer);
        }
    }
    uint32_t biased = 0;
    uint64_t lo = 0;
    if constexpr (BIASED) {
        lo = w.bias_offsets[row];
        uint64_t hi = w.bias_offsets[row + 1];
        hi = hi < w.n_bias ? hi : w.n_bias;
        if (lo < hi) {  // the same for the whole workgroup
            if (hi - lo > kScannedBiases) {
                lo = bias_from(w.bias_tokens, lo, hi, (int64_t)begin);
                hi = bias_from(w.bias_tokens, lo, hi, (int64_t)begin + kChunk);
            }
            if (t < kChunk / 32) lds.there[t] = 0;
            __syncthreads();
            for (uint64_t e = lo + t; e < hi; e += kBlock) {
                const uint64_t at = (uint64_t)((int64_t)w.bias_tokens[e] - (int64_t)begin);
                if (at < kChunk) {
                    lds.entry[at] = (uint16_t)(e - lo);
                    atomicOr(&lds.there[at / 32], 1u << (at % 32));
                }
            }
            __syncthreads();
#pragma unroll
            for (uint32_t i = 0; i < kSegments; ++i) biased |= (lds.there[(i * kSegment + own) / 32] >> (own % 32) & kBits) << (i * kPer);
        }
    }
    if constexpr (WHOLE) {
#pragma unroll
        for (uint32_t i = 0; i < kSegments; ++i) store16(to + i * kSegment + own, masked_words<TYPE>(v[i], allowed >> (i * kPer)));
    } else {
        for (uint32_t left = valid; left; left &= left - 1u) {
            const uint32_t b = (uint32_t)__ffs((int)left) - 1u, token = b / kPer * kSegment + own + b % kPer;
            to[token] = allowed >> b & 1u ? from[token] : (T)(-__builtin_inff());
        }
    }
    uint32_t special = (seen | biased) & allowed & valid;
    if (!special) return;
    const float repetition = a.repetition[a.has_repetition ? row : 0], frequency = a.frequency[a.has_frequency ? row : 0],
                presence = a.presence[a.has_presence ? row : 0];
    const uint32_t *counts = w.counts + (uint64_t)s * a.vocab + begin;
    do {
        const uint32_t b = (uint32_t)__ffs((int)special) - 1u, token = b / kPer * kSegment + own + b % kPer;
        special &= special - 1u;
        float x = Element<TYPE>::wide(from[token]);  // as it was: what is special has been stored unchanged
        if (seen >> b & 1u) {
            const uint32_t count = w.counts ? counts[token] : 0u;
            const float r = a.has_repetition ? repetition : 1.0f;
            x = x > 0.0f ? x / r : x * r;
            if (w.counts && a.has_frequency) x -= frequency * (float)count;
            if (count && a.has_presence) x -= presence;
        }
        if constexpr (BIASED) {
            if (biased >> b & 1u) x += w.bias_values[lo + lds.entry[token]];
        }
        to[token] = Element<TYPE>::narrow(x);
    } while (special);
}

// grid.x: chunks of the vocabulary, grid.y: rows.
template <int TYPE, bool BIASED, uint32_t kSegments>
__global__ void __launch_bounds__(kBlock) adjust_kernel(const AdjustArgs a) {
    constexpr uint32_t kChunk = kSegments * kBlock * 16 / sizeof(typename Element<TYPE>::type);
    __shared__ Biases<BIASED ? kChunk : 0> lds;
    const uint32_t begin = wg_x() * kChunk;
    for (uint64_t row = wg_y(); row < a.n; row += 32768) {
        if (begin + kChunk <= a.vocab)
            adjust_row<TYPE, BIASED, kSegments, true>(a, lds, row, begin);
        else
            adjust_row<TYPE, BIASED, kSegments, false>(a, lds, row, begin);
        if (BIASED && row + 32768 < a.n) __syncthreads();  // the biases are filled again
    }
}

template <int TYPE, uint32_t kSegments>
void adjust(const AdjustArgs &a, hipStream_t s) {
    constexpr uint32_t kChunk = kBlock * kSegments * (16 / sizeof(typename Element<TYPE>::type));
    const dim3 grid((unsigned)cnr_ceil_div(a.vocab, kChunk), (unsigned)(a.n < 32768 ? a.n : 32768));
    if (a.with.bias_offsets)
        hipLaunchKernelGGL((adjust_kernel<TYPE, true, kSegments>), grid, dim3(kBlock), 0, s, a);
    else
        hipLaunchKernelGGL((adjust_kernel<TYPE, false, kSegments>), grid, dim3(kBlock), 0, s, a);
}
// bfloat16 with everything, four, two and one segments: 512 x 131072 70, 82 and 120 us; 2048 x 8000, 38 % of the tokens seen, 93, 60 and 51.
template <int TYPE>
void adjust(const AdjustArgs &a, const cnr_ctx *ctx, hipStream_t s) {
    if (a.vocab >= 32768 && (float)a.n * (float)a.vocab >= 8.0f * (float)ctx->n_cu * 8192.0f)
        adjust<TYPE, 4>(a, s);
    else
        adjust<TYPE, 1>(a, s);
}

}  // namespace

extern "C" {

cnr_status cnr_count_tokens(cnr_ctx *ctx, uint32_t *seen, uint32_t *counts, uint64_t n_slots, uint64_t vocab,
                            const void *tokens, uint64_t n_tokens, cnr_index_type type, const uint64_t *offsets,
                            const int32_t *slots, uint64_t n, int prompt, int restart, void *stream) {
    if (!ctx || (type != CNR_IDX_I32 && type != CNR_IDX_I64)) return CNR_E_INVALID;
    if (!offsets && n_tokens != n) return CNR_E_INVALID;
    if (vocab > CNR_LM_MAX_SIZE || n > CNR_LM_MAX_SIZE || n_slots > CNR_LM_MAX_SIZE || n_tokens > CNR_LM_MAX_SIZE) return CNR_E_TOO_LARGE;
    if (n == 0) return CNR_OK;
    if (!seen && n_slots && vocab) return CNR_E_INVALID;
    if (!tokens && n_tokens) return CNR_E_INVALID;
    if (!cnr_aligned(seen, 4) || !cnr_aligned(counts, 4) || !cnr_aligned(tokens, type == CNR_IDX_I64 ? 8 : 4) || !cnr_aligned(offsets, 8) ||
        !cnr_aligned(slots, 4))
        return CNR_E_ALIGN;
    cnr_status st = cnr_enter(ctx);
    if (st != CNR_OK) return st;
    CountArgs a;
    a.seen = seen;
    a.counts = counts;
    a.n_slots = n_slots;
    a.vocab = vocab;
    a.words = cnr_bitmap_words(vocab);
    a.tokens = tokens;
    a.n_tokens = n_tokens;
    a.offsets = offsets;
    a.slots = slots;
    a.n = n;
    a.err = ctx->dev_err;
    hipStream_t s = as_stream(stream);
    const bool wide = type == CNR_IDX_I64;
    if (vocab == 0 || n_slots == 0) restart = 0;  // no state
    const uint64_t average = n_tokens / n;
    const unsigned slices = (unsigned)cnr_ceil_div(vocab, kSlice), rows = (unsigned)(n < 32768 ? n : 32768);
    if (restart && average <= kBeginUpTo && (!slots || n <= kLookedThrough)) {
        wide ? slice_kernel<int64_t, true><<<dim3(slices, rows), kCounting, 0, s>>>(a, prompt != 0, 1)
             : slice_kernel<int32_t, true><<<dim3(slices, rows), kCounting, 0, s>>>(a, prompt != 0, 1);
        return cnr_launch_status(ctx);
    }
    if (restart) {
        const uint32_t shares = (uint32_t)cnr_ceil_div(counts ? vocab : a.words, 16 * kBlock);
        hipLaunchKernelGGL(restart_kernel, dim3(shares, rows), dim3(kBlock), 0, s, a, shares);
        st = cnr_launch_status(ctx);
        if (st != CNR_OK) return st;
    }
    if (n_tokens == 0) return CNR_OK;
    if (vocab && n_slots && average >= kAddFrom) {
        const uint64_t wanted = cnr_ceil_div(average, kPart);
        const unsigned parts = (unsigned)(wanted < 32768 ? wanted : 32768);
        const dim3 grid(slices, rows, parts);
        wide ? slice_kernel<int64_t, false><<<grid, kCounting, 0, s>>>(a, prompt != 0, parts)
             : slice_kernel<int32_t, false><<<grid, kCounting, 0, s>>>(a, prompt != 0, parts);
        return cnr_launch_status(ctx);
    }
    if (prompt) a.counts = nullptr;
    const unsigned grid = (unsigned)cnr_ceil_div(n_tokens, kBlock);
    wide ? count_kernel<int64_t><<<grid, kBlock, 0, s>>>(a) : count_kernel<int32_t><<<grid, kBlock, 0, s>>>(a);
    return cnr_launch_status(ctx);
}

cnr_status cnr_adjust_logits(cnr_ctx *ctx, const void *logits, uint64_t stride, void *out, uint64_t out_stride,
                             cnr_float_type type, uint64_t n, uint64_t vocab, const cnr_adjustments *adjustments,
                             void *stream) {
    if (!ctx || !adjustments || !cnr_valid_float_type(type) || stride < vocab || out_stride < vocab) return CNR_E_INVALID;
    const cnr_adjustments &w = *adjustments;
    if (vocab > CNR_LM_MAX_SIZE || n > CNR_LM_MAX_SIZE || w.n_slots > CNR_LM_MAX_SIZE || w.n_masks > CNR_LM_MAX_SIZE) return CNR_E_TOO_LARGE;
    if (n == 0 || vocab == 0) return CNR_OK;
    if (!logits || !out || (logits == out && stride != out_stride)) return CNR_E_INVALID;
    if (w.bias_offsets && w.n_bias && (!w.bias_tokens || !w.bias_values)) return CNR_E_INVALID;
    const size_t element = cnr_float_bytes(type);
    if (!cnr_aligned(logits, element) || !cnr_aligned(out, element) || !cnr_aligned(w.seen, 4) || !cnr_aligned(w.counts, 4) ||
        !cnr_aligned(w.slots, 4) || !cnr_aligned(w.repetition, 4) || !cnr_aligned(w.frequency, 4) || !cnr_aligned(w.presence, 4) ||
        !cnr_aligned(w.bias_offsets, 8) || !cnr_aligned(w.bias_tokens, 4) || !cnr_aligned(w.bias_values, 4) || !cnr_aligned(w.masks, 4) ||
        !cnr_aligned(w.mask_of, 4))
        return CNR_E_ALIGN;
    cnr_status st = cnr_enter(ctx);
    if (st != CNR_OK) return st;
    AdjustArgs a;
    a.logits = logits;
    a.out = out;
    a.stride = stride;
    a.out_stride = out_stride;
    a.n = n;
    a.vocab = vocab;
    a.words = cnr_bitmap_words(vocab);
    a.with = w;
    a.err = ctx->dev_err;
    const void *something = ctx->dev_err;
    a.has_slots = w.slots != nullptr;
    a.has_mask_of = w.mask_of != nullptr;
    a.has_repetition = w.repetition != nullptr;
    a.has_frequency = w.frequency != nullptr;
    a.has_presence = w.presence != nullptr;
    a.slots = w.slots ? w.slots : (const int32_t *)something;
    a.mask_of = w.mask_of ? w.mask_of : (const int32_t *)something;
    a.repetition = w.repetition ? w.repetition : (const float *)something;
    a.frequency = w.frequency ? w.frequency : (const float *)something;
    a.presence = w.presence ? w.presence : (const float *)something;
    if (type == CNR_FLOAT_F32)
        adjust<CNR_FLOAT_F32>(a, ctx, as_stream(stream));
    else if (type == CNR_FLOAT_BF16)
        adjust<CNR_FLOAT_BF16>(a, ctx, as_stream(stream));
    else
        adjust<CNR_FLOAT_F16>(a, ctx, as_stream(stream));
    return cnr_launch_status(ctx);
}

}  // extern "C"
