// What the losses over the vocabulary (lm_loss.hip) take of memory and how they are split: sizes, plans and workspaces, on the host.
#pragma once

#include "lm_dense.h"
#include "cnr_loss.h"

namespace {

// (largest exponent to base 2, sum of 2^(exponent - largest)) of some of a row's logits; (-infinity, 0) of none.
struct Stats {
    float top, sum;
};
// What the backward pass knows of a row: log2 of its sum of exponentials and dloss / T, scaled (0: the row adds nothing), and its target where it has
// one (else kNoTarget).
constexpr uint32_t kNoTarget = dense::kNoIndex;
struct __attribute__((aligned(16))) RowGradient {
    float lse2, gradient;
    uint32_t target, unused;
};

constexpr uint64_t kMaxRows = CNR_LOSS_MAX_ROWS, kMaxVocabulary = CNR_LOSS_MAX_VOCABULARY, kMaxDim = CNR_LOSS_MAX_DIM;
// Up to how many rows the weight goes straight from memory into the products.  With more its rows are better shared through LDS, even where they have to be laid
// out first: 64 x 54656 x 6026 at an odd stride 608 us by four times as many rows to a workgroup, 534 laid out.
constexpr uint32_t kNarrowRows = 16;
// Floats are laid out in three parts otherwise, and tiles of few rows are few: a step of 32 x 15815 x 5312 1055 -> 500 us, of 64 x 32000 x 1024 351 -> 271; with as many
// rows again the fp32 instructions would take longer than six bfloat16 ones.
constexpr uint32_t kNarrowRowsOfFloats = 64;
// Up to how many rows of 16 bits dz is held in two parts, whatever the results' type: products that are bound by reading the weight and by writing its gradient
// nearly have the time (a step of 32 x 131072 x 4096 941 -> 1013 us), and sums of few rows do not average roundings.
constexpr uint32_t kTwoPartRows = 64;
// And up to how many rows of bfloat16 in three parts for a gradient in fp32, which is then as exact as by dz in fp32 (two parts: off by 2.5e-6, sums in fp32 by 3e-7): a step of
// 64 x 131072 x 1024 409 -> 431 us, of 128 x 75456 x 602 240 -> 255, but of 333 x 50257 x 1024 286 -> 333, of 8192 x 32000 x 4096 8280 -> 10490.
constexpr uint32_t kThreePartRows = 128;
// In the backward pass of larger weights that need not be laid out tiles are faster even for few rows: a step of 16 x 131072 x 4096 in bfloat16 1249 -> 1022 us, of 1 row
// 1197 -> 983, of 16 x 32000 x 2048 142 -> 133; 16 x 32000 x 1024 83.8 and 83.0, 16 x 16384 x 1024 55.8 and 55.1; but of 16 x 131072 x 256 89 against 113, of 16 x 131072 x 128
// 73 against 94, of 16 x 1249 x 6784 62 against 77.
constexpr uint64_t kTiledFrom = 3ull << 24;
constexpr uint64_t kPieceBytes = 256ull << 20;  // of a piece of the weight, of its dz twice as many, up to the next multiple of 256 tokens
constexpr uint64_t kPieceTokens = 1ull << 20;   // a row of its dz, in up to three parts, is below 2^23 bytes
constexpr uint64_t kStatsBytes = 512ull << 20;  // of the stats of as many rows as go at a time
constexpr uint64_t kPartBytes = 128ull << 20;   // of sums that are split

inline uint64_t rounded(uint64_t v, uint64_t to) { return cnr_ceil_div(v, to) * to; }
inline uint64_t least(uint64_t a, uint64_t b) { return a < b ? a : b; }

// Whether a product can read rows of dim elements where they are.
inline bool whole_rows(const cnr_float_type type, const void *base, uint64_t stride, uint64_t dim, uint64_t rows) {
    return type != CNR_FLOAT_F32 && dim && dim % 8 == 0 && cnr_aligned(base, 16) && (rows <= 1 || (stride % 8 == 0 && stride < 1u << 22));
}

// Places in a workspace, in order.
struct Room {
    uint64_t used = 0;
    uint64_t take(uint64_t bytes) {
        const uint64_t at = used;
        used += rounded(bytes, 256);
        return at;
    }
};

struct Sizes {
    uint64_t n, vocab, dim;
    cnr_float_type type;
    uint32_t parts, blocks;  // of a laid out row: of 16-bit elements each, at least one block
    uint64_t row;            // its bytes
};
inline Sizes sizes_of(uint64_t n, uint64_t vocab, uint64_t dim, cnr_float_type type) {
    Sizes s = {n, vocab, dim, type, type == CNR_FLOAT_F32 ? 3u : 1u, 0, 0};
    s.blocks = dim ? (uint32_t)cnr_ceil_div(dim, dense::kBlockElements) : 1;
    s.row = (uint64_t)s.parts * s.blocks * dense::kBlockBytes;
    return s;
}
// Pairs of parts, the smallest products of a block first.
struct Terms {
    uint32_t number, across, down;
};
constexpr Terms kOne = {1, 0, 0}, kOfFloats = {6, 0x001012, 0x010210}, kOfTwoParts = {2, 0, 0x01}, kOfThreeParts = {3, 0, 0x012};

// Of a row: its stats, and where the entries of each tile begin.
inline uint64_t part_bytes(uint64_t n_parts) { return n_parts * sizeof(Stats) + (n_parts + 1) * sizeof(uint16_t); }

struct ForwardPlan {
    bool narrow;
    uint32_t fragments;    // columns of a narrow workgroup, in sixteens
    uint64_t rows, piece;  // at a time
    uint32_t n_parts;      // of a row
    dense::Plan tiles;
    uint64_t parts, begins, picked, hidden, weight, bytes;  // in the workspace
};
inline uint64_t narrow_rows(const Sizes &s) { return s.parts == 3 ? kNarrowRowsOfFloats : kNarrowRows; }
inline uint64_t padded_rows(uint64_t n) { return n <= 16 ? 16 : n <= 32 ? 32 : 64; }
inline uint32_t narrow_fragments(uint64_t n, uint64_t vocab) {
    // Two fragments of the weight to a wave where that still gives every SIMD a wave.
    return n > 1 && vocab >= 16384 ? 2 : 1;
}
inline ForwardPlan forward_plan(const cnr_ctx *ctx, const Sizes &s) {
    ForwardPlan f = {};
    f.rows = s.n;
    if (s.vocab == 0) return f;
    f.narrow = s.n <= narrow_rows(s);
    f.fragments = narrow_fragments(s.n, s.vocab);
    f.tiles = dense::plan_of(ctx, s.vocab, s.n, (uint64_t)s.blocks * (s.parts == 3 ? kOfFloats.number : 1), 0.5f /* time for exponentials */, 0);
    const uint32_t columns = f.narrow ? 16 * f.fragments : dense::kTiles[f.tiles.kind].columns;
    f.n_parts = (uint32_t)cnr_ceil_div(s.vocab, columns);
    const uint64_t per_row = part_bytes(f.n_parts), most = kStatsBytes / (per_row + 1) / 256 * 256;
    f.rows = most < 256 ? 256 : most;
    if (f.rows > s.n) f.rows = s.n;
    f.piece = rounded(kPieceBytes / s.row, 256);
    if (f.piece > s.vocab) f.piece = s.vocab;
    Room room;
    f.parts = room.take(f.rows * f.n_parts * sizeof(Stats));
    f.begins = room.take(f.rows * (f.n_parts + 1) * sizeof(uint16_t));
    f.picked = room.take(f.rows * sizeof(float));
    if (!f.narrow) {
        f.hidden = room.take(f.rows * s.row);
        f.weight = room.take(f.piece * s.row);
    }
    f.bytes = room.used;
    return f;
}

// (wide: dweight in fp32 from 16-bit operands)
inline uint32_t dz_parts(const Sizes &s, bool wide) {
    if (s.parts == 3 || (wide && s.type == CNR_FLOAT_BF16 && s.n <= kThreePartRows)) return 3;
    return wide || s.n <= kTwoPartRows ? 2 : 1;
}
struct BackwardPlan {
    bool narrow;
    uint64_t piece, width;  // of the vocabulary; columns of dz, whole blocks
    uint64_t scale, rows, dz, hidden_at, weight_at, sum, partial, bytes;
};
// Tokens of a piece whose dz are held in fp32, for as many rows as the matrix instructions take.
inline uint64_t narrow_piece(uint64_t n) { return 2 * kPieceBytes / (padded_rows(n) * sizeof(float)); }
// (wide: see dz_parts.  in_place: the weight is read where it is.)
inline BackwardPlan backward_plan(const cnr_ctx *ctx, const Sizes &s, bool wide, bool in_place) {
    BackwardPlan b = {};
    const uint32_t parts = dz_parts(s, wide);
    b.narrow = s.n <= narrow_rows(s) && !(in_place && s.vocab * s.dim >= kTiledFrom) && s.n * rounded(s.dim, 4) * sizeof(float) <= kPartBytes;
    if (b.narrow) {
        b.piece = least(s.vocab, narrow_piece(s.n));
        Room room;
        b.scale = room.take(2 * sizeof(float));
        b.rows = room.take(256 * sizeof(RowGradient));
        b.dz = room.take(b.piece * padded_rows(s.n) * sizeof(float));
        b.sum = room.take(b.piece < s.vocab ? s.n * s.dim * sizeof(float) : 0);
        b.partial = room.take(kPartBytes);
        b.bytes = room.used;
        return b;
    }
    uint64_t piece = 2 * kPieceBytes / (s.n * 2 * parts);
    const uint64_t by_weight = kPieceBytes / s.row;
    if (!in_place && piece > by_weight) piece = by_weight;
    piece = rounded(least(piece ? piece : 1, kPieceTokens), 256);
    // pieces of one size
    const uint64_t pieces = cnr_ceil_div(s.vocab, piece);
    b.piece = rounded(cnr_ceil_div(s.vocab, pieces), 256);
    if (b.piece > s.vocab) b.piece = s.vocab;
    b.width = rounded(b.piece, dense::kBlockElements);
    Room room;
    b.scale = room.take(2 * sizeof(float));
    b.rows = room.take(rounded(s.n, 256) * sizeof(RowGradient));
    b.dz = room.take(s.n * b.width * 2 * parts);
    b.hidden_at = room.take(s.n * s.row);
    b.weight_at = room.take(in_place ? 0 : b.piece * s.row);
    b.sum = room.take(pieces > 1 ? s.n * s.dim * sizeof(float) : 0);
    b.partial = room.take(kPartBytes);
    b.bytes = room.used;
    return b;
}

// At least what the plans take for n rows or fewer: each part's largest size.
inline uint64_t room_for(const Sizes &s, bool training, bool wide) {
    const uint64_t most_weight = least(s.vocab, rounded(kPieceBytes / s.row, 256)), small = least(s.n, 256);
    Room f;
    const uint64_t stats = part_bytes(cnr_ceil_div(s.vocab, 64)), narrow = least(s.n, narrow_rows(s)) * part_bytes(cnr_ceil_div(s.vocab, 16));
    uint64_t parts = least(s.n * stats, kStatsBytes);
    parts = parts > small * stats ? parts : small * stats;
    f.take((parts > narrow ? parts : narrow) + 256);
    f.take(s.n * sizeof(float));
    if (s.n > narrow_rows(s)) {
        f.take(s.n * s.row);
        f.take(most_weight * s.row);
    }
    if (!training) return f.used;
    Room b;
    const uint64_t of_dz = s.n * 2 * dz_parts(s, wide);
    b.take(2 * sizeof(float));
    b.take(rounded(s.n, 256) * sizeof(RowGradient));
    const uint64_t few = least(s.n, kThreePartRows) * 2 * 3, vocab = rounded(s.vocab, dense::kBlockElements);
    uint64_t tiled = least(of_dz * vocab, 2 * kPieceBytes + 256 * of_dz);
    tiled = tiled > least(few * vocab, 2 * kPieceBytes + 256 * few) ? tiled : least(few * vocab, 2 * kPieceBytes + 256 * few);
    const uint64_t narrow_dz = least(s.vocab * padded_rows(least(s.n, narrow_rows(s))) * sizeof(float), 2 * kPieceBytes);
    b.take(tiled > narrow_dz ? tiled : narrow_dz);
    b.take(s.n * s.row);
    b.take(most_weight * s.row);
    b.take(s.n * s.dim * sizeof(float));
    b.take(kPartBytes);
    return b.used > f.used ? b.used : f.used;
}

// Grids count threads in 32 bits, and 2^20 rows of 2^15 elements are 2^32 pieces of 16 bytes: launch(first, groups) for a thread to each of `threads` things.
constexpr uint64_t kLaunchThreads = 1ull << 28;
template <typename Launch>
void in_launches(uint64_t threads, const Launch &launch) {
    for (uint64_t first = 0; first < threads; first += kLaunchThreads) launch(first, (unsigned)cnr_ceil_div(least(threads - first, kLaunchThreads), kBlock));
}

}  // namespace
