// How the operators of a stored layer in use (adapt.hip, loss.hip) are split
// into tiles, splits and launches, and the workspaces that takes: host code
// that goes by sizes alone.
//
// A plan of fewer tokens may split more and need more for its partial sums than
// one of many.  These sums have a limit each, and what a call asks for (the
// functions most_...) is a bound that grows with its tokens: a workspace for a
// program's most tokens serves its every call, and each call takes the same way
// whatever it is given.
//
// Times beside the rules are of one MI355X.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round_256(size_t bytes) { return (bytes + 255) / 256 * 256; }  // parts of a workspace

constexpr int kCUs = 256;

// A product in tiles of one size and splits of k, whose partial sums are
// written and read again.
enum Size { kLarge, kMiddle, kSmall };
struct Split {
    Size size;
    int64_t k;   // of a split, a multiple of 64
    int splits;
    int64_t side_m() const { return size == kSmall ? 128 : 256; }
    int64_t side_n() const { return size == kLarge ? 256 : 128; }
    int64_t units(int64_t m, int64_t n) const {
        return (m + side_m() - 1) / side_m() * ((n + side_n() - 1) / side_n());
    }
};

// Estimated time of it in us: rounds of up to 256 blocks, each with its start
// and end and its stages of 64 k.  A stage takes 1.2 to 1.6 us in the large
// tile, 0.75 to 1.0 in the middle one and 0.5 to 0.6 in the small one, by how
// many of the CUs share the L2s (measured at 1024 x 1024 to 8192 x 8192, 4096
// deep); sums go at 5 TB/s.
inline double split_us(int64_t m, int64_t n, int64_t k, const Split &p) {
    const int64_t units = p.units(m, n) * p.splits;
    const double full = units < kCUs ? (double)units / kCUs : 1.0;
    const double stage = p.size == kLarge ? 1.2 + 0.4 * full : p.size == kMiddle ? 0.75 + 0.25 * full
                                                                                 : 0.5 + 0.1 * full;
    const double stages = (double)(((k + 63) / 64 + p.splits - 1) / p.splits);
    return (units + kCUs - 1) / kCUs * (stages * stage + 3.0) + 3.0 +
           (p.splits > 1 ? 3.0 + p.splits * m * n * 8 / 5.0e6 : 0.0);
}

constexpr int kMostSplits = 32;
constexpr int64_t kLeastSplit = 256;  // k of one

// Limits of partial sums: of a product in tiles, of the layer for few tokens and
// of logits.  At 5 TB/s 256 MB take 107 us to write and read again, as long as
// 67 stages of the large tile; one round of 256 blocks has sums of 16 to 64 MB.
constexpr int64_t kTileSums = (int64_t)256 << 20, kFewSums = (int64_t)64 << 20, kLogitSums = (int64_t)32 << 20;

// The tile and the splits of the least estimated time, whose sums are at most
// `most` bytes (0: not split).
inline Split split_plan(int64_t m, int64_t n, int64_t k, int64_t most) {
    Split least{kLarge, k, 1};
    double best = split_us(m, n, k, least);
    for (int size = kLarge; size <= kSmall; ++size)
        for (int64_t s = 1; s == 1 || (s <= kMostSplits && cdiv(k, s) >= kLeastSplit && s * m * n * 4 <= most); ++s) {
            const Split p{(Size)size, (k + s - 1) / s, (int)s};
            const double us = split_us(m, n, k, p);
            if (us < best) {
                best = us;
                least = p;
            }
        }
    least.k = (least.k + 63) / 64 * 64;
    least.splits = (int)((k + least.k - 1) / least.k);
    return least;
}

inline size_t sum_bytes(const Split &p, int64_t m, int64_t n) {
    return p.splits > 1 ? round_256((size_t)p.splits * m * n * 4) : 0;
}

// Of split_plan(m, up to n, up to k, most).
inline size_t most_sums(int64_t m, int64_t n, int64_t k, int64_t most) {
    const int64_t splits = std::min<int64_t>(kMostSplits, (k - 1) / (kLeastSplit - 1));
    return splits > 1 ? round_256((size_t)std::min(splits * m * n * 4, most)) : 0;
}

// ---------------------------------------------------------------------------
// The layer and its adapters
// ---------------------------------------------------------------------------

constexpr int kLowStep = 256;                   // down to the rank: k of a split is a multiple of it
constexpr int kFewLowK = 1024;                  // k of a block of it for few tokens
constexpr int kFewK = 512, kFewRows = 128;      // few tokens: a split is a multiple of kFewK, output rows of a block
constexpr int kOuterCols = 256, kOuterTokens = 64;  // gradients of the adapters: columns of a block, tokens of a stage
constexpr int kTargetBlocks = 1024;

// Up to 1024 tokens the stored weights go straight into the product; above,
// they are converted once and multiplied in tiles.  That way (and the other),
// us: 512 tokens of 4096 -> 14336 75 (151); 1040 of 4096 -> 14336 153 (161),
// of 14336 -> 4096 191 (169), of 4096 -> 4096 71 (65), of 4096 -> 1024 27 (29);
// 2040 of 4096 -> 14336 274 (243).
constexpr int64_t kFewTokens = 1024;
// Up to 64 tokens a block takes them all, in sixteens, above it takes 128.  The
// adapters' part is computed beside the product and added at its end (fused)
// while tokens x outputs x rank are few: the end reads B once per token, where
// the product's own stages, after two kernels before it, read it once per block
// of tokens and adapter among them.  Fused (and not), us, 64 tokens with 1, 8
// and 32 adapters: 4096 -> 4096, rank 128 26 (29), 32 (45), 48 (103), rank 256
// 36 (34), 52 (66), 84 (161); 4096 -> 14336, rank 64 50 (35), 55 (43), 65 (77),
// rank 128 75 (37), 83 (53), 165 (114), rank 256 128 (42), 151 (74), 369 (214).
// The limit up to 64 tokens, 80 Mi, lies where no number of adapters loses much.
// 80 tokens of 4096 -> 14336 with eight of rank 16 take 38 us fused.
constexpr int64_t kFewTile = 64, kFewFused = 512;
constexpr int64_t kFewTileWork = (int64_t)80 << 20, kFewFusedWork = (int64_t)64 << 20;  // up to 64 tokens, and above

inline int rank_pad(int rank) { return (rank + 31) / 32 * 32; }
inline int low_pad(int rank) { return (rank + 15) / 16 * 16; }

struct Low {
    int64_t k_split;
    int splits, slots;
};

// Ranks that a block of the product down to the rank takes.
inline int rank_tile(int rank) { return rank <= 32 ? 32 : 64; }

// Splits of k for the product down to the rank: as many as fill the chip, of
// at least 512 k.
inline Low low_plan(int64_t tokens, int64_t width, int count, int rank) {
    Low p;
    const int64_t blocks = cdiv(tokens, 128) * cdiv(rank, rank_tile(rank));
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(kTargetBlocks / blocks, cdiv(width, 2 * kLowStep)));
    p.k_split = cdiv(cdiv(width, want), kLowStep) * kLowStep;
    p.splits = (int)cdiv(width, p.k_split);
    // a slot more costs blocks that find no adapter; few tiles leave room for them
    p.slots = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(count, 8), 2 * kTargetBlocks / (blocks * p.splits)));
    return p;
}

inline size_t low_partial_bytes(const Low &p, int64_t tokens, int rank) {
    return round_256((size_t)p.splits * tokens * rank_pad(rank) * 4);
}

// Of low_plan for up to `tokens`: splits x tokens are at most kTargetBlocks x 128
// over the rank's tiles, or the tokens.
inline size_t most_low_partial(int64_t tokens, int64_t width, int rank) {
    const int64_t rows = std::min(cdiv(width, 2 * kLowStep) * tokens,
                                  (int64_t)kTargetBlocks * 128 / cdiv(rank, rank_tile(rank)));
    return round_256((size_t)std::max(tokens, rows) * rank_pad(rank) * 4);
}

inline size_t low_bytes(int64_t tokens, int rank) { return round_256((size_t)tokens * 2 * low_pad(rank) * 2); }

struct FewPlan {
    int64_t k_split;
    int splits, low_splits, low_slots;
    bool fused;  // the adapters' part beside the weights' and in the end, not before and with them
    int tile;    // tokens a block, in sixteens
};

// A launch's threads are fewer than 2^32: of 512 each, half of that for these.
constexpr int64_t kMostLowBlocks = (int64_t)1 << 22;

// Blocks down to the rank: tiles of 32 tokens and 32 ranks, each split and slot.
inline int64_t few_low_blocks(const FewPlan &p, int64_t tokens, int rank) {
    return cdiv(tokens, 32) * (rank_pad(rank) / 32) * p.low_splits * p.low_slots;
}

// The splits of k of the least estimated time in us: rounds of one or two
// blocks a CU, 256 k of a block in 1.2 to 2.4 us by its tokens (128 tokens
// 2.3, measured at 512 tokens, 4096 -> 14336), partial sums at 5 TB/s.
inline FewPlan few_plan(int64_t tokens, int64_t in, int64_t out, int count, int rank) {
    FewPlan p;
    p.tile = tokens > 64 ? 8 : (int)cdiv(tokens, 16);
    p.low_splits = (int)cdiv(in, kFewLowK);
    p.low_slots = (int)std::min<int64_t>(count, std::min<int64_t>(tokens, 32));
    p.fused = count > 0 && tokens <= kFewFused && few_low_blocks(p, tokens, rank) <= kMostLowBlocks &&
              tokens * out * (rank + 8) <= (tokens <= kFewTile ? kFewTileWork : kFewFusedWork);
    const int64_t blocks = cdiv(out, kFewRows) * cdiv(tokens, 16 * p.tile), slots = p.tile > 4 ? kCUs : 2 * kCUs;
    double least = 0.0;
    for (int64_t s = 1; s <= kMostSplits && s <= cdiv(in, kFewK); ++s) {
        const int64_t k = cdiv(cdiv(in, s), kFewK) * kFewK, n = cdiv(in, k);
        if (n > 1 && n * tokens * out * 4 > kFewSums) continue;
        const double each = p.tile > 4 ? 2.3 : 0.9 + 0.35 * p.tile;
        const double us = cdiv(blocks * n, slots) * (k / 256 * each + 2.0) +
                          (n > 1 || p.fused ? 3.0 + n * tokens * out * 8 / 5.0e6 : 0.0);
        if (s > 1 && us >= least) continue;
        least = us;
        p.k_split = k;
        p.splits = (int)n;
    }
    return p;
}

struct LinearPlan {
    bool few;
    FewPlan base;
    Low low;
    Split tile;
    size_t weights, partial, low_partial, low_parts, total;
};

inline LinearPlan linear_plan(int64_t tokens, int64_t in, int64_t out, int count, int rank) {
    LinearPlan p{};
    p.few = tokens <= kFewTokens;
    if (p.few) {
        p.base = few_plan(tokens, in, out, count, rank);
        if (p.base.fused || p.base.splits > 1) p.partial = round_256((size_t)p.base.splits * tokens * out * 4);
    } else {
        p.weights = round_256((size_t)out * in * 2);
        p.tile = split_plan(out, tokens, in, kTileSums);
        p.partial = sum_bytes(p.tile, out, tokens);
    }
    if (p.few && p.base.fused) {
        p.low_partial = round_256((size_t)p.base.low_splits * tokens * rank_pad(rank) * 4);
    } else if (count > 0) {
        p.low = low_plan(tokens, in, count, rank);
        p.low_partial = low_partial_bytes(p.low, tokens, rank);
        p.low_parts = low_bytes(tokens, rank);
    }
    p.total = p.weights + p.partial + p.low_partial + p.low_parts;
    return p;
}

// Of linear_plan for up to `tokens`.
inline size_t most_linear(int64_t tokens, int64_t in, int64_t out, int count, int rank) {
    const int64_t t = std::min(tokens, kFewTokens), splits = std::min<int64_t>(kMostSplits, cdiv(in, kFewK));
    int64_t sums = splits > 1 ? std::min(splits * t * out * 4, kFewSums) : 0;
    size_t low = 0;
    if (count > 0) {  // fused, k may be whole
        sums = std::max(sums, std::min(std::min(t, kFewTile) * out, kFewTileWork / (rank + 8)) * 4);
        sums = std::max(sums, std::min(t * out, kFewFusedWork / (rank + 8)) * 4);
        const size_t fused = (size_t)cdiv(in, kFewLowK) * std::min(t, kFewFused) * rank_pad(rank) * 4;
        low = std::max(round_256(fused), most_low_partial(t, in, rank)) + low_bytes(t, rank);
    }
    const size_t few = round_256((size_t)sums) + low;
    if (tokens <= kFewTokens) return few;
    const size_t many = round_256((size_t)out * in * 2) + most_sums(out, tokens, in, kTileSums) +
                        (count > 0 ? most_low_partial(tokens, in, rank) + low_bytes(tokens, rank) : 0);
    return std::max(few, many);
}

struct GradPlan {
    int64_t width;  // columns of dY as the kernels read it
    bool widen;
    Low v, u;
    int64_t split_a, split_b;
    int splits_a, splits_b;
    Split tile;
    size_t weights, dy, turned, low_partial, low, outer, total;
};

// Up to 512 tokens are not split for the adapters' gradients, which saves the
// partial sums and the kernels that add them: 500 tokens of 1024 -> 4096, eight
// adapters of rank 32, 70 us so and 79 in two splits; 512 of 8192 -> 1024, one
// of rank 64, 83 and 82.
constexpr int64_t kOuterWhole = 512;

// Splits of the tokens for the adapters' gradients, and the most of them.
inline int64_t most_outer_splits(int64_t tokens, int64_t width, int count, int rank) {
    const int64_t blocks = cdiv(width, kOuterCols) * cdiv(rank, rank_tile(rank)) * count;
    return tokens <= kOuterWhole ? 1 : std::min(cdiv(kTargetBlocks, blocks), cdiv(tokens, 256));
}

inline void outer_plan(int64_t tokens, int64_t width, int count, int rank, int64_t &split, int &splits) {
    const int64_t want = most_outer_splits(tokens, width, count, rank);
    split = cdiv(cdiv(tokens, want), kOuterTokens) * kOuterTokens;
    splits = (int)cdiv(tokens, split);
}

inline GradPlan grad_plan(int64_t tokens, int64_t in, int64_t out, int count, int rank, bool widen) {
    GradPlan p{};
    p.width = cdiv(out, 16) * 16;
    p.widen = widen;
    p.weights = round_256((size_t)out * in * 2);
    p.dy = widen ? round_256((size_t)tokens * p.width * 2) : 0;
    p.turned = round_256((size_t)count * rank * p.width * 2);
    p.v = low_plan(tokens, p.width, count, rank);
    p.u = low_plan(tokens, in, count, rank);
    p.low_partial = std::max(low_partial_bytes(p.v, tokens, rank), low_partial_bytes(p.u, tokens, rank));
    p.low = low_bytes(tokens, rank);
    outer_plan(tokens, in, count, rank, p.split_a, p.splits_a);
    outer_plan(tokens, p.width, count, rank, p.split_b, p.splits_b);
    const size_t cols_a = p.splits_a > 1 ? (size_t)p.splits_a * in : 0;
    const size_t cols_b = p.splits_b > 1 ? (size_t)p.splits_b * p.width : 0;
    p.outer = round_256(std::max(cols_a, cols_b) * count * rank * 4);
    p.tile = split_plan(in, tokens, p.width, kTileSums);
    p.outer = std::max(p.outer, sum_bytes(p.tile, in, tokens));  // in turn
    p.total = p.weights + p.dy + p.turned + p.low_partial + 2 * p.low + p.outer;
    return p;
}

// Of grad_plan for up to `tokens`.
inline size_t most_grad(int64_t tokens, int64_t in, int64_t out, int count, int rank, bool widen) {
    const int64_t width = cdiv(out, 16) * 16;
    const int64_t a = most_outer_splits(tokens, in, count, rank), b = most_outer_splits(tokens, width, count, rank);
    const int64_t cols = std::max(a > 1 ? a * in : 0, b > 1 ? b * width : 0);
    const size_t outer = round_256((size_t)cols * count * rank * 4);
    return round_256((size_t)out * in * 2) + (widen ? round_256((size_t)tokens * width * 2) : 0) +
           round_256((size_t)count * rank * width * 2) +
           std::max(most_low_partial(tokens, width, rank), most_low_partial(tokens, in, rank)) +
           2 * low_bytes(tokens, rank) + std::max(outer, most_sums(in, tokens, width, kTileSums));
}

// ---------------------------------------------------------------------------
// The token loss and its gradient
// ---------------------------------------------------------------------------

constexpr int kMost = 256;  // parts of the largest weight

// k is split where 128 x 128 tiles leave half the chip without one.  Loss of 20
// tokens of 8192 over 500 words: 18 us so, 66 in one pass; of 300 over 2000: 29
// and 67; at 250 tiles (64 tokens of 4096 over 32000 words) both take 68.
inline Split logit_plan(int64_t words, int64_t tokens, int64_t d, bool one_piece) {
    return split_plan(words, tokens, d, one_piece && cdiv(words, 128) * cdiv(tokens, 128) <= kCUs / 2 ? kLogitSums : 0);
}

// Of logit_plan for up to `tokens`.
inline size_t most_logit_sums(int64_t words, int64_t tokens, int64_t d) {
    return cdiv(words, 128) <= kCUs / 2 ? most_sums(words, tokens, d, kLogitSums) : 0;
}

struct LossPlan {
    Split tile;
    size_t parts, at, total;  // parts: partial sums, if split
};

inline LossPlan loss_plan(int64_t tokens, int64_t d, int64_t vocab) {
    LossPlan p;
    const int64_t words = cdiv(vocab, 4) * 4;
    p.tile = logit_plan(words, tokens, d, true);
    if (p.tile.splits > 1) {
        p.parts = p.total = round_256((size_t)p.tile.splits * tokens * words * 4);
        p.at = 0;
        return p;
    }
    p.parts = round_256((size_t)cdiv(vocab, p.tile.side_m()) * tokens * 2 * sizeof(float));
    p.at = round_256((size_t)tokens * 4);
    p.total = p.parts + p.at;
    return p;
}

// Of loss_plan for up to `tokens`.
inline size_t most_loss(int64_t tokens, int64_t d, int64_t vocab) {
    const size_t parts = round_256((size_t)cdiv(vocab, 128) * tokens * 2 * sizeof(float));
    return std::max(parts + round_256((size_t)tokens * 4), most_logit_sums(cdiv(vocab, 4) * 4, tokens, d));
}

// Both parts of a piece of g take up to 380 MB, and at least 2048 of the
// vocabulary: so that a piece's products fill the chip many times over, and its
// sums in dX, read and written once a piece, stay below a twentieth of them.
constexpr int64_t kPieceBytes = (int64_t)380 << 20;
constexpr int64_t kLeastPiece = 2048;
constexpr int64_t kPieceStep = 256;

struct LossGradPlan {
    int64_t piece, pieces;
    Split dx, logits;  // logits: of a single piece, whose k may be split
    size_t g, sum, rows, factor, total;
};

inline LossGradPlan loss_grad_plan(int64_t tokens, int64_t d, int64_t vocab, bool dw) {
    LossGradPlan p;
    const int64_t fit = std::max(kLeastPiece, kPieceBytes / (4 * tokens) / kPieceStep * kPieceStep);
    p.pieces = cdiv(vocab, fit);
    p.piece = cdiv(cdiv(vocab, p.pieces), kPieceStep) * kPieceStep;
    p.pieces = cdiv(vocab, p.piece);
    p.dx = split_plan(d, tokens, 2 * p.piece, kTileSums);  // both parts
    p.dx.k = cdiv(cdiv(p.piece, p.dx.splits), 64) * 64;
    p.dx.splits = (int)cdiv(p.piece, p.dx.k);
    p.logits = logit_plan(p.piece, tokens, d, p.pieces == 1);
    p.g = round_256((size_t)tokens * p.piece * 4);
    p.sum = round_256((size_t)p.dx.splits * tokens * d * 4);
    if (p.logits.splits > 1)  // in turn
        p.sum = std::max(p.sum, round_256((size_t)p.logits.splits * tokens * p.piece * 4));
    p.rows = dw ? round_256((size_t)tokens * d * 2) : 0;
    p.factor = round_256((size_t)tokens * sizeof(float));
    p.total = p.g + p.sum + p.rows + p.factor + kMost * sizeof(float);
    return p;
}

// Of loss_grad_plan for up to `tokens`.
inline size_t most_loss_grad(int64_t tokens, int64_t d, int64_t vocab, bool dw) {
    const int64_t words = cdiv(vocab, kPieceStep) * kPieceStep;
    const int64_t g = std::min(std::max(kPieceBytes, 4 * tokens * kLeastPiece), 4 * tokens * words);
    const size_t sum = std::max(round_256((size_t)tokens * d * 4), most_sums(d, tokens, 2 * words, kTileSums));
    return round_256((size_t)g) + std::max(sum, most_logit_sums(words, tokens, d)) +
           (dw ? round_256((size_t)tokens * d * 2) : 0) + round_256((size_t)tokens * sizeof(float)) +
           kMost * sizeof(float);
}

// The tiles of a piece's slopes (`ldg` words) and of its rows of dW (`cols`).
inline Split slope_plan(int64_t ldg, int64_t tokens, int64_t d) { return split_plan(ldg, tokens, d, 0); }
inline Split dw_plan(int64_t d, int64_t cols, int64_t tokens) { return split_plan(d, cols, 2 * tokens, 0); }

}  // namespace
