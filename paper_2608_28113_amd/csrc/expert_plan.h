// How a layer of stored experts (experts.hip) goes in pieces, blocks and
// splits, and the workspace that takes: host code that goes by sizes alone.
//
// The order in which a token's products are added up - the waves that share a
// row of gate and up, the splits of the down product's k - is chosen once for a
// call, by the most tokens that one of its pieces may have.  How many slots a
// block takes is chosen for each piece: it changes no order of summation.  So a
// token's bits are the same in every piece, and X's stride, which makes pieces
// smaller, does not change them either.  A short last piece pays for it: 52
// tokens behind 2048 (2 of 8 experts of 2048 x 2048) take 13 us of 266 more than
// in four splits of their own, one behind 682 (6 of 64 of 2048 x 1024) 6 of 186.
//
// Times beside the rules are of one MI355X.
#pragma once

#include "plan.h"

namespace {

constexpr int kMaxExperts = 1024;
constexpr int kMaxChoices = 32;
constexpr int64_t kMaxWidth = (int64_t)1 << 21;
constexpr int64_t kMaxTokens = (int64_t)1 << 24;

constexpr int kPieceSlots = 4096;  // a call of more goes piece by piece

// Up to so many, each block finds its expert's slots itself: at 512 slots as fast
// as sorting them in a launch (306 us, 64 tokens over 128 experts of 4096 x 1536),
// and with room for 1024 all calls take 3 to 8 % longer.  One column of blocks
// then takes all slots of an expert, a tile after the other: 128 tokens over 2 of
// 8 experts of 4096 x 14336 take 371 us, 429 where all choose the same two, and
// 129 tokens, sorted, 324 and 281.
constexpr int kBlockSlots = 256;

// Up to a block's slots of one expert; count 0: none.
struct Share {
    int expert, first, count;
};

inline bool layer_sizes_ok(int64_t tokens, int64_t in, int64_t hidden, int32_t experts, int32_t k) {
    return tokens >= 0 && tokens <= kMaxTokens && in >= 0 && in % 16 == 0 && in <= kMaxWidth && hidden >= 0 &&
           hidden % 16 == 0 && hidden <= kMaxWidth && experts >= 1 && experts <= kMaxExperts && k >= 1 &&
           k <= kMaxChoices;
}

// The most tokens of a piece: h and the sums take no more than 1 GB each, and
// are addressed in 32 bits.
inline int64_t most_tokens(int64_t in, int64_t hidden, int32_t k) {
    return std::max<int64_t>(1, std::min<int64_t>(kPieceSlots / k, ((int64_t)1 << 28) / (std::max(in, hidden) * k)));
}

constexpr int kDownSplits = 16;
constexpr int64_t kSplitBytes = (int64_t)32 << 20;  // of their sums, unless one takes more

struct LayerSpace {
    size_t h, p, order, shares, total;
};

inline LayerSpace layer_space(int64_t tokens, int64_t in, int64_t hidden, int32_t experts, int32_t k) {
    const int64_t slots = std::min(tokens, most_tokens(in, hidden, k)) * k;
    LayerSpace s{};
    s.h = round_256((size_t)(slots * hidden * 4));
    // Splits of few tokens are more: a bound that does not fall with the tokens.
    s.p = round_256((size_t)std::min(slots * in * 4 * kDownSplits, std::max(slots * in * 4, kSplitBytes)));
    s.order = round_256((size_t)slots * 4);
    s.shares = round_256((size_t)(slots + experts) * sizeof(Share));
    s.total = s.h + s.p + s.order + s.shares;
    return s;
}

// Slots of a block: as many as an expert's share is likely to need.  us of the
// whole call in blocks of 16, 32 and 64, for 32 experts of 2048 x 1024 with on
// average
//   9 slots   48.3  49.0  62.4       24 slots  67.0  59.0  65.7
//   12 slots  52.4  49.4  63.0       32 slots  78.3  66.6  70.6
//   16 slots  55.5  51.3  64.8       40 slots  88.5  76.9  72.6
// and for 16 of 4096 x 1536 59.7, 69.6, 89.1 with 9 and 128, 101, 101 with 40.
inline int slots_of_block(int64_t tokens, int64_t slots, int64_t experts) {
    if (tokens <= 4) return 4;
    if (tokens <= 16 || slots <= 10 * experts) return 16;
    return tokens <= 32 || slots <= 34 * experts ? 32 : 64;
}

// Shares of the experts, or a bound of them: what a launch has blocks for.
inline int shares_of(int64_t slots, int tile, int32_t experts) {
    const int64_t most = slots > kBlockSlots ? slots / tile + experts : experts;
    return (int)std::min(slots, most);
}

// Waves of gate and up that share their rows.  A wave alone has its rows where
// they are many.  Where they are few, two waves share them, or four in blocks of
// 32 and 64 slots.  us of the whole call, one, two and four waves:
//   1 token through 6 of 64 experts of 2048 x 1024     28.4  24.2  25.2
//   12 tokens through 6 of 64 of 2048 x 1408           70.1  75.9  115
// Blocks of four waves take 16 rows: 512 of them, two a CU, are one round of 32
// slots.  More are two, and one wave alone is faster by then.  Blocks of 64
// slots have a CU each, and a few rounds of them still gain where k is long.
// In a graph, one and four waves, `u` rows / 128 x shares:
//   32 slots  in 1024  u 64  26.5  26.5     64 slots  in 1040  u 49  45.7  46.2
//             in 1040  u 64  28.2  26.9               in 1536  u 80  50.5  47.0
//             in 4096  u 64  42.1  35.9               in 2048  u 98  56.0  48.8
//             in 1040  u 66  29.2  32.4               in 4096  u 99  91.0  89.1
//             in 4096  u 66  44.7  46.4               in 2048 u 110  57.8  69.8
//             in 4096 u 110  52.9  61.1               in 4096 u 110  91.6   105
inline int waves_of_row(int64_t in, int64_t hidden, int shares, int tile) {
    const int64_t u = cdiv(hidden, 128) * shares, steps = cdiv(in, 256);
    if (tile <= 16) return cdiv(hidden, 16) * shares < 4096 && steps >= 2 ? 2 : 1;
    return (tile == 32 ? u <= 64 && steps >= 4 : u <= 100 && steps >= 6) ? 4 : 1;
}

// Splits of the down product's k, for `shares` shares of experts: two blocks a CU
// (37 tokens over 8 experts of 4096 x 14336, 256 blocks: 192 us in two splits, 204
// in one, 197 in four; one token over two of them, 64 blocks: 64 us in eight, 66 in
// four, 110 in one).
inline int down_splits(int64_t slots, int64_t in, int64_t hidden, int64_t shares) {
    const int64_t steps = cdiv(hidden, 256), blocks = cdiv(in, 128) * shares;
    int64_t n = cdiv(512, blocks);
    n = std::min({n, steps, (int64_t)kDownSplits, std::max<int64_t>(1, kSplitBytes / (slots * in * 4))});
    n = std::max<int64_t>(1, n);
    return (int)cdiv(steps, cdiv(steps, n));
}

struct LayerPlan {
    int64_t piece;     // tokens
    int waves, splits;
    int split;         // steps of 256 k of a split
};

inline LayerPlan plan_layer(int64_t tokens, int64_t in, int64_t hidden, int32_t experts, int32_t k, int64_t ldx) {
    const int64_t most = std::min(tokens, most_tokens(in, hidden, k)), slots = most * k;
    const int tile = slots_of_block(most, slots, experts), shares = shares_of(slots, tile, experts);
    LayerPlan p{};
    // Rows of X are addressed in 32 bits too.
    p.piece = std::min(most, std::max<int64_t>(1, ((int64_t)1 << 29) / ldx));
    p.waves = waves_of_row(in, hidden, shares, tile);
    p.splits = down_splits(slots, in, hidden, shares);
    p.split = (int)cdiv(cdiv(hidden, 256), p.splits);
    return p;
}

struct PiecePlan {
    int slots, tile, shares;
    bool many;  // slots are sorted first
};

inline PiecePlan plan_piece(const LayerPlan &p, int64_t tokens, int32_t experts, int32_t k) {
    PiecePlan q{};
    q.slots = (int)(tokens * k);
    q.tile = slots_of_block(tokens, q.slots, experts);
    if (p.waves == 4) q.tile = std::max(q.tile, 32);  // the least that four waves are built for
    q.shares = shares_of(q.slots, q.tile, experts);
    q.many = q.slots > kBlockSlots;
    return q;
}

}  // namespace
