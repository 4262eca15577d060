// The plans behind a layer of stored experts, alone (expert_plan.h is plain
// C++), over many sizes: what every launch writes lies within the part of the
// workspace that is meant for it, every token has a piece and every step of k a
// split, all pieces of a call add in one order, and what the kernels address in
// 32 bits and launch in one dimension fits.
// With an argument: reads calls from standard input, TOKENS IN HIDDEN EXPERTS K
// a line, and prints the ways they take, one of a kernel a word.
#include <cstdio>
#include <cstdlib>

#include "expert_plan.h"

static long calls = 0;

#define HOLDS(what)                                                                                             \
    if (!(what)) {                                                                                              \
        std::printf("%s: tokens %lld in %lld hidden %lld experts %d k %d ldx %lld\n", #what, (long long)tokens, \
                    (long long)in, (long long)hidden, experts, k, (long long)ldx);                              \
        std::exit(1);                                                                                           \
    }

static void piece_holds(const LayerPlan &p, const LayerSpace &s, int64_t n, int64_t tokens, int64_t in, int64_t hidden,
                        int experts, int k, int64_t ldx) {
    const PiecePlan q = plan_piece(p, n, experts, k);
    HOLDS(q.slots == n * k && q.slots >= 1);
    HOLDS((size_t)q.slots * hidden * 4 <= s.h && (size_t)p.splits * q.slots * in * 4 <= s.p);
    HOLDS(q.many == (q.slots > kBlockSlots));
    HOLDS(q.many || q.shares == std::min(q.slots, experts));
    HOLDS(!q.many || ((size_t)q.slots * 4 <= s.order && (size_t)q.shares * sizeof(Share) <= s.shares));
    // The most shares: a slot at each expert and the rest at few.
    const int64_t used = std::min(q.slots, experts), rest = q.slots - used;
    HOLDS(!q.many || used + rest / q.tile <= q.shares);
    // The kernels that there are.
    HOLDS(q.tile == 4 || q.tile == 16 || q.tile == 32 || q.tile == 64);
    HOLDS(p.waves == 1 || (p.waves == 2 && q.tile <= 16) || (p.waves == 4 && q.tile >= 32));
    // Splits of the down product, in its steps.
    const int64_t step = q.tile >= 32 ? 128 : 256, split = (int64_t)p.split * (256 / step), steps = cdiv(hidden, step);
    HOLDS(p.splits >= 1 && p.splits <= kDownSplits && (p.splits - 1) * split < steps && p.splits * split >= steps);
    // Reads of X and h stay below the offset that means none; launches below 2^16 blocks in y and z.
    HOLDS(((n - 1) * ldx + in) * 2 < 0x7FFF0000 && (int64_t)q.slots * hidden * 4 < 0x7FFF0000);
    HOLDS(q.shares <= 65535 && n <= 65535);
    ++calls;
}

static void call_holds(int64_t tokens, int64_t in, int64_t hidden, int experts, int k, int64_t ldx) {
    HOLDS(layer_sizes_ok(tokens, in, hidden, experts, k));
    const LayerSpace s = layer_space(tokens, in, hidden, experts, k);
    HOLDS(s.total == s.h + s.p + s.order + s.shares && s.h % 256 == 0 && s.p % 256 == 0 && s.order % 256 == 0);
    const LayerPlan p = plan_layer(tokens, in, hidden, experts, k, ldx);
    HOLDS(p.piece >= 1 && p.piece <= tokens);
    piece_holds(p, s, p.piece, tokens, in, hidden, experts, k, ldx);
    if (const int64_t last = tokens % p.piece) piece_holds(p, s, last, tokens, in, hidden, experts, k, ldx);
    const LayerPlan near = plan_layer(tokens, in, hidden, experts, k, in);  // rows one after another
    HOLDS(near.waves == p.waves && near.splits == p.splits && near.split == p.split && near.piece >= p.piece);
}

static void ways(int64_t tokens, int64_t in, int64_t hidden, int experts, int k) {
    const LayerPlan p = plan_layer(tokens, in, hidden, experts, k, in);
    for (int64_t n : {p.piece, tokens % p.piece}) {
        if (n == 0) continue;
        const PiecePlan q = plan_piece(p, n, experts, k);
        const int gate = q.tile == 4 && p.waves == 1 ? 16 : q.tile;  // four slots alone are built for two waves
        std::printf("slots:%s gate:%d:%d down:%d:%s ", q.many ? "sorted" : experts < q.slots ? "found" : "found-by-slot", gate,
                    p.waves, q.tile, p.splits > 1 ? "split" : "whole");
    }
    std::printf("\n");
}

int main(int argc, char **) {
    if (argc > 1) {
        long long t, in, hidden;
        int e, k;
        while (std::scanf("%lld %lld %lld %d %d", &t, &in, &hidden, &e, &k) == 5) ways(t, in, hidden, e, k);
        return 0;
    }
    const int64_t widths[] = {16, 32, 48, 112, 256, 272, 528, 1024, 1040, 2048, 4096, 14336, 1 << 16, (1 << 20) + 16, 1 << 21};
    const int64_t counts[] = {1, 2, 3, 4, 5, 12, 16, 17, 32, 33, 64, 100, 127, 128, 129, 255, 256, 257, 341, 342, 512, 682,
                              683, 1023, 1024, 1025, 2048, 2100, 4095, 4096, 4097, 5000, 8192, 8193, 100001, 1 << 24};
    for (int64_t tokens : counts)
        for (int64_t in : widths)
            for (int64_t hidden : widths)
                for (int experts : {1, 2, 3, 5, 8, 64, 127, 128, 300, 1024})
                    for (int k : {1, 2, 3, 6, 8, 31, 32})
                        for (int64_t ldx : {in, in + 8, (int64_t)1 << 19, kMaxWidth})
                            if (ldx >= in) call_holds(tokens, in, hidden, experts, k, ldx);
    std::printf("expert plans: ok, %ld pieces\n", calls);
    return calls < 1000 ? 1 : 0;
}
