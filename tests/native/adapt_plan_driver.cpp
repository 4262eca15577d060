// The plans behind the adapted layer, its gradients and the token loss, alone
// (plan.h is plain C++).  Without arguments: over many sizes, what a plan uses
// is at most what its call asks for, and that never falls with the tokens.
// And no launch of one dimension has 2^32 threads.
// With an argument: reads calls, one a line, from standard input and prints
// the ways they take, one of a kernel a word.
//   linear TOKENS IN OUT COUNT RANK | grad ... | loss TOKENS D VOCAB | loss_grad ...
#include <cstdio>
#include <cstring>
#include <string>

#include "plan.h"

static const char *size_of(const Split &p) { return p.size == kLarge ? "256x256" : p.size == kMiddle ? "256x128" : "128x128"; }
static std::string tiles(const char *kernel, const Split &p) {
    return std::string(kernel) + ":" + size_of(p) + (p.splits > 1 ? ":split " : ":whole ");
}
static std::string down(const char *of, const Low &p, int rank) {
    return std::string("shrink:") + of + (rank <= 32 ? ":32" : ":64") + (p.splits > 1 ? ":split " : ":whole ");
}

static std::string linear(int64_t t, int64_t in, int64_t out, int count, int rank) {
    const LinearPlan p = linear_plan(t, in, out, count, rank);
    std::string s;
    if (p.low_parts) s += down("bf16", p.low, rank);
    if (!p.few) return s + tiles(count ? "layer_along+adapters" : "layer_along", p.tile);
    return s + "few:" + std::to_string(p.base.tile) + (in % 32 ? ":odd" : ":even") +
           (!count ? ":alone" : p.base.fused ? ":fused" : ":adapters") + (p.base.splits > 1 ? ":split " : ":whole ");
}

static std::string grad(int64_t t, int64_t in, int64_t out, int count, int rank) {
    const GradPlan p = grad_plan(t, in, out, count, rank, out % 16 != 0);
    const auto outer = [&](const char *of, int splits) {
        return std::string("outer:") + of + (rank <= 32 ? ":32" : ":64") + (splits > 1 ? ":split " : ":whole ");
    };
    return down("bf16", p.v, rank) + down("int8", p.u, rank) + tiles("layer_across", p.tile) +
           outer("int8", p.splits_a) + outer("bf16", p.splits_b) + (p.widen ? "widen " : "");
}

static std::string loss(int64_t t, int64_t d, int64_t vocab) {
    const LossPlan p = loss_plan(t, d, vocab);
    return tiles(p.tile.splits > 1 ? "logit_sum" : "loss_tile", p.tile);
}

static std::string loss_grad(int64_t t, int64_t d, int64_t vocab) {
    const LossGradPlan p = loss_grad_plan(t, d, vocab, true);
    std::string s = p.pieces > 1 ? "pieces " : "";
    s += tiles("loss_dx", p.dx);
    for (int64_t v0 = 0; v0 < vocab; v0 += p.piece) {
        const int64_t cols = std::min(p.piece, vocab - v0), ldg = cdiv(cols, kPieceStep) * kPieceStep;
        s += p.logits.splits > 1 ? tiles("logit_sum+slope", p.logits) : tiles("loss_slope", slope_plan(ldg, t, d));
        s += tiles("loss_dw", dw_plan(d, cols, t));
    }
    return s;
}

static int bad = 0;

// The blocks of 512 threads of the layer for few tokens: those down to the rank,
// then those of the product.
static void launchable(int64_t t, int64_t in, int64_t out, int count, int rank) {
    const FewPlan p = few_plan(t, in, out, count, rank);
    const int64_t blocks = (p.fused ? few_low_blocks(p, t, rank) : 0) +
                           cdiv(out, kFewRows) * p.splits * cdiv(t, 16 * p.tile);
    if (blocks * 512 >= (int64_t)1 << 32 && bad++ < 10)
        std::printf("adapted_linear %lld x %lld, %d of rank %d, %lld tokens: %lld blocks\n", (long long)in,
                    (long long)out, count, rank, (long long)t, (long long)blocks);
}

template <class Used, class Most>
static void grows(const char *what, int64_t a, int64_t b, int count, int rank, const Used &used, const Most &most) {
    size_t before = 0;
    for (int64_t t = 1; t <= (1 << 24); t += t < 1300 ? 1 : t / 61) {
        const size_t u = used(t), m = most(t);
        if (u > m || m < before) {
            if (bad++ < 10)
                std::printf("%s %lld x %lld, %d of rank %d, %lld tokens: uses %zu, asks for %zu, %zu for fewer\n", what,
                            (long long)a, (long long)b, count, rank, (long long)t, u, m, before);
        }
        before = m;
    }
}

int main(int argc, char **) {
    if (argc > 1) {
        char what[16];
        long long t, a, b;
        int count = 0, rank = 0;
        while (std::scanf("%15s %lld %lld %lld %d %d", what, &t, &a, &b, &count, &rank) == 6)
            std::puts((!std::strcmp(what, "linear") ? linear(t, a, b, count, rank)
                       : !std::strcmp(what, "grad") ? grad(t, a, b, count, rank)
                       : !std::strcmp(what, "loss") ? loss(t, a, b)
                                                    : loss_grad(t, a, b))
                          .c_str());
        return 0;
    }
    const int64_t widths[] = {16, 64, 512, 1040, 4096, 14336, 1 << 21}, outs[] = {1, 24, 100, 1030, 4096, 14336, 1 << 21};
    const int adapters[][2] = {{0, 0}, {1, 8}, {8, 32}, {32, 16}, {3, 40}, {300, 256}, {4096, 8}};
    for (int64_t n : widths)
        for (int64_t m : outs) {
            for (const auto &a : adapters) {
                const int c = a[0], r = a[1];
                for (int64_t t = 1; t <= kFewTokens; ++t) launchable(t, n, m, c, r);
                grows("adapted_linear", n, m, c, r, [&](int64_t t) { return linear_plan(t, n, m, c, r).total; },
                      [&](int64_t t) { return most_linear(t, n, m, c, r); });
                if (c)
                    for (bool w : {false, true})
                        grows("adapted_linear_grad", n, m, c, r,
                              [&](int64_t t) { return grad_plan(t, n, m, c, r, w).total; },
                              [&](int64_t t) { return most_grad(t, n, m, c, r, w); });
            }
            for (int64_t vocab : {m, m * 9 + 3}) {
                if (vocab > (1 << 24)) continue;
                grows("token_loss", n, vocab, 0, 0, [&](int64_t t) { return loss_plan(t, n, vocab).total; },
                      [&](int64_t t) { return most_loss(t, n, vocab); });
                for (bool w : {false, true})
                    grows("token_loss_grad", n, vocab, 0, 0,
                          [&](int64_t t) { return loss_grad_plan(t, n, vocab, w).total; },
                          [&](int64_t t) { return most_loss_grad(t, n, vocab, w); });
            }
        }
    if (bad) return 1;
    std::puts("plans: ok");
    return 0;
}
