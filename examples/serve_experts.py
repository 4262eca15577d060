"""A layer of experts is quantized and serves a few requests under their rules.

    python examples/serve_experts.py [--steps 12]

An embedding, one layer of routed experts and an output head stand for a model.
The experts' matrices and the head are stored in NVFP4 by the Hessian-guided
search, all of a kind in one launch and written where they are served from.
Then requests answer token by token: router, experts, head, and on the logits a
penalty for repeated words, a request's biases and a mask of the words that its
grammar allows.  One decode step is captured in a graph and replayed.
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

import paper_2608_28113_amd as hs  # noqa: E402


def stored_experts(W, h):
    """(global scales, codes, packed) of bf16 W [experts, out, in] for activations with diagonal h."""
    E, m, n = W.shape
    codes = torch.empty((E, m, n // 16), dtype=torch.uint8, device=W.device)
    packed = torch.empty((E, m, n // 2), dtype=torch.uint8, device=W.device)
    scales = [w.float().abs().max().item() / (448.0 * 6.0) for w in W]
    hs.search_layers([(W[e], h, scales[e]) for e in range(E)], down=9, up=6,
                     outputs=[(codes[e], packed[e]) for e in range(E)])
    return torch.tensor(scales, dtype=torch.float32, device=W.device), codes, packed


class Model:
    def __init__(self, vocab, width, hidden, experts, k, generator, device):
        def make(*shape, std):
            return (torch.randn(shape, generator=generator) * std).bfloat16().to(device)

        self.k = k
        self.embedding = make(vocab, width, std=1.0)
        self.router = make(experts, width, std=width ** -0.5)
        self.W = [make(experts, hidden, width, std=width ** -0.5), make(experts, hidden, width, std=width ** -0.5),
                  make(experts, width, hidden, std=hidden ** -0.5)]
        calibration = make(512, width, std=1.0)
        inner = make(512, hidden, std=0.5)
        h, h_inner = hs.hdiag(calibration), hs.hdiag(inner)
        self.experts = [stored_experts(self.W[0], h), stored_experts(self.W[1], h), stored_experts(self.W[2], h_inner)]
        self.head_W = make(vocab, width, std=width ** -0.5)
        self.head_scale = self.head_W.float().abs().max().item() / (448.0 * 6.0)
        self.head = hs.search(self.head_W, h, self.head_scale, down=9, up=6)

    def logits(self, token):
        X = self.embedding[token]
        expert, weight = hs.route_tokens(X @ self.router.t(), self.k)
        Y = X + hs.expert_layer(X, expert, weight, *self.experts)
        return hs.adapted_linear(Y, self.head_scale, *self.head)


def main(steps=12, requests=5, vocab=1003, width=256, hidden=384, experts=8, k=2, seed=0, device="cuda:0"):
    g = torch.Generator().manual_seed(seed)
    model = Model(vocab, width, hidden, experts, k, g, device)

    # The last request may answer with even words only; the first never wants word 7.
    words = torch.arange(-(-vocab // 32) * 32).view(-1, 32)
    mask = ((words % 2 == 0).long() << (words % 32)).sum(-1)
    mask = torch.where(mask >= 2 ** 31, mask - 2 ** 32, mask).to(torch.int32)[None].to(device)
    bias = torch.zeros((1, vocab), device=device)
    bias[0, 7] = -100.0
    none = torch.full((requests,), -1, dtype=torch.int32)
    mask_row, bias_row = none.clone(), none.clone()
    mask_row[-1], bias_row[0] = 0, 0
    prompt_words = 4
    history = torch.full((requests, prompt_words + steps), -1, dtype=torch.int32, device=device)
    history[:, :prompt_words] = torch.randint(0, vocab, (requests, prompt_words), generator=g).int().to(device)
    length = torch.full((requests,), prompt_words, dtype=torch.int32, device=device)
    rules = dict(history=history, length=length, prompt=length.clone(), mask=mask, mask_row=mask_row.to(device), bias=bias,
                 bias_row=bias_row.to(device), repetition=torch.full((requests,), 1.3, device=device),
                 frequency=torch.full((requests,), 2.0, device=device), presence=torch.full((requests,), 4.0, device=device))
    token = history[:, prompt_words - 1].long()

    def step():
        logits = model.logits(token)
        hs.adjust_logits(logits, **rules, out=logits)
        chosen = logits.argmax(-1)
        history.scatter_(1, length[:, None].long(), chosen[:, None].int())
        length.add_(1)
        token.copy_(chosen)

    start = [t.clone() for t in (history, length, token)]
    step()  # once outside the graph, then from the start again
    for t, was in zip((history, length, token), start):
        t.copy_(was)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(steps):
        graph.replay()
    torch.cuda.synchronize()
    return model, rules, history[:, prompt_words:].cpu(), start


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=12)
    answers = main(steps=p.parse_args().steps)[2]
    for r, words in enumerate(answers.tolist()):
        print(f"request {r}: {words}")
