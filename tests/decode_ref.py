"""Plain 64-bit implementations of routing, a layer of stored experts and the
rules on logits, for the tests of the kernels (written from the formulas; they
share nothing with the library)."""
import torch

from tests import adapt_ref


def route(logits, k, normalize):
    """(expert, weight float64, max |l - max| of the chosen)."""
    l = logits.cpu().double()
    T, E = l.shape
    expert = torch.full((T, k), -1, dtype=torch.int32)
    weight = torch.zeros((T, k), dtype=torch.float64)
    for t in range(T):
        row = l[t].tolist()
        may = [e for e in range(E) if row[e] > float("-inf")]  # neither -inf nor NaN
        best = sorted(may, key=lambda e: (-row[e], e))[:k]
        expert[t, :len(best)] = torch.tensor(best, dtype=torch.int32)
        if torch.isnan(l[t]).any() or torch.isposinf(l[t]).any():
            weight[t] = float("nan")
        elif best:
            p = torch.exp(l[t] - row[best[0]])
            weight[t, :len(best)] = p[best] / (p[best].sum() if normalize else p.sum())
    return expert, weight


def matrix(stored, e):
    """float64 [out, in] of expert e."""
    scale, codes, packed = stored
    return adapt_ref.weights(float(scale[e]), codes[e], packed[e])


def experts(X, expert, weight, gate, up, down, sums):
    """(Y, how far a result may be off): `sums` bounds the error of an fp32 sum
    relative to the sum of its absolute terms.  With that, |silu'| <= 1.1 and two
    parts of 2^-8 each of the rest: h errs by at most
        1.1 sums |G||x| |u| + |silu(g)| sums |U||x| + (2^-16 + 2^-20) |h|
    (2^-20: the exponential, the quotient and the products), and y by |w||D| of
    that, by `sums` of its own terms and by one rounding to bf16, half a step of
    8 bits: 2^-8 of the value."""
    X, expert, weight = X.cpu().double(), expert.cpu(), weight.cpu().double()
    E = gate[0].shape[0]
    Y, off = torch.zeros_like(X), torch.zeros_like(X)
    for e in range(E):
        t, j = (expert == e).nonzero(as_tuple=True)
        if not t.numel():
            continue
        G, U, D = (matrix(m, e) for m in (gate, up, down))
        x, w = X[t], weight[t, j, None]
        g, u = x @ G.t(), x @ U.t()
        s = g * torch.sigmoid(g)
        h = s * u
        dh = 1.1 * sums * (x.abs() @ G.abs().t()) * u.abs() + s.abs() * sums * (x.abs() @ U.abs().t())
        dh += (2.0 ** -16 + 2.0 ** -20) * h.abs()
        Y.index_add_(0, t, w * (h @ D.t()))
        off.index_add_(0, t, w.abs() * ((dh + sums * h.abs()) @ D.abs().t()))
    none = (expert < 0) | (expert >= E)
    Y += torch.where(none, weight * 0.0, 0.0).sum(-1, keepdim=True)
    return Y, off + 2.0 ** -8 * Y.abs()


def logits(l, history=None, length=None, prompt=None, repetition=None, frequency=None, presence=None, bias=None,
           bias_row=None, mask=None, mask_row=None):
    """(float64 result, the sum of the absolute terms behind it)."""
    l = l.cpu().double().clone()
    R, V = l.shape
    size = l.abs()
    one = lambda t, r: float(t.cpu()[r])  # noqa: E731
    for r in range(R):
        if history is not None:
            L = history.shape[1]
            n = L if length is None else min(max(int(length[r]), 0), L)
            first = 0 if prompt is None else min(max(int(prompt[r]), 0), L)
            seen, count = set(), {}
            for i, v in enumerate(history[r, :n].cpu().tolist()):
                if 0 <= v < V:
                    seen.add(v)
                    if i >= first:
                        count[v] = count.get(v, 0) + 1
            for v in seen:
                if repetition is not None:
                    rho = one(repetition, r)
                    l[r, v] = l[r, v] / rho if l[r, v] > 0 else l[r, v] * rho
                    size[r, v] += l[r, v].abs()
                if v in count:
                    f = 0.0 if frequency is None else one(frequency, r) * count[v]
                    p = 0.0 if presence is None else one(presence, r)
                    l[r, v] = l[r, v] - f - p
                    size[r, v] += 2 * abs(f) + abs(p)
        if bias is not None:
            b = 0 if bias_row is None else int(bias_row[r])
            if 0 <= b < bias.shape[0]:
                l[r] += bias[b].cpu().double()
                size[r] += bias[b].cpu().double().abs()
        if mask is not None:
            m = 0 if mask_row is None else int(mask_row[r])
            if 0 <= m < mask.shape[0]:
                words = [w & 0xFFFFFFFF for w in mask[m].cpu().tolist()]
                for v in range(V):
                    if not words[v >> 5] >> (v & 31) & 1:
                        l[r, v] = float("-inf")
    return l, size
