"""A layer of stored experts on numbers that every order of summation keeps
exact, so that each output has one right value: all bits of the hidden values
and every round, wave and split of k show.  And every scale code, at both ends
of the global scales' range."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_experts import DEV, ROUTES, SIZES, _gen, hs  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

GRID = torch.tensor([s * v for s in (1.0, -1.0) for v in (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)], dtype=torch.float64)


def _values(codes):
    """float64 of E4M3 codes 0 .. 126."""
    c = codes.long()
    return torch.where(c < 8, (c & 7) * 2.0 ** -9, (8 + (c & 7)).double() * torch.exp2((c >> 3).double() - 10.0))


def _pack(q):
    return (q[..., 0::2] | (q[..., 1::2] << 4)).to(torch.uint8)


def _matrix(q, codes, scale):
    """float64 [E, m, n] of nibbles q, codes and global scales."""
    return GRID[q.long()] * (_values(codes) * scale.double()[:, None, None]).repeat_interleave(16, -1)


def _one_of(g, choices, shape):
    return torch.tensor(choices)[torch.randint(0, len(choices), shape, generator=g)]


def _gate(E, hidden, n, columns, g, codes):
    """Each row takes one of `columns` twice: a value times its scale code is 2 there, 0 elsewhere."""
    q = torch.zeros((E, hidden, n), dtype=torch.int32)
    at = columns[torch.randint(0, len(columns), (E, hidden, 1), generator=g)]
    which = torch.randint(0, 4, (E, hidden, 1), generator=g)
    q.scatter_(2, at, torch.tensor([4, 6, 2, 1], dtype=torch.int32)[which])  # 2, 4, 1, 0.5
    codes = codes.clone()
    codes.scatter_(2, at // 16, torch.tensor([56, 48, 64, 72], dtype=codes.dtype)[which])  # 1, 0.5, 2, 4
    return q, codes


def _reference(X, expert, weight, G, U, D):
    """Y in float64, silu(g) = g (it is, in fp32, from 18 on), the largest h, and
    the largest sums of absolute terms of u and of y."""
    X, weight = X.double(), weight.double()
    Y, most_h, most_u, most_y = torch.zeros_like(X), 0.0, 0.0, torch.zeros_like(X)
    for e in range(G.shape[0]):
        t, j = (expert == e).nonzero(as_tuple=True)
        if not t.numel():
            continue
        g, u = X[t] @ G[e].t(), X[t] @ U[e].t()
        assert (g == 32.0).all()
        h = g * u
        Y.index_add_(0, t, weight[t, j, None] * (h @ D[e].t()))
        most_y.index_add_(0, t, weight[t, j, None] * (h.abs() @ D[e].abs().t()))
        most_h, most_u = max(most_h, h.abs().max().item()), max(most_u, (X[t].abs() @ U[e].abs().t()).max().item())
    return Y, most_h, most_u, most_y.max().item()


def _on_gpu(*matrices):
    return [tuple(t.to(DEV) for t in (s, c.to(torch.uint8), _pack(q))) for s, c, q in matrices]


SMALL = [c for c in SIZES + ROUTES if c[1] * c[2] * c[3] < 10 ** 8]
WIDE = [(1, 2048, 1024, 7, 6), (3, 1024, 2064, 3, 2), (12, 2048, 1424, 9, 6), (64, 1024, 1536, 9, 8), (37, 1040, 3088, 4, 2),
        (300, 2048, 1024, 9, 6), (300, 2048, 528, 4, 4), (300, 2048, 272, 8, 2), (75, 3152, 848, 5, 3), (40, 2048, 528, 4, 2)]


@pytest.mark.parametrize("T,n,hidden,E,k", SMALL + WIDE)
def test_every_bit_of_the_hidden_values_counts(hs, T, n, hidden, E, k):  # noqa: F811
    """u is a whole multiple of 1/8 (of 1/4, or half as much again) and y's terms
    are whole multiples of 4: all sums are exact in fp32 while those of absolute
    terms are below 2^24 units.  h = 32 u has up to 17 bits, and two parts of 8
    bits hold them: what the first leaves is at most 256 units of 4.  All this is
    asserted.  With h rounded to 8 bits most outputs would differ."""
    g = _gen(T + n + hidden + E)
    columns = torch.randperm(n, generator=g)[:max(1, n // 8)].sort().values
    X = torch.randint(-3, 4, (T, n), generator=g).double()
    X[:, columns] = 16.0
    one = torch.ones(E)
    other = torch.where(torch.arange(E) % 2 == 1, 1.5, 1.0)
    qg, cg = _gate(E, hidden, n, columns, g, _one_of(g, [40, 56, 72], (E, hidden, n // 16)))
    qu, cu = torch.randint(0, 16, (E, hidden, n), generator=g), _one_of(g, [48, 56], (E, hidden, n // 16))
    few = max(2, 64 // k)  # of D's row are not 0: k rows' terms stay below 2^24 units
    qd = torch.zeros((E, n, hidden), dtype=torch.int32)
    at = torch.randint(0, hidden, (E, n, few), generator=g)
    qd.scatter_(2, at, _one_of(g, [2, 4, 10, 12], (E, n, few)).int())  # 1, 2, -1, -2
    cd = torch.full((E, n, hidden // 16), 56)
    expert = torch.randint(-1, E, (T, k), generator=g, dtype=torch.int32)
    weight = _one_of(g, [1.0, 2.0], (T, k)).float()
    want, most_h, most_u, most_y = _reference(X, expert, weight, _matrix(qg, cg, one), _matrix(qu, cu, other), _matrix(qd, cd, one))
    assert most_h <= 4 * 2.0 ** 17 and most_u < 2.0 ** 24 / 8 and most_y < 4 * 2.0 ** 24
    m = _on_gpu((one, cg, qg), (other, cu, qu), (one, cd, qd))
    print(f"[exact {T} {n} {hidden} {E} {k}]", flush=True)
    got = hs.expert_layer(X.bfloat16().to(DEV), expert.to(DEV), weight.to(DEV), *m)
    assert torch.equal(got.cpu(), want.float().bfloat16())


LOW, HIGH = 2.0 ** -117, 2.0 ** 119  # global scales, about the ends of what the search accepts


def _sparse(E, m, columns, n, g, signs=True):
    """One weight a row, in one of `columns`; every scale code from 0 to 126."""
    q = torch.zeros((E, m, n), dtype=torch.int32)
    at = columns[torch.randint(0, len(columns), (E, m, 1), generator=g)]
    q.scatter_(2, at, _one_of(g, [1, 2, 3, 4, 5, 6, 7] + [9, 10, 11, 12, 13, 14, 15] * signs, (E, m, 1)).int())
    codes = (torch.arange(E * m * (n // 16)).view(E, m, n // 16) + torch.randint(0, 127, (E, m, 1), generator=g)) % 127
    return q, codes


# Every tile of slots and every number of waves to a row.
CODED = [(1, 1040, 528, 2), (12, 528, 1056, 3), (12, 144, 272, 3), (40, 528, 272, 2), (160, 1040, 272, 2), (300, 144, 272, 3)]


@pytest.mark.parametrize("T,n,hidden,E", CODED)
@pytest.mark.parametrize("s_up,s_down,x", [(1.0, 1.0, 0), (1.5 * 2.0 ** 60, 1.0, -60), (1.0, 1.5 * 2.0 ** -40, 40),
                                           (LOW, 1.0, 110), (HIGH, 1.0, -120), (1.0, LOW, 90), (1.0, HIGH, -90),
                                           (LOW, HIGH, 30), (HIGH, LOW, -30)])
def test_every_scale_code_of_up_and_down(hs, T, n, hidden, E, s_up, s_down, x):  # noqa: F811
    """One term a sum, X about 2^x: at most 8 bits of X, 6 of a weight and 2 of a
    scale are 16 bits of h, and y's 24 bits are rounded once."""
    g = _gen(T + n + hidden)
    columns = torch.arange(0, n, 2)
    X = _one_of(g, [-255.0, -3.0, -1.0, 1.0, 2.0, 5.0, 131.0, 255.0], (T, n)).double() * 2.0 ** x
    X[:, columns] = 16.0
    qg, cg = _gate(E, hidden, n, columns, g, torch.randint(0, 127, (E, hidden, n // 16), generator=g))
    qu, cu = _sparse(E, hidden, columns + 1, n, g)
    qd, cd = _sparse(E, n, torch.arange(hidden), hidden, g)
    one, up, down = torch.ones(E), torch.full((E,), s_up), torch.full((E,), s_down)
    expert = torch.randint(0, E, (T, 1), generator=g, dtype=torch.int32)
    weight = torch.ones((T, 1))
    want, most_h, _, _ = _reference(X, expert, weight, _matrix(qg, cg, one), _matrix(qu, cu, up), _matrix(qd, cd, down))
    assert most_h < 2.0 ** 127 and want.abs().max() < 2.0 ** 127 and want[want != 0].abs().min() >= 2.0 ** -126
    m = _on_gpu((one, cg, qg), (up, cu, qu), (down, cd, qd))
    print(f"[codes {T} {n} {hidden} {E} {s_up} {s_down}]", flush=True)
    got = hs.expert_layer(X.bfloat16().to(DEV), expert.to(DEV), weight.to(DEV), *m)
    assert torch.equal(got.cpu(), want.float().bfloat16())


@pytest.mark.parametrize("T,n,hidden,E", CODED)
@pytest.mark.parametrize("s,x", [(1.0, -6), (LOW, 111), (HIGH, -125)])
def test_every_scale_code_of_gate(hs, T, n, hidden, E, s, x):  # noqa: F811
    """One term a sum: g is exact.  The exponential, the sum, the quotient and the
    product err by at most 2^-21 together, two parts of h by 2^-16, y's product
    and factors by 2^-22, and y by half a step of 8 bits: 2^-8."""
    g = _gen(T + n + hidden)
    columns = torch.arange(0, n, 2)
    X = _one_of(g, [-1.5, -1.0, 1.0, 1.75], (T, n)).double() * 2.0 ** x  # |g| up to 74
    X[:, columns] = 16.0
    qg, cg = _sparse(E, hidden, columns + 1, n, g, signs=False)
    qu, cu = _gate(E, hidden, n, columns, g, torch.randint(0, 127, (E, hidden, n // 16), generator=g))  # u is 32
    qd, cd = _sparse(E, n, torch.arange(hidden), hidden, g)
    one, gate = torch.ones(E), torch.full((E,), s)
    expert = torch.randint(0, E, (T, 1), generator=g, dtype=torch.int32)
    weight = 0.5 + torch.rand((T, 1), generator=g)
    G, U, D = _matrix(qg, cg, gate), _matrix(qu, cu, one), _matrix(qd, cd, one)
    want = torch.zeros_like(X)
    for e in range(E):
        t = (expert[:, 0] == e).nonzero()[:, 0]
        if not t.numel():
            continue
        v, u = X[t] @ G[e].t(), X[t] @ U[e].t()
        assert (u == 32.0).all() and v.abs().max() < 80.0
        want[t] = weight[t].double() * ((v * torch.sigmoid(v) * u) @ D[e].t())
    print(f"[gate codes {T} {n} {hidden} {E} {s}]", flush=True)
    got = hs.expert_layer(X.bfloat16().to(DEV), expert.to(DEV), weight.to(DEV),
                          *_on_gpu((gate, cg, qg), (one, cu, qu), (one, cd, qd)))
    assert ((got.cpu().double() - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * want.abs()).all()
