"""Routing and layers of stored experts against 64-bit plain implementations."""
from __future__ import annotations

import pytest
import torch

from tests import decode_ref as ref

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"

# An fp32 sum of up to 2^14 terms on the matrix cores and in four parts: at most
# (terms / 16) 2^-24 of the sum of absolute terms, 2^-14, and the roundings of
# the scale and of the routing weight.
SUMS = 2.0 ** -14


@pytest.fixture(scope="module")
def hs():
    import paper_2608_28113_amd as hs
    from paper_2608_28113_amd import _lib
    _lib.load()
    yield hs
    torch.cuda.empty_cache()  # what is cached here would serve later tests that bound the memory left


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bf(shape, std, g):
    return (torch.randn(shape, generator=g) * std).bfloat16().to(DEV)


def _stored(E, m, n, g, s=1.0):
    """Random codes; about 1 / sqrt(n) large where s is 1."""
    codes = torch.randint(40, 72, (E, m, n // 16), generator=g, dtype=torch.uint8)
    packed = torch.randint(0, 256, (E, m, n // 2), generator=g, dtype=torch.int32).to(torch.uint8)
    scale = s * n ** -0.5 / 6.0 * (0.5 + torch.rand(E, generator=g))
    return scale.to(DEV), codes.to(DEV), packed.to(DEV)


def _problem(T, n, hidden, E, k, seed=0, ids="distinct"):
    g = _gen(seed + 1000 * T + n + hidden)
    if ids == "distinct":
        expert = torch.rand((T, E), generator=g).argsort(-1)[:, :k].int()
    elif ids == "wild":  # none, past the end, and the same one twice
        expert = torch.randint(-2, E + 2, (T, k), generator=g, dtype=torch.int32)
    else:  # nearly all tokens at one expert
        expert = torch.randint(0, E, (T, k), generator=g, dtype=torch.int32)
        expert[torch.rand((T, k), generator=g) < 0.9] = E - 1
    weight = torch.rand((T, k), generator=g)
    return dict(X=_bf((T, n), 1.0, g), expert=expert.to(DEV), weight=weight.to(DEV), gate=_stored(E, hidden, n, g),
                up=_stored(E, hidden, n, g), down=_stored(E, n, hidden, g))


def _check(got, p, **changed):
    Y, off = ref.experts(**{**p, **changed}, sums=SUMS)
    worst = ((got.cpu().double() - Y).abs() - off).max().item()
    assert worst <= 0.0, worst


SIZES = [
    (1, 16, 16, 1, 1), (1, 64, 96, 8, 3), (2, 2064, 1424, 300, 6), (3, 48, 80, 5, 2), (5, 1024, 512, 64, 6),
    (17, 144, 208, 4, 4), (40, 96, 112, 200, 1), (33, 272, 304, 5, 2), (64, 512, 272, 128, 8), (70, 256, 144, 3, 2),
    (86, 64, 48, 1024, 3), (300, 128, 64, 16, 4), (513, 64, 48, 2, 1), (256, 32, 32, 1, 1), (257, 32, 32, 1, 1),
    (9, 1296, 2064, 3, 32),
]


@pytest.mark.parametrize("T,n,hidden,E,k", SIZES)
@pytest.mark.parametrize("ids", ["distinct", "wild", "one"])
def test_layer(hs, T, n, hidden, E, k, ids):
    p = _problem(T, n, hidden, E, min(k, E) if ids == "distinct" else k, ids=ids)
    print(f"[layer {T} {n} {hidden} {E} {k} {ids}]", flush=True)
    _check(hs.expert_layer(**p), p)


# Every tile of slots (4, 16, 32, 64), one, two and four waves to a row, with
# several rounds of k, and splits of the down product.
ROUTES = [(1, 64, 96, 8, 3), (1, 528, 4112, 8, 2), (4, 1040, 528, 64, 6), (12, 528, 1056, 64, 6), (16, 1104, 272, 7, 3),
          (40, 528, 1056, 100, 8), (160, 528, 1040, 12, 2), (160, 1040, 272, 12, 2), (160, 80, 2064, 12, 2),
          (300, 528, 1040, 8, 2), (300, 1040, 272, 8, 2), (300, 96, 3088, 6, 2)]


@pytest.mark.parametrize("T,n,hidden,E,k", ROUTES)
@pytest.mark.parametrize("odd", [0, 1])
def test_every_route(hs, T, n, hidden, E, k, odd):
    """`odd`: scales that start at an odd byte, packed weights at 8 bytes."""
    p = _problem(T, n, hidden, E, k)
    if odd:
        for m in ("gate", "up", "down"):
            s, c, w = p[m]
            codes = torch.full((c.numel() + 9,), 255, dtype=torch.uint8, device=DEV)  # a NaN on either side
            packed = torch.full((w.numel() + 16,), 0x77, dtype=torch.uint8, device=DEV)
            codes[1:-8] = c.flatten()
            packed[8:-8] = w.flatten()
            p[m] = s, codes[1:-8].view(c.shape), packed[8:-8].view(w.shape)
    print(f"[route {T} {n} {hidden} {E} {k} {odd}]", flush=True)
    _check(hs.expert_layer(**p), p)


def test_pieces(hs):
    """More slots than one piece of 4096 takes, the last piece a short one."""
    p = _problem(1500, 32, 48, 7, 3)
    _check(hs.expert_layer(**p), p)


def test_a_token_does_not_depend_on_its_neighbours(hs):
    """The same bits alone, among others, at every size of the call's tiles and in
    any order, for widths up to 256, which no call splits."""
    p = _problem(600, 144, 112, 12, 3)
    whole = hs.expert_layer(**p)
    for a, b in ((0, 1), (0, 5), (7, 60), (100, 200), (599, 600)):
        part = dict(p, X=p["X"][a:b], expert=p["expert"][a:b], weight=p["weight"][a:b])
        assert torch.equal(hs.expert_layer(**part), whole[a:b]), (a, b)
    order = torch.randperm(600, generator=_gen(3)).to(DEV)
    mixed = dict(p, X=p["X"][order], expert=p["expert"][order], weight=p["weight"][order])
    assert torch.equal(hs.expert_layer(**mixed), whole[order])
    for _ in range(3):
        assert torch.equal(hs.expert_layer(**p), whole)


@pytest.mark.parametrize("T", [1, 30, 400])
def test_rows_may_be_strided(hs, T):
    p = _problem(T, 80, 64, 6, 2)
    X = torch.full((T + 1, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    X[:T, 16:96] = p["X"]
    Y = torch.full((T + 2, 131), 7.0, dtype=torch.bfloat16, device=DEV)
    out = hs.expert_layer(**dict(p, X=X[:T, 16:96]), Y=Y[1:T + 1, 3:83])
    assert out.data_ptr() == Y[1:, 3:].data_ptr()
    _check(out, p)
    Y[1:T + 1, 3:83] = 7.0
    assert (Y == 7.0).all()


@pytest.mark.parametrize("T", [4, 300])
def test_what_is_not_finite_stays_with_its_token(hs, T):
    p = _problem(T, 64, 48, 5, 2)
    clean = hs.expert_layer(**p)
    X, w, e = p["X"].clone(), p["weight"].clone(), p["expert"].clone()
    X[1, 5], X[2] = float("nan"), float("inf")
    w[3, 1] = float("nan")
    e[3, 1] = -1  # no expert, but its weight shows
    got = hs.expert_layer(**dict(p, X=X, weight=w, expert=e))
    assert got[1].isnan().all() and not got[2].isfinite().any() and got[3].isnan().all()
    keep = [t for t in range(T) if t not in (1, 2, 3)]
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("T", [3, 200])
def test_tokens_without_experts(hs, T):
    p = _problem(T, 64, 48, 5, 2)
    p["expert"][T // 2] = -1
    p["expert"][0] = torch.tensor([5, 2 ** 31 - 1], dtype=torch.int32)
    got = hs.expert_layer(**p)
    assert (got[0] == 0).all() and (got[T // 2] == 0).all()
    _check(got, p)
    p["expert"].fill_(-7)
    assert (hs.expert_layer(**p) == 0).all()


def test_no_tokens(hs):
    p = _problem(2, 64, 48, 5, 2)
    got = hs.expert_layer(p["X"][:0], p["expert"][:0], p["weight"][:0], p["gate"], p["up"], p["down"])
    assert got.shape == (0, 64)


@pytest.mark.parametrize("big", [2.0 ** 110, 2.0 ** -110])
def test_ends_of_the_scales_range(hs, big):
    """The scales of gate and up at one end, those of X at the other."""
    p = _problem(5, 96, 64, 3, 2)
    for m in ("gate", "up"):
        p[m] = (p[m][0] * big, *p[m][1:])
    p["X"] = (p["X"].float() * (1.0 / big)).bfloat16()
    _check(hs.expert_layer(**p), p)


def test_hidden_values_at_the_end_of_the_range(hs):
    """h past bf16's largest is inf in its first part; the second adds nothing to it."""
    p = _problem(2, 32, 32, 2, 1)
    p["up"] = (torch.full_like(p["up"][0], 3e38 / 2688), torch.full_like(p["up"][1], 126),
               torch.full_like(p["up"][2], 0x77))
    p["gate"] = (torch.ones_like(p["gate"][0]), torch.full_like(p["gate"][1], 56), torch.full_like(p["gate"][2], 0x77))
    p["down"] = (p["down"][0], p["down"][1], torch.full_like(p["down"][2], 0x11))
    p["X"].fill_(1.0)
    assert torch.isposinf(hs.expert_layer(**p)).all()


def test_another_stream_and_a_given_workspace(hs):
    p = _problem(300, 64, 48, 6, 2)
    want = hs.expert_layer(**p)
    ws = torch.empty(hs.expert_layer_workspace_bytes(600, 64, 48, 6, 2), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for T in (300, 1, 40):  # a workspace for many tokens serves fewer
        ws.fill_(255)
        side.wait_stream(torch.cuda.current_stream())
        got = hs.expert_layer(p["X"][:T], p["expert"][:T], p["weight"][:T], p["gate"], p["up"], p["down"],
                              workspace=ws, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want[:T])


@pytest.mark.parametrize("T", [1, 24, 320])
def test_captured_and_replayed(hs, T):
    """Routing and layer in one graph, replayed on new inputs."""
    p = _problem(T, 128, 96, 16, 4)
    logits = torch.randn((T, 16), generator=_gen(1)).to(DEV)
    layer = (p["gate"], p["up"], p["down"])

    def step():
        return hs.expert_layer(p["X"], *hs.route_tokens(logits, 4), *layer)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = step()
    for seed in range(4):
        logits.copy_(torch.randn((T, 16), generator=_gen(seed)))
        p["X"].copy_(torch.randn((T, 128), generator=_gen(seed + 50)))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want)


def test_experts_past_32_bits(hs):
    """The last of 40 experts lies more than 2^32 bytes behind the first."""
    E, n, hidden = 40, 16384, 16384
    codes = torch.full((E, hidden, n // 16), 56, dtype=torch.uint8, device=DEV)
    packed = torch.zeros((E, hidden, n // 2), dtype=torch.uint8, device=DEV)
    scale = torch.full((E,), 2.0 ** -10, device=DEV)
    g = _gen(5)
    rows = torch.randint(0, 256, (hidden, n // 2), generator=g, dtype=torch.int32).to(torch.uint8)
    packed[E - 1] = rows.to(DEV)
    m = (scale, codes, packed)
    X = _bf((1, n), 1.0, g)
    expert = torch.tensor([[E - 1]], dtype=torch.int32, device=DEV)
    weight = torch.ones((1, 1), device=DEV)
    got = hs.expert_layer(X, expert, weight, m, m, m)
    last = tuple(t[E - 1:] for t in m)
    Y, off = ref.experts(X, torch.zeros_like(expert), weight, last, last, last, sums=2.0 ** -13)
    assert ((got.cpu().double() - Y).abs() <= off).all()


# ---------------------------------------------------------------------------
# Routing
# ---------------------------------------------------------------------------


def _check_route(logits, k, normalize, expert, weight):
    want, w = ref.route(logits, k, normalize)
    assert torch.equal(expert.cpu(), want)
    nan = w.isnan()
    assert torch.equal(weight.cpu().isnan(), nan)
    # exp of a difference d rounded to fp32 errs by |d| 2^-24, expf by 2 units,
    # a sum of E terms by E 2^-24 and the quotient by one rounding; shares below
    # 2^-126 may be flushed.
    E = logits.shape[1]
    d = torch.log(w.clamp(min=1e-45)).abs() + 8.0
    off = (w * (2 * d + 2 * E + 16) * 2.0 ** -24 + 2.0 ** -126)[~nan]
    assert ((weight.cpu().double() - w)[~nan].abs() <= off).all()


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (5, 64, 6), (130, 65, 8), (67, 128, 32), (33, 160, 8),
                                   (9, 257, 5), (3, 1024, 32), (1000, 40, 4)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("normalize", [True, False])
def test_route(hs, T, E, k, dtype, normalize):
    logits = (torch.randn((T, E), generator=_gen(T + E)) * 3).to(dtype).to(DEV)
    _check_route(logits, k, normalize, *hs.route_tokens(logits, k, normalize=normalize))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_route_ties_and_ends(hs, dtype):
    inf, nan = float("inf"), float("nan")
    rows = [[1, 1, 1, 1, 1], [0.0, -0.0, 0.0, -0.0, -1], [-inf, 2, -inf, 2, -inf], [-inf] * 5, [-inf, -3, -inf, -inf, -inf],
            [nan, 1, 2, 3, 4], [nan] * 5, [1, inf, 2, 3, 4], [inf, inf, 0, 0, -inf], [3e38, -3e38, 0, 1, 2],
            [-200, -200, 0, -300, -1e30], [nan, -inf, -inf, -inf, -inf]]
    logits = torch.tensor(rows).to(dtype).to(DEV)
    for k in (1, 3, 5):
        for normalize in (True, False):
            _check_route(logits, k, normalize, *hs.route_tokens(logits, k, normalize=normalize))


def test_route_strided_rows_and_given_outputs(hs):
    big = torch.randn((21, 50), generator=_gen(2)).to(DEV)
    expert = torch.full((22, 3), 99, dtype=torch.int32, device=DEV)
    weight = torch.full((22, 3), 9.0, device=DEV)
    hs.route_tokens(big[:, 7:40], 3, expert=expert[:21], weight=weight[:21])
    _check_route(big[:, 7:40], 3, True, expert[:21], weight[:21])
    assert (expert[21] == 99).all() and (weight[21] == 9.0).all()
    none = hs.route_tokens(big[:0], 3)
    assert none[0].shape == none[1].shape == (0, 3)


@pytest.mark.parametrize("T,n,hidden,E,k", [(1, 2048, 1024, 64, 6), (1, 4096, 2048, 8, 2), (9, 640, 1040, 33, 4)])
def test_many_small_calls_in_a_row(hs, T, n, hidden, E, k):
    """Calls that follow one another in the same workspace with other inputs give
    what each gives alone."""
    p = [_problem(T, n, hidden, E, k, seed=s) for s in (1, 2, 3)]
    for q in p[1:]:
        q.update(gate=p[0]["gate"], up=p[0]["up"], down=p[0]["down"])
    ws = torch.empty(hs.expert_layer_workspace_bytes(T, n, hidden, E, k), dtype=torch.uint8, device=DEV)
    want = [hs.expert_layer(**q, workspace=ws).clone() for q in p]
    for q, w in zip(p, want):
        _check(w, q)
    got = [hs.expert_layer(**p[i % 3], workspace=ws) for i in range(600)]
    assert all(torch.equal(y, want[i % 3]) for i, y in enumerate(got))
