"""Plain 64-bit implementations of a stored layer with adapters, its gradients
and the token loss, for the tests of the kernels (written from the formulas;
they share nothing with the library)."""
import numpy as np
import torch

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 128


def weights(s_g, codes, packed):
    """float64 [m, n] of stored codes."""
    codes, packed = codes.cpu().numpy().astype(np.int64), packed.cpu().numpy()
    e, f = codes >> 3, codes & 7
    S = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0)) * float(np.float32(s_g))
    q = np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[0], -1)
    v = np.array(GRID + tuple(-g for g in GRID))[q]
    return torch.from_numpy(v * np.repeat(S, 16, axis=1))


def chosen(adapter, count, T):
    """[(adapter, its token numbers)]."""
    if adapter is None:
        return [(0, torch.arange(T))] if count else []
    ids = adapter.cpu()
    return [(a, (ids == a).nonzero()[:, 0]) for a in range(count)]


def linear(X, W, A=None, B=None, alpha=None, adapter=None):
    """(Y, size): size bounds the sums of absolute terms behind each Y."""
    X = X.cpu().double()
    Y, size = X @ W.t(), X.abs() @ W.abs().t()
    if A is not None:
        A, B = A.cpu().double(), B.cpu().double()
        for a, t in chosen(adapter, A.shape[0], X.shape[0]):
            s = 1.0 if alpha is None else float(alpha[a])
            Y[t] += s * (X[t] @ A[a].t()) @ B[a].t()
            size[t] += abs(s) * (X[t].abs() @ A[a].abs().t()) @ B[a].abs().t()
    return Y, size


def linear_grad(dY, X, W, A, B, alpha=None, adapter=None):
    """((dX, dA, dB), their sizes as above)."""
    def once(dY, X, W, A, B, alpha):
        dX, dA, dB = dY @ W, torch.zeros_like(A), torch.zeros_like(B)
        for a, t in chosen(adapter, A.shape[0], X.shape[0]):
            s = 1.0 if alpha is None else float(alpha[a])
            v, u = s * dY[t] @ B[a], s * X[t] @ A[a].t()
            dX[t] += v @ A[a]
            dA[a], dB[a] = v.t() @ X[t], dY[t].t() @ u
        return dX, dA, dB

    args = [v.cpu().double() for v in (dY, X, W, A, B)]
    al = None if alpha is None else alpha.cpu().double()
    return once(*args, al), once(*(v.abs() for v in args), None if al is None else al.abs())


def pack(X):
    """(q int8, scale fp32, restored bf16), every step in numpy float32."""
    x = X.cpu().float().numpy()
    T, n = x.shape
    nb = -(-n // BLOCK)
    q, scale = np.zeros((T, n), np.int8), np.zeros((T, nb), np.float32)
    for b in range(nb):
        c = slice(b * BLOCK, min(n, (b + 1) * BLOCK))
        m = np.maximum(np.abs(x[:, c]).max(1, initial=0.0), np.float32(2.0 ** -100)).astype(np.float32)
        scale[:, b] = m * np.float32(1.0 / 127.0)
        q[:, c] = np.rint(x[:, c] * (np.float32(127.0) / m)[:, None]).astype(np.int8)
    back = q.astype(np.float32) * np.repeat(scale, BLOCK, axis=1)[:, :n]
    return torch.from_numpy(q), torch.from_numpy(scale), torch.from_numpy(back).bfloat16()


def loss(X, W, target):
    """(loss, lse, logits), float64; the rows of unscored tokens may hold anything."""
    X, W, target = X.cpu().double(), W.cpu().double(), target.cpu()
    logits = X @ W.t()
    lse = torch.logsumexp(logits, -1)
    ok = (target >= 0) & (target < W.shape[0])
    at = logits[torch.arange(len(target)), torch.where(ok, target, 0)]
    return torch.where(ok, lse - at, 0.0), lse, logits


def loss_grad(X, W, target, weight):
    """(dX, dW) and the sums of the absolute terms behind them."""
    ok = (target.cpu() >= 0) & (target.cpu() < W.shape[0]) & (weight.cpu() != 0)
    X = torch.where(ok[:, None], X.cpu().double(), 0.0)
    W = W.cpu().double()
    g = torch.softmax(X @ W.t(), -1)
    t = ok.nonzero()[:, 0]
    g[t, target.cpu()[t]] -= 1.0
    g *= torch.where(ok, weight.cpu().double(), 0.0)[:, None]
    return (g @ W, g.t() @ X), (g.abs() @ W.abs(), g.abs().t() @ X.abs())
