"""64-bit references for the operators at a network's end, and how far fp32 and
bf16 arithmetic may be from them (no test functions here).

The bounds are elementwise and follow from the operations: a sum of n products
in fp32 is off by at most (n + 8) u sum|a b| with u = 2^-24 whatever its order;
rounding to bf16 is off by at most 2^-8 of the value.  SLACK covers second-order
terms and the exponential's and logarithm's own few roundings.
"""
import numpy as np
import torch

U32 = 2.0 ** -24
U16 = 2.0 ** -8
SLACK = 2.0
TINY = 1e-37          # below fp32's normal range, where values may flush to 0


def xent(X, W, target, dloss):
    """(loss, lse, G, dX, dW) in float64; rows whose target is outside 0..V-1
    have loss 0 and G = 0, and their X reaches no gradient."""
    X, W, dloss = X.double(), W.double(), dloss.double()
    V = W.shape[0]
    has = (target >= 0) & (target < V)
    S = X @ W.t()
    lse = torch.logsumexp(S, 1)
    rows = torch.nonzero(has)[:, 0]
    at = target[rows]
    loss = torch.zeros(X.shape[0], dtype=torch.float64, device=X.device)
    loss[rows] = lse[rows] - S[rows, at]
    G = torch.zeros_like(S)
    P = torch.exp(S[rows] - lse[rows, None])
    P[torch.arange(len(rows), device=X.device), at] -= 1.0
    G[rows] = P * dloss[rows, None]
    Xv = torch.where(has[:, None], X, torch.zeros_like(X))
    return loss, lse, G, G @ W, G.t() @ Xv


def xent_bounds(X, W, target, dloss, lse, G, dX, dW, bf16):
    """Bounds of (loss, lse, G, dX, dW), elementwise, for finite rows with a
    target (lse: all rows)."""
    X, W = X.double(), W.double()
    V, D = W.shape
    T = X.shape[0]
    has = ((target >= 0) & (target < V))[:, None]
    X = torch.nan_to_num(X)
    d = torch.where(has[:, 0], dloss.double().abs(), torch.zeros_like(lse))
    ds = (D + 8) * U32 * (X.abs() @ W.abs().t())               # a logit's error
    worst = ds.max(1).values
    dl = worst + 16 * U32 * (1 + torch.nan_to_num(lse).abs() + torch.nan_to_num(X).abs() @ W.abs().max(0).values)
    P = torch.where(has, G.abs(), torch.zeros_like(G)) + 0.0   # |p - onehot| d; p d itself is at most this + d at the target
    hot = torch.zeros_like(G)
    rows = torch.nonzero(has[:, 0])[:, 0]
    hot[rows, target[rows]] = d[rows]
    dG = (P + hot) * (ds + dl[:, None] + 16 * U32) + 4 * U32 * hot + TINY
    dG = torch.where(has, dG, torch.zeros_like(dG))
    aW, aX, aG = W.abs(), torch.where(has, X.abs(), torch.zeros_like(X)), G.abs() + dG
    bX = dG @ aW + (V + 8) * U32 * (aG @ aW) + TINY
    if bf16:
        bX = bX + U16 * (aG @ aW) + U16 * dX.abs()
    bW = dG.t() @ aX + (T + 8) * U32 * (aG.t() @ aX) + TINY
    return SLACK * 2 * dl, SLACK * dl, SLACK * dG, SLACK * bX, SLACK * bW


def keep(seed, offset, rows, cols, p):
    """The kept elements: Philox4x32 with seven rounds in numpy's integers, one
    call per group of eight neighbours, 16 bits an element."""
    thr = int(np.floor(p * 65536 + 0.5))
    u, m32 = np.uint64, np.uint64(0xFFFFFFFF)
    per = (cols + 7) // 8
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    g = np.arange(rows * per, dtype=u)
    c = [g & m32, g >> u(32), np.full(g.shape, offset & 0xFFFFFFFF, u), np.full(g.shape, offset >> 32, u)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(7):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k0), b & m32, (a >> u(32)) ^ c[3] ^ u(k1), a & m32]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    bits = np.empty((rows * per, 8), dtype=np.uint32)
    for w in range(4):
        bits[:, 2 * w] = (c[w] & u(0xFFFF)).astype(np.uint32)
        bits[:, 2 * w + 1] = (c[w] >> u(16)).astype(np.uint32)
    return torch.from_numpy(bits.reshape(rows, per * 8)[:, :cols] >= thr), thr


def dropped(x, mask, thr):
    """keep * x / (1 - p) in float64."""
    if thr == 0:
        return x.double()
    scale = 0.0 if thr >= 65536 else 65536.0 / (65536 - thr)
    return torch.where(mask, x.double() * scale, torch.zeros((), dtype=torch.float64))


def norm_forward(h, gamma, beta, eps):
    """(y, mean, rstd) of float64 rows."""
    mean = h.mean(1)
    rstd = ((h - mean[:, None]).square().mean(1) + eps) ** -0.5
    return (h - mean[:, None]) * rstd[:, None] * gamma.double() + beta.double(), mean, rstd


def norm_backward(dy, h, gamma, mean, rstd, dres):
    """(dh, dgamma, dbeta) in float64."""
    dy, h, mean, rstd = dy.double(), h.double(), mean.double()[:, None], rstd.double()[:, None]
    n = (h - mean) * rstd
    g = dy * gamma.double()
    dh = rstd * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    return dh + (dres.double() if dres is not None else 0.0), (dy * n).sum(0), dy.sum(0)
