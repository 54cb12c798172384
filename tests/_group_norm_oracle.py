"""Group norm with an activation, and its gradient, in 64 bits, with bounds of what
fp32 arithmetic may add (no test functions here).

Bounds count roundings: u = 2^-24 each, relative, and half a step of the result's
type for the last.  Forward, a thread sums at most 64 rows of differences from one of
the group's values or from a first mean.  Those sums are joined by their means in 64
bits, or in fp32 in at most 3 + 64 / piece + 6 steps (eight channels, the partial
sums that one of 64 lanes adds up, the lanes), piece >= 1.  So `k` = min(L, 64) + 80
roundings bound a mean of such differences.  Backward, fp32 sums have a thread's at
most 64 rows, six shuffles and at most 256 teams of a workgroup."""
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8
TINY = 1e-37


def sigmoid(z):
    return 1 / (1 + torch.exp(-z))


def act_of(z, act):
    return z.clamp(min=0.0) if act == "relu" else z * sigmoid(z) if act == "silu" else z


def slope_of(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        q = sigmoid(z)
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def shaped(x, groups):
    """(N, L, G, D) in 64 bits."""
    return x.double().reshape(x.shape[0], -1, groups, x.shape[-1] // groups)


def forward(x, gamma, beta, groups, eps, act, u):
    """{name: (value, bound)} of y, mean and rstd."""
    v = shaped(x, groups)
    N, L, G, D = v.shape
    w, b = gamma.double().view(G, D), beta.double().view(G, D)
    mean = v.mean((1, 3), keepdim=True)
    c = v - mean
    var = c.square().mean((1, 3), keepdim=True)
    rstd = (var + eps) ** -0.5
    most = c.abs().amax((1, 3), keepdim=True)
    k = min(L, 64) + 80
    # differences from the pivot: at most 2 most, their mean square var + most^2
    d_mean = k * U32 * 2 * most + 2 * U32 * mean.abs()
    d_rstd = 0.5 * (2 * k * U32 * (var + most.square()) + d_mean.square()) / (var + eps) + 2 * U32   # relative
    n = c * rstd
    z = n * w + b
    d_z = w.abs() * (rstd * d_mean + n.abs() * (d_rstd + 4 * U32)) + 2 * U32 * (z.abs() + b.abs())
    y = act_of(z, act)
    # silu: slope at most 1.1; e^-z within (2 |z| + 4) u, which |z| q (1 - q) <= 0.28 halves at least
    d_y = d_z if act != "silu" else 1.1 * d_z + 6 * U32 * z.abs()
    return {"y": (y.reshape(x.shape), (d_y + u * (y.abs() + d_y)).reshape(x.shape) + TINY),
            "mean": (mean.view(N, G), d_mean.view(N, G) + TINY),
            "rstd": (rstd.view(N, G), (rstd * d_rstd).view(N, G))}


def backward(dy, x, gamma, beta, mean, rstd, act, u):
    """{name: (value, bound)} of dx, dgamma and dbeta from fp32 mean and rstd."""
    groups = mean.shape[1]
    v, t = shaped(x, groups), shaped(dy, groups)
    N, L, G, D = v.shape
    w, b = gamma.double().view(G, D), beta.double().view(G, D)
    mu, r = mean.double()[:, None, :, None], rstd.double()[:, None, :, None]
    n = (v - mu) * r
    z = n * w + b
    dz = t * slope_of(z, act)
    d_n = 2 * U32 * n.abs()
    # silu: the slope's slope is at most 0.5, its own arithmetic 10 roundings of
    # terms below 1.5, and e^-z within (2 |z| + 4) u, damped by q (1 - q) (1 + |z|) <= 0.5
    d_dz = t.abs() * (0.5 * 4 * U32 * ((n * w).abs() + b.abs()) + 20 * U32) if act == "silu" else torch.zeros_like(t)
    g = dz * w
    count = L * D
    a1, a2 = (x_.sum((1, 3), keepdim=True) / count for x_ in (g, g * n))
    # (a sum with 0 rounds nothing: no more teams count than rows)
    k = min(L, 64) + min(L, 256) + 8
    e1 = (w.abs() * (d_dz + k * U32 * dz.abs())).sum((1, 3), keepdim=True) / count + 2 * U32 * a1.abs()
    e2 = (w.abs() * (d_dz * n.abs() + dz.abs() * d_n + k * U32 * (dz * n).abs())).sum((1, 3), keepdim=True) / count \
        + 2 * U32 * a2.abs()
    dx = r * (g - a1 - n * a2)
    d_dx = r * (w.abs() * d_dz + e1 + n.abs() * e2 + d_n * a2.abs() +
                5 * U32 * (g.abs() + a1.abs() + (n * a2).abs()))
    sums = {}
    for name, term, err in (("dgamma", dz * n, d_dz * n.abs() + dz.abs() * d_n), ("dbeta", dz, d_dz)):
        sums[name] = (term.sum((0, 1)).view(-1),
                      (err + k * U32 * term.abs()).sum((0, 1)).view(-1) + U32 * term.sum((0, 1)).abs().view(-1) + TINY)
    return {"dx": (dx.reshape(x.shape), (d_dx + u * (dx.abs() + d_dx)).reshape(x.shape) + TINY), **sums}
