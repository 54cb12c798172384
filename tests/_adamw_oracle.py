"""AdamW, its 8-bit moments and the gradients' norm in 64 bits, on the CPU (no
test functions here)."""
import math

import numpy as np
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8   # half a step of fp32 and of bf16, relative
BLOCK = 128


def bits16(seed, offset, first_group, n):
    """Each value's 16 random bits: Philox4x32 with seven rounds in numpy."""
    u = np.uint64
    low = u(0xFFFFFFFF)
    g = np.arange(first_group, first_group + (n + 7) // 8, dtype=u)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    w = [g & low, g >> u(32), np.full(g.shape, offset % 2 ** 32, u), np.full(g.shape, offset >> 32, u)]
    key = [seed % 2 ** 32, seed >> 32]
    for _ in range(7):
        x, y = w[0] * u(0xD2511F53), w[2] * u(0xCD9E8D57)
        w = [(y >> u(32)) ^ w[1] ^ u(key[0]), y & low, (x >> u(32)) ^ w[3] ^ u(key[1]), x & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack([v.astype("<u4") for v in w], 1).view("<u2").reshape(-1)[:n].astype(np.int64)


def exchanged(bits):
    return (bits & 255) * 256 + (bits >> 8)


def decode(codes, exponents, signed):
    """The values of codes (numpy bytes), by the header's formula."""
    top = 127 if signed else 255
    c = codes.astype(np.int64)
    e = np.repeat(exponents.astype(np.int64), BLOCK)[:len(c)]
    k = c & top
    word = ((e + 1) << 23) - ((top - k) << 20)
    v = np.where(k == 0, 0, word).astype(np.uint32).view(np.float32).astype(np.float64)
    if signed:
        v = np.where(c & 128, -v, v)
    return np.where(e == 255, np.nan, v)


def encode(x, bits, signed):
    """Codes and exponent bytes of fp64 values: the number of code points at or
    below each magnitude (found in a table of all 126 or 254 of them), one more
    where its share of the way to the next reaches 1 - bits / 65536."""
    top, least = (127, 16) if signed else (255, 32)
    codes, exponents = np.zeros(len(x), np.uint8), np.zeros(-(-len(x) // BLOCK), np.uint8)
    for b in range(len(exponents)):
        at = slice(b * BLOCK, min(len(x), (b + 1) * BLOCK))
        a = np.abs(x[at])
        a = np.where(a < 2.0 ** -126, 0.0, a)
        most = a.max()
        if not most < 2.0 ** 128:
            exponents[b] = 255
            codes[at] = np.where(np.signbit(x[at]), 128, 0) if signed else 0
            continue
        e = max(least, math.frexp(most)[1] + 126 if most > 0 else 0)
        exponents[b] = e
        # code points 0 .. top + 1: 2^(E + 1 - 127) times eighths of binades
        point = np.array([(1 + (k - top) % 8 / 8) * 2.0 ** (e - 126 + (k - top) // 8) for k in range(top + 2)])
        k = np.searchsorted(point, a, side="right") - 1     # -1: below code 0's place
        inside = k >= 0
        q = np.maximum(k, 0)
        share = (a - point[q]) / (point[np.minimum(q + 1, top + 1)] - point[q])
        k = np.where(inside, q + (share + bits[at] / 65536 >= 1), 0)
        k = np.where(a == 0, 0, np.maximum(k, 0 if signed else 1))
        codes[at] = k + (np.where(np.signbit(x[at]), 128, 0) if signed else 0)
    return codes, exponents


def adamw(W, rows, m, v, *, lr, step, betas, eps, decay, scale=1.0):
    """(W, m, v, bound of W's error, of m's, of v's) of one step from fp64 moments,
    rows (P, n) summed in order.

    The bounds count roundings to fp32 (u each, relative) where the moments are
    fp32: g one, its factor and product two, the other product's factor one, the sum
    one; g^2 two more.  The update u = rate m / (sqrt(v) root + eps): rate, product,
    root, product with the sum, square root and division one each, and half of v's;
    decay: its factor and product two; the sum of the two and W's difference one
    each.  16 units of |u| and 4 of the decay's term hold all of them."""
    g = np.zeros(rows.shape[1])
    for r in rows:
        g = g + r
    g = g * float(scale)
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * (g * g)
    c1, c2 = 1 - b1 ** step, 1 - b2 ** step
    den = np.sqrt(v / c2) + eps
    u = lr * (m / c1) / den
    w = W - lr * decay * W - u
    dm = U32 * (np.abs(m) + 4 * (1 - b1) * np.abs(g) + 2 * np.abs(m - (1 - b1) * g))
    dv = U32 * 8 * v
    dw = U32 * (np.abs(w) + 16 * np.abs(u) + 4 * np.abs(lr * decay * W)) + lr / c1 * dm / den
    return w, m, v, dw, dm, dv
