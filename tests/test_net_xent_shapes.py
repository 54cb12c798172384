"""The classifier loss on every tile shape that a call can take for each of its
products: alone, for the rows or columns that another shape leaves, with k split,
and adding to the pieces before; each case says which shapes it is there for."""
import re

import pytest
import torch

import _net_oracle as O
from _helpers import dev, log, whole_kernel_names

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

# Rows, classes, features, type, and the tiles that the forward pass, the backward
# pass and the factor form take: S logits into running sums, L logits into memory,
# G logits into their gradient, X dX, W dW.  Together they are all that 60000
# random sizes of up to 8192 x 70000 x 4200 took.
CASES = [
    (1, 2, 2, BF16, "L32x64",
     "G32x64 W32x64 X32x64", "L32x64 X32x64"),
    (5815, 518, 2, BF16, "S64x128",
     "G64x128 W64x64 X64x64", "L64x128 X64x64"),
    (2089, 2, 4110, BF16, "S64x64",
     "G64x64 W32x64 X256x192", "L64x64 X256x192"),
    (1, 6283, 2794, BF16, "L32x64",
     "G32x64 W256x256 W64x64 X32x64", "L32x64 X32x64"),
    (149, 66670, 2, BF16, "S256x192",
     "G256x192 G64x128 W64x64 X64x64", "L256x192 L64x128 X64x64"),
    (2, 7176, 2284, BF16, "L32x64",
     "G32x64 W256x256 W32x64 X32x64", "L32x64 X32x64"),
    (7164, 2, 2466, BF16, "S64x64",
     "G64x64 W32x64 X256x256 X64x64", "L64x64 X256x256 X64x64"),
    (1, 61456, 618, BF16, "L64x128",
     "G64x128 W128x128 W256x256 X64x64", "L64x128 X64x64"),
    (4865, 4, 3686, BF16, "S64x64",
     "G64x64 W32x64 X256x256 X64x128", "L64x64 X256x256 X64x128"),
    (327, 59550, 4, BF16, "S256x256",
     "G128x128 G256x256 W64x64 X64x64", "L128x128 L256x256 X64x64"),
    (2, 28140, 1794, BF16, "L32x64",
     "G32x64 W256x192 W64x128 X64x128", "L32x64 X64x128"),
    (868, 24737, 6, BF16, "S256x256",
     "G128x128 G256x256 W64x64 X64x64", "L128x128 L256x256 X64x64"),
    (5941, 12, 2770, BF16, "S64x64",
     "G64x64 W32x64 X256x256 X64x64", "L64x64 X256x256 X64x64"),
    (148, 28760, 70, BF16, "S128x128",
     "G128x128 W64x128 X64x64", "L128x128 X64x64"),
    (6907, 68, 1128, BF16, "S64x64",
     "G64x64 W64x128 X128x128", "L64x64 X128x128"),
    (259, 63967, 70, BF16, "S256x256 S64x128",
     "G256x256 G64x128 W128x128 X64x64", "L256x256 L64x128 X64x64"),
    (69, 8271, 4008, BF16, "S64x64",
     "G64x64 W256x256 W64x64 X64x128", "L64x128 X64x128"),
    (1876, 14027, 144, BF16, "S256x256",
     "G256x192 G256x256 W64x64 X256x192", "L256x256 X256x192"),
    (2593, 6324, 324, BF16, "S256x256 S64x64",
     "G256x256 G64x64 W256x192 X64x128", "L256x256 L64x64 X64x128"),
    (1806, 8984, 400, BF16, "S256x256 S32x64",
     "G256x256 G32x64 W256x256 X128x128", "L256x256 L32x64 X128x128"),
    (8118, 2065, 396, BF16, "S256x256 S64x64",
     "G256x256 G64x64 W128x128 X64x128", "L256x256 L64x64 X64x128"),
    (2085, 43959, 76, BF16, "S256x256 S64x64",
     "G256x256 G64x64 W64x64 X64x128", "L256x256 L64x64 X128x128"),
    (357, 53851, 382, BF16, "S128x128 S256x256",
     "G128x128 W256x192 X64x128", "L128x128 X64x128"),
    (3094, 29850, 84, BF16, "S256x256",
     "G256x256 W128x128 X128x128", "L256x256 X128x128"),
    (4184, 944, 3958, BF16, "S64x64",
     "G64x64 W256x192 X128x128", "L256x192 X128x128"),
    (626, 33237, 814, BF16, "S128x128 S256x256",
     "G128x128 G256x256 W256x192 X128x128", "L128x128 L256x256 X128x128"),
    (4152, 25637, 200, BF16, "S256x256",
     "G128x128 G256x256 G64x64 W256x256 X256x256", "L256x256 X256x256"),
    (7011, 863, 3626, BF16, "S128x128",
     "G128x128 W256x256 X256x192 X256x256", "L128x128 X256x192 X256x256"),
    (890, 10656, 2530, BF16, "S256x192",
     "G256x192 W256x192 W256x256 X256x256", "L256x192 X256x256"),
    (1369, 68189, 264, BF16, "S256x256 S64x128",
     "G256x256 G64x128 W256x192 W64x64 X256x192 X64x64", "L256x256 L64x128 X256x192"),
    (301, 24226, 3466, BF16, "S256x192",
     "G64x128 W128x128 W256x256 X256x256 X64x128", "L256x192 X256x256 X64x128"),
    (2651, 34010, 336, BF16, "S256x256",
     "G256x256 G64x128 W256x192 W64x64 X256x192 X64x64", "L256x256 X256x192"),
    (3482, 7349, 1390, BF16, "S256x256",
     "G256x192 G256x256 W256x192 X256x256", "L256x192 L256x256 X256x256"),
    (6446, 25014, 298, BF16, "S256x256",
     "G256x256 W128x128 W256x192 X256x192", "L256x256 X128x128 X256x192"),
    (361, 38171, 3776, BF16, "S128x128",
     "G128x128 W256x256 X128x128 X256x256", "L128x128 X128x128 X256x256"),
    (788, 23315, 3152, BF16, "S256x192",
     "G256x192 W256x192 W256x256 X256x192 X32x64", "L256x192 X256x192 X32x64"),
    (4097, 16384, 1024, BF16, "S256x256 S32x64",
     "G256x256 G32x64 W256x256 X256x256 X32x64", "L256x256 L32x64 X256x256 X32x64"),
    (1, 2, 1, F32, "L32x64",
     "G32x64 W32x64 X32x64", "L32x64 X32x64"),
    (6591, 2, 459, F32, "S64x64",
     "G64x64 W32x64 X64x128", "L64x64 X64x128"),
    (1, 47022, 265, F32, "L32x64",
     "G32x64 W128x128 W64x64 X32x64", "L32x64 X32x64"),
    (2, 5014, 1646, F32, "L32x64",
     "G32x64 W128x128 W32x64 X32x64", "L32x64 X32x64"),
    (1, 9016, 3645, F32, "L32x64",
     "G32x64 W128x128 W64x64 X32x64", "L32x64 X32x64"),
    (6200, 3, 2561, F32, "S64x64",
     "G64x64 W32x64 X128x128 X64x64", "L64x64 X128x128 X64x64"),
    (5640, 4, 2840, F32, "S64x64",
     "G64x64 W32x64 X128x128 X32x64", "L64x64 X128x128 X32x64"),
    (6494, 20495, 1, F32, "S128x128",
     "G128x128 W64x64 X64x64", "L128x128 X64x64"),
    (5811, 41, 1439, F32, "S64x64",
     "G64x64 W64x64 X128x128 X64x64", "L64x64 X128x128 X64x64"),
    (77, 1964, 4180, F32, "S64x64",
     "G64x64 W64x128 X64x128", "L64x64 X64x128"),
    (2695, 3049, 79, F32, "S128x128 S32x64",
     "G128x128 G32x64 W64x64 X64x64", "L128x128 L32x64 X64x64"),
    (1082, 7683, 91, F32, "S128x128 S64x64",
     "G128x128 G64x64 W64x64 X64x64", "L128x128 L64x64 X64x64"),
    (417, 24855, 77, F32, "S128x128",
     "G128x128 G64x128 W128x128 X64x64", "L128x128 L64x128 X64x64"),
    (428, 9074, 231, F32, "S64x128",
     "G64x128 W64x64 X128x128", "L64x128 X128x128"),
    (964, 608, 1669, F32, "S64x64",
     "G64x64 W128x128 X64x64", "L64x128 X64x64"),
    (2057, 206, 2584, F32, "S64x64",
     "G64x64 W64x128 X128x128", "L128x128 X128x128"),
    (209, 34204, 173, F32, "S128x128 S64x64",
     "G128x128 G64x64 W64x64 X64x64", "L128x128 L64x64 X64x64"),
    (162, 58309, 131, F32, "S128x128 S64x128",
     "G128x128 G64x128 W128x128 X64x64", "L128x128 L64x128 X64x64"),
    (4170, 32076, 65, F32, "S128x128",
     "G128x128 G64x64 W128x128 X128x128", "L128x128 X128x128"),
    (163, 20074, 2761, F32, "S64x128",
     "G64x128 W128x128 X128x128 X64x128", "L128x128 L64x128 X128x128 X64x128"),
    (811, 23505, 839, F32, "S128x128 S64x128",
     "G128x128 G64x128 W128x128 X128x128", "L128x128 L64x128 X128x128"),
    (3383, 66034, 261, F32, "S128x128",
     "G128x128 G64x64 W128x128 W64x64 X128x128 X64x64", "L128x128 X128x128"),
]


def tiles(call):
    """The tiles of a call's products, as in CASES.  (The profiler does not know
    bf16's name: it takes the operand flag after it, if that is true, for part of
    it, and else leaves the whole name as the compiler has it.)"""
    found = set()
    for name in whole_kernel_names(call):
        if "product_kernel" not in name:
            continue
        name = name.replace("Tile<bool _Accum, bool, E, ", "Tile<bf16, true, ")
        m = (re.search(r"Tile<\w+, (true|false), (true|false), (\d+), (\d+), .*?>, \(Use\)(\d)>", name) or
             re.search(r"TileI\w+?Lb(\d)ELb(\d)ELi(\d+)ELi(\d+)E\w+?3UseE(\d)E", name))
        assert m, name
        a, b = m[1] in ("true", "1"), m[2] in ("true", "1")
        found.add(f"{'SGL'[int(m[5])] if a and b else 'X' if a else 'W'}{m[3]}x{m[4]}")
    return " ".join(sorted(found))


def make(T, V, D, dtype):
    g = torch.Generator(device=dev()).manual_seed(T + 3 * V + 5 * D)
    X = torch.randn(T, D, generator=g, device=dev()).to(dtype)
    W = (torch.randn(V, D, generator=g, device=dev()) * 2 / D ** 0.5).to(dtype)
    target = torch.randint(0, V, (T,), generator=g, device=dev())
    if T > 8:
        target[torch.rand(T, generator=g, device=dev()) < 0.1] = -1
    return X, W, target, torch.rand(T, generator=g, device=dev()) + 0.5


def within(got, want, bound, what):
    over = (got.double() - want).abs() / bound.clamp(min=1e-300)
    assert bool(torch.isfinite(got).all()) and float(over.max()) <= 1.0, f"{what}: {float(over.max()):.2f} of its bound"


def near(got, want, scale, k, D, bf16, what):
    """The error's rms.  fp32 sums of k terms: each of k roundings is up to u of a
    partial sum no larger (rms) than the whole's scale, the root of the terms'
    squares, and they add as a random walk: u sqrt(k / 3) of it, and a few more
    that do not grow.  G's own come from its logits, sums of D terms of scale about
    2, and from the exponential of up to 16: u of it each.  A bf16 result is also
    off by its rounding, up to 2^-8 and evenly spread."""
    u = O.U32
    limit = u * ((k / 3) ** 0.5 + 2 * ((D / 3) ** 0.5 + 4) + 24) * float(scale.square().mean().sqrt())
    if bf16:
        limit = (limit ** 2 + float(want.square().mean()) * (O.U16 ** 2 / 3)) ** 0.5
    err = float((got.double() - want).square().mean().sqrt())
    assert err <= limit + O.TINY, f"{what}: {err / limit:.2f} of its limit"


@pytest.mark.parametrize("T,V,D,dtype,forward,backward,factor", CASES,
                         ids=[f"{c[0]}x{c[1]}x{c[2]}-{'f32' if c[3] == F32 else 'bf16'}" for c in CASES])
def test_every_tile_shape(T, V, D, dtype, forward, backward, factor):
    from paper_1706_03292_amd import api
    log(f"xent shapes {T}x{V}x{D} {dtype}")
    X, W, target, dloss = make(T, V, D, dtype)
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    bl, be, bG, bX, bW = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, dtype == BF16)
    G2 = G.square()
    sX = (G2 @ W.double().square()).sqrt()
    sW = (G2.t() @ X.double().square()).sqrt()
    del G2
    l1, e1 = api.xent_forward(X, W, target)
    x1, w1 = api.xent_backward(X, W, target, e1, dloss)
    l2, u2, x2 = api.xent_factor(X, W, target, dloss)
    within(l1, loss, bl, "loss")
    within(e1, lse, be, "lse")
    within(x1, dX, bX, "dX")
    within(w1, dW, bW, "dW")
    within(l2, loss, bl, "factor loss")
    within(u2, G, bG, "U")
    within(x2, dX, bX, "factor dX")
    near(x1, dX, sX, V, D, dtype == BF16, "dX")
    near(x2, dX, sX, V, D, dtype == BF16, "factor dX")
    near(w1, dW, sW, T, D, False, "dW")
    assert tiles(lambda: api.xent_forward(X, W, target)) == forward
    assert tiles(lambda: api.xent_backward(X, W, target, e1, dloss)) == backward
    assert tiles(lambda: api.xent_factor(X, W, target, dloss)) == factor
