"""Softmax cross entropy fused with the classifier's product: forward, backward
and factor form against a 64-bit reference within bounds derived from the
arithmetic (tests/_net_oracle.py), at the sizes where tiles, steps, splits and
pieces end."""
import pytest
import torch

import _net_oracle as O
from _helpers import dev, kernels, log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

# Rows, classes, features: single ones, below, at and past tile (32, 64, 128)
# and step (32, 64) ends, features off the 16-byte boundaries, many rows of few
# classes and the reverse.
SIZES = [(1, 1, 1), (1, 1000, 64), (2, 7, 3), (31, 63, 65), (32, 64, 32), (33, 65, 129), (64, 128, 64), (128, 128, 8),
         (129, 257, 72), (200, 1000, 100), (257, 300, 256), (300, 2000, 513), (1000, 40, 16), (5, 21841, 40),
         (700, 513, 1030), (1174, 10709, 640), (2308, 6801, 320)]


def make(T, V, D, dtype, seed, ignore=0.2):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(T, D, generator=g).to(dtype)
    W = (torch.randn(V, D, generator=g) * 2 / D ** 0.5).to(dtype)
    target = torch.randint(0, V, (T,), generator=g)
    none = torch.rand(T, generator=g) < ignore
    target = torch.where(none, torch.where(torch.rand(T, generator=g) < 0.5, torch.full_like(target, -100),
                                           target + V), target)
    dloss = torch.rand(T, generator=g) + 0.5
    return X, W, target, dloss


def within(got, want, bound, what):
    got = got.double().cpu()
    want, bound = want.cpu(), bound.cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - want).abs() / bound.clamp(min=1e-300)
    assert got.numel() == 0 or float(over.max()) <= 1.0, f"{what}: {float(over.max()):.2f} of its bound"


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_against_64_bits(T, V, D, dtype):
    from paper_1706_03292_amd import api
    log(f"xent {T}x{V}x{D} {dtype}")
    X, W, target, dloss = make(T, V, D, dtype, 11 * T + V + D)
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    bl, be, bG, bX, bW = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, dtype == BF16)
    Xd, Wd, td, dd = (v.to(dev()) for v in (X, W, target, dloss))
    l1, e1 = api.xent_forward(Xd, Wd, td)
    x1, w1 = api.xent_backward(Xd, Wd, td, e1, dd)
    l2, u2, x2 = api.xent_factor(Xd, Wd, td, dd)
    assert x1.dtype == dtype and w1.dtype == F32 and u2.dtype == F32
    within(l1, loss, bl, "loss")
    within(e1, lse, be, "lse")
    within(x1, dX, bX, "dX")
    within(w1, dW, bW, "dW")
    within(l2, loss, bl, "factor loss")
    within(u2, G, bG, "U")
    within(x2, dX, bX, "factor dX")
    none = (target < 0) | (target >= V)
    assert (l1.cpu()[none] == 0).all() and (u2.cpu()[none] == 0).all() and (x1.cpu()[none] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", [(9, 130, 64), (150, 300, 72)])
def test_rows_without_a_target_reach_nothing(T, V, D, dtype):
    """NaN and infinity in the X and dloss of ignored rows, all rows ignored,
    and the lse of an ignored row."""
    from paper_1706_03292_amd import api
    log(f"xent ignored {T}x{V}x{D} {dtype}")
    X, W, target, dloss = make(T, V, D, dtype, 5, ignore=0.4)
    target[0], target[1], target[T - 1] = -1, V, 2 ** 40
    none = (target < 0) | (target >= V)
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    _, _, bG, bX, bW = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, dtype == BF16)
    bad = X.clone()
    bad[none] = float("nan")
    bad[0, ::2] = float("inf")
    dbad = dloss.clone()
    dbad[none] = float("nan")
    Xd, Wd, td, dd = (v.to(dev()) for v in (bad, W, target, dbad))
    l1, e1 = api.xent_forward(Xd, Wd, td)
    assert torch.isfinite(l1).all() and (l1.cpu()[none] == 0).all()
    x1, w1 = api.xent_backward(Xd, Wd, td, e1, dd)
    within(x1, dX, bX, "dX")
    within(w1, dW, bW, "dW")
    _, u2, x2 = api.xent_factor(Xd, Wd, td, dd)
    within(u2, G, bG, "U")
    within(x2, dX, bX, "factor dX")
    all_out = torch.full_like(td, -1)
    l3, e3 = api.xent_forward(Xd, Wd, all_out)
    x3, w3 = api.xent_backward(Xd, Wd, all_out, e3, dd)
    assert (l3 == 0).all() and (x3 == 0).all() and (w3 == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_no_rows(dtype):
    from paper_1706_03292_amd import api
    log(f"xent T=0 {dtype}")
    X, W = torch.empty(0, 40, dtype=dtype, device=dev()), torch.randn(70, 40, device=dev()).to(dtype)
    t, z = torch.empty(0, dtype=torch.int64, device=dev()), torch.empty(0, device=dev())
    loss, lse = api.xent_forward(X, W, t)
    assert loss.shape == (0,) and lse.shape == (0,)
    dW = torch.full((70, 40), 3.0, device=dev())
    dX, dW = api.xent_backward(X, W, t, z, z, dW=dW)
    assert dX.shape == (0, 40) and (dW == 0).all()
    loss, U, dX = api.xent_factor(X, W, t, z)
    assert loss.shape == (0,) and U.shape == (0, 70) and dX.shape == (0, 40)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_large_logits(dtype):
    """Rows whose softmax is all but one-hot, at the target and elsewhere, and
    logits of several hundred: the running maximum keeps every sum finite."""
    from paper_1706_03292_amd import api
    log(f"xent large logits {dtype}")
    T, V, D = 40, 500, 64
    X, W, target, dloss = make(T, V, D, dtype, 3, ignore=0.0)
    X = (X.double() * 60).to(dtype)
    S = X.double() @ W.double().t()
    target[:20] = S[:20].argmax(1)
    assert float(S.abs().max()) > 200
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    bl, be, bG, bX, bW = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, dtype == BF16)
    Xd, Wd, td, dd = (v.to(dev()) for v in (X, W, target, dloss))
    l1, e1 = api.xent_forward(Xd, Wd, td)
    x1, w1 = api.xent_backward(Xd, Wd, td, e1, dd)
    _, u2, x2 = api.xent_factor(Xd, Wd, td, dd)
    for got, want, b, what in ((l1, loss, bl, "loss"), (e1, lse, be, "lse"), (x1, dX, bX, "dX"), (w1, dW, bW, "dW"),
                               (u2, G, bG, "U"), (x2, dX, bX, "factor dX")):
        within(got, want, b, what)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", [(32, 1000, 64), (300, 2100, 200), (1300, 5000, 264), (5, 21841, 40)])
def test_classes_at_the_lowest_value(T, V, D, dtype):
    """Classes kept out by a weight of the type's lowest value at a feature that
    is 1 (a padded vocabulary): whole tiles of them and odd ones, results as
    without them."""
    from paper_1706_03292_amd import api
    log(f"xent lowest {T}x{V}x{D} {dtype}")
    X, W, target, dloss = make(T, V, D, dtype, 21)
    out = (torch.arange(V) // 256 % 2 == 1) | (torch.arange(V) % 7 == 3) | (torch.arange(V) >= V - 90)
    X[:, 0], W[:, 0] = 1, 0
    W[out] = 0
    W[out, 0] = torch.finfo(dtype).min
    kept = torch.nonzero(~out)[:, 0]
    none = (target < 0) | (target >= V)
    place = torch.randint(0, len(kept), (T,), generator=torch.Generator().manual_seed(22))
    target = torch.where(none, target, kept[place])
    small = torch.where(none, torch.full_like(place, -1), place)
    loss, lse, G, dX, dW = O.xent(X, W[kept], small, dloss)
    bl, be, bG, bX, bW = O.xent_bounds(X, W[kept], small, dloss, lse, G, dX, dW, dtype == BF16)
    Xd, Wd, td, dd = (v.to(dev()) for v in (X, W, target, dloss))
    l1, e1 = api.xent_forward(Xd, Wd, td)
    x1, w1 = api.xent_backward(Xd, Wd, td, e1, dd)
    l2, u2, x2 = api.xent_factor(Xd, Wd, td, dd)
    assert (w1.cpu()[out] == 0).all() and (u2.cpu()[:, out] == 0).all()
    for got, want, b, what in ((l1, loss, bl, "loss"), (e1, lse, be, "lse"), (x1, dX, bX, "dX"),
                               (w1.cpu()[kept], dW, bW, "dW"), (l2, loss, bl, "factor loss"),
                               (u2.cpu()[:, kept], G, bG, "U"), (x2, dX, bX, "factor dX")):
        within(got, want, b, what)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_any_element_boundary(dtype):
    """Arrays that start one element past a boundary of 16 bytes give the bits
    that aligned ones give."""
    from paper_1706_03292_amd import api
    log(f"xent boundary {dtype}")
    T, V, D = 70, 333, 64
    X, W, target, dloss = (v.to(dev()) for v in make(T, V, D, dtype, 8))

    def off(x):
        y = torch.empty(x.numel() + 1, dtype=x.dtype, device=x.device)[1:].view(x.shape)
        return y.copy_(x)

    l1, e1 = api.xent_forward(X, W, target)
    x1, w1 = api.xent_backward(X, W, target, e1, dloss)
    l2, e2 = api.xent_forward(off(X), off(W), off(target))
    x2, w2 = api.xent_backward(off(X), off(W), off(target), off(e1), off(dloss), dW=off(torch.zeros_like(w1)))
    assert torch.equal(l1, l2) and torch.equal(e1, e2) and torch.equal(x1, x2) and torch.equal(w1, w2)
    l3, u3, x3 = api.xent_factor(X, W, target, dloss)
    l4, u4, x4 = api.xent_factor(off(X), off(W), target, dloss, U=off(torch.zeros_like(u3)))
    assert torch.equal(l3, l4) and torch.equal(u3, u4) and torch.equal(x3, x4)


@pytest.mark.parametrize("T,V,D,dtype", [(2050, 65536 + 77, 16, BF16), (2050, 65536 + 77, 16, F32)],
                         ids=["bf16", "f32"])
def test_several_pieces_of_the_vocabulary(T, V, D, dtype):
    """More logits than one piece of the backward pass holds (the last piece
    ragged), so dX is summed over pieces."""
    from paper_1706_03292_amd import api
    log(f"xent pieces {T}x{V}x{D} {dtype}")
    X, W, target, dloss = (v.to(dev()) for v in make(T, V, D, dtype, 21))
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    bl, be, _, bX, bW = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, dtype == BF16)
    l1, e1 = api.xent_forward(X, W, target)
    names = kernels(lambda: api.xent_backward(X, W, target, e1, dloss))
    assert sum("product_kernel" in n for n in names) >= 6, names
    x1, w1 = api.xent_backward(X, W, target, e1, dloss)
    within(l1, loss, bl, "loss")
    within(x1, dX, bX, "dX")
    within(w1, dW, bW, "dW")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_same_bits_every_time_and_on_another_stream(dtype):
    from paper_1706_03292_amd import api
    log(f"xent repeat {dtype}")
    X, W, target, dloss = (v.to(dev()) for v in make(150, 2000, 96, dtype, 2))

    def all_of(stream=None):
        l, e = api.xent_forward(X, W, target, stream=stream)
        if stream is not None:
            e.record_stream(stream)
        return (l, e, *api.xent_backward(X, W, target, e, dloss, stream=stream),
                *api.xent_factor(X, W, target, dloss, stream=stream))

    first = all_of()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    again, there = all_of(), all_of(other)
    torch.cuda.current_stream().wait_stream(other)
    raw = all_of()
    for a, b, c, d in zip(first, again, there, raw):
        assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, d)


def test_captured_graph_replays():
    """A captured training step of the classifier, replayed on new inputs with
    eager work in between, gives what the eager call gives."""
    from paper_1706_03292_amd import api
    log("xent graph")
    X, W, target, dloss = (v.to(dev()) for v in make(64, 1500, 128, BF16, 4))
    eager = lambda: (api.xent_factor(X, W, target, dloss),  # noqa: E731
                     api.xent_backward(X, W, target, api.xent_forward(X, W, target)[1], dloss))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = eager()
    for seed in (41, 42, 43):
        fresh = make(64, 1500, 128, BF16, seed)
        for dst, src in zip((X, W, target, dloss), fresh):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        want = eager()
        torch.cuda.synchronize()
        for h, w in zip(held, want):
            for a, b in zip(h, w):
                assert torch.equal(a, b)


def test_gradient_against_differences():
    """The fp32 gradients against central differences of the kernel's own loss
    along random directions: off by the third-order term and by the loss's
    rounding over the step."""
    from paper_1706_03292_amd import api
    log("xent differences")
    T, V, D, eps = 48, 300, 80, 0.02
    X, W, target, dloss = (v.to(dev()) for v in make(T, V, D, F32, 6))
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    bl = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, False)[0]
    _, e = api.xent_forward(X, W, target)
    gX, gW = api.xent_backward(X, W, target, e, dloss)
    gen = torch.Generator(device=dev()).manual_seed(1)
    for which in ("X", "W"):
        x, grad = (X, gX) if which == "X" else (W, gW)
        step = torch.randn(x.shape, generator=gen, device=dev())
        step = step / step.norm(dim=1, keepdim=True)

        def value(sign, of):
            moved = x + sign * eps * step
            a = (moved, W) if which == "X" else (X, moved)
            return float((of(*a).double() * dloss.double()).sum())

        kernel = lambda a, b: api.xent_forward(a, b, target)[0]  # noqa: E731
        exact = lambda a, b: O.xent(a, b, target, dloss)[0]  # noqa: E731
        slope = (value(1, kernel) - value(-1, kernel)) / (2 * eps)
        # the differences' own error, from the 64-bit loss
        third = abs((value(1, exact) - value(-1, exact)) / (2 * eps) -
                    float((((dX if which == "X" else dW)) * step.double()).sum()))
        rounding = float((bl * dloss.double()).sum()) / eps
        assert abs(slope - float((grad.double() * step.double()).sum())) <= third + 2 * rounding + 1e-6


@pytest.mark.parametrize("dtype,D", [(F32, 37), (F32, 64), (BF16, 100), (BF16, 64)], ids=str)
def test_a_class_masked_by_minus_infinity(dtype, D):
    """A class whose weights are -inf has logit -inf for positive features and
    leaves every other class as if it were not there -- also the class before
    it, whose row ends inside the 16 bytes that hold the masked row's start."""
    from paper_1706_03292_amd import api
    log(f"xent masked class {dtype} D={D}")
    T, V = 9, 150
    X, W, target, dloss = make(T, V, D, dtype, 7, ignore=0.0)
    X = X.abs() + torch.finfo(dtype).eps
    for v in (1, 64, V - 1):
        W[v] = -float("inf")
    left = torch.tensor([v for v in range(V) if v not in (1, 64, V - 1)])
    target = left[target % len(left)]
    place = torch.searchsorted(left, target)
    loss, lse, G, dX, dW = O.xent(X, W[left], place, dloss)
    bl, be, bG, _, _ = O.xent_bounds(X, W[left], place, dloss, lse, G, dX, dW, dtype == BF16)
    Xd, Wd, td, dd = (v.to(dev()) for v in (X, W, target, dloss))
    l1, e1 = api.xent_forward(Xd, Wd, td)
    within(l1, loss, bl, "loss")
    within(e1, lse, be, "lse")
    l2, u2, _ = api.xent_factor(Xd, Wd, td, dd)
    within(l2, loss, bl, "factor loss")
    within(u2.cpu()[:, left], G, bG, "U")
    assert (u2.cpu()[:, [1, 64, V - 1]] == 0).all()
