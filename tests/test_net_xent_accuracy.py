"""What the classifier loss's products keep of their operands, seen where a
worst-case bound over a whole sum would not see it."""
import pytest
import torch

import _net_oracle as O
from _helpers import dev, kernels, log, sf_arithmetic
from test_net_xent import make, within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


# fp32 sizes whose logits are products of bf16 parts, with a rest of rows in a
# launch of fp32 products and without.
SPLIT_SIZES = [(2308, 6801, 320), (1300, 5000, 264)]


def rms(x):
    return float(x.double().square().mean().sqrt())


def in_parts(call):
    """How many of a call's launches multiply fp32 in bf16 parts."""
    return sum("product_kernel<Tile<Split32" in n.replace("poseidon::", "") for n in kernels(call))


@pytest.mark.parametrize("T,V,D", [(24, 900, 136), (24, 20000, 64), (300, 2100, 200), (700, 4100, 513)])
def test_bf16_input_gradient_of_classes_that_share_a_component(T, V, D):
    """Classes whose weights are 30 times as large as they differ, as a trained
    classifier's may be, and rows whose softmax is concentrated.  A row of G sums
    to 0, so the shared component cancels in dX: what G's own rounding left of it
    would not.  The reference takes the kernel's fp32 U.  G in two bf16 parts is
    off by at most 2^-16 of each entry (rms 2^-16 / sqrt(3) of 30 times dX's
    size: 0.16 of the rounding of dX to bf16, 2^-8 / sqrt(3) * 0.7 of it), and
    fp32 sums by less: 1.05 times dX's rounding holds them.  One part, the
    target's entry made exact, is 3.6 to 5.8 times it at these sizes."""
    from paper_1706_03292_amd import api
    log(f"xent shared component {T}x{V}x{D}")
    g = torch.Generator().manual_seed(T + V + D)
    W = torch.randn(V, D, generator=g) / D ** 0.5
    W[:, ::2] += 30 / D ** 0.5
    X = torch.randn(T, D, generator=g)
    X[:, 1::2] *= 4
    W, X = W.to(BF16).to(dev()), X.to(BF16).to(dev())
    target = torch.randint(0, V, (T,), generator=g).to(dev())
    dloss = (torch.rand(T, generator=g) + 0.5).to(dev())
    _, U, x2 = api.xent_factor(X, W, target, dloss)
    _, lse = api.xent_forward(X, W, target)
    x1, _ = api.xent_backward(X, W, target, lse, dloss)
    want = U.double() @ W.double()
    rounding = rms(want.to(BF16).double() - want)
    for got, what in ((x2, "factor dX"), (x1, "dX")):
        err = rms(got.double() - want)
        assert err <= 1.05 * rounding, f"{what}: {err / rounding:.2f} times the rounding of dX"


@pytest.mark.parametrize("T,V,D", SPLIT_SIZES)
def test_classes_masked_by_minus_infinity_where_fp32_is_multiplied_in_parts(T, V, D):
    """An infinite weight has no finite bf16 parts: classes masked by one still
    leave every other class as if they were not there, whichever tile a size
    takes.  (dX is not checked: 0 times infinity is its value.)"""
    from paper_1706_03292_amd import api
    log(f"xent masked classes {T}x{V}x{D} f32")
    X, W, target, dloss = make(T, V, D, F32, 7)
    X = X.abs() + torch.finfo(F32).eps
    out = (torch.arange(V) % 997 == 1) | (torch.arange(V) >= V - 70)
    W[out] = -float("inf")
    kept = torch.nonzero(~out)[:, 0]
    none = (target < 0) | (target >= V)
    place = torch.randint(0, len(kept), (T,), generator=torch.Generator().manual_seed(22))
    target = torch.where(none, target, kept[place])
    small = torch.where(none, torch.full_like(place, -1), place)
    loss, lse, G, dX, dW = O.xent(X, W[kept], small, dloss)
    bl, be, bG, _, bW = O.xent_bounds(X, W[kept], small, dloss, lse, G, dX, dW, False)
    Xd, Wd, td, dd = (v.to(dev()) for v in (X, W, target, dloss))
    assert in_parts(lambda: api.xent_forward(Xd, Wd, td)) >= 1
    l1, e1 = api.xent_forward(Xd, Wd, td)
    within(l1, loss, bl, "loss")
    within(e1, lse, be, "lse")
    _, w1 = api.xent_backward(Xd, Wd, td, e1, dd)
    assert (w1.cpu()[out] == 0).all()
    within(w1.cpu()[kept], dW, bW, "dW")
    l2, u2, _ = api.xent_factor(Xd, Wd, td, dd)
    within(l2, loss, bl, "factor loss")
    within(u2.cpu()[:, kept], G, bG, "U")
    assert (u2.cpu()[:, out] == 0).all()


@pytest.mark.parametrize("T,V,D", SPLIT_SIZES)
def test_bad_rows_where_fp32_is_multiplied_in_parts(T, V, D):
    """NaN, infinities and the type's ends in rows without a target leave the
    tile's other rows as they are, and in rows with one too."""
    from paper_1706_03292_amd import api
    log(f"xent bad rows {T}x{V}x{D} f32")
    X, W, target, dloss = make(T, V, D, F32, 9)
    none = (target < 0) | (target >= V)
    bad = X.clone()
    at = torch.nonzero(none)[:, 0]
    bad[at[0::4]] = float("nan")
    bad[at[1::4], ::2] = float("inf")
    bad[at[2::4], 1::3] = -float("inf")
    bad[at[3::4], ::5] = torch.finfo(F32).max
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    bl, be, bG, bX, bW = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, False)
    Xd, Wd, td, dd = (v.to(dev()) for v in (bad, W, target, dloss))
    l1, e1 = api.xent_forward(Xd, Wd, td)
    within(l1, loss, bl, "loss")
    within(e1.cpu()[~none], lse[~none], be[~none], "lse")
    x1, w1 = api.xent_backward(Xd, Wd, td, e1, dd)
    within(x1, dX, bX, "dX")
    within(w1, dW, bW, "dW")
    l2, u2, x2 = api.xent_factor(Xd, Wd, td, dd)
    within(l2, loss, bl, "factor loss")
    within(u2, G, bG, "U")
    within(x2, dX, bX, "factor dX")
    seen = (int(at[0]) + 1) % T       # a row with a target, made NaN: its own loss is NaN, no other row's
    while bool(none[seen]):
        seen = (seen + 1) % T
    bad[seen] = float("nan")
    l3, _ = api.xent_forward(bad.to(dev()), Wd, td)
    others = torch.arange(T) != seen
    assert torch.isnan(l3[seen])
    within(l3.cpu()[others], loss[others], bl[others], "loss beside a NaN row")


def any_mantissa(n, g):
    """fp32 values of either sign, any mantissa and a few orders."""
    v = (1 + torch.rand(n, generator=g, dtype=torch.float64)) * 2.0 ** torch.randint(-3, 4, (n,), generator=g)
    return (v * (2 * torch.randint(0, 2, (n,), generator=g) - 1)).float()


def below_a_step(n, g):
    """fp32 values a little less than one bf16 step above 1.  To nearest, their
    first part is that step and two parts hold them; cut off, it is 1, the second
    part is as large as it can be, and so is nearly the third."""
    third = 2.0 ** -16 * (0.5 + 0.5 * torch.rand(n, generator=g, dtype=torch.float64))
    return (1 + 2.0 ** -7 - 2.0 ** -15 + third).float()


@pytest.mark.parametrize("values,worst,mean", [(any_mantissa, 12.0, None), (below_a_step, None, 2.0)],
                         ids=["any", "below_a_step"])
def test_single_fp32_products_in_parts(values, worst, mean):
    """Each result is one product, the other terms 0, of operands that the call
    leaves as they are: with logits 0 and lse 0, G is dloss (its column at the
    target 0), and a row whose one large logit is above all others has it as its
    lse.  In units of 2^-24 of the product: what the six products of parts drop is
    below 1 (2 * 2^-8 * 2^-17), their five sums round by at most 1 each, to
    nearest, or 2, and lse once more: 12.  Without any of the six it is 60 or more.
    Where two parts hold a value nothing is dropped and three sums round, each by
    half a unit on average: 2.  With the first part cut off, the dropped products
    come to 3 there."""
    from paper_1706_03292_amd import api
    log(f"xent single products {values.__name__}")
    T, V, D = SPLIT_SIZES[0]
    g = torch.Generator().manual_seed(5)
    one_class, one_row = torch.randperm(V - 1, generator=g)[:D], torch.randperm(T, generator=g)[:D]
    feature = torch.arange(D)
    w, d, x = values(D, g), values(T, g), values(D, g)
    target, lse = torch.full((T,), V - 1, device=dev()), torch.zeros(T, device=dev())
    dloss = d.to(dev())

    def check(got, want, what):
        units = ((got.double().cpu() - want) / want).abs() * 2 ** 24
        assert worst is None or float(units.max()) <= worst, f"{what}: {float(units.max()):.1f} units"
        assert mean is None or float(units.mean()) <= mean, f"{what}: {float(units.mean()):.2f} units on average"

    # dX[t, k] = dloss_t * W[class of k, k]
    X, W = torch.zeros(T, D, device=dev()), torch.zeros(V, D)
    W[one_class, feature] = w
    W = W.to(dev())
    assert in_parts(lambda: api.xent_backward(X, W, target, lse, dloss)) == 3
    check(api.xent_backward(X, W, target, lse, dloss)[0], d.double()[:, None] * w.double(), "dX")
    # dW[v, k] = dloss of k's row * X[that row, k]
    X, W = torch.zeros(T, D), torch.zeros(V, D, device=dev())
    X[one_row, feature] = x
    X = X.to(dev())
    assert in_parts(lambda: api.xent_backward(X, W, target, lse, dloss)) == 3
    dW = api.xent_backward(X, W, target, lse, dloss)[1]
    check(dW[:-1], (d[one_row].double() * x.double()).expand(V - 1, D), "dW")
    # lse_t = X[t, k] * W[class of k, k] for the row's one feature k
    X, W, k = torch.zeros(T, D), torch.zeros(V, D), torch.randint(0, D, (T,), generator=g)
    W[one_class, feature] = w.abs()
    X[torch.arange(T), k] = 128 * d.abs()
    want = 128 * d.double().abs() * w.double().abs()[k]
    large = want > 60                          # the other classes' e^-60 is nothing beside 1
    assert int(large.sum()) > T // 2
    check(api.xent_forward(X.to(dev()), W.to(dev()), target)[1][large.to(dev())], want[large], "lse")


def test_single_bf16_products_of_the_weight_gradient():
    """dW of bf16 inputs from G in three exact parts: each result is one product
    of an fp32 dloss and a bf16 X (as above).  Two sums round, each by at most a
    unit of 2^-24, to nearest, or 2: 4.  Two parts of G leave up to 128."""
    from paper_1706_03292_amd import api
    log("xent single bf16 products")
    T, V, D = SPLIT_SIZES[0]
    g = torch.Generator().manual_seed(6)
    d, x, one_row = any_mantissa(T, g), any_mantissa(D, g).to(BF16), torch.randperm(T, generator=g)[:D]
    X = torch.zeros(T, D, dtype=BF16)
    X[one_row, torch.arange(D)] = x
    target, lse = torch.full((T,), V - 1, device=dev()), torch.zeros(T, device=dev())
    _, dW = api.xent_backward(X.to(dev()), torch.zeros(V, D, dtype=BF16, device=dev()), target, lse, d.to(dev()))
    want = (d[one_row].double() * x.double()).expand(V - 1, D)
    units = ((dW[:-1].double().cpu() - want) / want).abs() * 2 ** 24
    assert float(units.max()) <= 4.0, f"{float(units.max()):.1f} units"


@pytest.mark.parametrize("T,V,D", SPLIT_SIZES)
def test_fp32_products_where_the_process_asks_for_them(T, V, D):
    """poseidon_sf_set_arithmetic reaches the loss's fp32 products, on workspaces
    of the same size, and setting it back gives the former bits."""
    from paper_1706_03292_amd import api
    log(f"xent arithmetic {T}x{V}x{D}")
    X, W, target, dloss = make(T, V, D, F32, 13)
    loss, lse, G, dX, dW = O.xent(X, W, target, dloss)
    bounds = O.xent_bounds(X, W, target, dloss, lse, G, dX, dW, False)
    Xd, Wd, td, dd = (v.to(dev()) for v in (X, W, target, dloss))

    def everything():
        l1, e1 = api.xent_forward(Xd, Wd, td)
        x1, w1 = api.xent_backward(Xd, Wd, td, e1, dd)
        return (l1, e1, x1, w1) + tuple(api.xent_factor(Xd, Wd, td, dd))

    before = everything()
    with sf_arithmetic(api.SF_FP32):
        assert in_parts(everything) == 0
        l1, e1, x1, w1, l2, u2, x2 = everything()
    assert in_parts(everything) >= 3
    for got, want, b, what in ((l1, loss, bounds[0], "loss"), (e1, lse, bounds[1], "lse"), (u2, G, bounds[2], "U"),
                               (x1, dX, bounds[3], "dX"), (w1, dW, bounds[4], "dW"), (l2, loss, bounds[0], "factor loss"),
                               (x2, dX, bounds[3], "factor dX")):
        within(got, want, b, what)
    for a, b in zip(before, everything()):
        assert torch.equal(a, b)
