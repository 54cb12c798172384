"""Layer norm with residual and dropout, its backward pass, and dropout alone,
against a 64-bit reference with the generator written out in numpy."""
import pytest
import torch

import _net_oracle as O
from _helpers import dev, log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DTYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])

# One value, rows that end inside a group of eight, each team size's ends (128,
# 512, 1024, 2048, 4096, 8192 and 32768 values) and rows past the longest.
SHAPES = [(1, 1), (3, 7), (2, 8), (70, 100), (17, 128), (5, 129), (9, 512), (4, 1000), (33, 1024), (6, 2047),
          (3, 2049), (5, 4096), (2, 5001), (2, 8192), (3, 9000), (1, 32768), (2, 32777)]
SEED, OFFSET = 0x123456789ABCDEF, -3


def rounding(dtype):
    return O.U16 if dtype == BF16 else O.U32


def state():
    return torch.tensor([SEED, OFFSET], dtype=torch.int64, device=dev())


def rows_of(rows, cols, dtype, seed, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, cols, generator=g) * std + mean).to(dtype)


def within(got, want, bound, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - want).abs() / bound
    assert float(over.max()) <= 1.0, f"{what}: {float(over.max()):.2f} of its bound"


@DTYPES
@pytest.mark.parametrize("residual", [False, True], ids=["", "residual"])
@pytest.mark.parametrize("p", [0.1, 0.5])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (64, 64), (5, 1001), (1, 100003), (40, 4096)])
def test_dropout(rows, cols, p, residual, dtype):
    from paper_1706_03292_amd import api
    log(f"dropout {rows}x{cols} p={p} {dtype}")
    x, res = rows_of(rows, cols, dtype, 1), rows_of(rows, cols, dtype, 2) if residual else None
    mask, thr = O.keep(SEED, OFFSET, rows, cols, p)
    want = O.dropped(x, mask, thr) + (res.double() if residual else 0.0)
    y = api.dropout(x.to(dev()), p, state(), residual=res.to(dev()) if residual else None)
    scale = O.dropped(x, mask, thr).abs() + (res.double().abs() if residual else 0.0)
    within(y, want, 4 * O.U32 * scale + rounding(dtype) * want.abs() + O.TINY, "y")
    if not residual:
        assert torch.equal(y.cpu() == 0, (~mask) | (x == 0))


def test_dropout_generator_known_answer():
    """Key and counter 0: the first group's 128 bits, as seven rounds of
    Philox4x32 give them (published test vector of the generator)."""
    words = [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    bits = [b for w in words for b in (w & 0xFFFF, w >> 16)]
    for i, b in enumerate(bits):
        below, at = b / 65536, (b + 1) / 65536
        assert bool(O.keep(0, 0, 1, 8, below)[0][0, i]) and not bool(O.keep(0, 0, 1, 8, at)[0][0, i])


@DTYPES
def test_dropout_ends_and_what_is_dropped(dtype):
    """p = 0 copies without a generator, p = 1 leaves the residual; infinity and
    NaN in dropped places leave nothing."""
    from paper_1706_03292_amd import api
    log(f"dropout ends {dtype}")
    x, res = rows_of(5, 333, dtype, 3).to(dev()), rows_of(5, 333, dtype, 4).to(dev())
    assert torch.equal(api.dropout(x, 0.0, None), x)
    assert torch.equal(api.dropout(x, 1.0, state(), residual=res), res)
    mask, _ = O.keep(SEED, OFFSET, 5, 333, 0.5)
    bad = torch.where(mask.to(dev()), x, torch.full_like(x, float("nan")))
    bad[:, ::3] = torch.where(mask.to(dev()), x, torch.full_like(x, float("inf")))[:, ::3]
    assert torch.equal(api.dropout(bad, 0.5, state()), api.dropout(x, 0.5, state()))
    assert api.dropout(x[:0], 0.5, state()).shape == (0, 333)
    assert api.dropout(x[:, :0].contiguous(), 0.5, state()).shape == (5, 0)


def test_dropout_masks_differ_and_keep_their_share():
    from paper_1706_03292_amd import api
    log("dropout share")
    n, p = 1 << 20, 0.3
    x = torch.ones(16, n // 16, device=dev())
    a = api.dropout(x, p, state()) != 0
    b = api.dropout(x, p, torch.tensor([SEED, OFFSET + 1], dtype=torch.int64, device=dev())) != 0
    sd = (p * (1 - p) / n) ** 0.5
    for m in (a, b):
        assert abs(float(m.double().mean()) - (1 - p)) < 6 * sd
    both = float((a & b).double().mean())
    assert abs(both - (1 - p) ** 2) < 6 * ((1 - p) ** 2 / n) ** 0.5


@DTYPES
@pytest.mark.parametrize("p,residual", [(0.0, False), (0.0, True), (0.1, True), (0.5, False), (1.0, True)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_forward(rows, cols, p, residual, dtype):
    from paper_1706_03292_amd import api
    log(f"norm_forward {rows}x{cols} p={p} {residual} {dtype}")
    eps = 1e-5
    x, res = rows_of(rows, cols, dtype, 5, 1.5, 0.5), rows_of(rows, cols, dtype, 6) if residual else None
    gamma, beta = rows_of(1, cols, F32, 7, 0.1, 1.0)[0], rows_of(1, cols, F32, 8, 0.1)[0]
    mask, thr = O.keep(SEED, OFFSET, rows, cols, p)
    h = O.dropped(x, mask, thr) + (res.double() if residual else 0.0)
    y, mean, rstd = O.norm_forward(h, gamma, beta, eps)
    y1, h1, m1, r1 = api.norm_forward(x.to(dev()), gamma.to(dev()), beta.to(dev()), eps,
                                      residual=None if res is None else res.to(dev()), p=p, rng=state() if p else None)
    u = O.U32
    # errors: h 2 roundings; the mean a sum of cols values; the variance a sum of
    # their squares (with the mean's error squared); rstd half the variance's.
    dh = 4 * u * ((res.double().abs() if residual else 0.0) + O.dropped(x, mask, thr).abs()) + O.TINY
    dm = dh.mean(1) + (cols + 8) * u * h.abs().mean(1) + O.TINY
    c = (h - mean[:, None]).abs()
    dc = dh + dm[:, None] + u * c
    dv = (2 * c * dc + dc * dc).mean(1) + (cols + 8) * u * c.square().mean(1)
    dr = 0.5 * rstd ** 3 * dv + 4 * u * rstd
    dy = (dc * rstd[:, None] + c * dr[:, None]) * gamma.double().abs() + 4 * u * (
        c * rstd[:, None] * gamma.double().abs() + beta.double().abs())
    within(m1, mean, O.SLACK * dm, "mean")
    within(r1, rstd, O.SLACK * dr + O.TINY, "rstd")
    within(h1, h, O.SLACK * dh + rounding(dtype) * h.abs(), "h")
    within(y1, y, O.SLACK * dy + rounding(dtype) * y.abs() + O.TINY, "y")
    if not residual and p == 0.0:
        assert torch.equal(h1.cpu(), x)


@DTYPES
@pytest.mark.parametrize("p,residual", [(0.0, False), (0.0, True), (0.1, True), (0.5, False), (1.0, True)])
@pytest.mark.parametrize("rows,cols", SHAPES + [(1500, 24), (2100, 264), (1100, 4100)])
def test_norm_backward(rows, cols, p, residual, dtype):
    from paper_1706_03292_amd import api
    log(f"norm_backward {rows}x{cols} p={p} {residual} {dtype}")
    h, dy = rows_of(rows, cols, dtype, 9, 1.5, 0.25), rows_of(rows, cols, dtype, 10, 0.1)
    dres = rows_of(rows, cols, dtype, 11, 0.1) if residual else None
    gamma = rows_of(1, cols, F32, 12, 0.1, 1.0)[0]
    mean = h.double().mean(1).float()
    rstd = ((h.double() - mean.double()[:, None]).square().mean(1) + 1e-5).rsqrt().float()
    dh, dgamma, dbeta = O.norm_backward(dy, h, gamma, mean, rstd, dres)
    mask, thr = O.keep(SEED, OFFSET, rows, cols, p)
    to = lambda t: None if t is None else t.to(dev())  # noqa: E731
    # into shards of a larger array
    shards = torch.full((3, 2, cols), 7.0, device=dev())
    x1, h1, g1, b1 = api.norm_backward(to(dy), to(h), to(gamma), to(mean), to(rstd), dresidual=to(dres), p=p,
                                       rng=state() if p else None, dgamma=shards[1, 0], dbeta=shards[1, 1])
    u = O.U32
    n = ((h.double() - mean.double()[:, None]) * rstd.double()[:, None]).abs()
    a = (h.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]   # what cancels in n
    g = (dy.double() * gamma.double()).abs()
    R = rstd.double()[:, None]
    dn = 4 * u * a
    avg = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    d1 = (cols + 8) * u * avg(g)
    d2 = (cols + 8) * u * avg(g * n) + avg(g * dn)
    bound = R * (4 * u * g + d1 + n * d2 + dn * avg(g * n) + 4 * u * (avg(g) + n * avg(g * n))) + 4 * u * dh.abs() + O.TINY
    if residual:
        bound = bound + 2 * u * dres.double().abs()
    within(h1, dh, O.SLACK * bound + rounding(dtype) * dh.abs(), "dh")
    wx = O.dropped(dh, mask, thr)
    scale = 1.0 if thr == 0 else 0.0 if thr >= 65536 else 65536.0 / (65536 - thr)
    within(x1, wx, O.SLACK * scale * bound + (rounding(dtype) + 4 * u) * wx.abs() + O.TINY, "dx")
    ady = dy.double().abs()
    within(g1, dgamma, O.SLACK * ((rows + 8) * u * (ady * n).sum(0) + (ady * dn).sum(0)) + O.TINY, "dgamma")
    within(b1, dbeta, O.SLACK * (rows + 8) * u * ady.sum(0) + O.TINY, "dbeta")
    assert (shards[0] == 7).all() and (shards[2] == 7).all()
    assert g1.data_ptr() == shards[1, 0].data_ptr()


@DTYPES
def test_no_rows(dtype):
    from paper_1706_03292_amd import api
    log(f"norm no rows {dtype}")
    x = torch.empty(0, 72, dtype=dtype, device=dev())
    one = torch.ones(72, device=dev())
    y, h, mean, rstd = api.norm_forward(x, one, one)
    assert y.shape == (0, 72) and mean.shape == (0,)
    full = torch.full((2, 72), 5.0, device=dev())
    _, _, dgamma, dbeta = api.norm_backward(x, x, one, mean, rstd, dgamma=full[0], dbeta=full[1])
    assert (dgamma == 0).all() and (dbeta == 0).all()


@pytest.mark.parametrize("shape", [(4, 0), (2, 3, 0)])
def test_no_columns(shape):
    """A row of no values has no mean; dropout of nothing is nothing."""
    from paper_1706_03292_amd import api
    log(f"norm no columns {shape}")
    x, none = torch.empty(shape, device=dev()), torch.empty(0, device=dev())
    with pytest.raises(api.PoseidonError):
        api.norm_forward(x, none, none)
    assert api.dropout(x, 0.5, state()).shape == shape


@DTYPES
@pytest.mark.parametrize("cols", [96, 1000, 4096])
def test_any_boundary_and_leading_shape(cols, dtype):
    """Arrays one element past a 16-byte boundary and inputs of three
    dimensions give the bits that aligned two-dimensional ones give."""
    from paper_1706_03292_amd import api
    log(f"norm boundary {cols} {dtype}")
    x, res, dy = (rows_of(12, cols, dtype, s).to(dev()) for s in (1, 2, 3))
    gamma, beta = rows_of(1, cols, F32, 4, 0.1, 1.0)[0].to(dev()), rows_of(1, cols, F32, 5).to(dev())[0]

    def off(t):
        return torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape).copy_(t)

    def both(f):
        y, h, m, r = api.norm_forward(f(x), f(gamma), f(beta), residual=f(res), p=0.25, rng=state())
        return (y, h, m, r, *api.norm_backward(f(dy), f(h), f(gamma), f(m), f(r), dresidual=f(res), p=0.25,
                                               rng=state()), api.dropout(f(x), 0.25, state(), residual=f(res)))

    plain = both(lambda t: t)
    for a, b in zip(plain, both(off)):
        assert torch.equal(a, b)
    y3 = api.norm_forward(x.view(3, 4, cols), gamma, beta, residual=res.view(3, 4, cols), p=0.25, rng=state())
    assert y3[2].shape == (3, 4)
    for a, b in zip(plain[:4], y3):
        assert torch.equal(a.flatten(), b.flatten())


def test_gradient_against_differences():
    """sum(dy * y) along random directions of x, gamma and beta: the kernel's
    gradients against central differences of the 64-bit formula, whose own
    third-order error is below eps^2 of the slope's scale."""
    from paper_1706_03292_amd import api
    log("norm differences")
    rows, cols, eps = 20, 200, 1e-3
    x, dy = rows_of(rows, cols, F32, 1, 1.5), rows_of(rows, cols, F32, 2)
    gamma, beta = rows_of(1, cols, F32, 3, 0.1, 1.0)[0], rows_of(1, cols, F32, 4)[0]
    mask, thr = O.keep(SEED, OFFSET, rows, cols, 0.25)
    y, h, m, r = api.norm_forward(x.to(dev()), gamma.to(dev()), beta.to(dev()), p=0.25, rng=state())
    dx, _, dgamma, dbeta = api.norm_backward(dy.to(dev()), h, gamma.to(dev()), m, r, p=0.25, rng=state())

    def value(x, gamma, beta):
        return float((O.norm_forward(O.dropped(x, mask, thr), gamma, beta, 1e-5)[0] * dy.double()).sum())

    for k, grad in enumerate((dx, dgamma, dbeta)):
        at = [x.double(), gamma.double(), beta.double()]
        step = torch.randn(at[k].shape, generator=torch.Generator().manual_seed(k)).double()
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + eps * step, at[k] - eps * step
        slope = (value(*up) - value(*down)) / (2 * eps)
        got = float((grad.double().cpu() * step).sum())
        scale = float((grad.double().cpu().abs() * step.abs()).sum())
        assert abs(slope - got) <= 1e-4 * scale, (k, slope, got)


@DTYPES
def test_repeated_on_another_stream_and_in_a_graph(dtype):
    """The same bits each time; a captured graph's replays each take the
    generator's state of their time."""
    from paper_1706_03292_amd import api
    log(f"norm graph {dtype}")
    x, res, dy = (rows_of(300, 520, dtype, s).to(dev()) for s in (1, 2, 3))
    gamma, beta = torch.ones(520, device=dev()), torch.zeros(520, device=dev())
    rng = state()

    def both(stream=None):
        y, h, m, r = api.norm_forward(x, gamma, beta, residual=res, p=0.25, rng=rng, stream=stream)
        return (y, h, m, r, *api.norm_backward(dy, h, gamma, m, r, p=0.25, rng=rng, stream=stream))

    first = both()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    there = both(other)
    torch.cuda.current_stream().wait_stream(other)
    for a, b in zip(first, there):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for _ in range(3):
        rng[1] += 1
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, both()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


@DTYPES
@pytest.mark.parametrize("cols", [40, 2000, 9000])
def test_norm_backward_of_no_rows_needs_no_generator(cols, dtype):
    """A C call without rows may leave every array of rows and the generator
    NULL, with dropout too: dgamma and dbeta are 0."""
    import ctypes

    from paper_1706_03292_amd import _lib as L
    log(f"norm_backward no rows, no generator {cols} {dtype}")
    lib, size = L.lib(), ctypes.c_int64()
    assert lib.poseidon_norm_workspace(0, cols, ctypes.byref(size)) == L.OK
    dgamma, dbeta = torch.full((2, cols), 3.0, device=dev())
    ws = torch.empty(max(size.value, 16), dtype=torch.uint8, device=dev())
    code = L.F32 if dtype == F32 else L.BF16
    for p in (0.0, 0.5, 1.0):
        assert lib.poseidon_norm_backward(None, None, None, None, None, None, 0, cols, code, p, None, None, None,
                                          dgamma.data_ptr(), dbeta.data_ptr(), ws.data_ptr(), size.value,
                                          torch.cuda.current_stream().cuda_stream) == L.OK
        assert (dgamma == 0).all() and (dbeta == 0).all()
        dgamma.fill_(3.0), dbeta.fill_(3.0)


@pytest.mark.parametrize("rows,cols", [(6, 2 ** 23 + 5), (5, 2 ** 27)])
def test_norm_backward_of_the_longest_rows(rows, cols):
    """More columns than one launch of the partial sums' workgroups covers (2^23),
    and as many as would ask for 2^32 threads: dgamma and dbeta are sums of a few
    products of bf16 values, each fp32."""
    from paper_1706_03292_amd import api
    log(f"norm_backward long {rows}x{cols}")
    g = torch.Generator(device=dev()).manual_seed(cols)
    dy = torch.randn(rows, cols, generator=g, device=dev(), dtype=BF16)
    h = torch.randn(rows, cols, generator=g, device=dev(), dtype=BF16)
    gamma = torch.ones(cols, device=dev())
    mean, rstd = torch.linspace(-0.1, 0.2, rows, device=dev()), torch.linspace(0.5, 1.5, rows, device=dev())
    _, _, dgamma, dbeta = api.norm_backward(dy, h, gamma, mean, rstd)
    for at in range(0, cols, 1 << 23):
        c = slice(at, at + (1 << 23))
        d = dy[:, c].double()
        n = (h[:, c].double() - mean.double()[:, None]) * rstd.double()[:, None]
        # rows sums, and two roundings of n in each
        over = (dgamma[c].double() - (d * n).sum(0)).abs() - (rows + 4) * O.U32 * (
            d.abs() * (h[:, c].double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]).sum(0)
        assert float(over.max()) <= 0, f"dgamma from {at}"
        over = (dbeta[c].double() - d.sum(0)).abs() - rows * O.U32 * d.abs().sum(0)
        assert float(over.max()) <= 0, f"dbeta from {at}"
