"""Group norm with an activation, channels last, and its backward pass, against a
64-bit reference."""
import pytest
import torch

import _group_norm_oracle as O
from _helpers import dev, log

F32, BF16 = torch.float32, torch.bfloat16
gpu = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
ACTS = pytest.mark.parametrize("act", [None, "relu", "silu"], ids=["none", "relu", "silu"])
EPS = 1e-5

# (N, L, C, groups): one value; channels that end inside a vector of eight; groups of
# 1, 3, 9 and 5 channels; one group; as many groups as channels; more channels than a
# workgroup holds (2048), and odd ones; few rows of many samples; many rows; a last
# chunk of one row.
SHAPES = [(1, 1, 1, 1), (2, 17, 1, 1), (2, 3, 7, 7), (3, 5, 36, 12), (2, 49, 64, 32), (1, 196, 512, 32),
          (2, 50, 45, 9), (1, 33, 288, 32), (3, 2, 2056, 8), (1, 7, 4100, 4), (2, 1, 300, 1), (300, 2, 16, 4),
          (2, 20001, 8, 2), (1, 4099, 24, 8), (5, 65, 768, 16), (1, 1025, 2048, 1), (2, 3136, 256, 32)]


def api():
    from paper_1706_03292_amd import api as a
    return a


def rounding(dtype):
    return O.U16 if dtype == BF16 else O.U32


def drawn(N, L, C, dtype, seed, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, L, C, generator=g) * (0.5 + torch.rand(C, generator=g)) + torch.randn(C, generator=g) + mean
    return (x.to(dtype), 1 + 0.2 * torch.randn(C, generator=g), 0.3 * torch.randn(C, generator=g),
            (0.01 * torch.randn(N, L, C, generator=g)).to(dtype))


def within(got, want, what):
    value, bound = want
    got = got.double().cpu()
    assert got.shape == value.shape, what
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - value).abs() / bound
    assert float(over.max()) <= 1.0, f"{what}: {float(over.max()):.2f} of its bound"


@gpu
@DTYPES
@ACTS
@pytest.mark.parametrize("N,L,C,groups", SHAPES)
def test_forward_and_backward(N, L, C, groups, act, dtype):
    log(f"group norm {N} {L} {C} {groups} {act} {dtype}")
    x, gamma, beta, dy = drawn(N, L, C, dtype, N + L + C)
    d = [t.to(dev()) for t in (x, gamma, beta, dy)]
    y, mean, rstd = api().group_norm_forward(d[0], d[1], d[2], groups, EPS, act=act)
    want = O.forward(x, gamma, beta, groups, EPS, act, rounding(dtype))
    for name, got in (("mean", mean), ("rstd", rstd), ("y", y)):
        within(got, want[name], name)
    dx, dgamma, dbeta = api().group_norm_backward(d[3], d[0], d[1], d[2], mean, rstd, act=act)
    want = O.backward(dy, x, gamma, beta, mean.cpu(), rstd.cpu(), act, rounding(dtype))
    for name, got in (("dx", dx), ("dgamma", dgamma), ("dbeta", dbeta)):
        within(got, want[name], name)


@pytest.mark.parametrize("act", [None, "relu", "silu"])
def test_the_gradient_formula_against_differences(act):
    """The 64-bit gradient is that of sum(dy * y) by central differences."""
    N, L, C, groups = 2, 6, 12, 4
    x, gamma, beta, dy = (t.double() for t in drawn(N, L, C, F32, 4))

    def y_of(x, gamma, beta):
        return (dy * O.forward(x, gamma, beta, groups, EPS, act, 0.0)["y"][0]).sum()

    f = O.forward(x, gamma, beta, groups, EPS, act, 0.0)
    want = O.backward(dy, x, gamma, beta, f["mean"][0], f["rstd"][0], act, 0.0)
    h = 1e-6
    for k, name in enumerate(("dx", "dgamma", "dbeta")):
        args = [x, gamma, beta]
        flat = args[k].reshape(-1)
        for i in range(0, flat.numel(), 5):
            pair = []
            for s in (h, -h):
                moved = flat.clone()
                moved[i] += s
                args[k] = moved.view(flat.shape if k else x.shape)
                pair.append(y_of(*args))
            # terms of size 0.05 in 64 bits over 2 h, and h^2 of the third derivative
            assert abs((pair[0] - pair[1]) / (2 * h) - want[name][0].reshape(-1)[i]) <= 1e-8


@gpu
@DTYPES
def test_a_mean_far_from_zero(dtype):
    """Spreads of a thousandth of the mean (of a tenth in bf16, whose own step is
    2^-8): the statistics keep their digits."""
    log(f"group norm far mean {dtype}")
    x, gamma, beta, dy = drawn(2, 3000, 64, F32, 1)
    x = (1000.0 + (x if dtype == F32 else 100 * x)).to(dtype)
    d = [t.to(dev()) for t in (x, gamma, beta)]
    want = O.forward(x, gamma, beta, 8, EPS, "relu", rounding(dtype))
    for got, name in zip(api().group_norm_forward(*d, 8, EPS, act="relu"), ("y", "mean", "rstd")):
        within(got, want[name], name)


@gpu
@DTYPES
def test_a_first_value_far_from_the_others(dtype):
    log(f"group norm outlier {dtype}")
    x, gamma, beta, dy = drawn(2, 3000, 64, dtype, 2)
    x[:, 0] = 3e4
    want = O.forward(x, gamma, beta, 8, EPS, None, rounding(dtype))
    for got, name in zip(api().group_norm_forward(*[t.to(dev()) for t in (x, gamma, beta)], 8, EPS),
                         ("y", "mean", "rstd")):
        within(got, want[name], name)


@gpu
def test_constant_values_and_no_eps():
    """No spread: y is beta, and without eps NaN, as the formula says."""
    log("group norm constant")
    x = torch.full((2, 50, 16), 3.0, device=dev())
    gamma, beta = torch.ones(16, device=dev()), torch.arange(16.0, device=dev())
    y, mean, rstd = api().group_norm_forward(x, gamma, beta, 4, EPS)
    assert (mean == 3).all() and torch.equal(y, beta.expand_as(y))
    assert ((rstd - EPS ** -0.5).abs() <= 2 * O.U32 * EPS ** -0.5).all()
    assert torch.isinf(api().group_norm_forward(x, gamma, beta, 4, 0.0)[2]).all()


@gpu
@ACTS
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_group(bad, act):
    log(f"group norm {bad} {act}")
    x, gamma, beta, dy = (t.to(dev()) for t in drawn(3, 300, 24, F32, 5))
    good = api().group_norm_forward(x, gamma, beta, 4, EPS, act=act)
    x[1, 77, 8] = bad
    y, mean, rstd = api().group_norm_forward(x, gamma, beta, 4, EPS, act=act)
    hit = torch.zeros(3, 4, dtype=torch.bool, device=dev())
    hit[1, 1] = True
    assert torch.equal(mean[~hit], good[1][~hit]) and not torch.isfinite(rstd[hit]).any()
    cells = hit[:, None, :, None].expand(3, 300, 4, 6).reshape(3, 300, 24)
    assert torch.equal(y[~cells], good[0][~cells]) and torch.isnan(y[cells]).all()
    dx, dgamma, dbeta = api().group_norm_backward(dy, x, gamma, beta, mean, rstd, act=act)
    assert torch.isfinite(dx[~cells]).all()


# Of maps that no workgroup holds: in two launches, three and four.
SPREAD = [(3, 5000, 72, 9), (3, 5000, 70, 1), (2, 9000, 520, 1)]


@gpu
@pytest.mark.parametrize("N,L,C,groups", SPREAD)
def test_far_means_and_bad_values_over_many_workgroups(N, L, C, groups):
    """Spreads of a thousandth of the mean, then a NaN in the last chunk of a sample."""
    log(f"group norm spread {N} {L} {C} {groups}")
    x, gamma, beta, dy = drawn(N, L, C, F32, 12)
    x = 1000.0 + x
    want = O.forward(x, gamma, beta, groups, EPS, "relu", rounding(F32))
    x, gamma, beta, dy = (t.to(dev()) for t in (x, gamma, beta, dy))
    good = api().group_norm_forward(x, gamma, beta, groups, EPS, act="relu")
    for got, name in zip(good, ("y", "mean", "rstd")):
        within(got, want[name], name)
    back = api().group_norm_backward(dy, x, gamma, beta, good[1], good[2], act="relu")
    x[1, L - 1, C - 1] = float("nan")
    y, mean, rstd = api().group_norm_forward(x, gamma, beta, groups, EPS, act="relu")
    hit = torch.zeros(N, groups, dtype=torch.bool, device=dev())
    hit[1, groups - 1] = True
    assert torch.equal(mean[~hit], good[1][~hit]) and torch.equal(rstd[~hit], good[2][~hit])
    assert torch.isnan(mean[hit]).all() and torch.isnan(rstd[hit]).all()
    cells = hit[:, None, :, None].expand(N, L, groups, C // groups).reshape(N, L, C)
    assert torch.equal(y[~cells], good[0][~cells]) and torch.isnan(y[cells]).all()
    dx, dgamma, dbeta = api().group_norm_backward(dy, x, gamma, beta, mean, rstd, act="relu")
    assert torch.equal(dx[~cells], back[0][~cells]) and torch.isnan(dx[cells]).all()
    free = C - C // groups      # channels of the groups before the last
    assert torch.equal(dgamma[:free], back[1][:free]) and torch.equal(dbeta[:free], back[2][:free])


@gpu
def test_relu_at_zero_passes_nothing():
    """gamma = 0 makes z = beta: the gradient passes where beta > 0 only."""
    log("group norm relu border")
    x, _, _, dy = (t.to(dev()) for t in drawn(2, 40, 16, F32, 6))
    gamma = torch.zeros(16, device=dev())
    beta = torch.tensor([0.0, -0.0, 1e-30, -1e-30] * 4, device=dev())
    _, mean, rstd = api().group_norm_forward(x, gamma, beta, 4, EPS, act="relu")
    dx, dgamma, dbeta = api().group_norm_backward(dy, x, gamma, beta, mean, rstd, act="relu")
    on = beta > 0
    assert (dx == 0).all() and (dgamma[~on] == 0).all() and (dbeta[~on] == 0).all() and (dbeta[on] != 0).all()


@gpu
def test_relu_border_in_64_bits():
    """beta puts z next to 0 (far below fp32's step of its terms): each value falls
    on the side that 64 bits say."""
    log("group norm relu border 64 bits")
    x, gamma, beta, dy = drawn(1, 64, 32, F32, 7)
    d = [t.to(dev()) for t in (x, gamma, beta, dy)]
    _, mean, rstd = api().group_norm_forward(*d[:3], 8, EPS)
    n = (x.double() - mean.cpu().double().repeat_interleave(4, 1)[:, None]) * rstd.cpu().double().repeat_interleave(4, 1)[:, None]
    for row in range(64):
        beta = (-n[0, row] * gamma.double()).float()     # z of this row: its own rounding alone
        z = n * gamma.double() + beta.double()
        got = api().group_norm_backward(d[3], d[0], d[1], beta.to(dev()), mean, rstd, act="relu")[2].cpu()
        want = torch.where(z > 0, dy.double(), 0.0).sum((0, 1))
        assert ((got.double() - want).abs() <= 70 * O.U32 * dy.double().abs().sum((0, 1))).all()


@gpu
@DTYPES
def test_odd_boundaries_and_given_outputs(dtype):
    """Arrays one value past a 16-byte boundary, gradients into a worker's shards,
    and nothing written beside the results."""
    log(f"group norm boundaries {dtype}")
    N, L, C, groups = 2, 37, 36, 6
    x, gamma, beta, dy = drawn(N, L, C, dtype, 8)

    def odd(t):
        base = torch.full((t.numel() + 9,), 5.0, dtype=t.dtype, device=dev())
        v = base[1:1 + t.numel()].view(t.shape)
        v.copy_(t)
        return base, v

    (_, xo), (_, go), (_, bo), (_, do) = (odd(t) for t in (x, gamma, beta, dy))
    base, y = odd(torch.zeros_like(x))
    got, mean, rstd = api().group_norm_forward(xo, go, bo, groups, EPS, act="silu", y=y)
    ref = api().group_norm_forward(x.to(dev()), gamma.to(dev()), beta.to(dev()), groups, EPS, act="silu")
    assert got is y and torch.equal(y, ref[0]) and torch.equal(mean, ref[1]) and torch.equal(rstd, ref[2])
    assert base[0] == 5 and (base[1 + x.numel():] == 5).all()
    shards = torch.full((3, 2 * C + 1), 5.0, device=dev())
    dg, db = shards[1, 1:1 + C], shards[1, 1 + C:]
    dx, a, b = api().group_norm_backward(do, xo, go, bo, mean, rstd, act="silu", dgamma=dg, dbeta=db)
    want = api().group_norm_backward(dy.to(dev()), x.to(dev()), gamma.to(dev()), beta.to(dev()), mean, rstd, act="silu")
    assert torch.equal(dx, want[0]) and torch.equal(dg, want[1]) and torch.equal(db, want[2])
    assert (shards[0] == 5).all() and (shards[2] == 5).all() and shards[1, 0] == 5


@gpu
def test_no_samples():
    log("group norm no samples")
    gamma = torch.ones(12, device=dev())
    x = torch.empty(0, 5, 5, 12, device=dev())
    y, mean, rstd = api().group_norm_forward(x, gamma, gamma, 3)
    assert y.shape == x.shape and mean.shape == (0, 3)
    dx, dgamma, dbeta = api().group_norm_backward(x, x, gamma, gamma, mean, rstd)
    assert dx.shape == x.shape and (dgamma == 0).all() and (dbeta == 0).all()


@gpu
def test_channels_last_tensors_of_torch():
    """An (N, C, H, W) tensor in torch's channels_last layout, by its view."""
    log("group norm channels_last")
    g = torch.Generator(device=dev()).manual_seed(1)
    t = torch.randn(3, 32, 9, 11, generator=g, device=dev()).to(memory_format=torch.channels_last)
    gamma, beta = torch.rand(32, device=dev()), torch.rand(32, device=dev())
    y = api().group_norm_forward(t.permute(0, 2, 3, 1), gamma, beta, 8)[0].permute(0, 3, 1, 2)
    v = t.double().reshape(3, 8, -1)
    n = ((v - v.mean(2, keepdim=True)) * (v.var(2, correction=0, keepdim=True) + EPS) ** -0.5).view(t.shape)
    want = n * gamma.double().view(1, -1, 1, 1) + beta.double().view(1, -1, 1, 1)
    assert float((y - want).abs().max()) < 2e-5    # 70 roundings of differences below 10, times rstd


@gpu
@DTYPES
@pytest.mark.parametrize("N,L,C,groups", [(4, 999, 72, 9)] + SPREAD)
def test_same_bits_on_another_stream_and_in_a_graph(N, L, C, groups, dtype):
    log(f"group norm streams {N} {L} {C} {groups} {dtype}")
    x, gamma, beta, dy = (t.to(dev()) for t in drawn(N, L, C, dtype, 9))

    def both(stream=None):
        y, mean, rstd = api().group_norm_forward(x, gamma, beta, groups, EPS, act="silu", stream=stream)
        return [y, mean, rstd, *api().group_norm_backward(dy, x, gamma, beta, mean, rstd, act="silu", stream=stream)]

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = both(side)
    torch.cuda.synchronize()
    for a, b in zip(first, other):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        x.mul_(1.5), dy.neg_()
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), f"replay {i}"


@gpu
def test_a_map_past_32_bits():
    """2^31 values and more: the groups of both samples' ends."""
    log("group norm 2^31 values")
    N, L, C, groups = 2, 2 ** 21 + 3, 516, 3
    g = torch.Generator(device=dev()).manual_seed(3)
    x = torch.empty(N, L, C, dtype=BF16, device=dev())
    for n in range(N):
        for r in range(0, L, 1 << 18):
            x[n, r:r + (1 << 18)] = torch.randn(min(L - r, 1 << 18), C, generator=g, device=dev(), dtype=BF16)
    gamma, beta = torch.rand(C, generator=g, device=dev()), torch.rand(C, generator=g, device=dev())
    y, mean, rstd = api().group_norm_forward(x, gamma, beta, groups, EPS, act="relu")
    dx, dgamma, dbeta = api().group_norm_backward(x, x, gamma, beta, mean, rstd, act="relu")
    D = C // groups
    s1, s2 = (torch.zeros(C, dtype=torch.float64, device=dev()) for _ in range(2))
    avg = torch.zeros(N, groups, 3, dtype=torch.float64, device=dev())
    for n in range(N):
        for r in range(0, L, 1 << 18):
            v = x[n, r:r + (1 << 18)].double()
            mu, rs = (t[n].double().repeat_interleave(D) for t in (mean, rstd))
            k = (v - mu) * rs
            dz = torch.where(k * gamma.double() + beta.double() > 0, v, 0.0)
            s1 += (dz * k).sum(0)
            s2 += dz.sum(0)
            for q, t in enumerate((v, (dz * gamma), (dz * gamma * k))):
                avg[n, :, q] += t.view(-1, groups, D).sum((0, 2)) / (L * D)
    assert float((mean - avg[:, :, 0]).abs().max()) < 70 * O.U32 * 10
    # at most 300 roundings of each term of about 1; the sums have 4e6 of them
    assert float((dgamma - s1).abs().max()) <= 300 * O.U32 * 2 * N * L
    assert float((dbeta - s2).abs().max()) <= 300 * O.U32 * 2 * N * L
    for n in range(N):
        for rows in (slice(0, 100), slice(L - 100, L)):
            v = x[n, rows].double()
            mu, rs = (t[n].double().repeat_interleave(D) for t in (mean, rstd))
            k = (v - mu) * rs
            z = k * gamma.double() + beta.double()
            a1, a2 = (avg[n, :, q].repeat_interleave(D) for q in (1, 2))
            want = rs * (torch.where(z > 0, v, 0.0) * gamma.double() - a1 - k * a2)
            # 2^-8 of the result's rounding, and 300 roundings of averages below 1
            assert ((dx[n, rows] - want).abs() <= O.U16 * want.abs() + 1e-4).all()
            assert ((y[n, rows] - z.clamp(min=0)).abs() <= O.U16 * z.abs() + 1e-5).all()


def launched(call):
    """The group norm kernels that `call` launches: names, with the threads and rows
    of those that hold a map."""
    import re

    from _helpers import whole_kernel_names
    out = []
    for name in whole_kernel_names(call):
        m = re.search(r"(held_\w+?_kernel)<[^>]*?, (\d+), (\d+)>", name)
        if m:
            out.append((m[1], int(m[2]), int(m[3])))
        else:
            m = re.search(r"(chunk_stats|chunk_sums|join_chunks|join_channels|group_stats|join_sums|average|forward|backward|weights)_kernel", name)
            if m:
                out.append(m[1])
    return out


# (sizes, workgroup that holds them): one for each shape, none, none with groups too
# wide for one workgroup's sums, and none with few enough chunks for two launches.
FORWARD_BF16 = [((1, 49, 512, 32), (256, 2)), ((1, 400, 512, 32), (256, 4)), ((1, 900, 512, 32), (256, 8)),
                ((1, 1800, 512, 32), (512, 8)), ((4, 3500, 512, 32), (512, 16)), ((4, 8000, 512, 32), (512, 32)),
                ((1, 2000, 288, 32), "late"), ((1, 8000, 512, 32), "wide"), ((1, 3000, 100, 1), None), ((64, 1, 4096, 32), (256, 2)),
                ((2, 4000, 1029, 3), "wide"), ((1, 9000, 520, 1), "wide"), ((1, 9000, 64, 32), "late"),
                ((3, 1300, 1800, 8), "late"), ((17, 500, 249, 249), "late"), ((1, 2500, 57, 57), "late")]
FORWARD_F32 = [((1, 49, 512, 32), (256, 2)), ((1, 400, 512, 32), (256, 4)), ((1, 900, 512, 32), (256, 8)),
               ((2, 1800, 512, 32), (512, 8)), ((4, 3500, 512, 32), (512, 16)), ((5, 3500, 520, 65), None),
               ((17, 700, 288, 32), "late"), ((3, 4000, 8, 8), "late")]
BACKWARD_BF16 = [((1, 49, 512, 32), (256, 2)), ((1, 400, 512, 32), (256, 4)), ((1, 900, 512, 32), (256, 8)),
                 ((2, 1800, 512, 32), (512, 8)), ((4, 3500, 512, 32), (512, 16)), ((1, 3500, 512, 32), None),
                 ((3, 33, 57, 19), (256, 2)), ((2, 4000, 1029, 3), "wide"), ((1, 9000, 130, 2), "wide"),
                 ((1, 9000, 128, 2), None), ((24, 6000, 57, 19), None), ((3, 1300, 1800, 8), "late"), ((17, 500, 249, 249), "late"),
                 ((1, 2500, 57, 57), "late")]
BACKWARD_F32 = [((1, 49, 512, 32), (256, 2)), ((1, 400, 512, 32), (256, 4)), ((2, 900, 512, 32), (256, 8)),
                ((4, 1800, 512, 32), (512, 8)), ((1, 1800, 512, 32), "late"), ((1, 3500, 512, 32), None),
                ((17, 700, 288, 32), "late"), ((3, 4000, 8, 8), "late")]


@gpu
@pytest.mark.parametrize("op,dtype,sizes,held", [(op, dt, s, h) for op, dt, rows in (
    ("forward", BF16, FORWARD_BF16), ("forward", F32, FORWARD_F32), ("backward", BF16, BACKWARD_BF16),
    ("backward", F32, BACKWARD_F32)) for s, h in rows])
def test_each_workgroup(op, dtype, sizes, held):
    """Every shape of workgroup that holds a map, and what is left to two, three and four
    launches: that these sizes take it, and their results."""
    N, L, C, groups = sizes
    log(f"group norm workgroup {op} {dtype} {sizes}")
    x, gamma, beta, dy = drawn(N, L, C, dtype, 11)
    d = [t.to(dev()) for t in (x, gamma, beta, dy)]
    y, mean, rstd = api().group_norm_forward(d[0], d[1], d[2], groups, EPS, act="relu")
    if op == "forward":
        names = launched(lambda: api().group_norm_forward(d[0], d[1], d[2], groups, EPS, act="relu"))
        want = {None: ["chunk_stats", "group_stats", "forward"], "late": ["chunk_stats", "forward"],
                "wide": ["chunk_stats", "join_chunks", "group_stats", "forward"]}.get(held) or [("held_forward_kernel", *held)]
        checked, results = O.forward(x, gamma, beta, groups, EPS, "relu", rounding(dtype)), {"y": y, "mean": mean, "rstd": rstd}
    else:
        call = lambda: api().group_norm_backward(d[3], d[0], d[1], d[2], mean, rstd, act="relu")  # noqa: E731
        names = launched(call)
        want = {None: ["chunk_sums", "join_sums", "backward"], "late": ["chunk_sums", "backward"],
                "wide": ["chunk_sums", "join_channels", "average", "backward"]}.get(held) or \
            [("held_backward_kernel", *held)] + ["weights"] * (N > 1)
        checked = O.backward(dy, x, gamma, beta, mean.cpu(), rstd.cpu(), "relu", rounding(dtype))
        results = dict(zip(("dx", "dgamma", "dbeta"), call()))
    assert names == want
    for name, got in results.items():
        within(got, checked[name], name)
