"""AdamW over many tensors with fp32 and 8-bit moments, the moments' values and
the gradients' norm, against a 64-bit reference."""
import numpy as np
import pytest
import torch

import _adamw_oracle as O
from _helpers import dev, log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DTYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
BITS = pytest.mark.parametrize("bits", [32, 8])
# Nothing, one value, ends of a group, of a block and of a workgroup's 2048.
SIZES = [1, 7, 0, 8, 9, 127, 128, 129, 255, 2047, 2048, 2049, 5003]
SEED, OFFSET = 0x123456789ABCDEF, -3
TINY = 1e-44   # a denormal fp32's step


def api():
    from paper_1706_03292_amd import api as a
    return a


def np64(t):
    return t.detach().cpu().double().numpy()


class Net:
    """Tensors in flat buffers with a gap of `odd` values before each and a value
    to watch after it; the oracle's copy beside them."""

    def __init__(self, sizes, P, dtype, bits, odd=0, seed=0, copy=True, sums=False, spread=1.0, decay=0.1):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.P, self.dtype, self.bits = sizes, P, dtype, bits
        self.places, at = [], 0
        for n in sizes:
            at += odd
            self.places.append(at)
            at += n + 1
        total = max(at, 1)
        sigma = 1e-3 * (spread * torch.randn(total, generator=g)).exp()
        self.G = (sigma * torch.randn(P, total, generator=g)).to(dtype).to(dev())
        self.W = (0.05 * torch.randn(total, generator=g)).to(dev())
        m, v = 0.3 * sigma * torch.randn(total, generator=g), sigma.square() * (0.5 + torch.rand(total, generator=g))
        self.decays = [decay * (i % 2) for i in range(len(sizes))]
        self.copy = torch.full((total,), 7.0, dtype=BF16, device=dev()) if copy else None
        self.sum = torch.full((total,), 7.0, device=dev()) if sums else None
        if bits == 32:
            self.m, self.v, self.x = m.to(dev()), v.to(dev()), None
        else:
            self.m = torch.full((total,), 77, dtype=torch.uint8, device=dev())
            self.v = torch.full((total,), 77, dtype=torch.uint8, device=dev())
            self.xat, x = [], 0
            for n in sizes:
                self.xat.append(x)
                x += 2 * -(-n // O.BLOCK) + 1
            self.x = torch.full((max(x, 1),), 77, dtype=torch.uint8, device=dev())
            for i, n in enumerate(sizes):
                for k, (arr, src, signed) in enumerate(((self.m, m, True), (self.v, v, False))):
                    at = self.places[i]
                    c, e = O.encode(np64(src[at:at + n]), np.full(n, 32768), signed)
                    arr[at:at + n] = torch.from_numpy(c).to(dev())
                    self.x[self.xat[i] + k:self.xat[i] + k + 2 * len(e):2] = torch.from_numpy(e).to(dev())

    def slot(self, arr, i):
        return arr[self.places[i]:self.places[i] + self.sizes[i]]

    def exps(self, i):
        return self.x[self.xat[i]:self.xat[i] + 2 * -(-self.sizes[i] // O.BLOCK)]

    def tensors(self):
        out = []
        for i, n in enumerate(self.sizes):
            t = {"W": self.slot(self.W, i), "shards": self.G[:, self.places[i]:self.places[i] + n],
                 "m": self.slot(self.m, i), "v": self.slot(self.v, i), "weight_decay": self.decays[i]}
            if self.copy is not None:
                t["copy"] = self.slot(self.copy, i)
            if self.sum is not None:
                t["sum"] = self.slot(self.sum, i)
            if self.bits == 8:
                t["exponents"] = self.exps(i)
            out.append(t)
        return out

    def arrays(self):
        return [a for a in (self.W, self.m, self.v, self.x, self.copy, self.sum) if a is not None]

    def moments(self, i):
        if self.bits == 32:
            return np64(self.slot(self.m, i)), np64(self.slot(self.v, i))
        e = self.exps(i).cpu().numpy()
        return (O.decode(self.slot(self.m, i).cpu().numpy(), e[0::2], True),
                O.decode(self.slot(self.v, i).cpu().numpy(), e[1::2], False))

    def first_groups(self):
        at, out = 0, []
        for n in self.sizes:
            out.append(at)
            at += -(-n // O.BLOCK) * 16
        return out

    def expected(self, rng=None, rows=None, **kw):
        """What each tensor's arrays hold after a step."""
        out = []
        for i, n in enumerate(self.sizes):
            m0, v0 = self.moments(i)
            r = np64(self.G[:, self.places[i]:self.places[i] + n]) if rows is None else rows[i]
            decay = float(np.float32(self.decays[i]))
            w, m, v, dw, dm, dv = O.adamw(np64(self.slot(self.W, i)), r, m0, v0, decay=decay, **kw)
            if self.bits == 8:
                b = O.bits16(*rng, self.first_groups()[i], n) if rng else np.full(n, 32768)
                (cm, em), (cv, ev) = O.encode(m, b, True), O.encode(v, O.exchanged(b) if rng else b, False)
                out.append((w, dw, cm, em, cv, ev))
            else:
                out.append((w, dw, m, dm, v, dv))
        return out

    def check(self, want):
        for i, n in enumerate(self.sizes):
            if n == 0:
                continue
            w, dw = want[i][:2]
            got = np64(self.slot(self.W, i))
            assert np.all(np.abs(got - w) <= dw + TINY), f"tensor {i}: W {np.max(np.abs(got - w) / (dw + TINY))}"
            if self.copy is not None:
                assert torch.equal(self.slot(self.copy, i), self.slot(self.W, i).to(BF16)), f"tensor {i}: copy"
            if self.bits == 32:
                _, _, m, dm, v, dv = want[i]
                for name, a, x, d in (("m", self.m, m, dm), ("v", self.v, v, dv)):
                    over = np.abs(np64(self.slot(a, i)) - x) - d - TINY
                    assert np.all(over <= 0), f"tensor {i}: {name}"
            else:
                _, _, cm, em, cv, ev = want[i]
                e = self.exps(i).cpu().numpy()
                assert np.array_equal(e[0::2], em) and np.array_equal(e[1::2], ev), f"tensor {i}: exponents"
                assert np.array_equal(self.slot(self.m, i).cpu().numpy(), cm), f"tensor {i}: m's codes"
                assert np.array_equal(self.slot(self.v, i).cpu().numpy(), cv), f"tensor {i}: v's codes"

    def between(self):
        """The values that belong to no tensor."""
        out = []
        for a in self.arrays():
            keep = torch.ones(a.numel(), dtype=torch.bool)
            for i, n in enumerate(self.sizes):
                at, length = ((self.xat[i], 2 * -(-n // O.BLOCK)) if a is self.x else (self.places[i], n))
                keep[at:at + length] = False
            out.append(a.cpu()[keep].clone())
        return out


def state(offset=OFFSET):
    return torch.tensor([SEED, offset], dtype=torch.int64, device=dev())


KW = {"betas": (0.9, 0.999), "eps": 1e-8}


@DTYPES
@BITS
@pytest.mark.parametrize("P", [1, 2, 3, 5, 8, 10])
@pytest.mark.parametrize("odd", [0, 1, 5])
def test_step(P, odd, bits, dtype):
    """Two steps of tensors of every end, on boundaries of 1 and 5 values too,
    with all of what lies between them left as it was."""
    log(f"adamw step P={P} odd={odd} bits={bits} {dtype}")
    net = Net(SIZES, P, dtype, bits, odd, seed=P + 10 * odd)
    opt = api().AdamW(net.tensors(), **KW)
    between = net.between()
    for step in (1, 2):
        rng = (SEED, OFFSET + step) if step == 2 else None
        want = net.expected(rng, lr=0.01, step=step, **KW)
        opt.step(0.01, step, rng=state(OFFSET + step) if rng else None)
        net.check(want)
    for a, b in zip(between, net.between()):
        assert torch.equal(a, b)


@BITS
def test_more_tensors_than_a_launch_holds(bits):
    log(f"adamw many tensors bits={bits}")
    net = Net([1 + (37 * i) % 300 for i in range(131)], 2, F32, bits, seed=3, copy=False)
    opt = api().AdamW(net.tensors(), **KW)
    want = net.expected((SEED, OFFSET), lr=0.01, step=7, **KW)
    opt.step(0.01, 7, rng=state())
    net.check(want)


def test_both_kinds_of_moments_in_one_optimizer():
    """The random numbers count fp32 tensors too."""
    log("adamw mixed")
    a, b = Net([300, 129], 2, F32, 32, seed=1), Net([200, 1000], 2, F32, 8, seed=2)
    ta, tb = a.tensors(), b.tensors()
    opt = api().AdamW([ta[0], tb[0], ta[1], tb[1]], **KW)
    wa = a.expected(lr=0.01, step=3, **KW)
    groups = [3 * 16, 3 * 16 + 2 * 16 + 2 * 16]
    b.first_groups = lambda: groups
    wb = b.expected((SEED, OFFSET), lr=0.01, step=3, **KW)
    opt.step(0.01, 3, rng=state())
    a.check(wa), b.check(wb)


@BITS
@pytest.mark.parametrize("betas,eps,step", [((0.0, 0.0), 1e-3, 1), ((0.95, 0.98), 1e-6, 50), ((0.9, 0.9999), 1e-15, 10 ** 7)])
def test_rules(betas, eps, step, bits):
    """Other rules, by value and from the device's clock, with a scale."""
    log(f"adamw rules {betas} {eps} {step} bits={bits}")
    kw = {"betas": betas, "eps": eps}
    clock = torch.tensor([0.003, step], dtype=torch.float64, device=dev())
    for use in (None, clock):
        net = Net([500, 1029], 3, F32, bits, seed=step)
        opt = api().AdamW(net.tensors(), **kw)
        scale = torch.tensor([0.3], device=dev())
        want = net.expected((SEED, OFFSET), lr=0.003, step=step, scale=float(scale), **kw)
        opt.step(0.003, step, clock=use, scale=scale, rng=state())
        net.check(want)


@BITS
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_step_is_left_out_for_a_scale_that_is_not_finite(value, bits):
    log(f"adamw skip {value} bits={bits}")
    net = Net(SIZES, 2, F32, bits)
    before = [a.clone() for a in net.arrays()]
    api().AdamW(net.tensors(), **KW).step(0.01, 5, scale=torch.tensor([value], device=dev()), rng=state())
    for a, b in zip(net.arrays(), before):
        assert torch.equal(a, b)


@BITS
def test_zero_gradients_and_moments(bits):
    """Nothing but the decay moves the weights; moments stay 0."""
    log(f"adamw zeros bits={bits}")
    W = torch.randn(1000, device=dev())
    old = W.clone()
    t = {"W": W, "shards": torch.zeros(2, 1000, device=dev()), "weight_decay": 0.5, **api().AdamW.moments(W, bits)}
    opt = api().AdamW([t])
    opt.step(0.1, 1)
    # the factor lr * decay and the product, then the difference: one rounding each
    want = old.double() * (1 - 0.1 * 0.5)
    assert ((W.double() - want).abs() <= 3 * O.U32 * old.double().abs()).all()
    m, v = opt.values()[0]
    assert (m == 0).all() and (v == 0).all()


def test_codes_over_the_whole_range():
    """Magnitudes from denormals to 2^60 in one block, and blocks of few: every
    code, each border and both signs."""
    log("adamw codes range")
    n = 128 * 70
    g = torch.Generator().manual_seed(5)
    grads = torch.randn(1, n, generator=g) * torch.exp2(torch.randint(-70, 60, (n,), generator=g).float())
    grads[:, 128:256] = torch.randn(1, 128, generator=g) * 1e-30     # v far below 2^-126
    grads[:, 256:384] = torch.randn(1, 128, generator=g) * 1e-40     # denormal gradients
    grads[:, 384:512] = 0.0
    grads[:, 512:5120] *= 0.0
    grads[:, 512:5120] += torch.randn(4608, generator=g) * torch.exp2(torch.rand(4608, generator=g) * 30 - 40)
    W = torch.zeros(n, device=dev())
    t = {"W": W, "shards": grads.to(dev()), **api().AdamW.moments(W, 8)}
    opt = api().AdamW([t], betas=(0.5, 0.75))
    m, v = np.zeros(n), np.zeros(n)
    for step in range(1, 5):
        _, m, v, *_ = O.adamw(np.zeros(n), np64(grads), m, v, lr=0.0, step=step, betas=(0.5, 0.75), eps=1e-8, decay=0)
        bits = O.bits16(SEED, step, 0, n)
        (cm, em), (cv, ev) = O.encode(m, bits, True), O.encode(v, O.exchanged(bits), False)
        opt.step(0.0, step, rng=state(step))
        e = t["exponents"].cpu().numpy()
        assert np.array_equal(e[0::2], em) and np.array_equal(e[1::2], ev)
        assert np.array_equal(t["m"].cpu().numpy(), cm) and np.array_equal(t["v"].cpu().numpy(), cv)
        m, v = O.decode(cm, em, True), O.decode(cv, ev, False)
        gm, gv = opt.values()[0]
        assert np.array_equal(np64(gm), m) and np.array_equal(np64(gv), v)
        assert ((v > 0) == (cv > 0)).all()
    assert (W == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_gradients_that_are_not_finite(bad):
    """fp32 moments: the value itself.  8 bits: its block reads as NaN, the others
    are as without it."""
    log(f"adamw not finite {bad}")
    for bits in (32, 8):
        nets = [Net([600], 1, F32, bits, seed=9) for _ in range(2)]
        nets[1].G[0, nets[1].places[0] + 300] = bad
        values = []
        for net in nets:
            opt = api().AdamW(net.tensors(), **KW)
            opt.step(0.01, 2)
            values.append(opt.values()[0])
        touched = torch.zeros(600, dtype=torch.bool)
        touched[300 if bits == 32 else slice(256, 384)] = True
        for a, b in zip(*values):
            assert torch.equal(a.cpu()[~touched], b.cpu()[~touched])
            assert not torch.isfinite(b.cpu()[touched]).any()
            if bits == 8:
                assert torch.isnan(b.cpu()[touched]).all()
        others = torch.arange(600) != 300
        assert torch.equal(nets[0].slot(nets[0].W, 0).cpu()[others], nets[1].slot(nets[1].W, 0).cpu()[others])


def test_eight_bit_variance_follows_its_gradients():
    """A hundred steps at gradients far below those that v came from: rounded at
    random, v falls as 0.999^t on average (rounded to nearest it would not move).
    A step's rounding has a variance of at most f (1 - f) of a code's distance
    squared, f the way to the next code: v's 0.1 % of codes 6 to 12 % apart, so the
    mean over 65536 values of a hundred steps is off by less than 0.1 %
    (sqrt(100 * 0.017) * 0.125 / 256 = 0.06 %)."""
    log("adamw 8-bit variance")
    n = 65536
    W = torch.zeros(n, device=dev())
    t = {"W": W, "shards": torch.full((1, n), 1.0, device=dev()), **api().AdamW.moments(W, 8)}
    opt = api().AdamW([t])
    opt.step(0.0, 1, rng=state(0))
    t["shards"].fill_(0.01)
    start = opt.values()[0][1].double().mean()
    for i in range(100):
        opt.step(0.0, 2 + i, rng=state(1 + i))
    f = 0.999 ** 100
    want = float(start) * f + (1 - f) * 1e-4
    assert abs(float(opt.values()[0][1].double().mean()) / want - 1) < 2e-3


@DTYPES
@pytest.mark.parametrize("P", [1, 4, 7])
@pytest.mark.parametrize("sums", [False, True], ids=["", "sums"])
def test_clip(sums, P, dtype):
    log(f"adamw clip P={P} sums={sums} {dtype}")
    net = Net(SIZES + [70001] + 90 * [33], P, dtype, 32, odd=1, seed=P, sums=sums)
    opt = api().AdamW(net.tensors(), **KW)
    between = net.between()
    rows = [np64(net.G[:, at:at + n]) for at, n in zip(net.places, net.sizes)]
    square = sum(float((r.sum(0) ** 2).sum()) for r in rows)
    for most in (1e-3, 1e9, float("inf")):
        r = opt.clip(most).cpu().double()
        norm = square ** 0.5
        # sums in 64 bits, one rounding to fp32
        assert abs(float(r[0]) - norm) <= 1.01 * O.U32 * norm
        assert abs(float(r[1]) - min(1.0, most / norm)) <= 1.01 * O.U32
    if sums:
        for i, n in enumerate(net.sizes):
            s = rows[i].sum(0)
            assert np.all(np.abs(np64(net.slot(net.sum, i)) - s) <= 1.01 * O.U32 * np.abs(s) + TINY)
    for a, b in zip(between, net.between()):
        assert torch.equal(a, b)


def test_clip_of_nothing_and_of_what_is_not_finite():
    log("adamw clip ends")
    a = api()
    empty = a.AdamW([])
    assert empty.clip(1.0).tolist() == [0.0, 1.0]
    empty.step(0.1, 1)
    assert empty.values() == []
    W = torch.zeros(3000, device=dev())
    t = {"W": W, "shards": torch.zeros(1, 3000, device=dev()), **a.AdamW.moments(W)}
    opt = a.AdamW([t])
    assert opt.clip(1.0).tolist() == [0.0, 1.0]
    t["shards"][0, 2999] = 3e38      # its square passes fp32's range
    r = opt.clip(1.0)
    assert abs(float(r[0]) / 3e38 - 1) < 1e-6 and abs(float(r[1]) * 3e38 - 1) < 1e-5
    for bad in (float("inf"), float("nan")):
        t["shards"][0, 5] = bad
        r = opt.clip(1.0)
        assert not torch.isfinite(r[0]) and torch.isnan(r[1])
        opt.step(0.1, 1, scale=r[1:2])
        assert (W == 0).all() and (t["v"] == 0).all()


@DTYPES
@BITS
def test_step_from_sums(bits, dtype):
    log(f"adamw from sums bits={bits} {dtype}")
    net = Net(SIZES, 5, dtype, bits, odd=1, seed=4, sums=True)
    opt = api().AdamW(net.tensors(), **KW)
    r = opt.clip(0.01)
    rows = [np64(net.slot(net.sum, i))[None] for i in range(len(net.sizes))]
    want = net.expected((SEED, OFFSET), rows=rows, lr=0.01, step=9, scale=float(r[1]), **KW)
    opt.step(0.01, 9, scale=r[1:2], rng=state(), from_sums=True)
    net.check(want)


def test_same_bits_every_time_and_on_another_stream():
    log("adamw deterministic")
    nets = [Net(SIZES + [40001], 3, BF16, bits, seed=6, sums=True) for bits in (32, 8, 32, 8)]
    side = torch.cuda.Stream()
    for k, net in enumerate(nets):
        opt = api().AdamW(net.tensors(), **KW)
        s = side if k >= 2 else None
        if s is not None:
            side.wait_stream(torch.cuda.current_stream())
        r = opt.clip(0.02, stream=s)
        opt.step(0.01, 3, scale=r[1:2], rng=state(), stream=s)
        opt.values(stream=s)
        net.r = r
    torch.cuda.synchronize()
    for a, b in ((0, 2), (1, 3)):
        assert torch.equal(nets[a].r, nets[b].r)
        for x, y in zip(nets[a].arrays(), nets[b].arrays()):
            assert torch.equal(x, y)


@BITS
def test_replayed_from_a_graph(bits):
    """Clip and step in one graph, clock and random numbers on the device: every
    replay is the eager step, with eager work of another optimizer in between."""
    log(f"adamw graph bits={bits}")
    a = api()
    nets = [Net(SIZES + [30011], 3, BF16, bits, seed=8, sums=True) for _ in range(2)]
    opts = [a.AdamW(n.tensors(), **KW) for n in nets]
    clocks = [torch.tensor([0.01, 1.0], dtype=torch.float64, device=dev()) for _ in range(2)]
    rngs = [state(1) for _ in range(2)]

    def one(k):
        r = opts[k].clip(0.02)
        opts[k].step(clock=clocks[k], scale=r[1:2], rng=rngs[k], from_sums=True)
        clocks[k][1:] += 1
        rngs[k][1:] += 1

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    before = [x.clone() for x in nets[0].arrays() + [clocks[0], rngs[0]]]
    with torch.cuda.stream(side):
        one(0)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        one(0)
    for x, y in zip(nets[0].arrays() + [clocks[0], rngs[0]], before):
        x.copy_(y)
    for i in range(4):
        for n in nets:
            n.G.mul_(-1.25)
        graph.replay()
        one(1)
        torch.cuda.synchronize()
        for x, y in zip(nets[0].arrays(), nets[1].arrays()):
            assert torch.equal(x, y), f"replay {i}"


def test_workers_rows_far_apart():
    """Two workers' gradients more than 2^32 values apart."""
    log("adamw far rows")
    n, far = 3001, 2 ** 32 + 2 ** 20
    flat = torch.empty(far + n, dtype=BF16, device=dev())
    G = flat.as_strided((2, n), (far, 1))
    g = torch.Generator(device=dev()).manual_seed(1)
    G.copy_(torch.randn(2, n, generator=g, device=dev()))
    W = torch.randn(n, generator=g, device=dev())
    t = {"W": W, "shards": G, "sum": torch.empty(n, device=dev()), **api().AdamW.moments(W)}
    w, m, v, dw, dm, dv = O.adamw(np64(W), np64(G), np.zeros(n), np.zeros(n), lr=0.01, step=1, decay=0, **KW)
    opt = api().AdamW([t], **KW)
    r = opt.clip(1.0)
    assert abs(float(r[0]) / np.linalg.norm(np64(G).sum(0)) - 1) <= 1.01 * O.U32
    opt.step(0.01, 1)
    assert np.all(np.abs(np64(W) - w) <= dw) and np.all(np.abs(np64(t["m"]) - m) <= dm)


def test_a_tensor_past_32_bits():
    """2^31 + 1000 values in 8 bits: the last ones, checked alone, and the first."""
    log("adamw 2^31 values")
    n = 2 ** 31 + 1000
    W = torch.zeros(n, device=dev())
    t = {"W": W, "shards": torch.zeros(1, n, dtype=BF16, device=dev()), **api().AdamW.moments(W, 8)}
    places = [slice(0, 128), slice(2 ** 31 - 128, 2 ** 31 + 256), slice(n - n % 128, n)]
    g = torch.Generator(device=dev()).manual_seed(2)
    for p in places:
        t["shards"][0, p] = torch.randn(p.stop - p.start, generator=g, device=dev()).to(BF16)
    opt = api().AdamW([t], **KW)
    r = opt.clip(1.0)
    grads = [np64(t["shards"][:, p]) for p in places]
    assert abs(float(r[0]) / sum(float((x ** 2).sum()) for x in grads) ** 0.5 - 1) <= 1.01 * O.U32
    opt.step(0.01, 1, rng=state())
    for p, x in zip(places, grads):
        k = p.stop - p.start
        w, m, v, dw, _, _ = O.adamw(np.zeros(k), x, np.zeros(k), np.zeros(k), lr=0.01, step=1, decay=0, **KW)
        bits = O.bits16(SEED, OFFSET, p.start // 8, k)
        (cm, em), (cv, ev) = O.encode(m, bits, True), O.encode(v, O.exchanged(bits), False)
        assert np.array_equal(t["m"][p].cpu().numpy(), cm) and np.array_equal(t["v"][p].cpu().numpy(), cv)
        assert np.all(np.abs(np64(W[p]) - w) <= dw)
    for p in (slice(128, 2 ** 20), slice(2 ** 31 + 256, 2 ** 31 + 512)):
        assert (W[p] == 0).all() and (t["m"][p] == 0).all()
