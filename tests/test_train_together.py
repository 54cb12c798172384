"""Group norm, the classifier's loss, clipping and AdamW as a training program runs
them, by P workers on one GPU, against 64 bits; and the network's end trained by
AdamW."""
import numpy as np
import pytest
import torch

import _adamw_oracle as A
import _group_norm_oracle as G
import _net_oracle as O
from _helpers import dev, log

pytestmark = pytest.mark.gpu

KW = {"betas": (0.9, 0.999), "eps": 1e-8}
SEED = 77


def np64(t):
    return t.detach().cpu().double().numpy()


class Run:
    """One block of a convolution network's end: feature maps of P workers through
    group norm and SiLU, averaged over their positions, into a classifier."""

    N, H, C, groups, classes, P = 4, 5, 24, 6, 40, 3

    def __init__(self, bits):
        from paper_1706_03292_amd import api
        self.api, self.bits = api, bits
        g = torch.Generator().manual_seed(1)
        self.host = {"gamma": 1 + 0.1 * torch.randn(self.C, generator=g), "beta": 0.1 * torch.randn(self.C, generator=g),
                     "W": 0.3 * torch.randn(self.classes, self.C, generator=g)}
        self.p = {k: v.to(dev()) for k, v in self.host.items()}
        self.shards = {k: torch.zeros(self.P, *v.shape, device=dev()) for k, v in self.p.items()}
        self.x = torch.randn(self.P, self.N, self.H, self.H, self.C, generator=g)
        self.target = torch.randint(0, self.classes, (self.P, self.N), generator=g)
        self.dloss = torch.full((self.N,), 1.0 / (self.N * self.P), device=dev())
        self.tensors = {k: {"W": v, "shards": self.shards[k], "weight_decay": 0.1 * (k == "W"),
                            "sum": torch.zeros_like(v), **api.AdamW.moments(v, bits if k == "W" else 32)}
                        for k, v in self.p.items()}
        self.opt = api.AdamW(list(self.tensors.values()), **KW)
        self.clock = torch.tensor([0.02, 1.0], dtype=torch.float64, device=dev())
        self.rng = torch.tensor([SEED, 0], dtype=torch.int64, device=dev())
        self.device_x, self.device_target = self.x.to(dev()), self.target.to(dev())

    def step(self):
        api, p, positions = self.api, self.p, self.H * self.H
        losses = []
        for w in range(self.P):
            x = self.device_x[w]
            y, mean, rstd = api.group_norm_forward(x, p["gamma"], p["beta"], self.groups, act="silu")
            pooled = y.mean((1, 2))
            loss, lse = api.xent_forward(pooled, p["W"], self.device_target[w])
            d, _ = api.xent_backward(pooled, p["W"], self.device_target[w], lse, self.dloss, dW=self.shards["W"][w])
            dy = (d / positions)[:, None, None, :].expand_as(x).contiguous()
            api.group_norm_backward(dy, x, p["gamma"], p["beta"], mean, rstd, act="silu",
                                    dgamma=self.shards["gamma"][w], dbeta=self.shards["beta"][w])
            losses.append(loss)
        norm = self.opt.clip(0.05)
        self.opt.step(clock=self.clock, scale=norm[1:2], rng=self.rng, from_sums=True)
        self.clock[1:] += 1
        self.rng[1:] += 1
        return torch.cat(losses), norm

    def state(self):
        return [t[k] for t in self.tensors.values() for k in ("W", "m", "v", "exponents", "sum") if k in t] + [
            self.clock, self.rng]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_against_64_bits(bits):
    """The gradients of the whole chain, within a few hundred fp32 roundings of the
    largest; then AdamW from the gradients as they are."""
    log(f"train together bits={bits}")
    run = Run(bits)
    loss, norm = run.step()
    gamma, beta, W = (run.host[k].double() for k in ("gamma", "beta", "W"))
    want = {k: np.zeros(v.shape) for k, v in run.host.items()}
    for w in range(run.P):
        f = G.forward(run.x[w], gamma, beta, run.groups, 1e-5, "silu", 0.0)
        pooled = f["y"][0].mean((1, 2))
        rows, _, _, d, dW = O.xent(pooled, W, run.target[w], run.dloss.cpu().double())
        assert float((loss.view(run.P, -1)[w].cpu().double() - rows).abs().max()) < 1e-5
        dy = (d / run.H ** 2)[:, None, None, :].expand(run.x[w].shape)
        b = G.backward(dy, run.x[w], gamma, beta, f["mean"][0], f["rstd"][0], "silu", 0.0)
        for k, v in (("gamma", b["dgamma"][0]), ("beta", b["dbeta"][0]), ("W", dW)):
            want[k] += v.numpy()
            got = run.shards[k][w].cpu().double()
            assert float((got - v).abs().max()) < 1e-4 * float(v.abs().max()), k
    total = sum(float((v ** 2).sum()) for v in want.values()) ** 0.5
    assert abs(float(norm[0]) / total - 1) < 1e-4 and abs(float(norm[1]) * total / 0.05 - 1) < 1e-4
    first = 0
    for k, t in run.tensors.items():
        n = t["W"].numel()
        rows = np64(t["sum"]).reshape(1, -1)
        w, m, v, dw, dm, dv = A.adamw(np64(run.host[k]).ravel(), rows, np.zeros(n), np.zeros(n), lr=0.02, step=1,
                                      decay=float(np.float32(t.get("weight_decay", 0))), scale=float(norm[1]), **KW)
        assert np.all(np.abs(np64(t["W"]).ravel() - w) <= dw + 1e-44), k
        if "exponents" in t:
            r = A.bits16(SEED, 0, first, n)
            (cm, em), (cv, ev) = A.encode(m, r, True), A.encode(v, A.exchanged(r), False)
            e = t["exponents"].cpu().numpy()
            assert np.array_equal(e[0::2], em) and np.array_equal(e[1::2], ev)
            assert np.array_equal(t["m"].cpu().numpy(), cm) and np.array_equal(t["v"].cpu().numpy(), cv)
        else:
            assert np.all(np.abs(np64(t["m"]).ravel() - m) <= dm) and np.all(np.abs(np64(t["v"]).ravel() - v) <= dv)
        first += -(-n // 128) * 16


@pytest.mark.parametrize("bits", [32, 8])
def test_replayed_from_a_graph(bits):
    """Whole steps in a graph, replayed beside the same steps run eagerly."""
    log(f"train together graph bits={bits}")
    runs = [Run(bits) for _ in range(2)]
    start = [t.clone() for t in runs[0].state()]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        runs[0].step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        held = runs[0].step()
    for a, b in zip(runs[0].state(), start):
        a.copy_(b)
    for i in range(4):
        graph.replay()
        want = runs[1].step()
        torch.cuda.synchronize()
        for a, b in zip(held + tuple(runs[0].state()), want + tuple(runs[1].state())):
            assert torch.equal(a, b), f"replay {i}"


@pytest.mark.parametrize("classes,features,B,P", [(300, 40, 8, 3), (40, 16, 64, 2)], ids=["factors", "shards"])
@pytest.mark.parametrize("bits", [32, 8])
def test_network_end_by_adamw(classes, features, B, P, bits):
    """Its step is AdamW on the gradient that its SGD step applies (lr 1, no
    momentum, no decay: the weights' difference), clipped.  At the first step the
    update is the gradient over its size: where the gradient is above 1e-3 of its
    largest, fp32 roundings of it (a few hundred) move it by less than 1e-2."""
    from paper_1706_03292_amd import api
    from paper_1706_03292_amd.network_end import NetworkEnd
    log(f"network end adamw {classes} bits={bits}")
    g = torch.Generator().manual_seed(1)
    x, res = (torch.randn(P * B, features, generator=g).to(dev()) for _ in range(2))
    target = torch.randint(0, classes, (P * B,), generator=g).to(dev())
    sgd = NetworkEnd(classes, features, B, P, lr=1.0, momentum=0.0, p=0.25, seed=3)
    adam = NetworkEnd(classes, features, B, P, lr=0.01, p=0.25, seed=3,
                      adamw={"bits": bits, "max_norm": 0.5, "weight_decay": 0.0})
    assert sgd.scheme == adam.scheme == (api.SFB if classes == 300 else api.PS)
    before = {k: getattr(sgd, k).double() for k in ("W", "gamma", "beta")}
    a, b = sgd.step(x, res, target), adam.step(x, res, target)
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    grads = {k: before[k] - getattr(sgd, k).double() for k in before}
    norm = sum(float((v ** 2).sum()) for v in grads.values()) ** 0.5
    scale = min(1.0, 0.5 / norm)
    for k, grad in grads.items():
        moved = (before[k] - getattr(adam, k).double()) / 0.01
        # before - after of the SGD step: the gradient to fp32's step of the weights
        big = grad.abs() > max(1e-3 * float(grad.abs().max()), 2e-4)
        assert big.any()
        want = grad * scale / ((grad * scale).abs() + 1e-8)
        assert float((moved - want)[big].abs().max()) < 1e-2, k
    for _ in range(2):
        adam.step(x, res, target)
    assert torch.isfinite(adam.W).all() and adam.steps == 3
    sgd.close(), adam.close()
    with pytest.raises(ValueError):
        NetworkEnd(classes, features, B, P, lr=0.01, adamw={"bits": 4})


def test_network_end_by_adamw_in_bf16():
    """Activations in bf16 from the copy of the classifier that the step leaves."""
    from paper_1706_03292_amd.network_end import NetworkEnd
    log("network end adamw bf16")
    end = NetworkEnd(64, 96, 16, 4, lr=0.01, dtype=torch.bfloat16, seed=5, adamw={"bits": 8})
    g = torch.Generator(device=dev()).manual_seed(2)
    for _ in range(3):
        x = torch.randn(64, 96, generator=g, device=dev()).bfloat16()
        loss, dx, _ = end.step(x, torch.zeros_like(x), torch.randint(0, 64, (64,), generator=g, device=dev()))
        assert torch.isfinite(loss) and torch.isfinite(dx).all()
        assert torch.equal(end.copy, end.W.bfloat16())
    end.close()
