"""AdamW and group norm where a workgroup has more than one turn of its loop, and past
2^31 values in the forms that the operators' own tests take smaller."""
import numpy as np
import pytest
import torch

import _adamw_oracle as A
import _group_norm_oracle as G
from _helpers import dev, log
from test_group_norm import EPS, launched

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def api():
    from paper_1706_03292_amd import api as a
    return a


def holds(got, want, what):
    value, bound = want
    over = (got.double().reshape(value.shape) - value).abs() / bound
    assert float(over.max()) <= 1.0, f"{what}: {float(over.max()):.2f} of its bound"


# More samples than a launch has workgroups (2^20): four turns of each, in two launches
# (forward), three, and with groups too wide for one workgroup's sums.
MANY = [(2, 8, 8, ["chunk_stats", "forward"], ["chunk_sums", "join_sums", "backward"]),
        (2, 8, 1, ["chunk_stats", "group_stats", "forward"], ["chunk_sums", "join_sums", "backward"]),
        (1, 72, 1, ["chunk_stats", "group_stats", "forward"],
         ["chunk_sums", "join_channels", "average", "backward"])]


@pytest.mark.parametrize("L,C,groups,forward,backward", MANY, ids=["late", "groups", "wide"])
def test_group_norm_of_many_samples(L, C, groups, forward, backward):
    """Every sample against 64 bits; dgamma and dbeta, whose samples are added up in 64
    bits, against the sum of the parts' values and bounds."""
    N = 2 ** 22 + 5
    log(f"group norm {N} x {L} x {C} in {groups}")
    gen = torch.Generator(device=dev()).manual_seed(1)
    x = torch.randn(N, L, C, generator=gen, device=dev()).to(BF16)
    dy = torch.randn(N, L, C, generator=gen, device=dev()).to(BF16)
    gamma, beta = (torch.randn(C, generator=gen, device=dev()) for _ in range(2))
    y, mean, rstd = api().group_norm_forward(x, gamma, beta, groups, EPS, act="silu")
    dx, dgamma, dbeta = api().group_norm_backward(dy, x, gamma, beta, mean, rstd, act="silu")
    sums = {"dgamma": [0.0, 0.0], "dbeta": [0.0, 0.0]}
    for r in torch.arange(N, device=dev()).split(2 ** 18):
        s = slice(int(r[0]), int(r[-1]) + 1)
        want = G.forward(x[s], gamma, beta, groups, EPS, "silu", G.U16)
        holds(y[s], want["y"], "y"), holds(mean[s], want["mean"], "mean"), holds(rstd[s], want["rstd"], "rstd")
        want = G.backward(dy[s], x[s], gamma, beta, mean[s], rstd[s], "silu", G.U16)
        holds(dx[s], want["dx"], "dx")
        for name, total in sums.items():
            total[0], total[1] = total[0] + want[name][0], total[1] + want[name][1]
    holds(dgamma, sums["dgamma"], "dgamma"), holds(dbeta, sums["dbeta"], "dbeta")
    assert launched(lambda: api().group_norm_forward(x, gamma, beta, groups, EPS, act="silu")) == forward
    assert launched(lambda: api().group_norm_backward(dy, x, gamma, beta, mean, rstd, act="silu")) == backward


def test_group_norm_past_32_bits_in_two_launches():
    """2^31 values and more in 8193 samples: the first, the one across 2^31 and the last."""
    N, L, C, groups = 8193, 513, 516, 12
    log(f"group norm {N} x {L} x {C}")
    gen = torch.Generator(device=dev()).manual_seed(2)
    x = torch.empty(N, L, C, dtype=BF16, device=dev())
    for part in x.split(512):
        part.copy_(torch.randn(part.shape, generator=gen, device=dev(), dtype=BF16))
    gamma, beta = (torch.randn(C, generator=gen, device=dev()) for _ in range(2))
    y, mean, rstd = api().group_norm_forward(x, gamma, beta, groups, EPS, act="relu")
    dx, _, _ = api().group_norm_backward(x, x, gamma, beta, mean, rstd, act="relu")
    for n in (0, 2 ** 31 // (L * C), N - 1):
        s = slice(n, n + 1)
        want = G.forward(x[s], gamma, beta, groups, EPS, "relu", G.U16)
        holds(y[s], want["y"], "y"), holds(mean[s], want["mean"], "mean"), holds(rstd[s], want["rstd"], "rstd")
        holds(dx[s], G.backward(x[s], x[s], gamma, beta, mean[s], rstd[s], "relu", G.U16)["dx"], "dx")
    assert launched(lambda: api().group_norm_forward(x, gamma, beta, groups, EPS, act="relu")) == ["chunk_stats", "forward"]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("P", [1, 3])
def test_clip_of_several_turns(P, dtype):
    """More than 8192 workgroups' 2048 values: two turns each, the last one with a tail,
    of tensors on odd boundaries, the sums kept and nothing written beside them."""
    log(f"adamw clip of several turns P={P} {dtype}")
    sizes = [70001, 2 ** 24 + 33]
    gen = torch.Generator(device=dev()).manual_seed(3)
    total = sum(sizes) + 4
    shards = torch.empty(P, total, dtype=dtype, device=dev())
    for row in shards:
        row.copy_(torch.randn(total, generator=gen, device=dev()))
    sums = torch.full((total,), 7.0, device=dev())
    tensors, at = [], 1
    for n in sizes:
        W = torch.zeros(n, device=dev())
        tensors.append({"W": W, "shards": shards[:, at:at + n], "sum": sums[at:at + n], **api().AdamW.moments(W)})
        at += n + 1
    r = api().AdamW(tensors).clip(1.0).double()
    square = 0.0
    for t in tensors:
        want = t["shards"].double().sum(0)
        square += float(want.square().sum())
        # one rounding to fp32; P values add up in 64 bits
        assert ((t["sum"] - want).abs() <= 1.01 * A.U32 * want.abs()).all()
    assert abs(float(r[0]) - square ** 0.5) <= 1.01 * A.U32 * square ** 0.5
    assert abs(float(r[1]) * square ** 0.5 - 1) <= 1.01 * A.U32
    for i in (0, 1 + sizes[0], 2 + sum(sizes), 3 + sum(sizes)):
        assert sums[i] == 7


def test_adamw_past_32_bits_with_fp32_moments():
    """2^31 + 1000 values: the first, those across 2^31 and the last; clip, a step from
    the sums, the copy and the values."""
    log("adamw fp32 moments 2^31 values")
    n = 2 ** 31 + 1000
    W = torch.zeros(n, device=dev())
    t = {"W": W, "shards": torch.zeros(1, n, dtype=BF16, device=dev()), "sum": torch.empty(n, device=dev()),
         "copy": torch.empty(n, dtype=BF16, device=dev()), "weight_decay": 0.1, **api().AdamW.moments(W)}
    gen = torch.Generator(device=dev()).manual_seed(4)
    places = [slice(0, 128), slice(2 ** 31 - 128, 2 ** 31 + 256), slice(n - 100, n)]
    for p in places:
        t["shards"][0, p] = torch.randn(p.stop - p.start, generator=gen, device=dev()).to(BF16)
        W[p] = torch.randn(p.stop - p.start, generator=gen, device=dev())
    before = [W[p].cpu().double().numpy() for p in places]
    opt = api().AdamW([t])
    r = opt.clip(1.0)
    grads = [t["shards"][:, p].cpu().double().numpy() for p in places]
    assert abs(float(r[0]) / sum(float((x ** 2).sum()) for x in grads) ** 0.5 - 1) <= 1.01 * A.U32
    opt.step(0.01, 1, scale=r[1:2], from_sums=True)
    m_out, v_out = opt.values()[0]
    for p, x, w0 in zip(places, grads, before):
        zero = np.zeros(p.stop - p.start)
        w, m, v, dw, dm, dv = A.adamw(w0, x, zero, zero, lr=0.01, step=1, betas=(0.9, 0.999), eps=1e-8,
                                      decay=float(np.float32(0.1)), scale=float(r[1]))
        for got, value, bound in ((W, w, dw), (t["m"], m, dm), (t["v"], v, dv), (m_out, m, dm), (v_out, v, dv)):
            assert np.all(np.abs(got[p].cpu().double().numpy() - value) <= bound + 1e-44)
        assert torch.equal(t["copy"][p], W[p].to(BF16)) and torch.equal(t["sum"][p], t["shards"][0, p].float())
    for p in (slice(128, 2 ** 20), slice(2 ** 31 + 256, 2 ** 31 + 512)):
        assert (W[p] == 0).all() and (t["m"][p] == 0).all() and (t["sum"][p] == 0).all()
