"""AdamW's fp32 moments over many steps, at decay factors that fp32 cannot hold."""
import pytest
import torch

import _adamw_oracle as O
from _helpers import dev, log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P", [1, 2])
@pytest.mark.parametrize("beta", [0.9999, 0.99999])
def test_moments_follow_their_averages(beta, P):
    """Two thousand steps of gradients drawn anew (mean 1, spread 1/2), beside both
    moments in 64 bits: their ratio, averaged over n values.

    Every step rounds the new moment once, by at most u of it either way: a change is
    tens of fp32's steps, so the roundings' mean is 0 and (Hoeffding) the average of
    n values after T steps is off by u sqrt(2 T / n ln(2 / 1e-12)) = 5.3 u with one in
    10^12.  1 - beta, the square, the product and the sum that is added round once each,
    u of what a step adds: 4 u of the moment.  12 u holds both.  (A factor beta rounded
    to fp32 moves 1 - beta by up to 2^-25 / (1 - beta) of it; over these steps, of
    which 1 - beta^T is felt, that makes 3e-5: 500 u.)"""
    log(f"adamw decay beta={beta} P={P}")
    from paper_1706_03292_amd import api
    n, T = 4096, 2000
    gen = torch.Generator(device=dev()).manual_seed(3)
    W = torch.zeros(n, device=dev())
    shards = torch.zeros(P, n, device=dev())
    m, v = torch.full((n,), 1.0, device=dev()), torch.full((n,), 1.25, device=dev())
    m64, v64 = m.double(), v.double()
    opt = api.AdamW([{"W": W, "shards": shards, "m": m, "v": v}], betas=(beta, beta))
    for step in range(T):
        shards[P - 1] = 1 + 0.5 * torch.randn(n, generator=gen, device=dev())
        opt.step(0.0, 1 + step)
        g = shards[P - 1].double()
        m64 = beta * m64 + (1 - beta) * g
        v64 = beta * v64 + (1 - beta) * (g * g)
    for name, a, b in (("m", m, m64), ("v", v, v64)):
        off = float((a.double() / b - 1).mean())
        assert abs(off) <= 12 * O.U32, f"{name}: {off / O.U32:.1f} u"


@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.5, 0.75), (0.99999, 0.99999)])
def test_an_infinite_variance_stays_infinite(betas):
    """A finite gradient whose square passes fp32's range: v is infinite from then on, m
    is not, and the weight stands still."""
    log(f"adamw infinite variance {betas}")
    from paper_1706_03292_amd import api
    W = torch.ones(300, device=dev())
    t = {"W": W, "shards": torch.full((1, 300), 1e-3, device=dev()), **api.AdamW.moments(W)}
    opt = api.AdamW([t], betas=betas)
    t["shards"][0, 77] = 1e25
    opt.step(0.1, 1)
    assert torch.isinf(t["v"][77]) and W[77] == 1
    t["shards"][0, 77] = 1e-3
    for step in range(2, 6):
        opt.step(0.1, step)
    assert torch.isinf(t["v"][77]) and torch.isfinite(t["m"]).all() and W[77] == 1
    assert torch.isfinite(t["v"][:77]).all() and (W[:77] < 1).all()
