"""AdamW from the sums that clip leaves, where a sum does not fit fp32."""
import pytest
import torch

from _helpers import dev, log

pytestmark = pytest.mark.gpu

N = 5003


def made(P, sums, bits=32, at=N - 1, value=3e38):
    from paper_1706_03292_amd import api
    gen = torch.Generator(device=dev()).manual_seed(1)
    W = torch.randn(N, generator=gen, device=dev())
    G = 1e-3 * torch.randn(P, N, generator=gen, device=dev())
    G[:, at] = value
    t = {"W": W, "shards": G, **api.AdamW.moments(W, bits)}
    if sums:
        t["sum"] = torch.empty_like(W)
    return api.AdamW([t]), t


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("at", [0, 2047, N - 1])
def test_a_sum_past_fp32_leaves_the_step_out(at, bits):
    """Two workers' finite gradients whose sum is infinite in fp32."""
    log(f"adamw sum past fp32 at={at} bits={bits}")
    opt, t = made(2, True, bits, at)
    before = {k: t[k].clone() for k in ("W", "m", "v")}
    r = opt.clip(1.0)
    assert torch.isinf(t["sum"][at]) and torch.isinf(r[0]) and torch.isnan(r[1])
    opt.step(0.1, 1, scale=r[1:2], from_sums=True)
    for k, v in before.items():
        assert torch.equal(t[k], v), k


@pytest.mark.parametrize("P,sums", [(2, False), (1, True)])
def test_what_fits_is_stepped(P, sums):
    """Without sums, and where the sum itself is finite, the scale is max_norm over
    the norm: 1 / 6e38 and 1 / 3e38, of fp32's numbers below its normal range (steps of
    2^-149; the norm and its quotient are of 64 bits)."""
    log(f"adamw large norm P={P}")
    opt, t = made(P, sums)
    r = opt.clip(1.0)
    want = 1 / float(t["shards"].double().sum(0).norm())
    assert abs(float(r[1]) - want) <= 2.0 ** -150 + 1e-9 * want
    opt.step(0.1, 1, scale=r[1:2], from_sums=sums)
    assert all(torch.isfinite(t[k]).all() for k in ("W", "m", "v"))
