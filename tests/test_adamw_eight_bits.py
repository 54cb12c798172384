"""What 8-bit moments do over many steps: beside fp32 moments of the same gradients, and
where a value is small beside its block's largest."""
import pytest
import torch

from _helpers import dev, log

pytestmark = pytest.mark.gpu

SEED = 0x1234567


def made(n, bits):
    from paper_1706_03292_amd import api
    W = torch.zeros(n, device=dev())
    t = {"W": W, "shards": torch.zeros(1, n, device=dev()), **api.AdamW.moments(W, bits)}
    return api.AdamW([t], betas=(0.9, 0.999)), t


def test_beside_fp32_moments():
    """Three thousand steps of normal gradients, the same for both.  Of n = 65536 values:

    v.  A step moves v by 0.001 |g^2 - v|, 0.001 * 0.968 v on average, from a code; rounded
    at random between codes d apart that is a variance of that times d (a share of the way
    f is right on average with f (1 - f) d^2, f of about 1%).  d is an eighth of v's power of
    two, 0.0902 v on average over it.  What is left of all steps' is 1 / (1 - 0.999^2) of
    one's: 0.0437 v^2, a spread of 0.209 of v, which the average of n values has 256th of
    (six of them: 0.005).  16 random bits round down by 2^-17 of d a step more than up: 0.0007.

    m.  Codes are at most an eighth apart, so a step's rounding has a variance of at most
    1/4 of (m / 8)^2, all steps' 1 / (1 - 0.81) of it: spreads below 0.15 of m, a projection
    on fp32's m off by a 256th of that.  What falls below code 1, 2^-15 of the block's
    largest, counts for less."""
    log("adamw 8 bits beside 32")
    n = 65536
    (a, ta), (b, tb) = made(n, 8), made(n, 32)
    gen = torch.Generator(device=dev()).manual_seed(7)
    for step in range(3000):
        ta["shards"].copy_(torch.randn(1, n, generator=gen, device=dev()))
        tb["shards"].copy_(ta["shards"])
        a.step(0.0, 1 + step, rng=torch.tensor([SEED, step], device=dev()))
        b.step(0.0, 1 + step)
    (m8, v8), (m32, v32) = ([x.double() for x in o.values()[0]] for o in (a, b))
    ratio = v8 / v32
    assert abs(float(ratio.mean()) - 1) < 0.01
    assert 0.17 < float(ratio.std()) < 0.25
    assert abs(float((m8 * m32).sum() / m32.square().sum()) - 1) < 0.01


def test_small_first_moments():
    """After 200 steps in which only a block's first value has a gradient (of 1, so that m's
    code 1 is 1.9e-5 or 3.8e-5), its neighbours get one.  (1 - beta1) g of 1e-5 is below
    code 1, and m stays 0; of 6e-5 is above it, and m reaches g on average (codes at most
    an eighth apart: a spread below 0.15 of it, of 64 * 256 values together 0.0012)."""
    log("adamw 8 bits small m")
    blocks = 256
    opt, t = made(128 * blocks, 8)
    g = t["shards"].view(blocks, 128)
    g[:, 0] = 1.0
    for step in range(300):
        if step == 200:
            g[:, 1:64], g[:, 64:] = 1e-4, 6e-4
        opt.step(0.0, 1 + step, rng=torch.tensor([SEED, step], device=dev()))
    m = opt.values()[0][0].view(blocks, 128).double()
    assert (m[:, 1:64] == 0).all()
    assert abs(float(m[:, 64:].mean()) / 6e-4 - 1) < 0.01
