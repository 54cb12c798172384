"""The network's end trained by AdamW where a step is not like the others: weights
written between steps, and steps that are left out."""
import pytest
import torch

from _helpers import dev, log

pytestmark = pytest.mark.gpu

CLASSES, FEATURES, B, P = 64, 96, 16, 4


def end(dtype=torch.float32, seed=5, **adamw):
    from paper_1706_03292_amd.network_end import NetworkEnd
    return NetworkEnd(CLASSES, FEATURES, B, P, lr=0.01, p=0.0, dtype=dtype, seed=seed, adamw=adamw)


def batch(gen, dtype=torch.float32):
    x = torch.randn(P * B, FEATURES, generator=gen, device=dev()).to(dtype)
    return x, torch.zeros_like(x), torch.randint(0, CLASSES, (P * B,), generator=gen, device=dev())


@pytest.mark.parametrize("write", [lambda W, new: W.copy_(new), lambda W, new: W.data.copy_(new)],
                         ids=["copy_", "data"])
def test_weights_written_between_steps(write):
    """A bf16 network whose classifier is written from outside (a checkpoint, a
    broadcast) computes with what was written."""
    log("network end adamw written weights")
    a, b = end(torch.bfloat16), end(torch.bfloat16, seed=6)
    gen = torch.Generator(device=dev()).manual_seed(2)
    for e in (a, b):
        e.step(*batch(gen, torch.bfloat16))
    for name in ("gamma", "beta"):
        getattr(b, name).copy_(getattr(a, name))
    write(b.W, a.W)
    data = batch(gen, torch.bfloat16)
    for u, v in zip(a.step(*data), b.step(*data)):
        assert torch.equal(u, v)
    a.close(), b.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_that_is_left_out_is_not_counted(bits):
    """A first batch whose gradient is not finite changes nothing; the step after it is
    a fresh optimizer's first."""
    log(f"network end adamw left out bits={bits}")
    a, b = end(bits=bits, max_norm=1.0), end(bits=bits, max_norm=1.0)
    gen = torch.Generator(device=dev()).manual_seed(3)
    bad, good = batch(gen), batch(gen)
    bad[0][3, 5] = float("inf")
    before = [t.clone() for t in (a.W, a.gamma, a.beta)]
    a.step(*bad)
    for u, v in zip((a.W, a.gamma, a.beta), before):
        assert torch.equal(u, v)
    a.round_rng.copy_(b.round_rng)
    for e in (a, b):
        e.step(*good)
    for u, v in zip((a.W, a.gamma, a.beta), (b.W, b.gamma, b.beta)):
        assert torch.equal(u, v)
    for u, v in zip(a.optimizer.values(), b.optimizer.values()):
        assert torch.equal(u[0], v[0]) and torch.equal(u[1], v[1])
    a.close(), b.close()


def test_the_learning_rate_may_change():
    """`lr` is read at every step."""
    log("network end adamw lr")
    a = end()
    gen = torch.Generator(device=dev()).manual_seed(4)
    a.step(*batch(gen))
    before, a.lr = a.W.clone(), 0.0
    a.step(*batch(gen))
    assert torch.equal(a.W, before)
    a.close()
