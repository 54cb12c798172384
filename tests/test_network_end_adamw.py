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
