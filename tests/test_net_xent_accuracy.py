"""What the classifier loss's products keep of their operands, seen where a
worst-case bound over a whole sum would not see it."""
import pytest
import torch

from _helpers import dev, log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rms(x):
    return float(x.double().square().mean().sqrt())


@pytest.mark.parametrize("T,V,D", [(24, 900, 136), (24, 20000, 64), (300, 2100, 200), (700, 4100, 513)])
def test_bf16_input_gradient_of_classes_that_share_a_component(T, V, D):
    """Classes whose weights are 30 times as large as they differ, as a trained
    classifier's may be, and rows whose softmax is concentrated.  A row of G sums
    to 0, so the shared component cancels in dX: what G's own rounding left of it
    would not.  The reference takes the kernel's fp32 U.  G in two bf16 parts is
    off by at most 2^-16 of each entry (rms 2^-16 / sqrt(3) of 30 times dX's
    size: 0.16 of the rounding of dX to bf16, 2^-8 / sqrt(3) * 0.7 of it), and
    fp32 sums by less: 1.05 times dX's rounding holds them.  One part, the
    target's entry made exact, is 3.6 to 5.8 times it at these sizes."""
    from paper_1706_03292_amd import api
    log(f"xent shared component {T}x{V}x{D}")
    g = torch.Generator().manual_seed(T + V + D)
    W = torch.randn(V, D, generator=g) / D ** 0.5
    W[:, ::2] += 30 / D ** 0.5
    X = torch.randn(T, D, generator=g)
    X[:, 1::2] *= 4
    W, X = W.to(BF16).to(dev()), X.to(BF16).to(dev())
    target = torch.randint(0, V, (T,), generator=g).to(dev())
    dloss = (torch.rand(T, generator=g) + 0.5).to(dev())
    _, U, x2 = api.xent_factor(X, W, target, dloss)
    _, lse = api.xent_forward(X, W, target)
    x1, _ = api.xent_backward(X, W, target, lse, dloss)
    want = U.double() @ W.double()
    rounding = rms(want.to(BF16).double() - want)
    for got, what in ((x2, "factor dX"), (x1, "dX")):
        err = rms(got.double() - want)
        assert err <= 1.05 * rounding, f"{what}: {err / rounding:.2f} times the rounding of dX"
