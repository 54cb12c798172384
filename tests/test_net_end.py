"""The operators at a network's end together with the synchronisation they
feed: one step against 64 bits, and a short training."""
import pytest
import torch

import _net_oracle as O
from _helpers import dev, log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("classes,features,B,P", [(300, 40, 8, 3), (40, 16, 64, 2)], ids=["factors", "shards"])
def test_one_step_against_64_bits(classes, features, B, P):
    """The updated parameters of one fp32 step: lr times sums of T = P*B rows of
    products, each of them fp32, so within a few hundred fp32 roundings of the
    largest update."""
    from paper_1706_03292_amd import api
    from paper_1706_03292_amd.network_end import NetworkEnd
    log(f"network end {classes}x{features} B={B} P={P}")
    lr, p = 0.25, 0.25
    end = NetworkEnd(classes, features, B, P, lr, momentum=0.9, p=p, seed=3)
    assert end.scheme == (api.SFB if classes == 300 else api.PS)
    g = torch.Generator().manual_seed(1)
    x, res = torch.randn(P * B, features, generator=g), torch.randn(P * B, features, generator=g)
    target = torch.randint(0, classes, (P * B,), generator=g)
    target[::7] = -1
    W0, rng = end.W.double().cpu(), end.rng.cpu()
    loss, dx, dres = end.step(x.to(dev()), res.to(dev()), target.to(dev()))

    has = target >= 0
    dloss = has.double() / has.sum()
    masks = [O.keep(int(rng[w, 0]), int(rng[w, 1]), B, features, p) for w in range(P)]
    mask, thr = torch.cat([m for m, _ in masks]), masks[0][1]
    h = O.dropped(x, mask, thr) + res.double()
    one, zero = torch.ones(features), torch.zeros(features)
    y, mean, rstd = O.norm_forward(h, one, zero, 1e-5)
    want, _, _, dy, dW = O.xent(y, W0, target, dloss)
    dh, dgamma, dbeta = O.norm_backward(dy, h, one, mean, rstd, None)

    def near(got, want, what):
        err = float((got.double().cpu() - want).abs().max() / want.abs().max().clamp(min=1e-30))
        assert err < 1e-4, f"{what}: {err:.2e}"

    near(loss, (want * dloss).sum(), "loss")
    near(dres, dh, "dresidual")
    near(dx, O.dropped(dh, mask, thr), "dx")
    near(end.W - W0.float().to(dev()), -lr * dW, "classifier update")
    near(end.gamma - 1, -lr * dgamma, "gamma update")
    near(end.beta, -lr * dbeta, "beta update")
    assert (end.rng[:, 1] == 1).all()
    end.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_training_lowers_the_loss(dtype):
    from paper_1706_03292_amd.network_end import NetworkEnd
    log(f"network end training {dtype}")
    classes, features, B, P = 64, 96, 16, 4
    end = NetworkEnd(classes, features, B, P, lr=0.5, p=0.1, dtype=dtype, seed=5)
    g = torch.Generator(device=dev()).manual_seed(2)
    centre = torch.randn(classes, features, generator=g, device=dev())
    losses = []
    for _ in range(40):
        target = torch.randint(0, classes, (P * B,), generator=g, device=dev())
        x = (centre[target] + 0.5 * torch.randn(P * B, features, generator=g, device=dev())).to(dtype)
        losses.append(float(end.step(x, torch.zeros_like(x), target)[0]))
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5]), losses
    end.close()


@pytest.mark.parametrize("classes,features,B,P", [(300, 40, 8, 3), (40, 16, 64, 2)], ids=["factors", "shards"])
def test_rows_without_a_target_count_for_nothing(classes, features, B, P):
    """A step whose padding rows hold NaN and infinities gives the bits of one
    whose padding rows hold zeros."""
    from paper_1706_03292_amd.network_end import NetworkEnd
    log(f"network end padding {classes}x{features} B={B} P={P}")
    g = torch.Generator().manual_seed(4)
    x, res = torch.randn(P * B, features, generator=g), torch.randn(P * B, features, generator=g)
    target = torch.randint(0, classes, (P * B,), generator=g)
    target[::5], target[3] = -1, classes
    none = (target < 0) | (target >= classes)
    left = []
    for fill in (0.0, float("nan"), float("inf")):
        a, b = (torch.where(none[:, None], torch.full_like(v, fill), v).to(dev()) for v in (x, res))
        end = NetworkEnd(classes, features, B, P, 0.25, momentum=0.9, p=0.25, seed=3)
        loss, dx, dres = end.step(a, b, target.to(dev()))
        left.append((loss, dx, dres, end.W.clone(), end.gamma.clone(), end.beta.clone()))
        end.close()
    for now in left[1:]:
        for a, b in zip(left[0], now):
            assert torch.isfinite(b).all() and torch.equal(a, b)
