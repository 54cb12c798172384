"""AdamW's division where v is below fp32's normal range, or eps beyond it."""
import numpy as np
import pytest
import torch

import _adamw_oracle as O
from _helpers import dev, log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("beta2,eps,size", [(0.999, 2e-12, 3e-18), (0.99999, 1e-11, 2e-17), (0.99999, 1e-8, 2e-17),
                                            (0.0, 1.5e-12, 1e-19), (0.999, 1e-13, 3e-18), (0.999, 2e38, 1e19)])
def test_update_from_a_small_variance(beta2, eps, size, bits):
    """Weights of 0, so that the update alone counts, by value and from the clock: within
    the bound that counts roundings.  Of v (m): what is below 2^-126 has steps of 2^-149,
    so the root of v is off by up to half of 2^-149 over it, which eps is beside (8 bits:
    computed in 64 bits and rounded once).  Update values below 2^-126 have such steps too."""
    log(f"adamw small variance beta2={beta2} eps={eps} bits={bits}")
    from paper_1706_03292_amd import api
    n = 1000
    gen = torch.Generator().manual_seed(5)
    g = size * (0.5 + 0.5 * torch.rand(1, n, generator=gen))
    zero = np.zeros(n)
    kw = {"betas": (0.9, beta2), "eps": float(np.float32(eps))}
    w, m, v, dw, dm, dv = O.adamw(zero, g.double().numpy(), zero, zero, lr=0.5, step=1, decay=0.0, **kw)
    root = (1 - beta2) ** -0.5
    step = 2.0 ** -149
    # the root's error from v's, and m's, relative to what they are part of
    off = step / np.sqrt(v) * root / (np.sqrt(v) * root + eps) + step / np.abs(m)
    for clock in (None, torch.tensor([0.5, 1.0], dtype=torch.float64, device=dev())):
        W = torch.zeros(n, device=dev())
        t = {"W": W, "shards": g.to(dev()), **api.AdamW.moments(W, bits)}
        api.AdamW([t], **kw).step(0.5, 1, clock=clock)
        over = float((np.abs(W.cpu().double().numpy() - w) / (dw + off * np.abs(w) + step)).max())
        assert over <= 1.0, f"{over:.2f} of the bound"
