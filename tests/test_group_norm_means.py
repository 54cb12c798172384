"""Group norm of maps whose means are far above their spreads: the result, which the
mean's own rounding does not reach."""
import pytest
import torch

import _group_norm_oracle as O
from _helpers import dev, log
from test_group_norm import EPS, drawn, launched, within

pytestmark = pytest.mark.gpu

# (sizes, launches): held, held as a ragged row, in two launches, three and four.
FAR = [((2, 49, 64, 8), 1), ((3, 5, 45, 9), 1), ((1, 196, 512, 32), 1), ((3, 5000, 72, 9), 2), ((17, 1225, 288, 32), 2),
       ((3, 5000, 70, 1), 3), ((5, 3500, 520, 65), 3), ((2, 9000, 520, 1), 4), ((1, 4000, 4100, 4), 4)]


def centred(x, groups):
    """x without its groups' means, in 64 bits: group norm's y and rstd are those of x,
    and a bound that counts the mean's roundings counts none."""
    v = O.shaped(x, groups)
    return (v - v.mean((1, 3), keepdim=True)).reshape(x.shape)


@pytest.mark.parametrize("mean", [1000.0, 1e5])
@pytest.mark.parametrize("sizes,launches", FAR)
def test_the_means_rounding_does_not_reach_the_result(sizes, launches, mean):
    """fp32 values of spread about 1, of either sign in every other group.  Differences
    of near values are exact, so y's bound is that of the same values about 0; the mean
    itself is rounded once more."""
    from paper_1706_03292_amd import api
    N, L, C, groups = sizes
    log(f"group norm mean {mean} {sizes}")
    x, gamma, beta, _ = drawn(N, L, C, torch.float32, 21)
    x = x + mean * (1 - 2 * (torch.arange(C) // (C // groups) % 2))
    d = [t.to(dev()) for t in (x, gamma, beta)]
    y, m, rstd = api.group_norm_forward(*d, groups, EPS, act="silu")
    assert len(launched(lambda: api.group_norm_forward(*d, groups, EPS, act="silu"))) == launches
    want = O.forward(centred(x, groups), gamma, beta, groups, EPS, "silu", O.U32)
    within(y, want["y"], "y")
    within(rstd, want["rstd"], "rstd")
    exact = O.shaped(x, groups).mean((1, 3))
    within(m, (exact, want["mean"][1] + O.U32 * exact.abs()), "mean")


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("at", ["first", "middle", "last"])
@pytest.mark.parametrize("N,L,C,groups", [(3, 300, 24, 4), (3, 5000, 72, 9), (3, 5000, 70, 2), (2, 9000, 520, 2)])
def test_a_bad_value_where_differences_start(N, L, C, groups, at, bad):
    """Each group's first channel, in the rows that a difference may be taken from: its
    group's results are NaN, the others' as without it."""
    from paper_1706_03292_amd import api
    log(f"group norm bad value {at} {bad} {N} {L} {C}")
    x, gamma, beta, _ = (t.to(dev()) for t in drawn(N, L, C, torch.float32, 22))
    good = api.group_norm_forward(x, gamma, beta, groups, EPS, act="relu")
    for g in (0, groups - 1):
        z = x.clone()
        z[1, {"first": 0, "middle": L // 2, "last": L - 1}[at], g * (C // groups)] = bad
        y, mean, rstd = api.group_norm_forward(z, gamma, beta, groups, EPS, act="relu")
        hit = torch.zeros(N, groups, dtype=torch.bool, device=dev())
        hit[1, g] = True
        cells = hit[:, None, :, None].expand(N, L, groups, C // groups).reshape(N, L, C)
        assert torch.equal(y[~cells], good[0][~cells]) and torch.isnan(y[cells]).all()
        assert torch.equal(mean[~hit], good[1][~hit]) and torch.equal(rstd[~hit], good[2][~hit])
        assert not torch.isfinite(mean[hit]).any() and not torch.isfinite(rstd[hit]).any()
