"""Group norm without a GPU: what its entry points refuse before any device work,
their workspace query, and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_1706_03292_amd import _lib as L
from paper_1706_03292_amd import api

A, B, C, D, E, F, G, H, I, J = (ctypes.c_void_p(0x1000000 * (i + 1)) for i in range(10))   # never dereferenced
BAD = L.ERR_INVALID_ARG
NAN = float("nan")
SIZES = {"N": 2, "L_": 9, "C_": 24, "groups": 4, "dtype": L.F32}
WRONG = ({"N": -1}, {"N": 2 ** 24 + 1}, {"L_": 0}, {"L_": -1}, {"C_": 0}, {"C_": 2 ** 16 + 24}, {"groups": 0},
         {"groups": 5}, {"groups": -4}, {"groups": 48}, {"dtype": 2}, {"L_": 2 ** 40}, {"L_": 2 ** 62, "N": 0, "C_": 48})


def size_of(op, **kw):
    s = {**SIZES, **kw}
    size = ctypes.c_int64(-7)
    rc = L.lib().poseidon_group_norm_workspace(op, s["N"], s["L_"], s["C_"], s["groups"], s["dtype"], ctypes.byref(size))
    return rc, size.value


def fwd(x=A, gamma=B, beta=C, eps=1e-5, act=0, y=D, mean=E, rstd=F, ws=G, bytes=1 << 22, **kw):
    s = {**SIZES, **kw}
    return L.lib().poseidon_group_norm_forward(x, gamma, beta, s["N"], s["L_"], s["C_"], s["groups"], s["dtype"], eps,
                                               act, y, mean, rstd, ws, bytes, None)


def bwd(dy=H, x=A, gamma=B, beta=C, mean=E, rstd=F, act=0, dx=D, dgamma=I, dbeta=J, ws=G, bytes=1 << 22, **kw):
    s = {**SIZES, **kw}
    return L.lib().poseidon_group_norm_backward(dy, x, gamma, beta, mean, rstd, s["N"], s["L_"], s["C_"], s["groups"],
                                                s["dtype"], act, dx, dgamma, dbeta, ws, bytes, None)


def test_workspace():
    for op in (L.GROUP_NORM_FORWARD, L.GROUP_NORM_BACKWARD):
        rc, n = size_of(op)
        assert rc == L.OK and 0 <= n < 1 << 20
        assert size_of(op, N=0)[0] == L.OK
        for kw in WRONG:
            assert size_of(op, **kw)[0] == BAD, kw
    assert size_of(2)[0] == BAD and size_of(-1)[0] == BAD
    assert L.lib().poseidon_group_norm_workspace(0, 1, 1, 1, 1, 0, None) == BAD


def test_forward_refusals():
    for kw in WRONG + ({"eps": -1.0}, {"eps": NAN}, {"act": 3}, {"act": -1}, {"x": None}, {"gamma": None},
                       {"beta": None}, {"y": None}, {"mean": None}, {"rstd": None}, {"y": A}, {"y": B}, {"mean": C},
                       {"rstd": E}, {"mean": D}):
        assert fwd(**kw) == BAD, kw
    big = {"N": 40, "L_": 50000}
    need = size_of(L.GROUP_NORM_FORWARD, **big)[1]
    assert need > 0
    x, y = ctypes.c_void_p(0x80000000), ctypes.c_void_p(0x180000000)
    for kw in ({"ws": None}, {"ws": ctypes.c_void_p(0x7000008)}, {"bytes": need - 1}, {"ws": x}, {"ws": y}, {"ws": E}):
        assert fwd(**{**big, "x": x, "y": y, "bytes": need, **kw}) == BAD, kw
    assert fwd(x=None, gamma=None, beta=None, y=None, mean=None, rstd=None, ws=None, N=0) == L.OK


def test_backward_refusals():
    for kw in WRONG + ({"act": 3}, {"dy": None}, {"x": None}, {"gamma": None}, {"beta": None}, {"mean": None},
                       {"rstd": None}, {"dx": None}, {"dgamma": None}, {"dbeta": None}, {"dx": A}, {"dx": H},
                       {"dgamma": J}, {"dgamma": B}, {"dbeta": E}, {"dbeta": D}):
        assert bwd(**kw) == BAD, kw
    need = size_of(L.GROUP_NORM_BACKWARD, N=40, L_=50000)[1]
    dy, x, dx = (ctypes.c_void_p(0x100000000 * k) for k in (1, 2, 3))
    big = {"N": 40, "L_": 50000, "dy": dy, "x": x, "dx": dx}
    for kw in ({"ws": None}, {"ws": ctypes.c_void_p(0x7000008)}, {"bytes": need - 1}, {"ws": dy}, {"ws": dx}, {"ws": I}):
        assert bwd(**{**big, "bytes": need, **kw}) == BAD, kw


def test_the_binding_refuses():
    x, g = torch.zeros(2, 3, 8), torch.zeros(8)
    with pytest.raises(ValueError, match="HIP device"):
        api.group_norm_forward(x, g, g, 2)
    with pytest.raises(TypeError):
        api.group_norm_forward(x.half(), g, g, 2)
    with pytest.raises(TypeError):
        api.group_norm_forward([1.0], g, g, 2)
    with pytest.raises(ValueError, match="HIP device"):
        api.group_norm_backward(x, x, g, g, torch.zeros(2, 2), torch.zeros(2, 2))
    with pytest.raises(ValueError, match="act"):
        api._act("tanh")
