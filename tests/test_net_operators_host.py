"""The operators at a network's end, without a GPU: what their entry points
refuse before any device work, their workspace queries, and the binding's own
checks."""
import ctypes

import pytest
import torch

from paper_1706_03292_amd import _lib as L
from paper_1706_03292_amd import api

A, B, C, D, E, F, G = (ctypes.c_void_p(0x1000000 * (i + 1)) for i in range(7))   # never dereferenced
BAD = L.ERR_INVALID_ARG
NAN = float("nan")


def test_dropout_refusals():
    f = L.lib().poseidon_dropout
    assert f(A, None, -1, 8, L.F32, 0.1, B, C, None) == BAD
    assert f(A, None, 8, -1, L.F32, 0.1, B, C, None) == BAD
    assert f(A, None, 8, 8, 2, 0.1, B, C, None) == BAD
    for p in (-0.1, 1.5, NAN):
        assert f(A, None, 8, 8, L.F32, p, B, C, None) == BAD
    assert f(A, None, 8, 8, L.F32, 0.1, None, C, None) == BAD          # no generator
    assert f(None, None, 8, 8, L.F32, 0.1, B, C, None) == BAD
    assert f(A, None, 8, 8, L.F32, 0.1, B, None, None) == BAD
    assert f(A, None, 8, 8, L.F32, 0.1, B, A, None) == BAD             # in place
    assert f(A, C, 8, 8, L.BF16, 0.1, B, C, None) == BAD               # onto the residual
    assert f(A, None, 2 ** 40, 2 ** 30, L.F32, 0.1, B, C, None) == BAD
    assert f(None, None, 0, 8, L.F32, 0.1, None, None, None) == L.OK
    assert f(None, None, 8, 0, L.BF16, 0.1, None, None, None) == L.OK


def test_norm_refusals():
    lib = L.lib()

    def fwd(x=A, res=None, gamma=B, beta=C, rows=4, cols=8, dtype=L.F32, eps=1e-5, p=0.0, rng=None, h=None, y=D,
            mean=E, rstd=F):
        return lib.poseidon_norm_forward(x, res, gamma, beta, rows, cols, dtype, eps, p, rng, h, y, mean, rstd, None)

    for bad in (dict(rows=-1), dict(cols=-1), dict(cols=0), dict(cols=2 ** 28 + 1), dict(dtype=7), dict(eps=-1.0),
                dict(eps=NAN), dict(p=1.1), dict(p=0.5), dict(x=None), dict(gamma=None), dict(beta=None), dict(y=None),
                dict(mean=None), dict(rstd=None), dict(y=A), dict(h=D), dict(mean=F), dict(res=D), dict(h=C)):
        assert fwd(**bad) == BAD, bad
    assert fwd(rows=0) == L.OK

    n = ctypes.c_int64()
    assert lib.poseidon_norm_workspace(-1, 8, ctypes.byref(n)) == BAD
    assert lib.poseidon_norm_workspace(4, 8, None) == BAD

    def bwd(dy=A, h=B, gamma=C, mean=D, rstd=E, dres=None, rows=4, cols=8, dtype=L.F32, p=0.0, rng=None, dx=None, dh=F,
            dgamma=ctypes.c_void_p(0x20000000), dbeta=ctypes.c_void_p(0x21000000), ws=ctypes.c_void_p(0x22000000),
            size=1 << 20):
        return lib.poseidon_norm_backward(dy, h, gamma, mean, rstd, dres, rows, cols, dtype, p, rng, dx, dh, dgamma,
                                          dbeta, ws, size, None)

    for bad in (dict(rows=-1), dict(cols=-1), dict(cols=0), dict(dtype=-1), dict(p=NAN), dict(p=0.5, rng=G),
                dict(p=0.5, dx=G), dict(dy=None), dict(h=None), dict(gamma=None), dict(mean=None), dict(rstd=None),
                dict(dh=None), dict(dgamma=None), dict(dbeta=None), dict(ws=None), dict(size=8),
                dict(ws=ctypes.c_void_p(0x22000004)), dict(dh=A), dict(dgamma=C), dict(dbeta=F), dict(ws=A),
                dict(p=0.5, rng=G, dx=F)):
        assert bwd(**bad) == BAD, bad
    assert bwd(rows=0, cols=0) == L.OK


def test_xent_refusals():
    lib = L.lib()
    n = ctypes.c_int64()

    def size(op=L.XENT_FORWARD, T=4, V=9, D=8, dtype=L.F32, out=ctypes.byref(n)):
        return lib.poseidon_xent_workspace(op, A, B, T, V, D, dtype, out)

    assert size() == L.OK and n.value > 0
    sizes = (dict(T=-1), dict(V=0), dict(D=0), dict(dtype=3), dict(T=2 ** 24 + 1), dict(V=2 ** 24 + 1),
             dict(D=2 ** 20 + 1), dict(T=2 ** 20, V=2 ** 20))
    for bad in sizes + (dict(op=3), dict(op=-1), dict(out=None)):
        assert size(**bad) == BAD, bad
    big = 1 << 30
    w = ctypes.c_void_p(0x100000000)

    def fwd(X=A, W=B, t=C, T=4, V=9, D=8, dtype=L.F32, loss=ctypes.c_void_p(0x5000000), lse=E, ws=w, size=big):
        return lib.poseidon_xent_forward(X, W, t, T, V, D, dtype, loss, lse, ws, size, None)

    for bad in sizes + (dict(X=None), dict(W=None), dict(t=None), dict(loss=None), dict(lse=None), dict(ws=None),
                        dict(size=0), dict(ws=ctypes.c_void_p(0x100000008)), dict(loss=A), dict(loss=E), dict(lse=w)):
        if bad.get("loss") is E:
            bad = dict(loss=E, lse=E)
        assert fwd(**bad) == BAD, bad
    assert fwd(T=0) == L.OK

    def bwd(X=A, W=B, t=C, lse=D, dloss=E, T=4, V=9, D_=8, dtype=L.F32, dX=F, dW=G, ws=w, size=big):
        return lib.poseidon_xent_backward(X, W, t, lse, dloss, T, V, D_, dtype, dX, dW, ws, size, None)

    for bad in (dict(X=None), dict(W=None), dict(t=None), dict(lse=None), dict(dloss=None), dict(dX=None),
                dict(dW=None), dict(dX=A), dict(dW=B), dict(dW=F), dict(ws=A), dict(size=1), dict(T=-1), dict(V=0)):
        assert bwd(**bad) == BAD, bad

    def fac(X=A, W=B, t=C, dloss=D, T=4, V=9, D_=8, dtype=L.BF16, loss=E, U=F, dX=G, ws=w, size=big):
        return lib.poseidon_xent_factor(X, W, t, dloss, T, V, D_, dtype, loss, U, dX, ws, size, None)

    for bad in (dict(X=None), dict(W=None), dict(t=None), dict(dloss=None), dict(loss=None), dict(U=None),
                dict(dX=None), dict(U=A), dict(dX=F), dict(ws=B), dict(size=1), dict(D_=0), dict(dtype=9)):
        assert fac(**bad) == BAD, bad
    assert fac(T=0) == L.OK


def test_workspace_follows_the_arrays_boundaries():
    """A weight on 16-byte rows is read as it is; one that is not is laid out
    again, and the workspace says so."""
    lib, n = L.lib(), ctypes.c_int64()

    def size(W, D, dtype=L.BF16):
        assert lib.poseidon_xent_workspace(L.XENT_FORWARD, A, ctypes.c_void_p(W), 8, 1000, D, dtype,
                                           ctypes.byref(n)) == L.OK
        return n.value

    assert size(0x1000, 64) < 1000 * 64 * 2 <= size(0x1002, 64)
    assert size(0x1000, 65) >= 1000 * 65 * 2


def test_binding_refuses_what_it_cannot_hand_over():
    x, w, t = torch.zeros(4, 8), torch.zeros(9, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: api.xent_forward(x, w, t), lambda: api.norm_forward(x, torch.ones(8), torch.ones(8)),
                 lambda: api.dropout(x, 0.0, None)):
        with pytest.raises(ValueError, match="HIP device"):
            call()
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        api.dropout(x.double(), 0.0, None)
    with pytest.raises(TypeError):
        api.xent_forward([1.0], w, t)


@pytest.mark.parametrize("p", [-0.1, 1.1, NAN])
def test_binding_checks_p(p):
    with pytest.raises(ValueError, match="p must lie"):
        api._rng(None, p)


def test_binding_asks_for_the_generator():
    with pytest.raises(ValueError, match="rng"):
        api._rng(None, 0.1)
    assert api._rng(None, 0.0) is False
    with pytest.raises(TypeError):
        api._rng(torch.zeros(2), 0.1)


def test_xent_limits_each_on_its_own():
    """Rows, classes, features and logits at their limits and one past them, the
    others small."""
    lib, n = L.lib(), ctypes.c_int64()

    def size(T, V, D, dtype=L.BF16, op=L.XENT_FORWARD):
        return lib.poseidon_xent_workspace(op, A, B, T, V, D, dtype, ctypes.byref(n))

    for op in (L.XENT_FORWARD, L.XENT_BACKWARD, L.XENT_FACTOR):
        for dtype in (L.F32, L.BF16):
            assert size(2 ** 24, 2, 1, dtype, op) == L.OK and size(2 ** 24 + 1, 2, 1, dtype, op) == BAD
            assert size(2, 2 ** 21, 1, dtype, op) == L.OK and size(2, 2 ** 21 + 1, 1, dtype, op) == BAD
            assert size(2, 2, 2 ** 20, dtype, op) == L.OK and size(2, 2, 2 ** 20 + 1, dtype, op) == BAD
            assert size(2 ** 17, 2 ** 20, 1, dtype, op) == L.OK and size(2 ** 17 + 1, 2 ** 20, 1, dtype, op) == BAD


@pytest.mark.parametrize("W,D,copied", [(0x1000, 66, False), (0x1004, 66, False), (0x1002, 66, True), (0x1004, 64, False),
                                        (0x1000, 65, True), (0x1004, 65, True)])
def test_a_weight_on_rows_of_4_bytes_is_not_copied(W, D, copied):
    """bf16 rows that all start on 4-byte boundaries are read as they are, on
    16-byte boundaries or not; others are laid out again in the workspace.  fp32
    rows always are on them."""
    lib, n = L.lib(), ctypes.c_int64()
    V = 1000
    for op in (L.XENT_FORWARD, L.XENT_BACKWARD, L.XENT_FACTOR):
        got = []
        for at in (0x1000 if D % 2 == 0 else None, W):
            if at is None:
                got.append(None)
                continue
            assert lib.poseidon_xent_workspace(op, A, ctypes.c_void_p(at), 8, V, D, L.BF16, ctypes.byref(n)) == L.OK
            got.append(n.value)
        if copied:
            assert got[1] >= V * D * 2 + (got[0] or 0)
        else:
            assert got[1] == got[0]
        assert lib.poseidon_xent_workspace(op, A, ctypes.c_void_p(0x1000), 8, V, D, L.F32, ctypes.byref(n)) == L.OK
        aligned = n.value
        assert lib.poseidon_xent_workspace(op, A, ctypes.c_void_p(0x1004), 8, V, D, L.F32, ctypes.byref(n)) == L.OK
        assert n.value == aligned
