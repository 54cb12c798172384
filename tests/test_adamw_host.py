"""AdamW without a GPU: what its entry points refuse before any device work, and
the binding's own checks."""
import ctypes

import pytest
import torch

from paper_1706_03292_amd import _lib as L
from paper_1706_03292_amd import api

BAD = L.ERR_INVALID_ARG
NAN, INF = float("nan"), float("inf")
BASE = 0x100000000    # never dereferenced


def tensor(i=0, n=1000, **kw):
    at = BASE + i * 0x1000000
    f = {"W": at, "shards": at + 0x100000, "m": at + 0x200000, "v": at + 0x300000, "exponents": None, "copy": None,
         "sum": None, "n": n, "stride": n, "P": 2, "weight_decay": 0.1}
    f.update(kw)
    return L.PoseidonAdamwTensor(*[f[name] for name, _ in L.PoseidonAdamwTensor._fields_])


def create(*ts, dtype=L.F32, count=None):
    arr = (L.PoseidonAdamwTensor * max(1, len(ts)))(*ts)
    h = ctypes.c_void_p()
    rc = L.lib().poseidon_adamw_create(arr, len(ts) if count is None else count, dtype, ctypes.byref(h))
    assert (rc == L.OK) == bool(h.value)
    return rc, h


def made(*ts, **kw):
    rc, h = create(*ts, **kw)
    assert rc == L.OK
    return h


def test_descriptor_layout():
    assert ctypes.sizeof(L.PoseidonAdamwTensor) == 80 and L.PoseidonAdamwTensor.weight_decay.offset == 76
    assert ctypes.sizeof(L.PoseidonAdamwRule) == 72 and L.PoseidonAdamwRule.from_sums.offset == 64


def test_create():
    lib = L.lib()
    assert lib.poseidon_adamw_create(None, 0, L.F32, None) == BAD
    assert lib.poseidon_adamw_destroy(None) == L.OK
    for ts in ((), (tensor(),), (tensor(), tensor(1, n=0, W=None, shards=None, m=None, v=None), tensor(2, P=1, stride=0))):
        lib.poseidon_adamw_destroy(made(*ts))
    assert create(tensor(), count=-1)[0] == BAD
    assert create(tensor(), dtype=2)[0] == BAD
    h = ctypes.c_void_p()
    assert lib.poseidon_adamw_create(None, 1, L.F32, ctypes.byref(h)) == BAD
    for kw in ({"n": -1}, {"n": 2 ** 34 + 1}, {"P": 0}, {"P": 1025}, {"stride": 999}, {"stride": -1},
               {"stride": 2 ** 56}, {"W": None}, {"shards": None}, {"m": None}, {"v": None},
               {"weight_decay": -0.1}, {"weight_decay": NAN}, {"weight_decay": INF}):
        assert create(tensor(), tensor(1, **kw))[0] == BAD, kw


def test_written_arrays_may_not_meet():
    at = tensor().W
    for kw in ({"m": at + 3996}, {"v": at}, {"exponents": at + 4}, {"copy": at + 8}, {"sum": at},
               {"sum": at + 0x100000}, {"m": at + 0x300000}, {"shards": at + 3900}, {"shards": at - 4 * 1999}):
        assert create(tensor(**kw))[0] == BAD, kw
        assert create(tensor(), tensor(1, **kw))[0] == BAD, kw
    # side by side, and between two workers' rows
    ok = tensor(m=at + 4000, v=at + 8000, sum=at + 12000, copy=at + 16000)
    L.lib().poseidon_adamw_destroy(made(ok))
    L.lib().poseidon_adamw_destroy(made(tensor(shards=at - 4000, stride=2000)))
    # 8 bits: a byte a value
    L.lib().poseidon_adamw_destroy(made(tensor(m=at + 4000, v=at + 5000, exponents=at + 6000, copy=at + 6016)))
    assert create(tensor(m=at + 4000, v=at + 5000, exponents=at + 6000, copy=at + 6014))[0] == BAD
    # shards may be shared
    L.lib().poseidon_adamw_destroy(made(tensor(), tensor(1, shards=tensor().shards)))


def rule(**kw):
    f = {"lr": 0.1, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "step": 1, "clock": None, "scale": None, "rng": None,
         "from_sums": 0, "reserved": 0}
    f.update(kw)
    return L.PoseidonAdamwRule(*[f[name] for name, _ in L.PoseidonAdamwRule._fields_])


def test_step_refusals():
    f, h, empty = L.lib().poseidon_adamw_step, made(tensor()), made()
    assert f(None, rule(), None) == BAD and f(h, None, None) == BAD
    t = tensor()
    for kw in ({"lr": NAN}, {"lr": INF}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": NAN}, {"eps": 0.0},
               {"eps": -1.0}, {"eps": NAN}, {"eps": INF}, {"eps": 1e-60}, {"eps": 1e60}, {"step": 0}, {"step": -4},
               {"from_sums": 1}, {"from_sums": 2}, {"reserved": 1}, {"clock": t.W}, {"scale": t.m + 3996},
               {"rng": t.v - 8}):
        assert f(h, rule(**kw), None) == BAD, kw
    assert f(empty, rule(), None) == L.OK                       # nothing to launch
    assert f(empty, rule(from_sums=1), None) == L.OK
    assert f(empty, rule(step=0), None) == BAD
    assert f(empty, rule(step=0, lr=NAN, clock=64), None) == L.OK
    L.lib().poseidon_adamw_destroy(h), L.lib().poseidon_adamw_destroy(empty)


def test_values_refusals():
    f, h = L.lib().poseidon_adamw_values, made(tensor(), tensor(1, n=0))
    t = tensor()

    def ptrs(a, b=None):
        return (ctypes.c_void_p * 2)(a, b)

    far = BASE + 0x8000000
    assert f(None, ptrs(far), ptrs(far + 4000), None) == BAD
    assert f(h, None, ptrs(far), None) == BAD and f(h, ptrs(far), None, None) == BAD
    assert f(h, ptrs(far), ptrs(far + 3996), None) == BAD
    for p in (t.W, t.m, t.v + 3996, t.shards + 4000):
        assert f(h, ptrs(p), ptrs(far), None) == BAD and f(h, ptrs(far), ptrs(p), None) == BAD
    assert f(h, ptrs(None, far), ptrs(None, far), None) == L.OK     # nothing wanted of the tensor with values
    L.lib().poseidon_adamw_destroy(h)


def test_clip_refusals():
    lib = L.lib()
    h, size = made(tensor(), tensor(1, n=5000, stride=5000)), ctypes.c_int64()
    assert lib.poseidon_adamw_workspace(None, ctypes.byref(size)) == BAD
    assert lib.poseidon_adamw_workspace(h, None) == BAD
    assert lib.poseidon_adamw_workspace(h, ctypes.byref(size)) == L.OK and size.value > 0
    f, t, ws, out = lib.poseidon_adamw_clip, tensor(), BASE + 0x8000000, BASE + 0x9000000
    assert f(None, 1.0, out, ws, size, None) == BAD
    for most in (0.0, -1.0, NAN):
        assert f(h, most, out, ws, size, None) == BAD
    assert f(h, 1.0, None, ws, size, None) == BAD
    assert f(h, 1.0, out, None, size, None) == BAD
    assert f(h, 1.0, out, ws + 8, size, None) == BAD
    assert f(h, 1.0, out, ws, size.value - 1, None) == BAD
    assert f(h, 1.0, ws, ws, size, None) == BAD
    for p in (t.W, t.m, t.v, t.shards, t.shards + 4000):
        assert f(h, 1.0, p, ws, size, None) == BAD
        assert f(h, 1.0, out, p, size, None) == BAD
    lib.poseidon_adamw_destroy(h)


def test_the_binding_refuses():
    W = torch.zeros(8)
    t = {"W": W, "shards": torch.zeros(2, 8), **api.AdamW.moments(W)}
    with pytest.raises(ValueError, match="HIP device"):
        api.AdamW([t])
    with pytest.raises(TypeError):
        api.AdamW([{**t, "W": W.double()}])
    with pytest.raises(TypeError):
        api.AdamW([{**t, "W": [1.0]}])
    with pytest.raises(ValueError):
        api.AdamW.moments(W, 4)
    m = api.AdamW.moments(torch.zeros(3, 43), 8)
    assert m["m"].numel() == m["v"].numel() == 129 and m["exponents"].numel() == 4
