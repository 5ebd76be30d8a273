"""The float64 references of layer norm and attention: their gradients against differences of their values, and
the host-side refusals of the entry points."""
import ctypes as ct
import os

import numpy as np
import pytest

from tests import attention_ref as ref

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2007_16100_amd", "libspv.so")


def differences(f, x, h=1e-5):
    """d f / d x entry by entry, central differences."""
    g = np.zeros(x.shape)
    for idx in np.ndindex(x.shape):
        old = x[idx]
        x[idx] = old + h
        a = f()
        x[idx] = old - h
        b = f()
        x[idx] = old
        g[idx] = (a - b) / (2 * h)
    return g


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, dy, res = rng.normal(1.0, 2.0, (4, 7)), rng.normal(size=(4, 7)), rng.normal(size=(4, 7))
    g, b = rng.normal(1.0, 0.3, 7), rng.normal(size=7)
    dx, dg, db = ref.norm_backward(dy, x, g, 1e-5, res)

    def f():
        return (ref.norm(x, g, b, 1e-5)[2] * dy).sum() + (x * res).sum()
    for got, arg in ((dx, x), (dg, g), (db, b)):
        np.testing.assert_allclose(got, differences(f, arg), rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("cap", [0.0, 1.5])
@pytest.mark.parametrize("bias", [False, True])
def test_attention_gradient_against_differences(cap, bias):
    rng = np.random.default_rng(2)
    q_off, k_off = [0, 3, 3, 5, 6], [0, 4, 6, 6, 9]  # a scan without queries, one without keys
    q, dout = rng.normal(size=(6, 4, 3)), rng.normal(size=(6, 4, 3))
    k, v = rng.normal(size=(9, 2, 3)), rng.normal(size=(9, 2, 3))
    qc, kc = rng.integers(-5, 6, (6, 4)), rng.integers(-5, 6, (9, 4))
    kw = dict(scale=0.9, cap=cap)
    if bias:
        kw.update(qc=qc, kc=kc, slopes=np.array([0.1, 0.2, 0.3, 0.4]))
    R = ref.attention(q, k, v, q_off, k_off, dout=dout, **kw)
    assert np.all(R["out"][3:5] == 0) and np.all(R["lse"][3:5] == -np.inf) and np.all(R["dq"][3:5] == 0)
    assert np.all(R["dk"][4:6] == 0) and np.all(R["dv"][4:6] == 0)

    def f():
        return (ref.attention(q, k, v, q_off, k_off, **kw)["out"] * dout).sum()
    for got, arg in ((R["dq"], q), (R["dk"], k), (R["dv"], v)):
        np.testing.assert_allclose(got, differences(f, arg), rtol=1e-5, atol=1e-7)


@pytest.mark.skipif(not os.path.exists(LIB), reason="libspv.so not built")
def test_layer_norm_refusals():
    from paper_2007_16100_amd import spv
    L, P, big, ws = spv.lib(), ct.c_void_p(4096), 1 << 30, ct.c_void_p(256)
    bad = spv.SPV_ERR_INVALID_ARG

    def fwd(x=P, m=4, C=8, eps=1e-5, out=P, dt=1):
        return L.spv_layer_norm(None, x, None, m, C, None, None, eps, out, dt)
    for kw in (dict(x=None), dict(out=None), dict(m=-1), dict(m=1 << 31), dict(C=0), dict(eps=0.0), dict(eps=-1.0),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(dt=3)):
        assert fwd(**kw) == bad, kw
    assert fwd(x=None, out=None, m=0) == spv.SPV_OK

    def bwd(w=ws, nb=big, dy=P, x=P, m=4, C=8, eps=1e-5, dx=ct.c_void_p(8192), dg=P, dt=1):
        return L.spv_layer_norm_backward(None, w, nb, dy, x, None, m, C, None, eps, None, dx, dg, None, dt)
    for kw in (dict(w=None), dict(w=ct.c_void_p(16)), dict(dy=None), dict(x=None), dict(m=-1), dict(C=0),
               dict(eps=0.0), dict(dt=-1), dict(dx=P)):
        assert bwd(**kw) == bad, kw
    assert bwd(nb=16) == spv.SPV_ERR_CAPACITY
    assert bwd(w=None, dg=None, m=0) == spv.SPV_OK
    assert L.spv_layer_norm_backward_workspace_bytes(-1, 8) == 0
    assert L.spv_layer_norm_backward_workspace_bytes(4, 0) == 0
    assert L.spv_layer_norm_backward_workspace_bytes(1000, 96) > 0


@pytest.mark.skipif(not os.path.exists(LIB), reason="libspv.so not built")
def test_attention_refusals():
    from paper_2007_16100_amd import spv
    L, P, ws, big = spv.lib(), 1 << 20, ct.c_void_p(256), 1 << 40
    bad, unsup = spv.SPV_ERR_INVALID_ARG, spv.SPV_ERR_UNSUPPORTED

    def params(H=4, Hkv=2, D=32, B=2, scale=0.1, cap=0.0, q_off=P, k_off=P, qc=None, kc=None, slopes=None):
        return spv.AttentionParams(H, Hkv, D, B, scale, cap, q_off, k_off, qc, kc, slopes)

    def fwd(p=None, q=P, ldq=128, nq=4, k=2 * P, ldk=64, v=3 * P, ldv=64, nk=6, out=4 * P, ldo=128, dt=1, w=ws, nb=big,
            **kw):
        p = params(**kw) if p is None else p
        return L.spv_attention(None, w, nb, ct.byref(p), q, ldq, nq, k, ldk, v, ldv, nk, out, ldo, None, dt)
    for kw in (dict(H=0), dict(Hkv=0), dict(H=3), dict(D=0), dict(D=-8), dict(B=-1), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0),
               dict(cap=float("nan")), dict(cap=float("inf")), dict(q_off=None), dict(k_off=None), dict(qc=P),
               dict(qc=P, kc=P), dict(slopes=P), dict(qc=P + 4, kc=P, slopes=P), dict(q=None), dict(k=None),
               dict(v=None), dict(out=None), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8),
               dict(ldq=120), dict(ldq=132), dict(ldk=56), dict(ldv=56), dict(ldo=64), dict(nq=-1), dict(nk=-1),
               dict(nq=1 << 31), dict(nk=1 << 31), dict(dt=5), dict(out=P), dict(out=2 * P), dict(out=3 * P)):
        assert fwd(**kw) == bad, kw
    assert L.spv_attention(None, ws, big, None, P, 128, 4, P, 64, P, 64, 6, 4 * P, 128, None, 1) == bad
    for D in (12, 136, 256):
        assert fwd(D=D, ldq=4 * 256, ldk=2 * 256, ldv=2 * 256, ldo=4 * 256) == unsup
    assert fwd(nq=0, q=None, out=None) == spv.SPV_OK
    assert fwd(B=0, q_off=None, k_off=None) == spv.SPV_OK
    # rows of 32 MiB and more, and more workgroups than a grid is given
    for dt, ld in ((0, 1 << 23), (1, 1 << 24), (2, 1 << 24)):
        for name in ("ldq", "ldk", "ldv", "ldo"):
            assert fwd(dt=dt, **{name: ld}) == bad, (dt, name)
    assert fwd(nq=(1 << 31) - 1) == unsup and fwd(nk=(1 << 31) - 1) == unsup

    def bwd(dq=5 * P, dk=6 * P, dv=7 * P, lse=8 * P, dout=9 * P, lddo=128, lddq=128, lddk=64, lddv=64, w=ws, nb=big,
            nq=4):
        p = params()
        return L.spv_attention_backward(None, w, nb, ct.byref(p), P, 128, nq, 2 * P, 64, 3 * P, 64, 6, 4 * P, 128, lse,
                                        dout, lddo, dq, lddq, dk, lddk, dv, lddv, 1)
    for kw in (dict(dq=None), dict(dk=None), dict(dv=None), dict(lse=None), dict(dout=None), dict(dq=P),
               dict(dk=2 * P), dict(dv=9 * P), dict(dq=4 * P), dict(dk=7 * P), dict(dq=5 * P + 8), dict(dout=9 * P + 2),
               dict(lddo=120), dict(lddq=124), dict(lddk=32), dict(lddv=68), dict(w=None), dict(w=ct.c_void_p(64))):
        assert bwd(**kw) == bad, kw
    assert bwd(nb=8) == spv.SPV_ERR_CAPACITY
    p = params(D=12)
    assert L.spv_attention_workspace_bytes(ct.byref(p), 4, 6, 1) == 0
    p = params()
    assert L.spv_attention_backward_workspace_bytes(ct.byref(p), -1, 6, 1) == 0
    assert L.spv_attention_backward_workspace_bytes(ct.byref(p), 1000, 6, 1) >= 4 * 1000 * 4
