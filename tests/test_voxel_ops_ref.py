"""The float64 references of rotary positions, group norm and rows in 8 bits against differences and definitions, and
what their entry points refuse, on the CPU."""
import ctypes as ct
import os

import numpy as np
import pytest
import torch

from paper_2007_16100_amd import spv
from tests import voxel_ops_ref as ref

built = pytest.mark.skipif(not os.path.exists(spv.LIB_PATH), reason="libspv.so not built")
P, WS, BIG = ct.c_void_p(4096), ct.c_void_p(256), 1 << 40


def far(i):
    return ct.c_void_p(4096 * (2 + i))


@pytest.mark.parametrize("halves", [False, True])
def test_rotation_depends_on_where_rows_stand_to_each_other(halves):
    rng = np.random.default_rng(1)
    f, sec = rng.uniform(0.01, 1.0, 5).astype(np.float32), (2, 1, 2)
    q, k = rng.standard_normal((2, 1, 1, 12))
    c, d = rng.integers(-500, 500, (2, 1, 4))
    shift = rng.integers(-9000, 9000, (1, 4))
    products = [(ref.rope(q, c + s, f, sec, halves)[0] * ref.rope(k, d + s, f, sec, halves)[0]).sum() for s in (0, shift)]
    assert abs(products[0] - products[1]) < 1e-9
    y = ref.rope(q, c, f, sec, halves)[0]
    assert np.allclose(ref.rope(y, c, f, sec, halves, inverse=True)[0], q, atol=1e-12)
    assert np.array_equal(y[..., 10:], q[..., 10:]) and not np.allclose(y[..., :10], q[..., :10])
    # the backward of a product with g is the rotation back of g
    g = rng.standard_normal(q.shape)
    back = ref.rope(g, c, f, sec, halves, inverse=True)[0]
    for j in range(12):
        e = np.zeros_like(q)
        e[..., j] = 1e-6
        diff = ((ref.rope(q + e, c, f, sec, halves)[0] - ref.rope(q - e, c, f, sec, halves)[0]) * g).sum() / 2e-6
        assert abs(diff - back[..., j].sum()) < 1e-8


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_group_norm_gradients_by_differences(kind):
    rng = np.random.default_rng(2)
    off, G, m, C = [1, 4, 4, 9, 10], 3, 11, 6
    x, dy, dres = rng.standard_normal((3, m, C))
    ga, be = rng.standard_normal((2, C))

    def loss(x, ga, be):
        y = ref.group_norm(x, off, G, ga, be, 1e-2, kind, "f32")["y"]
        return np.nansum(y * dy)
    R = ref.group_norm(x, off, G, ga, be, 1e-2, kind, "f32", dy, dres)
    assert np.isnan(R["dx"][[0, 10]]).all()
    for (i, j), want in np.ndenumerate(np.nan_to_num(R["dx"] - dres)):
        e = np.zeros_like(x)
        e[i, j] = 1e-6
        assert abs((loss(x + e, ga, be) - loss(x - e, ga, be)) / 2e-6 - want) < 1e-6
    for j in range(C):
        e = np.zeros(C)
        e[j] = 1e-6
        assert abs((loss(x, ga + e, be) - loss(x, ga - e, be)) / 2e-6 - R["dgamma"][j]) < 1e-6
        assert abs((loss(x, ga, be + e) - loss(x, ga, be - e)) / 2e-6 - R["dbeta"][j]) < 1e-6


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_rows_in_8_bits_are_within_a_step(dtype):
    rng = np.random.default_rng(3)
    t = torch.from_numpy(rng.standard_normal((40, 75)) * np.exp(rng.uniform(-5, 5, (40, 1))))
    td = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    t = t.to(td)
    x = t.double().numpy()
    x[3], x[4, 5], x[5, 7] = 0.0, np.inf, np.nan
    q, e, y = ref.codes(x, dtype)
    assert q.shape == x.shape and e.shape == (40, 3) and not y[3].any()
    assert np.isnan(y[4, 5]) and np.isnan(y[5, 7]) and np.isfinite(np.delete(y[4], 5)).all()
    ok = np.isfinite(x)
    assert np.array_equal(torch.from_numpy(y).to(td).double().numpy()[ok], y[ok])  # exact in the type
    blocks = np.pad(np.where(ok, x, 0), ((0, 0), (0, 21))).reshape(40, 3, 32)
    step = np.ldexp(1.0, e.astype(int) - 127)[..., None]
    err = np.abs(np.pad(np.where(ok, y - x, 0), ((0, 0), (0, 21)))).reshape(40, 3, 32)
    assert np.all(err <= np.where(np.abs(blocks) > 127.5 * step, step, step / 2))
    top = np.abs(blocks).max(2)
    assert np.all(top[top > 0] >= 64 * step[..., 0][top > 0]) and np.all(top < 128 * step[..., 0])


def rope(n=4, D=32, sections=(6, 6, 4), q=far(0), ldq=64, H=2, k=far(1), ldk=32, K=1, qo=far(2), ldqo=64, ko=far(3),
         ldko=32, coords=P, freqs=4096, dt=1):
    p = spv.RopeParams(D, (ct.c_int32 * 3)(*sections), 0, freqs)
    return spv.lib().spv_rope(None, ct.byref(p), coords, None, n, q, ldq, H, k, ldk, K, qo, ldqo, ko, ldko, 0, dt)


@built
def test_rope_refusals():
    bad = spv.SPV_ERR_INVALID_ARG
    assert rope(n=0) == spv.SPV_OK
    for kw in (dict(sections=(0, 0, 0)), dict(sections=(6, 6, 5)), dict(sections=(-1, 6, 6)), dict(D=0), dict(H=0),
               dict(K=-1), dict(n=-1), dict(n=1 << 31), dict(dt=3), dict(q=None), dict(qo=None), dict(k=None),
               dict(ko=None), dict(coords=None), dict(coords=ct.c_void_p(4100)), dict(freqs=None), dict(ldq=63),
               dict(ldq=56), dict(ldk=31), dict(ldqo=60), dict(ldko=16), dict(q=ct.c_void_p(8194)), dict(K=0),
               dict(qo=far(0), ldqo=128), dict(qo=far(1)), dict(ko=far(0)), dict(ko=far(2)), dict(ldq=1 << 25)):
        assert rope(**kw) == bad, kw
    for D in (12, 136):
        assert rope(D=D, sections=(2, 2, 2), ldq=1024, ldk=1024, ldqo=1024, ldko=1024) == spv.SPV_ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        spv.make_rope_params(32, torch.ones(15), (6, 6, 4))
    with pytest.raises(ValueError):
        spv.make_rope_params(32, torch.ones(16, dtype=torch.float64), (6, 6, 4))
    with pytest.raises(ValueError):
        spv.make_rope_params(32, torch.ones(16), (8, 8))


@built
def test_rows_in_8_bits_refusals():
    L, bad = spv.lib(), spv.SPV_ERR_INVALID_ARG
    assert L.spv_checkpoint8(None, None, None, 0, 8, None, None, 1) == spv.SPV_OK
    assert L.spv_checkpoint8_read(None, None, None, None, 0, 8, None, 1) == spv.SPV_OK
    for x, m, C, q, e, dt in ((None, 4, 8, far(1), far(2), 1), (P, -1, 8, far(1), far(2), 1), (P, 1 << 31, 8, far(1), far(2), 1),
                              (P, 4, 0, far(1), far(2), 1), (P, 4, 8, None, far(2), 1), (P, 4, 8, far(1), None, 1),
                              (P, 4, 8, far(1), far(2), 3), (P, 4, 8, P, far(2), 1), (P, 4, 8, far(1), P, 1),
                              (P, 4, 8, far(1), far(1), 1)):
        assert L.spv_checkpoint8(None, x, None, m, C, q, e, dt) == bad
        if q is None or e is None or q.value != e.value:
            assert L.spv_checkpoint8_read(None, q, e, None, m, C, x, dt) == bad

    def wg(ws=WS, nb=BIG, q=far(0), e=far(1), m=4, ci=8, da=far(2), co=8, dW=far(3), dt=1):
        return L.spv_linear_backward8(None, ws, nb, q, e, None, m, ci, da, co, dW, dt)
    for kw in (dict(ws=None), dict(ws=P.value + 16 and ct.c_void_p(16)), dict(q=None), dict(e=None), dict(m=-1), dict(ci=0),
               dict(co=0), dict(da=None), dict(dW=None), dict(dt=5), dict(dW=far(2)), dict(dW=far(0)), dict(dW=far(1))):
        assert wg(**kw) == bad, kw
    assert wg(nb=8) == spv.SPV_ERR_CAPACITY
    assert wg(ci=2048, co=1024) == spv.SPV_ERR_UNSUPPORTED
    assert L.spv_linear_backward8_workspace_bytes(10, 2048, 1024) == 0
    assert L.spv_linear_backward8_workspace_bytes(0, 8, 8) > 0


@built
def test_group_norm_refusals():
    L, bad = spv.lib(), spv.SPV_ERR_INVALID_ARG

    def fwd(ws=WS, nb=BIG, x=far(0), m=4, C=8, off=P, B=1, G=2, eps=1e-5, act=1, out=far(1), q=None, e=None, dt=1):
        return L.spv_group_norm(None, ws, nb, x, m, C, off, B, G, None, None, ct.c_float(eps), act, out, None, q, e, dt)

    def bwd(ws=WS, nb=BIG, dy=far(0), x=far(1), q=None, e=None, m=4, C=8, off=P, B=1, G=2, stat=far(2), act=1, dx=far(3),
            dt=1):
        return L.spv_group_norm_backward(None, ws, nb, dy, x, q, e, m, C, off, B, G, None, None, stat, act, None, dx, P, P,
                                         dt)
    for kw in (dict(ws=None), dict(x=None), dict(m=-1), dict(C=0), dict(off=None), dict(B=-1), dict(G=0), dict(G=3),
               dict(eps=0.0), dict(eps=float("nan")), dict(act=3), dict(act=-1), dict(out=None), dict(q=far(4)), dict(e=far(4)),
               dict(q=far(4), e=far(4)), dict(q=far(0), e=far(4)), dict(q=far(4), e=far(1)), dict(dt=3)):
        assert fwd(**kw) == bad, kw
    for kw in (dict(ws=None), dict(dy=None), dict(x=None), dict(q=far(4), e=far(5)), dict(x=None, q=far(4)), dict(e=far(4)),
               dict(stat=None), dict(off=None), dict(G=3), dict(act=3), dict(dx=far(1)), dict(x=None, q=far(3), e=far(4)),
               dict(x=None, q=far(4), e=far(3)), dict(dt=-1)):
        assert bwd(**kw) == bad, kw
    for f in (fwd, bwd):
        assert f(nb=8) == spv.SPV_ERR_CAPACITY
        assert f(C=65538, G=1) == spv.SPV_ERR_UNSUPPORTED
        assert f(B=(1 << 24) + 1) == spv.SPV_ERR_UNSUPPORTED
        assert f(B=(1 << 22) + 1) == f(B=1 << 17, C=512, G=512) == spv.SPV_ERR_UNSUPPORTED  # past a launch's 2^32 threads
    assert fwd(B=0, off=None) == spv.SPV_OK
    for f in (L.spv_group_norm_workspace_bytes, L.spv_group_norm_backward_workspace_bytes):
        assert f(10, 8, 3, 1) == 0 and f(-1, 8, 2, 1) == 0 and f(0, 8, 2, 0) >= 0


def test_binding_refusals(monkeypatch):
    """Shapes and types that the calls would read past."""
    monkeypatch.setattr(spv, "_here", lambda: -1)  # where the tensors of the CPU are
    monkeypatch.setattr(spv, "lib", lambda: (_ for _ in ()).throw(AssertionError("a call was made")))
    ws = type("W", (), dict(ptr=None, nbytes=0))()
    BF = torch.bfloat16
    x, off = torch.zeros(6, 64, dtype=BF), torch.tensor([0, 6], dtype=torch.int32)
    saved = spv.Checkpoint8.empty(6, 64, BF, "cpu")
    wrong = [spv.Checkpoint8(saved.codes[:5], saved.exps, BF), spv.Checkpoint8(saved.codes, saved.exps[:, :1], BF),
             spv.Checkpoint8(saved.codes.view(torch.uint8), saved.exps, BF)]
    for bad in wrong:
        with pytest.raises(ValueError):
            spv.spv_checkpoint8_read(bad)
        with pytest.raises(ValueError):
            spv.spv_linear_backward8(ws, bad, x)
    for da in (x[:5], x.float(), x.view(-1)):
        with pytest.raises(ValueError):
            spv.spv_linear_backward8(ws, saved, da)
    with pytest.raises(ValueError):
        spv.spv_checkpoint8(x, out=spv.Checkpoint8.empty(6, 32, BF, "cpu"))
    with pytest.raises(ValueError):
        spv.spv_checkpoint8(x, m_dev=torch.tensor([3], dtype=torch.int32))
    for kw in (dict(off=off.long()), dict(off=off.view(1, 2)), dict(act="gelu"), dict(out=x.float()),
               dict(gamma=torch.ones(32)), dict(beta=torch.ones(64, dtype=BF))):
        with pytest.raises(ValueError):
            spv.spv_group_norm(ws, x, kw.pop("off", off), 4, **kw)
    stat = torch.zeros(1, 4, 2)
    for kw in (dict(x=x[:5]), dict(x=x.float()), dict(x=spv.Checkpoint8.empty(6, 64, torch.float16, "cpu")),
               dict(x=spv.Checkpoint8.empty(5, 64, BF, "cpu")), dict(stat=stat[:, :3]), dict(stat=stat.double()),
               dict(dres=x[:5]), dict(act="tanh")):
        with pytest.raises(ValueError):
            spv.spv_group_norm_backward(ws, x, kw.pop("x", x), off, 4, kw.pop("stat", stat), **kw)


def test_tensors_of_another_device(monkeypatch):
    """A call runs on the current device's stream; tensors of another one are refused before it."""
    monkeypatch.setattr(spv, "_here", lambda: 0)
    monkeypatch.setattr(spv, "lib", lambda: (_ for _ in ()).throw(AssertionError("a call was made")))
    ws = type("W", (), dict(ptr=None, nbytes=0))()
    x, off, c = torch.zeros(6, 64), torch.tensor([0, 6], dtype=torch.int32), torch.zeros(6, 4, dtype=torch.int32)
    saved, p = spv.Checkpoint8.empty(6, 64, torch.float32, "cpu"), spv.RopeParams(32)
    p._keep = torch.ones(16)
    for f in (lambda: spv.spv_checkpoint8(x), lambda: spv.spv_checkpoint8_read(saved),
              lambda: spv.spv_linear_backward8(ws, saved, x), lambda: spv.spv_group_norm(ws, x, off, 4),
              lambda: spv.spv_group_norm_backward(ws, x, x, off, 4, torch.zeros(1, 4, 2)),
              lambda: spv.spv_rope(p, c, x.view(6, 2, 32))):
        with pytest.raises(ValueError, match="current device"):
            f()


@built
@pytest.mark.parametrize("C,G,B", [(96, 8, 1), (96, 8, 4), (96, 96, 3), (4096, 1, 1), (19, 19, 2), (1, 1, 1), (5000, 5, 2)])
def test_a_workspace_for_more_rows_serves_fewer(C, G, B):
    """The bytes asked for never fall as rows are added: a program makes its workspace once, for its largest batch."""
    L = spv.lib()
    rows = sorted({*range(3000), *(240 * k + d for k in range(12, 1300) for d in (-1, 0, 1)), *(1 << k for k in range(12, 31))})
    for f in (lambda m: L.spv_group_norm_workspace_bytes(m, C, G, B), lambda m: L.spv_group_norm_backward_workspace_bytes(m, C, G, B),
              lambda m: L.spv_linear_backward8_workspace_bytes(m, min(C, 256), 64)):
        sizes = [f(m) for m in rows]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0


def test_workspaces_of_another_device(monkeypatch):
    """A workspace is where the call runs, too."""
    monkeypatch.setattr(spv, "_here", lambda: -1)  # where the tensors of the CPU are
    monkeypatch.setattr(spv, "lib", lambda: (_ for _ in ()).throw(AssertionError("a call was made")))
    ws = spv.Workspace(1024, "meta")
    ws.buf = type("Buffer", (), dict(get_device=lambda self: 1))()
    x, off = torch.zeros(6, 64), torch.tensor([0, 6], dtype=torch.int32)
    saved = spv.Checkpoint8.empty(6, 64, torch.float32, "cpu")
    for f in (lambda: spv.spv_linear_backward8(ws, saved, x), lambda: spv.spv_group_norm(ws, x, off, 4),
              lambda: spv.spv_group_norm_backward(ws, x, x, off, 4, torch.zeros(1, 4, 2))):
        with pytest.raises(ValueError, match="workspace of the current device"):
            f()
