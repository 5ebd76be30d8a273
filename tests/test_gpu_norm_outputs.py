"""Layer norm's backward through the C ABI with its outputs in place of its inputs, and without some of them: the same
bits as with all of them apart, on the 16-byte kernels and the plain ones."""
import pytest
import torch

from tests.test_gpu_norm import inputs, spv  # noqa: F401 (spv: a fixture)

pytestmark = pytest.mark.gpu
SHAPES = [(300, 96), (3, 8), (1000, 256), (41, 19), (700, 50), (9, 511)]


def backward(s, ws, dy, x, g, dres, dx, dg, db):
    st = s.lib().spv_layer_norm_backward(s._stream(), ws.ptr if ws else None, ws.nbytes if ws else 0, s._ptr(dy), s._ptr(x),
                                         None, x.shape[0], x.shape[1], s._ptr(g), 1e-5, s._ptr(dres), s._ptr(dx), s._ptr(dg),
                                         s._ptr(db), s._DT[x.dtype])
    assert st == s.SPV_OK


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,C", SHAPES)
def test_dx_in_place(spv, m, C, dtype):  # noqa: F811
    x, dy, res, g, _ = inputs(m, C, dtype, m + C)
    ws = spv.Workspace.for_layer_norm_backward(m, C)
    for dres in (None, res):
        want = spv.spv_layer_norm_backward(ws, dy, x, g, dres=dres)
        for at in ("dy", "dres"):
            if at == "dres" and dres is None:
                continue
            t = dict(dy=dy.clone(), dres=None if dres is None else dres.clone())
            dg, db = torch.full((C,), 7.0, device="cuda"), torch.full((C,), 7.0, device="cuda")
            backward(spv, ws, t["dy"], x, g, t["dres"], t[at], dg, db)
            for a, b in zip((t[at], dg, db), want):
                assert torch.equal(a, b), at


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,C", SHAPES)
def test_some_outputs(spv, m, C, dtype):  # noqa: F811
    x, dy, res, g, _ = inputs(m, C, dtype, m + C + 1)
    ws = spv.Workspace.for_layer_norm_backward(m, C)
    want = spv.spv_layer_norm_backward(ws, dy, x, g, dres=res)
    for keep in range(8):
        out = [torch.full_like(t, 7.0) if keep >> i & 1 else None for i, t in enumerate(want)]
        # dx alone takes no workspace
        backward(spv, ws if keep & 6 else None, dy, x, g, res, *out)
        for a, b in zip(out, want):
            assert a is None or torch.equal(a, b), keep
