"""Layer norm and its backward on the GPU against the float64 reference, within bounds derived from the kernels'
roundings (tests/attention_ref.py)."""
import numpy as np
import pytest
import torch

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def spv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2007_16100_amd import spv as s
    s.lib()
    return s


def arr(t):
    return t.detach().double().cpu().numpy()


def within(got, want, tol, what):
    err = np.abs(got - want)
    assert np.all(err <= tol), (what, float(np.max(err / tol)))


def inputs(m, C, dtype, seed, mean=0.5, std=2.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(m, C, generator=g) * std + mean).to(TD[dtype])
    dy, res = (torch.randn(m, C, generator=g).to(TD[dtype]) for _ in range(2))
    return [t.cuda() for t in (x, dy, res, 1.0 + 0.2 * torch.randn(C, generator=g), torch.randn(C, generator=g))]


SHAPES = [(1, 1), (1, 8), (3, 7), (5, 19), (2, 33), (64, 32), (65, 64), (127, 96), (1000, 96), (33, 100), (257, 128),
          (40, 192), (513, 256), (9, 520), (3, 1024), (5, 2048), (2, 4100), (70001, 16)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,C", SHAPES)
def test_norm_and_backward(spv, m, C, dtype):
    print(f"norm m={m} C={C} {dtype}", flush=True)
    x, dy, res, g, b = inputs(m, C, dtype, 7 * m + C)
    ws = spv.Workspace.for_layer_norm_backward(m, C)
    y = spv.spv_layer_norm(x, g, b)
    dx, dg, db = spv.spv_layer_norm_backward(ws, dy, x, g, dres=res)
    X, DY, R, G, B = map(arr, (x, dy, res, g, b))
    t = ref.norm_bounds(DY, X, G, B, 1e-5, R, dtype)
    within(arr(y), ref.norm(X, G, B, 1e-5)[2], t[0], "y")
    for got, want, tol, what in zip((dx, dg, db), ref.norm_backward(DY, X, G, 1e-5, R), t[1:], ("dx", "dg", "db")):
        within(arr(got), want, tol, what)
    again = spv.spv_layer_norm_backward(ws, dy, x, g, dres=res)
    for p, q in zip((dx, dg, db), again):
        assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_far_from_zero_and_flat_rows(spv, dtype):
    """Rows far from zero keep their deviations; a row of equal values gives beta and, with eps, a finite dx."""
    x, dy, _, g, b = inputs(50, 96, dtype, 3, mean=300.0, std=1.5)
    x[7] = 3.25
    x[8] = 0.0
    X, DY, G, B = map(arr, (x, dy, g, b))
    y = spv.spv_layer_norm(x, g, b)
    t = ref.norm_bounds(DY, X, G, B, 1e-5, None, dtype)
    within(arr(y), ref.norm(X, G, B, 1e-5)[2], t[0], "y")
    assert torch.equal(y[7], b.to(x.dtype)) and torch.equal(y[8], b.to(x.dtype))
    dx, dg, db = spv.spv_layer_norm_backward(spv.Workspace.for_layer_norm_backward(50, 96), dy, x, g)
    assert torch.isfinite(dx.float()).all() and torch.isfinite(dg).all()
    within(arr(db), DY.sum(0), t[3], "db")


def test_norm_options(spv):
    """No gamma or beta, in place, a row count on the device, non-finite rows that stay where they are, odd pointers."""
    for C in (96, 50):
        x, dy, res, g, b = inputs(300, C, "bf16", 11)
        ws = spv.Workspace.for_layer_norm_backward(300, C)
        one, zero = torch.ones_like(g), torch.zeros_like(b)
        assert torch.equal(spv.spv_layer_norm(x), spv.spv_layer_norm(x, one, zero))
        full = spv.spv_layer_norm(x, g, b)
        live = torch.tensor([211], dtype=torch.int64, device="cuda")
        out = torch.full_like(x, 9.0)
        spv.spv_layer_norm(x, g, b, m_dev=live, out=out)
        assert torch.equal(out[:211], full[:211]) and bool((out[211:] == 9.0).all())
        dx, dg, db = spv.spv_layer_norm_backward(ws, dy, x, g, dres=res, m_dev=live)
        dx2, dg2, db2 = spv.spv_layer_norm_backward(ws, dy[:211].contiguous(), x[:211].contiguous(), g,
                                                    dres=res[:211].contiguous())
        assert torch.equal(dx[:211], dx2)
        t = ref.norm_bounds(arr(dy[:211]), arr(x[:211]), arr(g), arr(b), 1e-5, arr(res[:211]), "bf16")
        for got, want, tol in ((dg, dg2, t[2]), (db, db2, t[3])):
            within(arr(got), arr(want), 2 * tol, "column sums under a device count")
        y = x.clone()
        assert torch.equal(spv.spv_layer_norm(y, g, b, out=y), full)
        x[5, 3], x[9, 0] = float("nan"), float("inf")
        bad = spv.spv_layer_norm(x, g, b)
        assert bool(torch.isnan(bad[5].float()).all()) and bool(torch.isnan(bad[9].float()).any())
        keep = [i for i in range(300) if i not in (5, 9)]
        assert torch.equal(bad[keep], full[keep])
    # a row start that is not 16-byte aligned takes the element-wise path: the same values within the bounds
    x, dy, res, g, b = inputs(40, 96, "bf16", 12)
    buf = torch.empty(40 * 96 + 1, dtype=x.dtype, device="cuda")
    odd = buf[1:].view(40, 96)
    odd.copy_(x)
    X = arr(x)
    t = ref.norm_bounds(arr(dy), X, arr(g), arr(b), 1e-5, None, "bf16")
    within(arr(spv.spv_layer_norm(odd, g, b)), ref.norm(X, arr(g), arr(b), 1e-5)[2], t[0], "unaligned")


def test_norm_empty_and_partial_outputs(spv):
    x, dy, _, g, b = inputs(0, 96, "f32", 1)
    ws = spv.Workspace.for_layer_norm_backward(0, 96)
    assert spv.spv_layer_norm(x, g, b).shape == (0, 96)
    dx, dg, db = spv.spv_layer_norm_backward(ws, dy, x, g)
    assert dx.shape == (0, 96) and not dg.any() and not db.any()
    with pytest.raises(ValueError):
        spv.spv_layer_norm(x, g[:5], b)
    with pytest.raises(ValueError):
        spv.spv_layer_norm(x, g, b, out=torch.empty(0, 96, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(spv.SpvError):
        spv.spv_layer_norm_backward(spv.Workspace(0), torch.zeros(9, 96, device="cuda"),
                                    torch.zeros(9, 96, device="cuda"), g)


def test_norm_gradient_against_differences(spv):
    """The slope of sum(y dy) along random directions, from the GPU's own float32 forward."""
    x, dy, _, g, b = inputs(30, 96, "f32", 21)
    ws = spv.Workspace.for_layer_norm_backward(30, 96)
    dx, dg, db = spv.spv_layer_norm_backward(ws, dy, x, g)

    def f(x, g, b):
        return (spv.spv_layer_norm(x, g, b).double() * dy.double()).sum().item()
    gen = torch.Generator().manual_seed(5)
    for grad, i in ((dx, 0), (dg, 1), (db, 2)):
        args = [x, g, b]
        d = torch.randn(args[i].shape, generator=gen).cuda()
        h = 1e-2
        up, dn = list(args), list(args)
        up[i], dn[i] = args[i] + h * d, args[i] - h * d
        slope = (f(*up) - f(*dn)) / (2 * h)
        want = (grad.double() * d.double()).sum().item()
        # third derivatives leave h^2, float32 noise sqrt(n) 2^-24 / h of the norms
        assert abs(slope - want) <= 2e-3 * (grad.double().norm() * d.double().norm()).item() / 10 + 0.05
