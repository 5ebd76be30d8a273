"""Rows past 2^31 elements: what the calls give for the last ones is what they give for those alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu
M, C, LAST = (1 << 26) + 1000, 32, 1000  # 2.1e9 values


@pytest.fixture(scope="module")
def spv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2007_16100_amd import spv as s
    s.lib()
    return s


def rows(seed, shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def test_rows_in_8_bits_and_their_weight_gradient(spv):
    x = torch.zeros(M, C, dtype=torch.bfloat16, device="cuda")
    x[-LAST:] = rows(1, (LAST, C))
    saved = spv.spv_checkpoint8(x)
    few = spv.spv_checkpoint8(x[-LAST:].contiguous())
    assert torch.equal(saved.codes[-LAST:], few.codes) and torch.equal(saved.exps[-LAST:], few.exps)
    assert not bool(saved.codes[:LAST].any())
    x.fill_(7.0)
    spv.spv_checkpoint8_read(saved, out=x)
    assert torch.equal(x[-LAST:], spv.spv_checkpoint8_read(few)) and not bool(x[:-LAST].any())
    da = x  # any rows: those of zeros in front add nothing
    dW = spv.spv_linear_backward8(spv.Workspace.for_linear_backward8(M, C, C), saved, da)
    want = spv.spv_checkpoint8_read(few).double().t() @ da[-LAST:].double()
    assert (dW.double() - want).abs().max() <= 2.0 ** -24 * 2 * (LAST + 16) * want.abs().max() * 8


def test_group_norm_and_its_backward(spv):
    x = torch.zeros(M, C, dtype=torch.bfloat16, device="cuda")
    x[-LAST:] = rows(2, (LAST, C))
    off = torch.tensor([0, M - LAST, M], dtype=torch.int32, device="cuda")
    ws = spv.Workspace.for_group_norm_backward(M, C, 4, 2)
    y, stat, saved = spv.spv_group_norm(ws, x, off, 4, act="silu", want_stat=True, want_checkpoint=True)
    few = x[-LAST:].double().view(LAST, 4, 8)
    var, mean = torch.var_mean(few, dim=(0, 2), correction=0, keepdim=True)
    r = 1.0 / torch.sqrt(var + 1e-5)
    z = ((few - mean) * r).view(LAST, C)
    want = torch.nn.functional.silu(z)
    assert (y[-LAST:].double() - want).abs().max() <= 2.0 ** -8 * want.abs().max()
    assert not bool(y[:-LAST].any()) and torch.equal(saved.codes[-LAST:], spv.spv_checkpoint8(x[-LAST:].contiguous()).codes)
    dy = y
    dx, dgamma, dbeta = spv.spv_group_norm_backward(ws, dy, x, off, 4, stat, act="silu")
    s = torch.sigmoid(z)
    gz = (dy[-LAST:].double() * s * (1 + z * (1 - s))).view(LAST, 4, 8)
    xh = z.view(LAST, 4, 8)
    g = (r * (gz - gz.mean((0, 2), keepdim=True) - xh * (gz * xh).mean((0, 2), keepdim=True))).view(LAST, C)
    assert (dx[-LAST:].double() - g).abs().max() <= 2.0 ** -8 * g.abs().max()
    assert (dbeta.double() - gz.sum(0).view(C)).abs().max() <= 2.0 ** -24 * LAST * gz.abs().max() * 8
    assert (dgamma.double() - (gz * xh).sum(0).view(C)).abs().max() <= 2.0 ** -24 * LAST * (gz * xh).abs().max() * 8


def test_rotary_positions(spv):
    n = (1 << 28) + 1000
    q = torch.zeros(n, 1, 8, dtype=torch.bfloat16, device="cuda")
    q[-LAST:] = rows(3, (LAST, 1, 8))
    c = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
    c[-LAST:] = torch.randint(-500, 500, (LAST, 4), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()
    p = spv.make_rope_params(8, spv.rope_freqs((2, 1, 1)), (2, 1, 1))
    want = spv.spv_rope(p, c[-LAST:].contiguous(), q[-LAST:].contiguous())
    got = spv.spv_rope(p, c, q, outs=(q,))
    assert torch.equal(got[-LAST:], want) and not bool(got[:-LAST].any())


def test_more_workgroups_than_an_axis_of_the_grid_holds(spv):
    """2^24 workgroups of 256 threads and more: short heads, and float32 rows of one vector."""
    n = (1 << 30) + 1000
    q = torch.zeros(n, 1, 8, dtype=torch.bfloat16, device="cuda")
    c = torch.zeros(n, 4, dtype=torch.int32, device="cuda")
    p = spv.make_rope_params(8, spv.rope_freqs((2, 1, 1)), (2, 1, 1))
    places = (0, (1 << 29) - LAST, 1 << 29, n - LAST)
    for i, r0 in enumerate(places):
        q[r0:r0 + LAST] = rows(5 + i, (LAST, 1, 8))
        c[r0:r0 + LAST] = torch.randint(-500, 500, (LAST, 4), generator=torch.Generator().manual_seed(i), dtype=torch.int32).cuda()
    want = [spv.spv_rope(p, c[r0:r0 + LAST].contiguous(), q[r0:r0 + LAST].contiguous()) for r0 in places]
    spv.spv_rope(p, c, q, outs=(q,))
    for r0, w in zip(places, want):
        assert torch.equal(q[r0:r0 + LAST], w)
    del q, c
    m = (1 << 31) - 1
    x = torch.zeros(m, 4, device="cuda")
    places = (0, (1 << 30) - LAST, 1 << 30, m - LAST)
    for i, r0 in enumerate(places):
        x[r0:r0 + LAST] = rows(9 + i, (LAST, 4), torch.float32)
    saved = spv.spv_checkpoint8(x)
    want = [spv.spv_checkpoint8(x[r0:r0 + LAST].contiguous()) for r0 in places]
    for r0, w in zip(places, want):
        assert torch.equal(saved.codes[r0:r0 + LAST], w.codes) and torch.equal(saved.exps[r0:r0 + LAST], w.exps)
    spv.spv_checkpoint8_read(saved, out=x)
    for r0, w in zip(places, want):
        assert torch.equal(x[r0:r0 + LAST], spv.spv_checkpoint8_read(w))


def test_group_norm_of_as_many_scans_as_it_takes(spv):
    """2^22 scans of one row and two by turns: the first and the last ones are what they are alone."""
    B, G, E = 1 << 22, 2, 2.0 ** -24
    off = (torch.arange(B + 1) * 3 // 2).to(torch.int32).cuda()
    m = B * 3 // 2
    x = torch.randn(m, 8, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    ws = spv.Workspace.for_group_norm_backward(m, 8, G, B)
    y, stat = spv.spv_group_norm(ws, x, off, G, want_stat=True)
    dx, dgamma, dbeta = spv.spv_group_norm_backward(ws, x, x, off, G, stat)
    for r0, b in ((0, 0), (m - 3000, B - 2000)):
        o, few, st = (off[b:b + 2001] - r0).contiguous(), x[r0:r0 + 3000].contiguous(), stat[b:b + 2000].contiguous()
        w = spv.Workspace.for_group_norm_backward(3000, 8, G, 2000)
        yw, sw = spv.spv_group_norm(w, few, o, G, want_stat=True)
        X, Y, R = float(few.abs().max()), float(yw.abs().max()), float(sw[..., 1].max())
        # of 8 values at most: a mean and a deviation off by d, r by d R + 16 E of itself, each side
        d = 10 * E * X
        assert (st[..., 0] - sw[..., 0]).abs().max() <= 2 * d
        assert ((st[..., 1] - sw[..., 1]) / sw[..., 1]).abs().max() <= 2 * (d * R + 16 * E)
        assert (y[r0:r0 + 3000] - yw).abs().max() <= 2 * (R * d + (d * R + 16 * E) * Y)
        # from the same stat: xh = x r - mu r off by h, the means by 8 E X and X h + 8 E X Y
        h = 3 * E * X * R
        dw = spv.spv_group_norm_backward(w, few, few, o, G, st)[0]
        assert (dx[r0:r0 + 3000] - dw).abs().max() <= 2 * R * X * (9 * E + 2 * h * Y + 8 * E * Y * Y + 4 * E * (2 + Y * Y))
    mu, r = (t.repeat_interleave(off.diff().long(), 0).repeat_interleave(4, 1).double() for t in (stat[..., 0], stat[..., 1]))
    xd, yd = x.double(), y.double()
    # a term x xh: xh off by roundings of x r, of mu r and of itself
    assert ((dgamma.double() - (xd * yd).sum(0)).abs() <= 8 * E * (xd.abs() * ((xd.abs() + mu.abs()) * r + yd.abs())).sum(0)).all()
    assert ((dbeta.double() - xd.sum(0)).abs() <= 8 * E * xd.abs().sum(0)).all()
