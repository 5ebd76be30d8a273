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
