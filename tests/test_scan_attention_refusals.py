"""What the attention layer refuses before any kernel runs: types, widths and rows that its calls would read past."""
import pytest
import torch

from paper_2007_16100_amd import scan_attention
from paper_2007_16100_amd.scan_attention import ScanAttention

BF, F32 = torch.bfloat16, torch.float32


def params(C=64, H=4, K=2, D=16, dtype=BF, **other):
    P = dict(gamma=torch.ones(C), beta=torch.zeros(C), Wq=torch.zeros(C, H * D, dtype=dtype),
             Wk=torch.zeros(C, K * D, dtype=dtype), Wv=torch.zeros(C, K * D, dtype=dtype),
             Wo=torch.zeros(H * D, C, dtype=dtype))
    return dict(P, **other)


@pytest.fixture
def no_calls(monkeypatch):
    """Every call that would launch a kernel or take device memory fails the test."""
    def fail(name):
        def f(*a, **k):
            raise AssertionError(f"{name} was called")
        return f
    for name in ("spv_layer_norm", "spv_layer_norm_backward", "spv_linear", "spv_linear_backward", "spv_attention",
                 "spv_attention_backward", "Workspace"):
        monkeypatch.setattr(scan_attention.spv, name, fail(name))


@pytest.mark.parametrize("other", [
    dict(Wk=torch.zeros(64, 32, dtype=F32)), dict(Wv=torch.zeros(64, 32, dtype=torch.float16)),
    dict(Wo=torch.zeros(64, 64, dtype=F32)), dict(gamma=torch.ones(64, dtype=BF)), dict(beta=torch.zeros(64, dtype=BF)),
    dict(gamma=torch.ones(32)), dict(beta=torch.ones(64, 1)), dict(Wq=torch.zeros(64, 64, dtype=torch.float64)),
    dict(Wo=torch.zeros(64, 32, dtype=BF))])
def test_parameters_of_other_types_and_widths(no_calls, other):
    with pytest.raises(ValueError):
        ScanAttention(params(**other), 4, 2)


@pytest.mark.parametrize("heads,kv", [(0, None), (4, 0), (4, 3), (-4, 2), (3, 3)])
def test_heads(no_calls, heads, kv):
    with pytest.raises(ValueError):
        ScanAttention(params(), heads, kv)


@pytest.mark.parametrize("slopes", [torch.zeros(3), torch.zeros(4, dtype=BF), torch.zeros(4, 1)])
def test_slopes(no_calls, slopes):
    with pytest.raises(ValueError):
        ScanAttention(params(), 4, 2, slopes=slopes)


def test_features_and_tokens_of_other_types_and_widths(no_calls):
    layer, off = ScanAttention(params(), 4, 2), torch.tensor([0, 10], dtype=torch.int32)
    x, tok = torch.zeros(10, 64, dtype=BF), torch.zeros(2, 64, dtype=BF)
    for bad in (x.float(), x.half(), x[:, :32], x[:, :32].contiguous(), x.view(2, 5, 64), x.t()):
        with pytest.raises(ValueError):
            layer.forward(bad, off)
    for bad in (tok.float(), tok[:, :48].contiguous(), tok[0]):
        with pytest.raises(ValueError):
            layer.forward(x, off, tokens=bad, token_off=off)
    with pytest.raises(ValueError):  # tokens of which scans?
        layer.forward(x, off, tokens=tok)


def test_a_bias_without_coordinates(no_calls):
    layer, off = ScanAttention(params(), 4, 2, slopes=torch.ones(4)), torch.tensor([0, 10], dtype=torch.int32)
    x, tok = torch.zeros(10, 64, dtype=BF), torch.zeros(2, 64, dtype=BF)
    c = torch.zeros(10, 4, dtype=torch.int32)
    for kw in (dict(), dict(coords=c[:9]), dict(coords=c.long()), dict(coords=c, tokens=tok, token_off=off),
               dict(coords=c, tokens=tok, token_off=off, token_coords=c[:1])):
        with pytest.raises(ValueError):
            layer.forward(x, off, **kw)


def test_incoming_gradients_that_do_not_fit(no_calls):
    """dy is read for as many rows as x has, as x's type."""
    layer, x = ScanAttention(params(), 4, 2), torch.zeros(10, 64, dtype=BF)
    rows = torch.zeros(10, 4, 16, dtype=BF)
    saved = dict(x=x, h=x, q=rows, k=rows[:, :2], v=rows[:, :2], o=rows, lse=torch.zeros(10, 4), p=None, own=True)
    for dy in (x[:9], torch.zeros(10, 64), torch.zeros(10, 32, dtype=BF), torch.zeros(20, 64, dtype=BF),
               x.t().contiguous().t(), torch.zeros(640, dtype=BF)):
        with pytest.raises(ValueError):
            layer.backward(saved, dy)
    with pytest.raises(ValueError):
        layer.backward(dict(saved, own=False), x)
