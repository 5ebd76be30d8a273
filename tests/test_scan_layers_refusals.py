"""What the layers with rotary positions, group norm and rows kept in 8 bits refuse before any kernel runs."""
import pytest
import torch

from paper_2007_16100_amd import scan_attention, scan_mlp, spv
from paper_2007_16100_amd.scan_attention import ScanAttention
from paper_2007_16100_amd.scan_mlp import ScanMLP

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture
def no_calls(monkeypatch):
    """Every call that would launch a kernel or take device memory fails the test."""
    def fail(name):
        def f(*a, **k):
            raise AssertionError(f"{name} was called")
        return f
    for name in [n for n in dir(spv) if n.startswith("spv_")] + ["Workspace"]:
        monkeypatch.setattr(scan_attention.spv, name, fail(name))


def mlp(C=64, F=128, dtype=BF, **other):
    P = dict(gamma1=torch.ones(C), beta1=torch.zeros(C), gamma2=torch.ones(F), beta2=torch.zeros(F),
             W1=torch.zeros(C, F, dtype=dtype), W2=torch.zeros(F, C, dtype=dtype))
    return dict(P, **other)


@pytest.mark.parametrize("other", [
    dict(W2=torch.zeros(128, 32, dtype=BF)), dict(W2=torch.zeros(128, 64)), dict(gamma1=torch.ones(128)),
    dict(gamma2=torch.ones(128, dtype=BF)), dict(beta1=torch.ones(64, 1)), dict(beta2=torch.ones(64)),
    dict(W1=torch.zeros(64, 128, dtype=torch.float64), W2=torch.zeros(128, 64, dtype=torch.float64))])
def test_parameters_of_other_types_and_widths(no_calls, other):
    with pytest.raises(ValueError):
        ScanMLP(mlp(**other), 8)


@pytest.mark.parametrize("groups,act", [(0, "silu"), (-2, "silu"), (3, "silu"), (128, "silu"), (8, "gelu"), (8, None)])
def test_groups_and_activations(no_calls, groups, act):
    with pytest.raises(ValueError):
        ScanMLP(mlp(), groups, act)


def test_features_and_gradients_that_do_not_fit(no_calls):
    layer, off, x = ScanMLP(mlp(), 8), torch.tensor([0, 10], dtype=torch.int32), torch.zeros(10, 64, dtype=BF)
    for bad in (x.float(), x[:, :32], x.t(), x.view(2, 5, 64), x.half()):
        with pytest.raises(ValueError):
            layer.forward(bad, off)
    for dy in (x[:9], x.float(), torch.zeros(10, 32, dtype=BF)):
        with pytest.raises(ValueError):
            layer.backward(dict(in1=x, off=off), dy)
        with pytest.raises(ValueError):
            layer.backward(dict(in1=spv.Checkpoint8.empty(10, 64, BF, "cpu"), off=off), dy)


def attention(**kw):
    P = dict(gamma=torch.ones(64), beta=torch.zeros(64), Wq=torch.zeros(64, 64, dtype=BF), Wk=torch.zeros(64, 32, dtype=BF),
             Wv=torch.zeros(64, 32, dtype=BF), Wo=torch.zeros(64, 64, dtype=BF))
    return ScanAttention(P, 4, 2, **kw)


def test_rotary_positions_without_coordinates(no_calls):
    with pytest.raises(ValueError):
        attention(rope=spv.RopeParams(32))
    layer, off = attention(rope=spv.RopeParams(16)), torch.tensor([0, 10], dtype=torch.int32)
    x, tok, c = torch.zeros(10, 64, dtype=BF), torch.zeros(2, 64, dtype=BF), torch.zeros(10, 4, dtype=torch.int32)
    for kw in (dict(), dict(coords=c[:9]), dict(coords=c.long()), dict(coords=c, tokens=tok, token_off=off),
               dict(coords=c, tokens=tok, token_off=off, token_coords=c[:1])):
        with pytest.raises(ValueError):
            layer.forward(x, off, **kw)


@pytest.fixture
def workspaces(monkeypatch):
    """(log, step): a step of a layer whose calls are replaced by ones that note their workspace, in order of use."""
    import ctypes as ct
    import types
    log = types.SimpleNamespace(used=[], stream=ct.c_void_p(None))

    class Workspace:
        def __init__(self, nbytes):
            self.nbytes = nbytes
    for n in ("for_ops", "for_linear_backward", "for_linear_backward8", "for_group_norm_backward"):
        setattr(Workspace, n, classmethod(lambda cls, *sizes: cls(sum(sizes))))

    def note(result):
        def f(ws, *a, **k):
            log.used.append(ws)
            return result(*a, **k)
        return f
    fake = types.SimpleNamespace(
        Workspace=Workspace, _stream=lambda: log.stream, Checkpoint8=spv.Checkpoint8,
        spv_linear=note(lambda x, W, res=None: torch.zeros(x.shape[0], W.shape[1])),
        spv_linear_backward=note(lambda x, W, da, want_dx=True: (None, torch.zeros_like(W))),
        spv_group_norm=note(lambda x, *a, want_stat=False, want_checkpoint=False: (x, torch.zeros(1, 2, 2)) if want_stat else x),
        spv_group_norm_backward=note(lambda dy, x, *a, dres=None: (dy, torch.zeros(1), torch.zeros(1))))
    monkeypatch.setattr(scan_attention, "spv", fake)
    monkeypatch.setattr(scan_mlp, "spv", fake)
    layer = ScanMLP(mlp(8, 16, F32), 2)

    def step():
        log.used.clear()
        saved, x = {}, torch.zeros(5, 8)
        layer.forward(x, torch.tensor([0, 5], dtype=torch.int32), save=saved)
        layer.backward(saved, x)
        return list(log.used)
    return log, step


def test_one_workspace_a_stream_and_thread(workspaces):
    """Two streams' and two threads' workspaces are apart."""
    import ctypes as ct
    import threading
    log, step = workspaces
    first = step()
    assert first and step() == first
    log.stream = ct.c_void_p(4096)
    other = step()
    assert len(other) == len(first) and not set(first) & set(other)
    log.stream, got = ct.c_void_p(None), []
    t = threading.Thread(target=lambda: got.extend(step()))
    t.start()
    t.join()
    assert len(got) == len(first) and not set(first) & set(got)


def test_captured_calls_have_workspaces_of_their_own(workspaces, monkeypatch):
    """A capture takes no workspace that the layer keeps, nor another capture's, and leaves none behind for later calls."""
    log, step = workspaces
    first, capturing = step(), [True]
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    one, two = step(), step()
    assert not set(first) & set(one) and not set(first) & set(two) and not set(one) & set(two)
    capturing[0] = False
    assert step() == first


@pytest.mark.parametrize("C,F", [(256, 512), (512, 256), (300, 260), (64, 128)])
def test_weight_gradients_of_wide_layers(workspaces, monkeypatch, C, F):
    """The linear layer's backward takes 65,536 weights: a layer of more has its weight gradient by blocks of outputs, each in a
    workspace that holds it."""
    calls = []

    def backward(ws, x, W, da, want_dx=True):
        assert W.shape[0] * W.shape[1] <= 65536 and W.is_contiguous() and da.is_contiguous() and not want_dx
        assert x.shape[1] == W.shape[0] and da.shape == (x.shape[0], W.shape[1]) and ws.nbytes >= sum(W.shape)
        calls.append(W.shape)
        return None, x.t() @ da
    fake = scan_attention.spv
    monkeypatch.setattr(fake, "spv_linear_backward", backward)
    layer, off = ScanMLP(mlp(C, F, F32), 2), torch.tensor([0, 5], dtype=torch.int32)
    x, dy, saved = torch.randn(5, C), torch.randn(5, C), {}
    layer.forward(x, off, save=saved)
    saved["out2"] = torch.randn(5, F)
    g = layer.backward(saved, dy)
    assert g["W2"].shape == (F, C) and torch.allclose(g["W2"], saved["out2"].t() @ dy, atol=1e-5)
    assert g["W1"].shape == (C, F) and len(calls) == (2 if C * F <= 65536 else 4)


def test_weight_gradients_of_wide_layers_from_8_bits(workspaces, monkeypatch):
    """The same from 8 bits, of 2^20 weights a call."""
    calls = []

    def backward(ws, saved, da):
        shape = (saved.codes.shape[1], da.shape[1])
        assert shape[0] * shape[1] <= 1 << 20 and da.is_contiguous()
        calls.append(shape)
        return saved.codes.float().t() @ da
    monkeypatch.setattr(scan_attention.spv, "spv_linear_backward8", backward, raising=False)
    layer = ScanMLP(mlp(1100, 1000, F32), 2)
    saved = spv.Checkpoint8(torch.randint(-127, 128, (5, 1100), dtype=torch.int8), torch.ones(5, 35, dtype=torch.uint8), F32)
    d = torch.randn(5, 1000)
    got = layer._weight_gradient(saved, layer.P["W1"], d)
    assert calls == [(1100, 944), (1100, 56)] and torch.allclose(got, saved.codes.float().t() @ d, atol=1e-2)
