"""The attention layer's workspaces on the CPU, with the calls replaced by ones that note the workspace they are given:
calls that may run at the same time, on two streams or from two threads, get different ones."""
import ctypes as ct
import threading
import types

import pytest
import torch

from paper_2007_16100_amd import scan_attention
from paper_2007_16100_amd.scan_attention import ScanAttention


@pytest.fixture
def calls(monkeypatch):
    """Fakes of the calls; .used: (call, workspace) in order, .stream: the current stream's handle."""
    log = types.SimpleNamespace(used=[], stream=ct.c_void_p(None), made=0)

    class Workspace:
        def __init__(self, nbytes):
            self.nbytes = nbytes
            log.made += 1

        @classmethod
        def for_ops(cls, n, C):
            return cls(n * C)

        @classmethod
        def for_linear_backward(cls, a, b):
            return cls(a * b)

        @classmethod
        def for_attention_backward(cls, p, m, n, dtype):
            return cls(m + n)

        @classmethod
        def for_layer_norm_backward(cls, m, C):
            return cls(m * C)

    def note(name, result):
        def f(ws, *a, **k):
            log.used.append((name, ws))
            return result(*a, **k)
        return f
    spv = types.SimpleNamespace(
        Workspace=Workspace, _stream=lambda: log.stream, spv_layer_norm=lambda x, *a: x,
        make_attention_params=lambda *a, **k: types.SimpleNamespace(B=1),
        spv_linear=note("linear", lambda x, W, res=None: torch.zeros(x.shape[0], W.shape[1])),
        spv_linear_backward=note("linear backward", lambda x, W, da, want_dx=True: (torch.zeros_like(x), torch.zeros_like(W))),
        spv_attention=note("attention", lambda p, q, k, v, want_lse=False: (q, q[..., 0]) if want_lse else q),
        spv_attention_backward=note("attention backward", lambda p, q, k, v, o, lse, do: (q, k, v)),
        spv_layer_norm_backward=note("norm backward", lambda dy, x, g, eps, dres=None: (dy, g, g)))
    monkeypatch.setattr(scan_attention, "spv", spv)
    return log


def layer():
    return ScanAttention(dict(gamma=torch.ones(8), beta=torch.zeros(8), Wq=torch.zeros(8, 8), Wk=torch.zeros(8, 8),
                              Wv=torch.zeros(8, 8), Wo=torch.zeros(8, 8)), 2)


def step(a, log):
    """The workspaces of a forward and backward of 5 rows."""
    log.used.clear()
    saved = {}
    a.forward(torch.zeros(5, 8), torch.tensor([0, 5], dtype=torch.int32), save=saved)
    a.backward(saved, torch.zeros(5, 8))
    return [(n, id(w), w) for n, w in log.used]


def test_one_workspace_a_stream(calls):
    a = layer()
    first = step(a, calls)
    made = calls.made
    assert step(a, calls) == first and calls.made == made  # kept from call to call
    calls.stream = ct.c_void_p(4096)
    other = step(a, calls)
    assert [n for n, _, _ in first] == [n for n, _, _ in other]
    assert not {w for _, w, _ in first} & {w for _, w, _ in other}
    calls.stream = ct.c_void_p(None)
    assert step(a, calls) == first


def test_one_workspace_a_thread(calls):
    a, got = layer(), []
    first = step(a, calls)
    t = threading.Thread(target=lambda: got.extend(step(a, calls)))
    t.start()
    t.join()
    assert len(got) == len(first) and not {w for _, w, _ in first} & {w for _, w, _ in got}
