"""Attention over packed scans where its numbers leave the ordinary range: caps far above the scores, scores of minus
infinity, scores of millions, weights and gradients far below one.  Oracles are the definition in float64; bounds are
given where they are used, in units of the type's half step (u) or of float32's (EPS)."""
import numpy as np
import pytest
import torch

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = ref.EPS


@pytest.fixture(scope="module")
def spv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2007_16100_amd import spv as s
    s.lib()
    return s


def arr(t):
    return t.detach().double().cpu().numpy()


def rnd(seed, *shape, std=1.0, dtype="f32"):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(TD[dtype]).cuda()


def off(*lens):
    return torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32).cuda()


def run(spv, q, k, v, dout=None, q_off=None, k_off=None, **kw):
    """out, lse and, with dout, dq, dk, dv; one scan where no offsets are given."""
    (nq, H, D), (nk, K, _) = q.shape, k.shape
    p = spv.make_attention_params(H, K, D, off(nq) if q_off is None else q_off, off(nk) if k_off is None else k_off, **kw)
    ws = spv.Workspace.for_attention_backward(p, nq, nk, q.dtype)
    ws.buf.fill_(255)
    out, lse = spv.spv_attention(ws, p, q, k, v, want_lse=True)
    got = dict(out=out, lse=lse)
    if dout is not None:
        got.update(zip(("dq", "dk", "dv"), spv.spv_attention_backward(ws, p, q, k, v, out, lse, dout)))
    return got


def rms(got, want):
    g = arr(got)
    assert not np.isnan(g).any()
    return np.sqrt(((g - want) ** 2).sum() / (want ** 2).sum())


# -- scores of minus infinity ------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("nq,nk,bad", [(40, 300, 150), (1, 5000, 1100), (200, 90, 64), (17, 129, 33)])
def test_keys_whose_score_is_minus_infinity(spv, nq, nk, bad, bias, dtype):
    """Keys in front of the others whose products overflow to minus infinity have no weight, in the forward and the
    backward: the rest of the row is as without them, within the bounds of that."""
    print(f"{nq}x{nk} bad={bad} bias={bias} {dtype}", flush=True)
    q, k, v, do = (rnd(i, n, h, 32, dtype=dtype) for i, (n, h) in enumerate(((nq, 2), (nk, 1), (nk, 1), (nq, 2))))
    q[..., 0], k[..., 0] = 1e25, 0.0
    k[:bad, :, 0] = -1e25
    kw, opt = {}, [None, None, None]
    if bias:
        g = torch.Generator().manual_seed(5)
        kw["q_coords"], kw["k_coords"] = (torch.randint(-9, 9, (n, 4), generator=g).to(torch.int32).cuda()
                                          for n in (nq, nk))
        kw["slopes"] = torch.tensor([0.25, 0.125]).cuda()
        opt = [kw["q_coords"].cpu().numpy(), kw["k_coords"][bad:].cpu().numpy(), arr(kw["slopes"])]
    got = run(spv, q, k, v, do, **kw)
    q0 = arr(q)
    q0[..., 0] = 0.0  # times the live keys' zeros
    want = ref.attention(q0, arr(k[bad:]), arr(v[bad:]), [0, nq], [0, nk - bad], float(np.float32(32 ** -0.5)), 0.0, *opt,
                         arr(do), dtype)
    for n in ("out", "lse", "dq"):
        assert np.all(np.abs(arr(got[n]) - want[n]) <= want[n + "_tol"]), n
    for n in ("dk", "dv"):
        assert not got[n][:bad].any(), n
        ch = slice(1, None) if n == "dk" else slice(None)  # channel 0 of dk is a sum of dz 1e25
        assert np.all(np.abs(arr(got[n][bad:]) - want[n])[..., ch] <= want[n + "_tol"][..., ch]), n


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nq,nk", [(40, 300), (2, 5000)])
def test_infinite_keys_and_rows_without_a_finite_score(spv, nq, nk, dtype):
    """Keys that are minus infinity in a channel where a query is positive have no weight for it; a query all of whose
    scores are minus infinity counts as one without a key, whichever way its keys are taken."""
    q, k, v = (rnd(i, n, 1, 32, dtype=dtype) for i, n in enumerate((nq, nk, nk)))
    q[..., 0] = 1.0
    k[: nk // 2, :, 0] = float("-inf")
    want = ref.attention(arr(q), arr(k[nk // 2:]), arr(v[nk // 2:]), [0, nq], [0, nk - nk // 2], float(np.float32(32 ** -0.5)),
                         dtype=dtype)
    got = run(spv, q, k, v)
    for n in ("out", "lse"):
        assert np.all(np.abs(arr(got[n]) - want[n]) <= want[n + "_tol"]), n
    k[..., 0] = float("-inf")
    got = run(spv, q, k, v)
    assert not got["out"].any() and bool((got["lse"] == -float("inf")).all())
