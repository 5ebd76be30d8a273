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


# -- caps ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("nq,nk", [(70, 513), (3, 4000)])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [1.0, 20.0, 50.0, 80.0, 1e3, 1e4, 1e6])
def test_a_caps_error_is_relative_to_the_score(spv, cap, bias, nq, nk, dtype):
    """Scores of ordinary size under caps up to the largest: where a cap is far above them it changes nothing.

    In float32 a weight takes a product of D steps (5 EPS in the root of the mean square), a tanh to a few EPS of scores
    of a few units (5), an exponent of up to 16 rounded once or twice (8) and its exponential (1): 11 EPS together.  The
    backward has lse's rounding too, and delta's.  In 16 bits the result's rounding is 0.5 u, that of the weights and of
    the scores' gradients as much again."""
    print(f"cap={cap} bias={bias} {nq}x{nk} {dtype}", flush=True)
    q, k, v, do = (rnd(i, n, h, 32, dtype=dtype) for i, (n, h) in enumerate(((nq, 2), (nk, 1), (nk, 1), (nq, 2))))
    kw = dict(cap=cap)
    opt = [None, None, None]
    if bias:
        g = torch.Generator().manual_seed(5)
        kw["q_coords"], kw["k_coords"] = (torch.randint(-9, 9, (n, 4), generator=g).to(torch.int32).cuda()
                                          for n in (nq, nk))
        kw["slopes"] = torch.tensor([0.0625, 0.03125]).cuda()
        opt = [kw["q_coords"].cpu().numpy(), kw["k_coords"].cpu().numpy(), arr(kw["slopes"])]
    got = run(spv, q, k, v, do, **kw)
    want = ref.attention(arr(q), arr(k), arr(v), [0, nq], [0, nk], float(np.float32(32 ** -0.5)), cap, *opt, arr(do), dtype)
    tol = 16 * EPS if dtype == "f32" else ref.UNIT[dtype]
    for n in ("out", "dq", "dk", "dv"):
        bound = tol if n == "out" or dtype != "f32" else 2 * tol
        assert rms(got[n], want[n]) <= bound, (n, rms(got[n], want[n]) / bound)


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


# -- large scores --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("slope", [2.0 ** 4, 2.0 ** 9, 2.0 ** 17, 2.0 ** 20])
@pytest.mark.parametrize("nq,nk", [(33, 700), (1, 6000), (300, 40)])
def test_tokens_far_from_every_key(spv, nq, nk, slope, cap, dtype):
    """Distances of some ten thousand under steep slopes: only the nearest keys have weight, each as much.  The scores are
    products of zero minus a distance, equal where the distances are, so the mean of the nearest keys' values is exact
    but for its own roundings; gradients are finite."""
    print(f"{nq}x{nk} slope={slope} cap={cap} {dtype}", flush=True)
    g = torch.Generator().manual_seed(11)
    q, k = torch.zeros(nq, 2, 32, dtype=TD[dtype]).cuda(), rnd(1, nk, 2, 32, dtype=dtype)
    v, do = rnd(2, nk, 2, 32, dtype=dtype), rnd(3, nq, 2, 32, dtype=dtype)
    kc = torch.randint(-30, 30, (nk, 4), generator=g).to(torch.int32).cuda()
    qc = torch.randint(-30, 30, (nq, 4), generator=g).to(torch.int32).cuda()
    qc[:, 1] += 20000
    qc[:, 2] -= 30000
    got = run(spv, q, k, v, do, cap=cap, scale=1.0, q_coords=qc, k_coords=kc, slopes=torch.tensor([slope, slope]).cuda())
    dist = np.abs(arr(qc)[:, None, 1:] - arr(kc)[None, :, 1:]).sum(-1)
    near = (dist == dist.min(1, keepdims=True)).astype(np.float64)
    V = arr(v)
    want = np.einsum("ij,jhd->ihd", near / near.sum(1, keepdims=True), V)
    # equal weights, so their rounding cancels; e^-16 = 1e-7 of each key a step further off
    n = nk * 2e-7 * (slope < 100) + (np.log2(nk) + 8) * EPS
    tol = ref.UNIT[dtype] * np.abs(want) + n * np.abs(V).max()
    assert not np.isnan(arr(got["out"])).any() and np.all(np.abs(arr(got["out"]) - want) <= tol)
    lse = -slope * dist.min(1) + np.log(near.sum(1))
    assert np.all(np.abs(arr(got["lse"]) - lse[:, None]) <= 4 * EPS * np.abs(lse[:, None]) + 1e-3)
    for name in ("dq", "dk", "dv"):
        assert bool(torch.isfinite(got[name].float()).all()), name


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [64.0, 4096.0, 1e6, 1e9])
@pytest.mark.parametrize("nq,nk,climb", [(40, 500, False), (40, 500, True), (1, 6000, True), (300, 70, True)])
def test_large_scales(spv, nq, nk, climb, scale, dtype):
    """Products of small whole numbers times a large scale: the keys with the largest product have all the weight, however
    often the largest so far moves up (climb: keys in ascending order)."""
    print(f"{nq}x{nk} scale={scale} climb={climb} {dtype}", flush=True)
    g = torch.Generator().manual_seed(12)
    q = torch.randint(1, 3, (nq, 1, 32), generator=g).to(TD[dtype]).cuda()
    k = torch.randint(-2, 3, (nk, 1, 32), generator=g).to(TD[dtype]).cuda()
    if climb:
        k = torch.randint(0, 2, (nk, 1, 32), generator=g).float().cuda()
        k += torch.arange(nk, device="cuda").div(64, rounding_mode="floor")[:, None, None] - 3.0
        k = k.to(TD[dtype])
    v, do = rnd(2, nk, 1, 32, dtype=dtype), rnd(3, nq, 1, 32, dtype=dtype)
    got = run(spv, q, k, v, do, scale=scale)
    z = np.einsum("ihd,jhd->ij", arr(q), arr(k))
    top = (z == z.max(1, keepdims=True)).astype(np.float64)
    V = arr(v)
    want = np.einsum("ij,jhd->ihd", top / top.sum(1, keepdims=True), V)
    tol = ref.UNIT[dtype] * np.abs(want) + (np.log2(nk) + 8) * EPS * np.abs(V).max()
    assert not np.isnan(arr(got["out"])).any() and np.all(np.abs(arr(got["out"]) - want) <= tol)
    # finite wherever the definition's gradient, of some hundred times the scale, is in the type's range
    want = ref.attention(arr(q), arr(k), V, [0, nq], [0, nk], scale, dout=arr(do))
    for name in ("dq", "dk", "dv"):
        held = torch.from_numpy(np.abs(want[name]) < 0.5 * torch.finfo(TD[dtype]).max)
        assert bool(torch.isfinite(got[name].float().cpu()[held]).all()), name


# -- float32 -----------------------------------------------------------------------------

@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("nq,nk", [(50, 300), (2, 5000)])
def test_float32_scores_far_below_zero(spv, nq, nk, D):
    """Tokens some 400 voxels from every key, at a slope of a half: the scores' sums are rounded a constant number of times
    at their size X (in units of log 2), not once for each of the product's D steps.  Three roundings of at most EPS X,
    evenly spread, are EPS X in the root of the mean square, so 1.5 EPS X ln 2 of the weights, and the products' own."""
    print(f"{nq}x{nk} D={D}", flush=True)
    g = torch.Generator().manual_seed(13)
    q, k, v, do = (rnd(i, n, 1, D) for i, n in enumerate((nq, nk, nk, nq)))
    kc = torch.randint(-4, 4, (nk, 4), generator=g).to(torch.int32).cuda()
    qc = torch.randint(-4, 4, (nq, 4), generator=g).to(torch.int32).cuda()
    qc[:, 1] += 400
    slopes = torch.tensor([0.5]).cuda()
    got = run(spv, q, k, v, do, q_coords=qc, k_coords=kc, slopes=slopes)
    want = ref.attention(arr(q), arr(k), arr(v), [0, nq], [0, nk], float(np.float32(D ** -0.5)), 0.0, qc.cpu().numpy(),
                         kc.cpu().numpy(), arr(slopes), arr(do))
    X = 200 * 1.4427
    bound = 1.5 * EPS * X * np.log(2.0) + 16 * EPS
    for n in ("out", "dq", "dk", "dv"):
        print(n, rms(got[n], want[n]) / EPS, bound / EPS, flush=True)
    assert rms(got["out"], want["out"]) <= bound
    for n in ("dq", "dk", "dv"):  # lse is rounded at that size too
        assert rms(got[n], want[n]) <= 1.5 * bound, n


@pytest.mark.parametrize("nq,nk", [(300, 300), (700, 3)])
def test_float32_gradients_without_a_bias(spv, nq, nk):
    """dv of heads of 128 channels: the weights' exponents, up to 16, are rounded three times (11 EPS), their products
    5 EPS, sums of some hundred rows 9."""
    q, k, v, do = (rnd(i, n, 1, 128) for i, n in enumerate((nq, nk, nk, nq)))
    got = run(spv, q, k, v, do)
    want = ref.attention(arr(q), arr(k), arr(v), [0, nq], [0, nk], float(np.float32(128 ** -0.5)), dout=arr(do))
    for n in ("out", "dq", "dk", "dv"):
        print(n, rms(got[n], want[n]) / EPS, flush=True)
    assert rms(got["dv"], want["dv"]) <= 24 * EPS


# -- float16 -----------------------------------------------------------------------------

@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("nk", [3000, 60000])
@pytest.mark.parametrize("score", [-12.0, -15.0, -17.5])
def test_f16_many_small_weights(spv, score, nk, nq):
    """One key at score 0 and thousands far below it: their weights, e^-17.5 each, are counted together.  Rounding one to
    float16 is off by 2^-11 of itself or, below the normal numbers, by 2^-25 of the largest that fits; the largest here
    is multiplied as 2^7 or more."""
    print(f"{nq}x{nk} score={score}", flush=True)
    q, k = torch.zeros(nq, 1, 32).half().cuda(), torch.zeros(nk, 1, 32).half().cuda()
    q[..., 0] = 1.0
    k[1:, :, 0] = score
    v = torch.ones(nk, 1, 32).half().cuda()
    v[0] = 0.0
    got = run(spv, q, k, v, scale=1.0)
    w = (nk - 1) * np.exp(score)
    want = w / (1 + w)
    tol = (nk - 1) * 2.0 ** -32 + 2.0 ** -11 * want * 2 + 2.0 ** -24
    assert np.all(np.abs(arr(got["out"]) - want) <= tol), (float(arr(got["out"]).mean()), want, tol)


# -- gradients in float16 -----------------------------------------------------------------

@pytest.mark.parametrize("std", [1e-4, 1e-3, 1e-2, 1.0])
@pytest.mark.parametrize("nq,nk", [(1500, 1500), (60, 6720), (2500, 40)])
def test_f16_small_gradients(spv, nq, nk, std):
    """Incoming gradients from 1e-4 up over long scans: dz, some 1e-8 each, keeps its eleven bits until it is summed.  Each
    gradient is off by the rounding of its weights and of dz (u each, as out's) and by its own last rounding, half a
    subnormal step where it is that small."""
    print(f"{nq}x{nk} std={std}", flush=True)
    q, k, v = (rnd(i, n, 2, 64, dtype="f16") for i, n in enumerate((nq, nk, nk)))
    do = rnd(3, nq, 2, 64, std=std, dtype="f16")
    got = run(spv, q, k, v, do)
    want = ref.attention(arr(q), arr(k), arr(v), [0, nq], [0, nk], 0.125, dout=arr(do), dtype="f16")
    for n in ("dq", "dk", "dv"):
        err, w = arr(got[n]) - want[n], want[n]
        # of a subnormal result: evenly spread over a step of 2^-24
        bound = 2 * ref.UNIT["f16"] * np.sqrt((w ** 2).sum()) + np.sqrt(w.size) * 2.0 ** -24 / np.sqrt(12.0)
        print(n, np.sqrt((err ** 2).sum()) / bound, flush=True)
        assert np.sqrt((err ** 2).sum()) <= bound, n


@pytest.mark.parametrize("nq,nk", [(3, 3), (200, 300), (5, 4000)])
def test_f16_gradients_past_its_range_on_the_way(spv, nq, nk):
    """Gradients scaled up: products dout . v of more than 65,504 whose dq and dk are in range again."""
    q, k = (rnd(i, n, 1, 64, std=2.0 ** -6, dtype="f16") for i, n in enumerate((nq, nk)))
    v, do = rnd(2, nk, 1, 64, std=128.0, dtype="f16"), rnd(3, nq, 1, 64, std=128.0, dtype="f16")
    got = run(spv, q, k, v, do)
    want = ref.attention(arr(q), arr(k), arr(v), [0, nq], [0, nk], 0.125, dout=arr(do), dtype="f16")
    for n in ("dq", "dk", "dv"):
        assert rms(got[n], want[n]) <= 4 * ref.UNIT["f16"], (n, rms(got[n], want[n]))


# -- means --------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("k_mean,v_mean", [(0.0, 4.0), (4.0, 0.0), (4.0, 4.0), (16.0, 4.0)])
@pytest.mark.parametrize("cap", [0.0, 30.0, 100.0])
@pytest.mark.parametrize("nq,nk,H,K,D", [(400, 1200, 1, 1, 32), (2, 6000, 2, 1, 64), (700, 45, 4, 2, 40), (90, 300, 1, 1, 96),
                                         (90, 300, 1, 1, 128)])
def test_gradients_of_keys_and_values_around_a_mean(spv, nq, nk, H, K, D, k_mean, v_mean, cap, dtype):
    """Keys and values that share a mean, as a layer's with biases do, or one without that centres its input: the rows of
    p (dout . v - delta) sum to zero, so nothing that is the same for all keys reaches dq.  A gradient is off by its own
    rounding and that of the weights or dz, 0.43 u each in the root of the mean square, 0.6 u together."""
    print(f"{nq}x{nk} H={H} K={K} D={D} means {k_mean} {v_mean} cap={cap} {dtype}", flush=True)
    q, do = rnd(0, nq, H, D, dtype=dtype), rnd(3, nq, H, D, dtype=dtype)
    k, v = ((rnd(i, nk, K, D) + m).to(TD[dtype]) for i, m in ((1, k_mean), (2, v_mean)))
    bias, opt = {}, [None, None, None]
    if D == 40:
        g = torch.Generator().manual_seed(5)
        bias["q_coords"], bias["k_coords"] = (torch.randint(-9, 9, (n, 4), generator=g).to(torch.int32).cuda()
                                              for n in (nq, nk))
        bias["slopes"] = torch.tensor([0.25, 0.125, 0.0625, 0.03125]).cuda()
        opt = [bias["q_coords"].cpu().numpy(), bias["k_coords"].cpu().numpy(), arr(bias["slopes"])]
    got = run(spv, q, k, v, do, cap=cap, **bias)
    want = ref.attention(arr(q), arr(k), arr(v), [0, nq], [0, nk], float(np.float32(D ** -0.5)), cap, *opt, arr(do), dtype)
    for n in ("dq", "dk", "dv"):
        print(n, rms(got[n], want[n]) / ref.UNIT[dtype], flush=True)
        assert rms(got[n], want[n]) <= ref.UNIT[dtype], n
