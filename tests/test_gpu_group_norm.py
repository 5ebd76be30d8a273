"""Group norm with an activation over packed scans, forward and backward, on the GPU against the float64 reference within
bounds derived from the kernels' roundings (tests/voxel_ops_ref.py)."""
import numpy as np
import pytest
import torch

from tests import voxel_ops_ref as ref

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
    err = np.abs(arr(got) - want)
    assert np.all(err <= tol), (what, float(np.nanmax(err / tol)))


def inputs(m, C, dtype, seed, mean=0.5, std=2.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(m, C, generator=g) * std + mean * torch.randn(C, generator=g)).to(TD[dtype])
    dy, res = (torch.randn(m, C, generator=g).to(TD[dtype]) for _ in range(2))
    return [t.cuda() for t in (x, dy, res, 1.0 + 0.2 * torch.randn(C, generator=g), torch.randn(C, generator=g))]


def offsets(lens, first=0):
    return torch.tensor(np.cumsum([first, *lens]), dtype=torch.int32, device="cuda")


def step(spv, x, dy, res, g, b, off, G, act, ckpt, ws=None):
    m, C = x.shape
    ws = ws or spv.Workspace.for_group_norm_backward(m, C, G, off.shape[0] - 1)
    got = spv.spv_group_norm(ws, x, off, G, g, b, act=act, want_stat=True, want_checkpoint=ckpt)
    saved = got[2] if ckpt else x
    return (*got[:2], *spv.spv_group_norm_backward(ws, dy, saved, off, G, got[1], g, b, act, res)), saved


def check(spv, x, dy, res, g, b, off, G, act, ckpt, dtype):
    (y, stat, dx, dg, db), saved = step(spv, x, dy, res, g, b, off, G, act, ckpt)
    o = off.tolist()
    X8 = None
    i, j = max(0, min(x.shape[0], o[0])), max(0, min(x.shape[0], o[-1]))
    if ckpt:
        q, e, X8 = ref.codes(arr(x), dtype)
        assert np.array_equal(saved.codes.cpu().numpy()[i:j], q[i:j])
        assert np.array_equal(saved.exps.cpu().numpy()[i:j], e[i:j])
    R = ref.group_norm(arr(x), o, G, arr(g), arr(b), 1e-5, act, dtype, arr(dy), None if res is None else arr(res), X8)
    within(stat[..., 0], R["mu"], R["mu_tol"] + ref.TINY["f32"], "mu")
    within(stat[..., 1], R["r"], R["r_tol"] + ref.EPS * R["r"], "r")
    within(y[i:j], R["y"][i:j], R["y_tol"][i:j], "y")
    within(dx[i:j], R["dx"][i:j], R["dx_tol"][i:j], "dx")
    within(dg, R["dgamma"], R["dgamma_tol"], "dgamma")
    within(db, R["dbeta"], R["dbeta_tol"], "dbeta")
    again, _ = step(spv, x, dy, res, g, b, off, G, act, ckpt)
    for p, q in zip((y[i:j], stat, dx[i:j], dg, db), (again[0][i:j], again[1], again[2][i:j], *again[3:])):
        assert torch.equal(p, q)


# lengths of the scans: one row, empty ones among them, many short ones, long ones
LENS = {"one": [1], "mixed": [0, 1, 5, 300, 0, 33, 0], "even": [64, 64], "none": [0, 0], "short": [3, 1, 0, 2] * 60,
        "long": [2777, 1, 1500], "crowd": [9, 0, 1, 4, 7] * 140, "many": [1, 0, 2, 1] * 1250, "six": [590, 10]}
SHAPES = [(1, 1, "mixed"), (7, 7, "mixed"), (8, 1, "one"), (8, 8, "mixed"), (19, 1, "mixed"), (19, 19, "long"), (32, 4, "even"),
          (96, 8, "mixed"), (96, 96, "mixed"), (96, 1, "long"), (96, 8, "one"), (96, 8, "none"), (96, 8, "short"), (100, 4, "mixed"),
          (36, 4, "long"), (64, 2, "short"), (256, 16, "long"), (256, 256, "even"), (520, 8, "mixed"), (1030, 2, "even"),
          (2049, 3, "one"), (2048, 32, "even"), (4096, 1, "even"), (5000, 5, "one"), (16, 16, "long"),
          # past what one launch takes: tiles joined by waves and by eights of lanes, by a launch of its own, searches over
          # hundreds and thousands of scans, rows by elements and too wide for a workgroup
          (96, 8, "crowd"), (96, 48, "crowd"), (96, 96, "crowd"), (51, 17, "crowd"), (51, 51, "crowd"), (32, 8, "many"),
          (33, 3, "many"), (256, 256, "six"), (256, 1, "six"), (250, 125, "six"), (2049, 3, "even"), (1030, 515, "even")]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C,G,lens", SHAPES)
def test_group_norm_and_backward(spv, C, G, lens, dtype):
    n = sum(LENS[lens])
    print(f"group norm C={C} G={G} {lens} {dtype}", flush=True)
    x, dy, res, g, b = inputs(n, C, dtype, C + G)
    act = ("none", "relu", "silu")[(C + G + len(lens)) % 3]
    check(spv, x, dy, res if G % 2 else None, g, b, offsets(LENS[lens]), G, act, C % 3 == 1, dtype)


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_activations_and_checkpoints(spv, dtype, act, ckpt):
    for C, G in ((96, 8), (50, 5), (32, 32)):
        x, dy, res, g, b = inputs(900, C, dtype, 5)
        check(spv, x, dy, res, g, b, offsets([500, 399, 1]), G, act, ckpt, dtype)


@pytest.mark.parametrize("m,C,G,scans", [(70001, 16, 4, 1), (40003, 96, 8, 4), (30011, 19, 1, 2), (9001, 256, 256, 3)])
def test_many_rows(spv, m, C, G, scans):
    x, dy, res, g, b = inputs(m, C, "bf16", m)
    cut = sorted(np.random.default_rng(m).integers(0, m, scans - 1).tolist())
    off = torch.tensor([0, *cut, m], dtype=torch.int32, device="cuda")
    for ckpt in (False, True):
        check(spv, x, dy, res, g, b, off, G, "silu", ckpt, "bf16")


def test_far_from_zero_flat_and_wild_rows(spv):
    """Scans far from zero keep their deviations; equal values give act(beta); a first row far from the rest; scales of 1e18 and
    1e-18."""
    for C, G in ((96, 8), (18, 3)):
        x, dy, res, g, b = inputs(400, C, "f32", 3, mean=0.0)
        x[:100] += 4000.0
        x[100:200] = 3.25
        x[200] = 3e4
        x[300:350] *= 1e17
        off = offsets([100, 100, 100, 50, 50])
        check(spv, x, dy, res, g, b, off, G, "none", False, "f32")
        y = spv.spv_group_norm(spv.Workspace.for_group_norm(400, C, G, 5), x, off, G, g, b, act="relu")
        assert torch.equal(y[100:200], b.clamp(min=0).expand(100, C))


def test_rows_of_no_scan_and_offsets_past_the_ends(spv):
    """Rows outside the scans stay as they were, in every output; offsets are clamped."""
    for C, G in ((96, 8), (21, 7)):
        m = 500
        x, dy, res, g, b = inputs(m, C, "bf16", 4)
        ws = spv.Workspace.for_group_norm_backward(m, C, G, 3)
        off = torch.tensor([37, 100, 100, 460], dtype=torch.int32, device="cuda")
        y = torch.full_like(x, 7.0)
        spv.spv_group_norm(ws, x, off, G, g, b, act="silu", out=y)
        assert bool((y[:37] == 7.0).all()) and bool((y[460:] == 7.0).all())
        check(spv, x, dy, res, g, b, off, G, "silu", True, "bf16")
        dx = res.clone()
        stat = spv.spv_group_norm(ws, x, off, G, g, b, act="silu", want_stat=True)[1]
        st = spv.lib().spv_group_norm_backward(spv._stream(), ws.ptr, ws.nbytes, spv._ptr(dy), spv._ptr(x), None, None, m, C,
                                               spv._ptr(off), 3, G, spv._ptr(g), spv._ptr(b), spv._ptr(stat), 2, spv._ptr(dx),
                                               spv._ptr(dx), None, None, 1)
        assert st == 0 and torch.equal(dx[:37], res[:37]) and torch.equal(dx[460:], res[460:])
        want = spv.spv_group_norm_backward(ws, dy, x, off, G, stat, g, b, "silu", res)[0]
        assert torch.equal(dx[37:460], want[37:460])
        saved = spv.Checkpoint8.empty(m, C, torch.bfloat16)
        saved.codes.fill_(3)
        saved.exps.fill_(9)
        st = spv.lib().spv_group_norm(spv._stream(), ws.ptr, ws.nbytes, spv._ptr(x), m, C, spv._ptr(off), 3, G, None, None, 1e-5,
                                      0, spv._ptr(y), None, *saved.addresses(0), 1)
        assert st == 0 and bool((saved.codes[:37] == 3).all()) and bool((saved.exps[460:] == 9).all())
        wide = torch.tensor([-50, 100, 100, 10 ** 6], dtype=torch.int32, device="cuda")
        check(spv, x, dy, res, g, b, wide, G, "relu", False, "bf16")
        none = torch.tensor([0], dtype=torch.int32, device="cuda")
        _, dg, db = spv.spv_group_norm_backward(ws, dy, x, none, G, stat[:0], g, b)
        assert not bool(dg.any()) and not bool(db.any())


def test_options(spv):
    """No gamma or beta, in place (with a checkpoint too), outputs left out, odd pointers, no rows."""
    for C, G in ((96, 8), (50, 2)):
        x, dy, res, g, b = inputs(300, C, "bf16", 11)
        off, ws = offsets([120, 180]), spv.Workspace.for_group_norm_backward(300, C, G, 2)
        one, zero = torch.ones_like(g), torch.zeros_like(b)
        assert torch.equal(spv.spv_group_norm(ws, x, off, G), spv.spv_group_norm(ws, x, off, G, one, zero))
        full, stat, saved = spv.spv_group_norm(ws, x, off, G, g, b, act="silu", want_stat=True, want_checkpoint=True)
        y = x.clone()
        got = spv.spv_group_norm(ws, y, off, G, g, b, act="silu", want_stat=True, want_checkpoint=True, out=y)
        assert torch.equal(y, full) and torch.equal(got[2].codes, saved.codes) and torch.equal(got[2].exps, saved.exps)
        alone = spv.spv_checkpoint8(x)
        assert torch.equal(alone.codes, saved.codes) and torch.equal(alone.exps, saved.exps)
        want = spv.spv_group_norm_backward(ws, dy, x, off, G, stat, g, b, "silu", res)
        p, L = spv._ptr, spv.lib()
        dx, dg = dy.clone(), torch.empty_like(g)
        tail = (300, C, p(off), 2, G, p(g), p(b), p(stat), 2, p(res))
        assert L.spv_group_norm_backward(spv._stream(), ws.ptr, ws.nbytes, p(dx), p(x), None, None, *tail, p(dx), None, None,
                                         1) == 0
        assert torch.equal(dx, want[0])
        assert L.spv_group_norm_backward(spv._stream(), ws.ptr, ws.nbytes, p(dy), p(x), None, None, *tail, None, p(dg), None,
                                         1) == 0
        assert torch.equal(dg, want[1])
        buf = torch.empty(300 * C + 1, dtype=x.dtype, device="cuda")
        odd = buf[1:].view(300, C)
        odd.copy_(x)
        check(spv, odd, dy, res, g, b, off, G, "silu", True, "bf16")
        none = offsets([0, 0])
        (y, stat, dx, dg, db), _ = step(spv, x[:0], dy[:0], None, g, b, none, G, "relu", True)
        assert y.shape == (0, C) and not bool(stat.any()) and not bool(dg.any()) and not bool(db.any())


def test_values_that_are_not_finite_stay_in_their_group(spv):
    """(In a checkpoint a value that is not finite no longer counts for its block's exponent, so its neighbours' codes may
    change, those of other groups among them: they stay finite.)"""
    for C, G in ((96, 8), (35, 5)):
        x, dy, res, g, b = inputs(300, C, "bf16", 12)
        off, w = offsets([100, 150, 50]), C // G
        clean, _ = step(spv, x, dy, res, g, b, off, G, "relu", False)
        x[110, 2 * w + 1], x[120, 0] = float("nan"), float("inf")
        (y, stat, dx, dg, db), _ = step(spv, x, dy, res, g, b, off, G, "relu", False)
        hit = torch.zeros(300, C, dtype=torch.bool, device="cuda")
        hit[100:250, :w] = hit[100:250, 2 * w:3 * w] = True
        assert bool(torch.isnan(y[hit].float()).all()) and torch.equal(y[~hit], clean[0][~hit])
        assert torch.equal(dx[~hit], clean[2][~hit])
        cols = torch.ones(C, dtype=torch.bool, device="cuda")
        cols[:w] = cols[2 * w:3 * w] = False
        assert torch.equal(dg[cols], clean[3][cols]) and torch.equal(db[cols], clean[4][cols])
        kept, _ = step(spv, x, dy, res, g, b, off, G, "relu", True)
        assert bool(torch.isfinite(kept[2][~hit].float()).all()) and bool(torch.isfinite(kept[3][cols]).all())


def test_group_norm_on_another_stream_and_in_a_graph(spv):
    """A captured step next to eager ones: every replay gives the eager results of its inputs."""
    m, C, G = 3001, 96, 8
    off = offsets([1000, 1, 2000])
    x, dy, res, g, b = inputs(m, C, "bf16", 1)
    want, _ = step(spv, x, dy, res, g, b, off, G, "silu", True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = step(spv, x, dy, res, g, b, off, G, "silu", True)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    ws = spv.Workspace.for_group_norm_backward(m, C, G, 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, _ = step(spv, x, dy, res, g, b, off, G, "silu", True, ws)
    for seed in (21, 22, 23):
        for t, s in zip((x, dy, res), inputs(m, C, "bf16", seed)):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = step(spv, x, dy, res, g, b, off, G, "silu", True)
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def equal_values(lens, C, G, seed, scale=1.0):
    """Rows whose groups hold one value each a scan, a whole number of 64 .. 127 (either sign) times scale / 16: exact in every
    type, and in 8 bits for powers of two."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(64, 128, (len(lens), G), generator=g) * (1 - 2 * torch.randint(0, 2, (len(lens), G), generator=g))
    return (v.double() * (scale / 16.0)).repeat_interleave(C // G, 1).repeat_interleave(torch.tensor(lens), 0)


def check_equal(spv, x, dy, res, gamma, beta, off, G, act, ckpt, dtype):
    """A group of equal values has xh = 0 to the last bit, in the forward and in the backward: y = act(beta), dgamma = 0, and
    without beta ReLU lets no gradient through; the others' slopes at 0 are 1 and 1/2."""
    m, C = x.shape
    (y, stat, dx, dg, db), _ = step(spv, x, dy, res, gamma, beta, off, G, act, ckpt)
    assert not bool(y.any()) and not bool(dg.any())
    o, E = off.tolist(), ref.EPS
    full = torch.tensor([b > a for a, b in zip(o, o[1:])], device="cuda")
    r = 1.0 / np.sqrt(1e-5)
    assert bool(((stat[full][..., 1].double() - r).abs() <= 4 * E * r).all())
    if act == "relu":
        assert not bool(db.any())
        assert torch.equal(dx, torch.zeros_like(dx) if res is None else res)
        return
    slope = {"none": 1.0, "silu": 0.5}[act]
    gz = arr(dy) * slope
    h = gz * (1.0 if gamma is None else arr(gamma))
    steps = 3 * min(m, 1024) + 16  # of a sum, as in the reference
    tol = E * (steps + 8) * np.abs(gz).sum(0) + ref.TINY["f32"]
    within(db, gz.sum(0), tol, "dbeta")
    for i, j in zip(o, o[1:]):
        if j <= i:
            continue
        t = h[i:j].reshape(j - i, G, C // G)
        mean, size = (f(t).mean((0, 2), keepdims=True) for f in (np.asarray, np.abs))
        want = (r * (t - mean)).reshape(j - i, C)
        err = r * (E * (steps + 16) * size + 8 * E * np.abs(t)).reshape(j - i, C) + 8 * E * np.abs(want)
        if res is not None:
            want = want + arr(res[i:j])
            err = err + E * np.abs(want)
        within(dx[i:j], want, err + ref.UNIT[dtype] * (np.abs(want) + err) + ref.TINY[dtype], "dx")


# scans of one row, of a few and of many tiles; vectors and elements, and rows too wide for a workgroup
EQUAL = [(96, 1, [1] * 40 + [700, 0, 5]), (96, 8, [3, 1, 2000, 1]), (96, 96, [1, 0, 3000, 2]), (96, 96, [1] * 300), (19, 19, [1, 900]),
         (51, 3, [1, 700, 0, 2]), (256, 16, [2500, 1]), (1030, 515, [1, 40, 2])]


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("act", ["relu", "silu", "none"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_equal_values_have_no_deviation_in_the_backward(spv, dtype, act, ckpt):
    for k, (C, G, lens) in enumerate(EQUAL):
        m = sum(lens)
        print(f"equal values C={C} G={G} {dtype} {act} {ckpt}", flush=True)
        x = equal_values(lens, C, G, 31 + k).to(TD[dtype]).cuda()
        _, dy, res, gamma, beta = inputs(m, C, dtype, 7 + k)
        gamma = gamma * torch.where(beta > 0, 1.0, -1.0)
        for p in ((gamma, None, res), (None, torch.zeros_like(beta), None)):
            check_equal(spv, x, dy, p[2], p[0], p[1], offsets(lens), G, act, ckpt, dtype)


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_equal_values_in_tiles_of_few_rows(spv, dtype, act, ckpt):
    """Values whose squares float32 does not hold (some 5e20), in tiles that have fewer rows than a workgroup takes at a time."""
    for k, (C, G, lens) in enumerate([(96, 1, [3, 1, 2000, 1]), (96, 8, [5, 2500, 2]), (36, 4, [1, 4000, 7]), (51, 3, [1, 1500, 2])]):
        m = sum(lens)
        print(f"large equal values C={C} G={G} {dtype} {act} {ckpt}", flush=True)
        x = equal_values(lens, C, G, 51 + k, 2.0 ** 66).to(TD[dtype]).cuda()
        _, dy, res, gamma, _ = inputs(m, C, dtype, 17 + k)
        check_equal(spv, x, dy, res, gamma, None, offsets(lens), G, act, ckpt, dtype)


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("act", ["relu", "none"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_values_at_the_end_of_the_type(spv, dtype, act, ckpt):
    """Values of 1.7e38 to 3.37e38, where float32 and bf16 end (3.40e38 and 3.39e38): not even two add up in float32."""
    for k, (C, G, lens) in enumerate([(96, 8, [1, 2500, 3]), (96, 96, [1, 3, 700]), (51, 3, [1, 1500, 4]), (36, 36, [40, 9, 1])]):
        m = sum(lens)
        print(f"equal values at the end C={C} G={G} {dtype} {act} {ckpt}", flush=True)
        x = equal_values(lens, C, G, 71 + k, 2.0 ** 125).to(TD[dtype]).cuda()
        assert bool(torch.isfinite(x).all()) and float(x.abs().min()) > 1.7e38
        _, dy, res, gamma, _ = inputs(m, C, dtype, 27 + k)
        check_equal(spv, x, dy, res, gamma, None, offsets(lens), G, act, ckpt, dtype)
