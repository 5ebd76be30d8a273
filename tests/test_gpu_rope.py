"""Rotary positions on the GPU against the float64 reference, within bounds derived from the kernel's roundings
(tests/voxel_ops_ref.py)."""
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


def within(got, want, tol, what):
    err = np.abs(got.detach().double().cpu().numpy() - want)
    assert np.all(err <= tol), (what, float(np.nanmax(err / tol)))


def rows(n, heads, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(n, heads, D, generator=g).to(TD[dtype]).cuda()


def places(n, seed):
    g = torch.Generator().manual_seed(seed)
    c = torch.randint(-32767, 32767, (n, 4), generator=g, dtype=torch.int32)
    c[: n // 2] = torch.randint(-40, 40, (n // 2, 4), generator=g, dtype=torch.int32)
    return c.cuda()


def check(spv, t, coords, freqs, sections, halves, inverse, got, dtype, what):
    want, e = ref.rope(t.double().cpu().numpy(), coords.cpu().numpy(), freqs.cpu().numpy(), sections, halves, inverse)
    within(got, want, ref.rounded(want, e, dtype), what)


# rows, heads, key heads, channels, sections: whole heads and parts, axes left out, a single pair, odd pairs of halves
SHAPES = [(1, 1, 0, 8, (1, 0, 0)), (1, 8, 8, 32, (6, 6, 4)), (2, 3, 1, 16, (0, 3, 5)), (33, 4, 2, 64, (8, 8, 8)),
          (40, 8, 0, 32, (6, 6, 4)), (7, 5, 5, 24, (4, 4, 4)), (65, 2, 1, 40, (5, 5, 3)), (100, 1, 1, 128, (22, 21, 21)),
          (129, 16, 4, 128, (16, 16, 16)), (1000, 3, 3, 96, (16, 16, 16)), (5003, 8, 8, 32, (8, 8, 0)),
          (257, 6, 2, 56, (9, 9, 9)), (31, 2, 2, 88, (12, 12, 8)), (3, 70, 9, 128, (32, 16, 16))]


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,H,K,D,sections", SHAPES)
def test_rope_and_inverse(spv, n, H, K, D, sections, dtype, halves):
    print(f"rope n={n} H={H} K={K} D={D} {sections} {dtype} halves={halves}", flush=True)
    q, k = rows(n, H, D, dtype, n + D), rows(n, K, D, dtype, n + D + 1) if K else None
    c, f = places(n, n), torch.from_numpy(np.random.default_rng(n).uniform(1e-3, 2.0, sum(sections)).astype(np.float32)).cuda()
    p = spv.make_rope_params(D, f, sections, halves)
    for inverse in (False, True):
        got = spv.spv_rope(p, c, q, k, inverse=inverse)
        got = (got,) if k is None else got
        for t, g in zip((q, k), got):
            check(spv, t, c, f, sections, halves, inverse, g, dtype, (inverse, t.shape))
            if 2 * sum(sections) < D:
                assert torch.equal(g[..., 2 * sum(sections):], t[..., 2 * sum(sections):])


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rope_in_place_and_parts_of_a_buffer(spv, dtype, halves):
    """q and k as views of one buffer, in place; what is beside them, and rows past a device count, stay as they were."""
    n, H, K, D, sec = 300, 4, 2, 48, (8, 8, 4)
    buf = rows(n, H + 2 * K + 1, D, dtype, 5)
    c, f = places(n, 9), spv.rope_freqs(sec)
    p = spv.make_rope_params(D, f, sec, halves)
    q, k = buf[:, :H], buf[:, H:H + K]
    want = spv.spv_rope(p, c, q, k)
    check(spv, q, c, f, sec, halves, False, want[0], dtype, "packed")
    again = spv.spv_rope(p, c, q.contiguous(), k.contiguous())
    assert all(torch.equal(a, b) for a, b in zip(want, again))
    live = torch.tensor([211], dtype=torch.int64, device="cuda")
    old = buf.clone()
    got = spv.spv_rope(p, c, q, k, outs=(q, k), m_dev=live)
    assert got[0].data_ptr() == buf.data_ptr()
    assert torch.equal(buf[:211, :H], want[0][:211]) and torch.equal(buf[:211, H:H + K], want[1][:211])
    assert torch.equal(buf[211:], old[211:]) and torch.equal(buf[:, H + K:], old[:, H + K:])
    for count in (-3, 0, 10 ** 12):
        live.fill_(count)
        out = torch.full_like(want[0], 7.0)
        spv.spv_rope(p, c, old[:, :H], outs=(out,), m_dev=live)
        assert torch.equal(out, want[0]) if count > 0 else bool((out == 7.0).all())
    none = spv.spv_rope(p, c[:0], q[:0], k[:0])
    assert none[0].shape == (0, H, D) and none[1].shape == (0, K, D)


def test_rope_far_places_and_odd_numbers(spv):
    """Angles of thousands of turns, coordinates outside the voxel range, frequencies of 0 and below, and values that are not
    finite: they reach their own pair alone."""
    n, D, sec = 64, 32, (6, 6, 4)
    c = torch.full((n, 4), 32766, dtype=torch.int32)
    c[::3], c[1::7], c[2::5] = -32767, 2 ** 31 - 1, -2 ** 31
    c = c.cuda()
    f = torch.tensor([0.0, -1.0, 1.0, 3.14159274, 1.57079637, 0.785398185, 100.0, 9999.0, 1e-30, 1e-4, 0.5, 0.25, 2.0, 7.0,
                      11.0, -0.1], device="cuda")
    q = rows(n, 2, D, "f32", 3)
    p = spv.make_rope_params(D, f, sec)
    got = spv.spv_rope(p, c, q)
    check(spv, q, c, f, sec, False, False, got, "f32", "far")
    q[5, 1, 6], q[9, 0, 3] = float("inf"), float("nan")
    bad = spv.spv_rope(p, c, q)
    differ = (bad != got).nonzero().tolist()
    assert all(i in ([5, 1, 6], [5, 1, 7], [9, 0, 2], [9, 0, 3]) for i in differ) and len(differ) >= 3
    f[4] = float("nan")
    bad = spv.spv_rope(p, c, rows(n, 2, D, "f32", 3))
    assert bool(torch.isnan(bad[..., 8:10]).all()) and torch.equal(bad[..., :8], got[..., :8])
    assert torch.equal(bad[..., 10:], got[..., 10:])


def test_rope_on_another_stream_and_in_a_graph(spv):
    n, H, D, sec = 4001, 8, 32, (6, 6, 4)
    q, k, c = rows(n, H, D, "bf16", 1), rows(n, 2, D, "bf16", 2), places(n, 3)
    p = spv.make_rope_params(D, spv.rope_freqs(sec), sec)
    want = spv.spv_rope(p, c, q, k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = spv.spv_rope(p, c, q, k)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = spv.spv_rope(p, c, q, k)
    for seed in (11, 12, 13):
        q.copy_(rows(n, H, D, "bf16", seed))
        graph.replay()
        want = spv.spv_rope(p, c, q, k)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
