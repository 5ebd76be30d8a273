"""Every form of the attention kernels that a large call runs, at sizes a float64 reference can follow: many short and a
few longer scans, so that there are workgroups enough for one wave or two on a block of columns.  shape() is the rule by
which a call takes its form, written out again; each test asserts what its sizes reach, in both directions."""
import pytest
import torch

from tests.test_gpu_attention import Case, spv  # noqa: F401 (spv: a fixture)

pytestmark = pytest.mark.gpu


def waves(dtype, D, mode):
    """Waves on a block of 32 columns."""
    width = (D + 31) // 32 * 32 * (2 if dtype == "f32" else 1)
    return min(1 << mode, 4 if width <= 64 else 2 if width <= 128 else 1)


def shape(dtype, D, n, per, B, K, rows):
    """(mode, parts) of n rows of `per` columns against scans of `rows` rows on average."""
    for mode in range(3):
        tiles = n * per // (128 // waves(dtype, D, mode)) + B
        if mode == 2 or tiles * K * 4 >= 2048:
            break
    parts = 1
    if tiles * K < 256:
        parts = min(512 // max(tiles * K, 1), rows // 256, 256)
        parts = parts // 8 * 8 if parts > 8 else max(parts, 1)
    return mode, parts


def shapes(c, dtype):
    """Of the forward and dq, and of dk, dv."""
    nq, nk, B, G = sum(c.ql), sum(c.kl), len(c.kl), c.H // c.K
    return (shape(dtype, c.D, nq, G, B, c.K, nk // B), shape(dtype, c.D, nk, 1, B, c.K, nq // B * G))


EDGES = [0, 1, 31, 32, 33, 63, 64, 65, 70, 5]  # around the tiles' edges


def scans(mode):
    """Lengths whose tiles leave two waves to each SIMD (2048) with one wave on a block, or only with two."""
    return [700, 257, 129, 128, 127] + EDGES * (28 if mode == 0 else 16)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cap", [0.0, 3.0, 100.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
@pytest.mark.parametrize("mode", [0, 1])
def test_one_or_two_waves_on_a_block_of_columns(spv, mode, D, bias, cap, dtype):  # noqa: F811
    print(f"mode={mode} D={D} bias={bias} cap={cap} {dtype}", flush=True)
    c = Case(scans(mode), None, 2, 2, D, dtype, cap=cap, bias=bias, packed=True, seed=D + mode)
    for m, parts in shapes(c, dtype):  # wide heads have one form in float32
        assert waves(dtype, D, m) == waves(dtype, D, mode) and parts == 1
    c.check(spv)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H,K,D", [(8, 8, 32), (6, 2, 40), (8, 2, 64), (4, 1, 32)])
def test_shared_heads_and_other_queries_in_large_launches(spv, H, K, D, dtype):  # noqa: F811
    """Queries of other numbers than the keys, scans with none of either, several query heads on a key head."""
    print(f"H={H} K={K} D={D} {dtype}", flush=True)
    kl = [300, 0, 1, 257] + EDGES * (30 if K == 2 else 60 if K == 1 else 8)
    ql = [64, 33, 0, 500] + (EDGES[3:] + EDGES[:3]) * (30 if K == 2 else 60 if K == 1 else 8)
    c = Case(kl, ql, H, K, D, dtype, cap=5.0 if H == 6 else 0.0, bias=True, seed=H)
    assert [s[0] for s in shapes(c, dtype)] == [0, 0]
    c.check(spv)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_far_apart_voxels_in_large_launches(spv, dtype):  # noqa: F811
    """Coordinates past a cube of 256, whose distances take two words, in the kernels of two 32-row steps."""
    c = Case(scans(0), None, 2, 2, 32, dtype, bias=True, seed=3, extent=3000)
    c.slopes.mul_(0.01)
    assert shapes(c, dtype) == ((0, 1), (0, 1))
    c.check(spv)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("ql,kl,H,K,D", [([1], [30001], 4, 4, 32), ([2, 1], [20000, 11], 2, 1, 64), ([1], [17000], 1, 1, 128)])
def test_keys_in_more_than_sixteen_parts(spv, ql, kl, H, K, D, dtype):  # noqa: F811
    """Rows that four waves join, with lse and the gradients."""
    print(f"queries {ql} keys {kl} {dtype}", flush=True)
    c = Case(kl, ql, H, K, D, dtype, bias=True, seed=1)
    assert shapes(c, dtype)[0][1] > 16
    c.check(spv)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("ql,kl,H,K", [([9000], [2], 2, 2), ([5000, 0], [3, 1], 4, 1)])
def test_rows_of_dk_and_dv_in_parts(spv, ql, kl, H, K, dtype):  # noqa: F811
    c = Case(kl, ql, H, K, 32, dtype, bias=True, seed=2)
    assert shapes(c, dtype)[1][1] > 8
    c.check(spv)


def test_large_launches_repeat_their_bits(spv):  # noqa: F811
    for mode in (0, 1):
        c = Case(scans(mode), None, 4, 2, 32, "bf16", bias=True, seed=4)
        first, again = c.run(spv), c.run(spv)
        assert all(torch.equal(first[n], again[n]) for n in first)
