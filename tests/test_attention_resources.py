"""What the built attention kernels take of a compute unit, read from the metadata of the library's code object."""
import re

from tests.test_kernel_resources import built  # noqa: F401 (a fixture)

LDS = 160 * 1024
ARGS = r"%s<(\d), (\d+), (\d), (true|false), (\d)>\("  # type, padded channels, waves on a block, bias, cap's form


def attention(built, name):  # noqa: F811
    """{(type, channels, waves, bias, cap): metadata}"""
    found = {}
    for n, k in built.items():
        m = re.search(ARGS % name, n)
        if m:
            found[int(m[1]), int(m[2]), int(m[3]), m[4] == "true", int(m[5])] = k
    return found


def test_every_form_is_built(built):  # noqa: F811
    """Three types, four widths, the waves that a width has room for, with and without a bias, three forms of the cap."""
    forms = {(dt, dp, kw, bias, cap) for dt in range(3) for dp in (32, 64, 96, 128) for kw in (1, 2, 4)
             if kw <= (4 if dp * (2 if dt == 0 else 1) <= 64 else 2 if dp * (2 if dt == 0 else 1) <= 128 else 1)
             for bias in (False, True) for cap in range(3)}
    for name in ("k_attn", "k_attn_dq", "k_attn_dkv"):
        assert set(attention(built, name)) == forms, name


def test_attention_kernels_keep_their_registers(built):  # noqa: F811
    """Up to 96 channels a form spills some dozens of registers at most (with the exact cap up to a hundred), the widest
    heads more: a change that makes a form spill shows here.  All fit a compute unit's LDS."""
    for name in ("k_attn", "k_attn_dq", "k_attn_dkv"):
        for (dt, dp, kw, bias, cap), k in attention(built, name).items():
            form = (name, dt, dp, kw, bias, cap)
            assert k[".group_segment_fixed_size"] <= LDS, form
            spills = k[".vgpr_spill_count"]
            most = (64, 64, 128) if dp < 128 else (160, 160, 256)
            assert spills <= most[cap], (form, spills)
