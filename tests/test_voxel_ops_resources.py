"""What the built kernels of rotary positions, group norm and rows in 8 bits take of a compute unit, read from the metadata of
the library's code object."""
import re

from tests.test_kernel_resources import built  # noqa: F401 (a fixture)

LDS = 160 * 1024
NAMES = ("k_rope_rows", "k_rope_pairs", "k_gn_few", "k_gn_tile_stat", "k_gn_tile_apply", "k_gn_tile_sums", "k_gn_tile_dx",
         "k_gn_join", "k_code8", "k_code8_read", "k_code8_short", "k_code8_any", "k_wgrad8", "k_wgrad8_any", "k_wgrad8_join")


def test_kernels_keep_their_registers(built):  # noqa: F811
    """No form spills a register, all fit a compute unit's LDS, and the tiles' kernels leave room for two workgroups."""
    for name in NAMES:
        found = {n: k for n, k in built.items() if re.search(r"spv::%s[<(]" % name, n)}
        assert found, name
        for n, k in found.items():
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n
            assert k[".group_segment_fixed_size"] <= LDS, n
            if "k_gn_tile" in n:  # 512 threads: two waves a SIMD each
                assert k[".vgpr_count"] <= 128 and 2 * k[".group_segment_fixed_size"] <= LDS, n
