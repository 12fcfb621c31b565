"""The sizes at which test_gpu_kvq_tiles.py runs the attention over the 4-bit cache, and that they are run as it says."""
import pytest

import paper_2512_16483_amd as fv
from test_kvq_host import ways

# dtype, head_dim, heads, kv heads, samples, queries, keys, way (rows of a block, wavefronts of its workgroup, shares of a divided block),
# and for how many wavefronts to a SIMD the kernel is built that runs it
TILES = {
    "one group, 64, 3 waves": ("bf16", 64, 8, 8, 40, 250, 421, (128, 4, 1), 3),
    "one group, 64": ("bf16", 64, 8, 2, 32, 200, 421, (128, 4, 1), 2),
    "one group, 128": ("bf16", 128, 8, 8, 32, 200, 421, (128, 4, 1), 2),
    "one group divided, 64, 3 waves": ("bf16", 64, 16, 16, 31, 200, 777, (128, 4, 3), 3),
    "one group divided, 128": ("bf16", 128, 4, 4, 70, 200, 777, (128, 4, 3), 2),
    "two groups, 64": ("bf16", 64, 8, 8, 14, 240, 777, (128, 8, 1), 2),
    "two groups, 128": ("bf16", 128, 4, 4, 20, 230, 1100, (128, 8, 1), 2),
    "two groups divided, 64": ("bf16", 64, 4, 4, 4, 500, 2100, (128, 8, 4), 2),
    "two groups divided, 128": ("bf16", 128, 8, 2, 4, 250, 2100, (128, 8, 4), 2),
}
SIXTEEN = {
    "16 rows": ("bf16", 128, 4, 2, 20, 33, 421, (16, 4, 1), 3),
    "16 rows, 3 shares": ("bf16", 64, 8, 2, 4, 30, 900, (16, 4, 3), 3),
    "16 rows, 19 shares": ("bf16", 128, 4, 4, 1, 1, 5000, (16, 4, 19), 3),
    "16 rows, fp32": ("f32", 64, 4, 4, 9, 60, 421, (16, 4, 1), 2),
    "16 rows, fp32, 3 shares": ("f32", 128, 4, 2, 4, 20, 900, (16, 4, 3), 2),
    "16 rows, fp32, 19 shares": ("f32", 64, 2, 2, 1, 3, 5000, (16, 4, 19), 2),
}


def check_way(name):
    dtype, dh, H, heads, B, n, L, expect, waves = {**TILES, **SIXTEEN}[name]
    built = fv.load_library()["_ZN4fvar28kvq_attention_waves_per_simdEiiiiiiii"]
    for ragged in (False, True):
        assert ways(dtype, B, n, H, heads, dh, L, ragged) == expect
        assert built(dtype == "bf16", B, n, H, heads, dh, L, ragged) == waves


@pytest.mark.parametrize("name", sorted(TILES) + sorted(SIXTEEN))
def test_sizes_are_run_as_the_tests_want_them(name):
    check_way(name)
