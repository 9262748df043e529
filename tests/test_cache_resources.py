"""What the compiler reports of the cache kernels in libminf.so."""
from tests.test_kernel_resources import kernels  # noqa: F401  (a fixture)


def test_cache_kernels_use_no_scratch_memory(kernels):  # noqa: F811
    """Two waves a SIMD leave 256 registers, and a rare path that needs more would spill in the tile loop."""
    names = [n for n in kernels if "cache_" in n]
    assert {n.split("cache_")[1].split("_kernel")[0] for n in names} == {"attn", "shared", "prefix", "join", "column", "select", "count",
                                                                          "emit", "move"}
    for n in names:
        assert kernels[n][".private_segment_fixed_size"] == 0 and kernels[n][".vgpr_spill_count"] == 0, n
