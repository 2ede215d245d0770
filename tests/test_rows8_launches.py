"""What launches ternary products over 8-bit rows make (CPU, no launch)."""
import ctypes

import pytest

import paper_2506_23025_amd as tl

_launches = tl.raw().tl_internal_rows8_launches           # not in tl.h: for the tests alone
_launches.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int]
_launches.restype = ctypes.c_int


def launches(*sizes, most=4096):
    """Of products of (M, N, K) in one call: a dict for each launch."""
    flat, out = (ctypes.c_int64 * (3 * len(sizes)))(*[v for s in sizes for v in s]), (ctypes.c_int64 * (7 * most))()
    n = _launches(flat, len(sizes), out, most)
    assert 0 <= n <= most
    return [dict(zip(("few", "way", "ragged", "jobs", "rows", "groups", "threads"), out[7 * i:7 * i + 7])) for i in range(n)]


# A grid counts its threads in 32 bits.  The narrowest matrices have the most workgroups for what they write, whatever the tile.
@pytest.mark.parametrize("sizes", [[(1 << 29, 1, 160)], [(1 << 30, 1, 16)], [((1 << 31) - 1, 1, 129)], [((1 << 31) - 1, 16, 100)], [((1 << 31) - 1, 511, 500)], [(1 << 27, 8, 1000)],
                                   [(1 << 16, (1 << 24) - 1, 64)], [(70000, 5000000, 1 << 18)], [(16, (1 << 24) - 1, 4096)] * 16, [(1, (1 << 24) - 1, 64)] * 64,
                                   [(1 << 26, 1, 160)] * 16, [(1 << 25, 3, 129), (1 << 28, 2, 1024), (5, 1 << 23, 64)] * 5])
def test_a_launch_counts_its_threads_in_32_bits(sizes):
    found = launches(*sizes, most=1 << 16)
    assert all(0 < launch["groups"] * launch["threads"] < 1 << 32 for launch in found)
    assert sum(launch["rows"] for launch in found) == sum(M for M, _, _ in sizes)
