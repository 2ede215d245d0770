"""What launches ternary products over 8-bit rows make (CPU, no launch)."""
import ctypes

import pytest

import paper_2506_23025_amd as tl
import test_gpu_rows8_ways as on_gpu

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


def ways(few, calls):
    """The (way, odd packed rows) of calls that make one launch each."""
    found = set()
    for sizes in calls:
        (launch,) = launches(*sizes)
        assert launch["few"] == few and launch["jobs"] == len(sizes), sizes
        found.add((launch["way"], launch["ragged"]))
    return found


def test_calls_of_the_gpu_tests_reach_every_way():
    every = {(way, ragged) for way in range(11) for ragged in (0, 1)}
    for calls in ([(s,) for s in on_gpu.MANY], [(s,) for s in on_gpu.LONG], on_gpu.JOINT):
        assert ways(0, calls) == every
    every = {(way, 0) for way in range(19)}
    assert ways(1, [(s,) for s in on_gpu.FEW]) == every
    assert ways(1, [((M, N - N // 3, K), (max(1, M - 1), N // 3, K)) for M, N, K in on_gpu.FEW]) == every
