"""Which way the fitted times send a product with 4-bit weights (CPU, no launch)."""
import ctypes

import paper_2506_23025_amd as tl
import test_gpu_four_ways as on_gpu

_way = tl.raw().tl_internal_four_way                      # not in tl.h: for the tests alone
_way.argtypes = [ctypes.c_int64] * 3
_way.restype = ctypes.c_int


def test_calls_of_the_gpu_tests_reach_every_way():
    for more in (0, 37):
        assert {_way(M, N, K + more) for M, N, K in on_gpu.WAYS} == set(range(23))
    assert all(_way(M, 1000, K) == -1 for M in (1, 5, 70) for K in (1, 7)) and _way(1, 16, 8) >= 0
