"""Products with 4-bit weights in every way to deal rows and columns to workgroups, with every form of groups and zero points: test_four_ways.py holds that these calls reach each."""
import pytest

from test_gpu_rows import check_four

pytestmark = pytest.mark.gpu

WAYS = [(2, 65, 520), (5, 65, 1100), (17, 65, 2600), (17, 2501, 1900), (2, 9000, 520), (5, 65, 520), (33, 1501, 520), (33, 4097, 1100), (49, 4097, 520), (65, 65, 520), (65, 65, 1100),
        (100, 3201, 520), (100, 4097, 520), (130, 65, 520), (130, 3201, 1100), (130, 3201, 520), (211, 65, 520), (211, 2501, 1100), (211, 2501, 520), (1, 65, 4100), (1, 9000, 520), (1, 13001, 520),
        (1, 25001, 520), (1, 65, 520)]


@pytest.mark.parametrize("group,zeros", [(32, False), (96, True), (64, False), (192, True), (128, True), (384, False)])
@pytest.mark.parametrize("M,N,K", WAYS)
def test_four_in_every_way(M, N, K, group, zeros):
    check_four(M + N + group, M, N, K, group, zeros, wide=True)
    check_four(M + N + group + 1, M, N, K + 37, group, zeros)
