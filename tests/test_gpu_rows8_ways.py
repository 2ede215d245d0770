"""Ternary products over 8-bit rows in every way that a launch of them has: test_rows8_launches.py holds that these calls reach each."""
import numpy as np
import pytest

import paper_2506_23025_amd as tl
from test_gpu_rows import gamma_bits, on, rows8_of, same

pytestmark = pytest.mark.gpu

# More than 16 rows: odd sizes of a few steps along K, and longer ones with whole pieces of 16 bytes to a row of y; packed rows that are a multiple of 16 bytes, and others.
MANY = [(19, 19, 53), (21, 17, 16), (33, 2079, 51), (33, 2147, 17), (19, 17, 5368), (17, 17, 5577), (33, 4149, 1152), (17, 9281, 1102), (1423, 653, 320), (1423, 653, 264), (35, 8199, 50),
        (35, 8383, 16), (75, 11107, 1856), (105, 8707, 1802), (103, 10299, 183), (165, 6959, 129), (193, 11457, 2496), (195, 10081, 2884), (129, 13275, 192), (129, 13809, 132), (65, 10887, 54),
        (71, 10903, 16)]
LONG = [(17, 16, 4032), (17, 16, 4007), (33, 2056, 3839), (33, 2112, 4010), (19, 16, 5440), (17, 16, 5517), (33, 4288, 3840), (33, 4240, 4035), (33, 8440, 4032), (33, 8816, 3888), (65, 8432, 4096),
        (65, 9072, 4010), (67, 11320, 3968), (65, 11736, 3851), (71, 11280, 2816), (67, 11600, 2765), (133, 13728, 3968), (131, 13360, 4097), (131, 14992, 2929), (199, 10232, 2608),
        (389, 13464, 2112), (399, 13608, 2149), (100, 4096, 11008)]
# Two products that share a launch.
JOINT = [((19, 17, 3008), (19, 16, 512)), ((19, 17, 2736), (19, 16, 238)), ((21, 21, 2496), (17, 4140, 256)), ((33, 41, 2847), (17, 5071, 227)), ((21, 17, 5184), (17, 17, 384)),
         ((21, 17, 5643), (17, 17, 576)), ((17, 95, 4032), (17, 8524, 256)), ((71, 39, 4849), (35, 5907, 208)), ((65, 21, 3136), (65, 6049, 256)), ((33, 33, 4168), (33, 8667, 444)),
         ((81, 21, 2304), (81, 8299, 256)), ((91, 27, 2301), (91, 8351, 266)), ((157, 119, 3136), (157, 7217, 1088)), ((145, 25, 3317), (145, 6880, 1444)), ((117, 83, 1728), (117, 8241, 320)),
         ((633, 23, 1430), (633, 1645, 200)), ((193, 4639, 3136), (193, 4639, 1344)), ((341, 3483, 2729), (341, 3483, 230)), ((163, 6927, 2432), (163, 6927, 256)),
         ((195, 4725, 2409), (195, 4725, 301)), ((397, 6447, 1723), (397, 6447, 250)), ((399, 6691, 2651), (399, 6691, 1430))]
# Up to 16 rows.
FEW = [(1, 17, 17), (4, 1001, 3000), (1, 17, 4099), (3, 8000, 4352), (2, 12845, 16), (4, 22016, 2000), (3, 12573, 2126), (4, 14336, 4096), (5, 17, 16), (8, 10001, 1000), (6, 17, 1067), (8, 6000, 5000), (7, 14399, 16),
       (8, 16384, 4096), (5, 33307, 16), (8, 36000, 2100), (5, 24811, 17), (7, 26000, 3000), (9, 17, 16), (16, 4096, 2000), (13, 17, 2096), (16, 4000, 4000), (9, 4243, 17), (16, 8000, 1800), (9, 4253, 2066),
       (15, 8192, 3000), (9, 8253, 17), (16, 12288, 1500), (9, 8965, 2114), (16, 12288, 4096), (9, 12755, 17), (16, 16000, 1000), (9, 12943, 2186), (15, 15001, 3000), (9, 16385, 17), (16, 24000, 4000),
       (11, 16397, 4316), (16, 22016, 5000)]


def check(seed, *sizes):
    """The products are summed in 64 bits on the host, where these sums are exact, and so is the kernels'."""
    import torch
    rng = np.random.default_rng(seed)
    calls, wants, outs = [], [], []
    for M, N, K in sizes:
        codes = np.clip(np.rint(rng.standard_normal((M, K)) * 40), -127, 127).astype(np.int8)
        scales = (0.01 + rng.random(M) / 30).astype(np.float32)
        W = rng.integers(-1, 2, (N, K), dtype=np.int8)
        gamma = np.float16(0.01 + 0.04 * rng.random())
        y = torch.full((M * N + 128,), 77.0, dtype=torch.float16, device="cuda")
        calls.append((rows8_of(codes, scales), on(tl.tl_pack_2bit(W).view(np.int32)), gamma_bits(gamma), y[64:64 + M * N].view(M, N)))
        outs.append(y)
        a = codes.astype(np.float64) @ W.astype(np.float64).T
        wants.append((a.astype(np.float32) * (scales * np.float32(gamma))[:, None]).astype(np.float16))
    tl.tl_ternary_gemm_rows8_grouped(calls)
    for y, want in zip(outs, wants):
        got = y.cpu().numpy()
        assert (got[:64] == 77).all() and (got[64 + want.size:] == 77).all(), "written outside of the output"
        same(got[64:64 + want.size].reshape(want.shape), want)


@pytest.mark.parametrize("M,N,K", MANY + LONG)
def test_more_than_16_rows(M, N, K):
    check(M + N + K, (M, N, K))


@pytest.mark.parametrize("one,two", JOINT)
def test_two_products_of_one_launch(one, two):
    check(sum(one), one, two)


@pytest.mark.parametrize("M,N,K", FEW)
def test_up_to_16_rows(M, N, K):
    check(M + N + K, (M, N, K))
    check(M + N + K + 1, (M, N - N // 3, K), (max(1, M - 1), N // 3, K))


def test_a_decode_batch_of_three_products():
    check(3, *[(16, 4096, 4096)] * 3)
