"""The gate over the ranges of fp16 as fp32 has it, and 4-bit products with zero points of any byte."""
import numpy as np
import pytest

import paper_2506_23025_amd as tl
import rows as ref
from test_gpu_rows import on, same

pytestmark = pytest.mark.gpu


def gated(g, u):
    """tl_gate's scales of rows of one place each: fl(|v| / 127), which shows v as it is in 32 bits."""
    import torch
    n = len(g)
    rows = torch.zeros((n, 16), dtype=torch.float16, device="cuda")         # gate and up of a row, 16 bytes each
    rows[:, 0], rows[:, 8] = on(g), on(u)
    codes, scales = torch.zeros((n, 16), dtype=torch.int8, device="cuda"), torch.full((n,), 77.0, device="cuda")
    tl.tl_gate(tl.make_gate_job(rows[:, :1], rows[:, 8:9], None, tl.make_rows8(codes, scales, 1)))
    c = codes.cpu().numpy()
    v = c[:, 0]
    assert (c[:, 1:] == 0).all()
    return v, scales.cpu().numpy()


# In 64 bits the kernel is off by less than 2^-50 of its result from g = -1 on and by less than 2^-47 at the least g that leaves one in fp32, since log(2) is held in one number and moves e^-g by 2^-55.2 for every
# power of 2 in it.  So its fp32 rounding is the exact value's where that is further than 2^-46 of itself from the middle between two fp32 numbers, and one of the two otherwise.  The exact value
# is taken in 80 bits here, off by 2^-62.
@pytest.mark.parametrize("lo,hi", [(-104.0, -10.0), (-10.0, -1.0), (-1.0, 0.0), (0.0, 65504.0)])
def test_gate_in_32_bits(lo, hi):
    g = np.arange(65536, dtype=np.uint16).view(np.float16)
    g = g[np.isfinite(g)]
    g = g[(g > lo) & (g <= hi) & (g != 0)]
    rng = np.random.default_rng(int(-lo) + 1)
    each = max(1, (1 << 21) // len(g))
    u = (1 + rng.integers(0, 1024, (len(g), each)) / 1024).astype(np.float16)
    g, u = np.repeat(g, each), u.reshape(-1)
    codes, scales = gated(g, u)
    wide = g.astype(np.longdouble)
    exact = wide / (1 + np.exp(-wide)) * u.astype(np.longdouble)
    v = exact.astype(np.float32)
    other = np.nextafter(v, np.where(v.astype(np.longdouble) < exact, np.float32(np.inf), np.float32(-np.inf)), dtype=np.float32)
    near = np.abs(exact - (v.astype(np.longdouble) + other.astype(np.longdouble)) / 2) <= 2.0 ** -46 * np.abs(exact)
    assert near.mean() < 2.0 ** -12                         # few, but where g is so small that the gate is g / 2 to 40 bits
    least = np.float32(2.0) ** -100                         # below it a row is 0
    with np.errstate(all="ignore"):
        a, b = ((np.where(np.abs(t) >= least, np.abs(t) / np.float32(127), np.float32(0))).astype(np.float32) for t in (v, other))
    assert ((scales == a) | (near & (scales == b))).all(), f"{int((scales != a).sum())} differ, {int(near.sum())} near"
    same(codes, np.where(scales > 0, np.where(v < 0, -127, 127), 0).astype(np.int8))


@pytest.mark.parametrize("M,N,K,group", [(1, 40, 5, 32), (1, 70, 520, 128), (3, 70, 500, 64), (20, 70, 500, 32), (70, 33, 300, 256), (130, 65, 260, 64)])
def test_four_of_any_zero_point(M, N, K, group):
    import torch
    rng = np.random.default_rng(M + N + K)
    x, codes = rng.standard_normal((M, K)).astype(np.float16), rng.integers(0, 16, (N, K)).astype(np.uint8)
    G = -(-K // group)
    scales, zeros = ((0.5 + rng.random((G, N))) / 16).astype(np.float16), rng.integers(0, 256, (G, N)).astype(np.uint8)
    zeros[0, :4] = 255, 254, 16, 128
    y = torch.empty((M, N), device="cuda")
    tl.tl_gemm_4bit(tl.make_4bit_job(on(x), on(tl.tl_pack_4bit(codes).view(np.int32)), on(scales), on(zeros), group, y))
    want, off = ref.gemm4(x, ref.weights4(codes, scales, zeros, group))     # code - zero is exact in fp16 for any byte: 1024 + 255 is below 2048
    assert (np.abs(y.cpu().numpy() - want) <= off + 2.0 ** -24 * np.abs(want)).all()
