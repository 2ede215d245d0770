"""Norm, gate and plain rows in every form that the kernel has: 1 to 16 waves to a row, 1 to 8 pieces a lane, by the rows' length and by whether there are 256 of them."""
import numpy as np
import pytest

from test_gpu_rows import check_gate, check_norm, values

pytestmark = pytest.mark.gpu

# below and at the ends of the forms, and whole pieces
DIMS = [509, 512, 1021, 2045, 2999, 4091, 4097, 8187, 8192, 12283, 12288, 16381, 16384, 32765, 65533]


@pytest.mark.parametrize("rows", [3, 257])
@pytest.mark.parametrize("dim", DIMS)
def test_norm_in_every_form(dim, rows):
    if rows * dim > 1 << 22:
        rows = 256                                         # as many as make the difference
    check_norm(rows, dim, np.float16, seed=1)
    check_norm(rows, dim, np.float32, weight=dim % 2 == 1, seed=2)
    check_norm(rows, dim, np.float16, residual=False, seed=3)


def not_finite(rng, g, u):
    """An infinity or a NaN in every other row, at its ends, where pieces meet, and anywhere."""
    rows, dim = u.shape
    at = [0, dim - 1, dim // 2, 7, 8, min(dim - 1, 511), min(dim - 1, 512), min(dim - 1, 4096)] + list(rng.integers(0, dim, rows))
    kinds = [(np.inf, 1), (-np.inf, 1), (1, np.inf), (np.nan, 2), (3, np.nan), (-np.inf, np.inf), (0, np.inf), (-2, -np.inf)]
    for i, r in enumerate(range(0, rows, 2)):
        g[r, at[i % len(at)]], u[r, at[i % len(at)]] = kinds[i % len(kinds)]


@pytest.mark.parametrize("rows", [17, 257])
@pytest.mark.parametrize("dim", DIMS)
def test_gate_in_every_form(dim, rows):
    if rows * dim > 1 << 22:
        rows = 256
    check_gate(rows, dim, seed=4)
    check_gate(rows, dim, True, seed=5)
    rng = np.random.default_rng(dim)
    g, u = values(rng, rows, dim, scale=2.0), values(rng, rows, dim)
    not_finite(rng, g, u)
    check_gate(rows, dim, g=g, u=u)
    check_gate(rows, dim, True, u=u)


@pytest.mark.parametrize("rows", [17, 257])
@pytest.mark.parametrize("dim", [509, 4091, 8187, 12283, 16381, 65533])
def test_norm_of_infinities_in_every_form(dim, rows):
    rng = np.random.default_rng(dim + 1)
    x, r = values(rng, rows, dim), values(rng, rows, dim, np.float32)
    not_finite(rng, x, r)
    check_norm(rows, dim, np.float32, x=x, r=r)
