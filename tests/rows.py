"""Plain forms of the operators on 8-bit rows and 4-bit weights, numpy in 64 bits, and their layouts."""
import numpy as np

F32 = np.float32


def up(x, to):
    return -(-x // to) * to


# ---- 8-bit rows --------------------------------------------------------------------------------

def in_order(codes):
    """int8 [rows][dim] -> the bytes of tl_rows8, [rows][ceil(dim / 16) * 16]: place 4 i + s of a block is byte 4 s + i."""
    rows, dim = codes.shape
    c = np.zeros((rows, up(dim, 16)), dtype=np.int8)
    c[:, :dim] = codes
    return np.ascontiguousarray(c.reshape(rows, -1, 4, 4).transpose(0, 1, 3, 2)).reshape(rows, -1)


def out_of_order(bytes_, dim):
    rows = bytes_.shape[0]
    return bytes_.reshape(rows, -1, 4, 4).transpose(0, 1, 3, 2).reshape(rows, -1)[:, :dim]


def coded(v):
    """float32 rows -> (int8 codes [rows][dim], float32 scales), each step as IEEE fp32 has it."""
    v = v.astype(F32)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(1)
        bad = ~np.isfinite(v).all(1)
        some = ~bad & (top >= F32(2.0) ** -100)
        scale = np.where(bad, F32(np.nan), np.where(some, top / F32(127), F32(0))).astype(F32)
        inverse = np.where(some, F32(127) / np.where(some, top, F32(1)), F32(0)).astype(F32)
        codes = np.where(some[:, None], np.rint(v * inverse[:, None]), 0).astype(np.int8)
    return codes, scale


def norm(x, residual=None, weight=None, eps=1e-5, kind=np.float16):
    """(sum, v): the sum in `kind`, the normed rows in float32.  The mean is taken in 64 bits."""
    with np.errstate(all="ignore"):
        s = x.astype(F32) if residual is None else (residual.astype(F32) + x.astype(F32)).astype(kind)
        f = s.astype(F32)
        r = (1.0 / np.sqrt((f.astype(np.float64) ** 2).sum(1) / f.shape[1] + np.float64(F32(eps)))).astype(F32)
        v = f * r[:, None]
        return s, v if weight is None else v * weight.astype(F32)


def gate(g, u):
    """float32 rows; the gate in 64 bits."""
    if g is None:
        return u.astype(F32)
    with np.errstate(all="ignore"):
        g, u = g.astype(np.float64), u.astype(np.float64)
        return (g / (1.0 + np.exp(-g)) * u).astype(F32)


def ternary(codes, scale, W, gamma):
    """float16 [M][N]: the sum in whole numbers, products and rounding as IEEE has them."""
    a = codes.astype(np.int64) @ W.astype(np.int64).T
    with np.errstate(all="ignore"):
        return (a.astype(F32) * (scale.astype(F32) * F32(gamma))[:, None]).astype(np.float16)


# ---- 4-bit weights -----------------------------------------------------------------------------

def pack4(codes):
    N, K = codes.shape
    c = np.zeros((N, up(K, 128)), dtype=np.uint32)
    c[:, :K] = codes
    at = np.array([0, 16, 4, 20, 8, 24, 12, 28], dtype=np.uint32)
    w = (c.reshape(N, -1, 8) << at).sum(-1, dtype=np.uint64).astype(np.uint32)
    return np.ascontiguousarray(w.reshape(N, -1, 4, 4).transpose(0, 1, 3, 2)).reshape(N, -1)


def weights4(codes, scales, zeros, group):
    """float64 [N][K]."""
    g = np.arange(codes.shape[1]) // group
    z = 8.0 if zeros is None else zeros.T.astype(np.float64)[:, g]
    return (codes.astype(np.float64) - z) * scales.T.astype(np.float64)[:, g]


def gemm4(x, w):
    """(y, how far a sum in 32 bits may be off): K additions whose partial sums are as a random walk's, each off by up to 2^-23 of it (matrix instructions may cut off), and four times that."""
    x = x.astype(np.float64)
    return x @ w.T, 4 * 2.0 ** -23 * np.sqrt(x.shape[1]) * np.sqrt((x ** 2) @ (w ** 2).T)
