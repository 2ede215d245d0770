"""8-bit rows and 4-bit weights without a GPU: the plain forms, the packers and the quantiser, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest

import paper_2506_23025_amd as tl
import rows as ref

P = 0x1000                                                 # an aligned address that no refusal reads


# ---- plain forms and layouts --------------------------------------------------------------------

def test_order_of_codes_meets_that_of_packed_words():
    rng = np.random.default_rng(0)
    W = rng.integers(-1, 2, (3, 50)).astype(np.int8)
    words = tl.tl_pack_2bit(W)
    for s in range(4):                                     # two bits of every byte of a word, against 4 bytes of a row's block
        two = (words[:, :, None] >> (2 * s + 8 * np.arange(4, dtype=np.uint32)) & 3).astype(np.int8) - 1
        assert np.array_equal(two, ref.in_order(W).reshape(3, -1, 4, 4)[:, :, s])
    assert np.array_equal(ref.out_of_order(ref.in_order(W), 50), W)


def test_codes_of_a_row():
    v = np.array([[0.0, -127.0, 63.5, 0.5, 1.5], [1e-31, -2e-31, 0, 0, 0], [0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0], [np.nan, 1, 2, 3, 4]], dtype=np.float32)
    c, s = ref.coded(v)
    assert c[0].tolist() == [0, -127, 64, 0, 2] and s[0] == 1
    assert (c[1:] == 0).all() and s[1:3].tolist() == [0, 0] and np.isnan(s[3:]).all()


@pytest.mark.parametrize("N,K", [(1, 1), (3, 7), (2, 128), (5, 129), (4, 1000)])
def test_packing_in_4_bits(N, K):
    rng = np.random.default_rng(N * 1000 + K)
    codes = rng.integers(0, 16, (N, K)).astype(np.uint8)
    packed = tl.tl_pack_4bit(codes)
    assert tl.tl_row_stride_4bit(K) == 64 * -(-K // 128) == packed.nbytes // N
    assert np.array_equal(packed, ref.pack4(codes)) and np.array_equal(tl.tl_unpack_4bit(packed, N, K), codes)


def test_a_block_of_4_bits_written_out():
    codes = np.zeros((1, 128), dtype=np.uint8)
    codes[0, 8 * 6 + 3] = 9                                # weight 3 of word 6: place 4 * 2 + 1, bits 16 + 4
    packed = tl.tl_pack_4bit(codes)
    assert packed[0, 9] == 9 << 20 and packed.astype(np.int64).sum() == 9 << 20


def test_quantising_to_4_bits():
    W = np.array([[0.7, -0.3, 0.05, -0.8] + [0] * 60], dtype=np.float32)
    codes, scales, zeros = tl.tl_quantize_4bit(W, 32)
    s = np.float16(np.float64(np.float32(0.8)) / 7)
    assert zeros is None and scales.shape == (2, 1) and scales[0, 0] == s and scales[1, 0] == 0 and (codes[0, 4:] == 8).all()
    assert codes[0, :4].tolist() == [8 + int(np.rint(float(w) / float(s))) for w in W[0, :4]]
    codes, scales, zeros = tl.tl_quantize_4bit(W, 32, True)
    s = np.float16((np.float64(np.float32(0.7)) + np.float64(np.float32(0.8))) / 15)
    assert scales[0, 0] == s and zeros[0, 0] == 8 and zeros[1, 0] == 8 and codes[0, :4].tolist() == [15, 5, 9, 0] or codes[0, 3] in (0, 1)


def test_quantising_to_4_bits_with_zero_points():
    codes, scales, zeros = tl.tl_quantize_4bit(np.array([[0.7, -0.3, 0.05, -0.8] + [0] * 60], dtype=np.float32), 32, True)
    s = np.float16((np.float64(np.float32(0.7)) + np.float64(np.float32(0.8))) / 15)
    assert scales[:, 0].tolist() == [s, 0] and zeros[:, 0].tolist() == [8, 8]
    assert codes[0, :4].tolist() == [15, 5, 9, 0]          # 8 + round(w / s): w / s is 7.0, -3.0, 0.5001 (s is below 0.1) and -8.0
    assert (codes[0, 4:] == 8).all()
    codes, scales, zeros = tl.tl_quantize_4bit(np.array([[3.0, 6.0, 15.0] + [3.0] * 29, [-15.0, -2.0, -7.0] + [-2.0] * 29], dtype=np.float32), 32, True)
    assert scales[0].tolist() == [1, 1] and zeros[0].tolist() == [0, 15]                # 0 is always among what a group can be
    assert codes[0, :4].tolist() == [3, 6, 15, 3] and codes[1, :4].tolist() == [0, 13, 8, 13]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 96, 4096])
def test_quantised_weights_are_near(group, zeros):
    rng = np.random.default_rng(group)
    W = (rng.standard_normal((6, 300)) + 0.3 * zeros).astype(np.float32)
    codes, scales, z = tl.tl_quantize_4bit(W, group, zeros)
    w = ref.weights4(codes, scales, z, group)
    s = scales.T.astype(np.float64)[:, np.arange(300) // group]
    # half a step; a scale rounded to fp16 moves the outermost codes by 15 * 2^-11 of a step more, and one held at the end of its range by as much again
    assert (np.abs(w - W) <= s * (0.5 + 2 * 15 * 2.0 ** -11 + (0.5 if zeros else 0))).all()


def test_4_bit_refusals():
    L, codes, scales = tl.raw(), np.zeros((1, 64), np.uint8), np.zeros(8, np.uint16)
    W = np.zeros((1, 64), np.float32)

    def quantize(W=W, N=1, K=64, group=32, codes=codes, scales=scales):
        return L.tl_quantize_4bit(None if W is None else W.ctypes.data, N, K, group, None if codes is None else codes.ctypes.data, None if scales is None else scales.ctypes.data, None)
    assert quantize() == tl.TL_OK
    for kw in ({"W": None}, {"codes": None}, {"scales": None}):
        assert quantize(**kw) == tl.TL_ERR_NULL
    for kw in ({"N": 0}, {"K": 0}, {"group": 0}, {"group": 48}, {"group": -32}, {"N": 1 << 40}):
        assert quantize(**kw) == tl.TL_ERR_SHAPE, kw
    for bad in (np.nan, np.inf, 1e6):
        V = W.copy()
        V[0, 40] = bad
        assert quantize(W=V) == tl.TL_ERR_VALUE
    out = np.zeros(64, np.uint32)
    bad = codes.copy()
    bad[0, 63] = 16
    assert L.tl_pack_4bit(bad.ctypes.data, 1, 64, out.ctypes.data) == tl.TL_ERR_VALUE
    for f in (L.tl_pack_4bit, L.tl_unpack_4bit):
        assert f(None, 1, 64, out.ctypes.data) == tl.TL_ERR_NULL and f(out.ctypes.data, 1, 64, None) == tl.TL_ERR_NULL
        assert f(out.ctypes.data, 0, 64, out.ctypes.data) == tl.TL_ERR_SHAPE and f(out.ctypes.data, 1, -1, out.ctypes.data) == tl.TL_ERR_SHAPE
    assert tl.tl_row_stride_4bit(0) == tl.tl_row_stride_4bit(-5) == 0


# ---- refusals of the entry points -----------------------------------------------------------------
#
# Calls of no rows pass all checks and do nothing, so what is refused can be told from what is not without a GPU.

def rows(**kw):
    return tl.tl_rows(**{**dict(ptr=P, stride=256), **kw})


def rows8(**kw):
    return tl.tl_rows8(**{**dict(codes=P, scales=P, stride=256), **kw})


NONE, NONE8 = tl.tl_rows(None, 0), tl.tl_rows8(None, None, 0)
BAD_ROWS = [({"ptr": P + 8}, tl.TL_ERR_ALIGN), ({"stride": 252}, tl.TL_ERR_ALIGN), ({"stride": -256}, tl.TL_ERR_SHAPE), ({"stride": 1 << 40}, tl.TL_ERR_SHAPE)]
BAD_ROWS8 = [({"scales": None}, tl.TL_ERR_NULL), ({"codes": P + 8}, tl.TL_ERR_ALIGN), ({"scales": P + 2}, tl.TL_ERR_ALIGN), ({"stride": 264}, tl.TL_ERR_ALIGN),
             ({"stride": -256}, tl.TL_ERR_SHAPE), ({"stride": 1 << 40}, tl.TL_ERR_SHAPE)]


def norm(**kw):
    job = tl.tl_norm_job(**{**dict(x=rows(), residual=rows(), sum=rows(), y=rows(), out=rows8(), weight=P, rows=0, dim=250, eps=1e-5, real=0), **kw})
    return tl.raw().tl_norm(ctypes.byref(job), None)


def gate(**kw):
    job = tl.tl_gate_job(**{**dict(gate=rows(), up=rows(), y=rows(), out=rows8(), rows=0, dim=250), **kw})
    return tl.raw().tl_gate(ctypes.byref(job), None)


def test_norm_refusals():
    assert norm() == norm(real=1) == norm(residual=NONE) == norm(weight=None) == norm(y=NONE, out=NONE8) == norm(sum=NONE, y=NONE) == tl.TL_OK
    assert tl.raw().tl_norm(None, None) == tl.TL_ERR_NULL
    assert norm(x=NONE) == norm(sum=NONE, y=NONE, out=NONE8) == norm(residual=NONE, y=NONE, out=NONE8) == tl.TL_ERR_NULL
    for name in ("x", "residual", "sum", "y"):
        for bad, status in BAD_ROWS:
            assert norm(**{name: rows(**bad)}) == status, (name, bad)
    for bad, status in BAD_ROWS8:
        assert norm(out=rows8(**bad)) == status, bad
    assert norm(residual=rows(stride=252), real=1) == tl.TL_OK            # 16 bytes are 4 places of 32 bits
    assert norm(weight=P + 8) == tl.TL_ERR_ALIGN
    for kw in ({"rows": -1}, {"rows": 1 << 31}, {"dim": 0}, {"dim": 65537}):
        assert norm(**kw) == tl.TL_ERR_SHAPE, kw
    for name in ("sum", "y"):
        assert norm(rows=2, **{name: rows(stride=248)}) == tl.TL_ERR_SHAPE
    assert norm(rows=2, out=rows8(stride=240)) == tl.TL_ERR_SHAPE
    for eps in (-1.0, float("nan"), float("inf")):
        assert norm(eps=eps) == tl.TL_ERR_VALUE
    assert norm(real=2) == tl.TL_ERR_UNSUPPORTED


def test_gate_refusals():
    assert gate() == gate(gate=NONE) == gate(y=NONE) == gate(out=NONE8) == tl.TL_OK
    assert tl.raw().tl_gate(None, None) == gate(up=NONE) == gate(y=NONE, out=NONE8) == tl.TL_ERR_NULL
    for name in ("gate", "up", "y"):
        for bad, status in BAD_ROWS:
            assert gate(**{name: rows(**bad)}) == status, (name, bad)
    for bad, status in BAD_ROWS8:
        assert gate(out=rows8(**bad)) == status, bad
    for kw in ({"rows": -1}, {"rows": 1 << 31}, {"dim": 0}, {"dim": 65537}, {"rows": 2, "y": rows(stride=248)}, {"rows": 2, "out": rows8(stride=240)}):
        assert gate(**kw) == tl.TL_ERR_SHAPE, kw


def test_rows8_product_refusals():
    def status(jobs=None, count=1, **kw):
        job = tl.tl_gemm_rows8_job(**{**dict(x=rows8(), Wpacked=P, y=P, M=2, N=16, K=250, gamma_fp16_bits=0), **kw})
        arr = (tl.tl_gemm_rows8_job * 1)(job)
        one = tl.raw().tl_ternary_gemm_rows8(ctypes.byref(job), None)
        assert count != 1 or tl.raw().tl_ternary_gemm_rows8_grouped(arr, count, None) == one
        return one if count == 1 else tl.raw().tl_ternary_gemm_rows8_grouped(arr, count, None)
    assert status(count=0) == tl.TL_OK and status(count=-1) == tl.TL_ERR_SHAPE
    assert tl.raw().tl_ternary_gemm_rows8(None, None) == tl.raw().tl_ternary_gemm_rows8_grouped(None, 2, None) == tl.TL_ERR_NULL
    assert status(Wpacked=None) == status(y=None) == status(x=NONE8) == tl.TL_ERR_NULL
    assert status(Wpacked=P + 4) == status(y=P + 2) == tl.TL_ERR_ALIGN
    for bad, s in BAD_ROWS8:
        assert status(x=rows8(**bad)) == s, bad
    for kw in ({"M": 0}, {"N": 0}, {"K": 0}, {"M": 1 << 31}, {"N": 1 << 24}, {"K": 1 << 24}, {"x": rows8(stride=240)}, {"M": 1 << 30, "N": 1 << 30}):
        assert status(**kw) == tl.TL_ERR_SHAPE, kw


def test_4_bit_product_refusals():
    def status(**kw):
        job = tl.tl_gemm_4bit_job(**{**dict(x=P, Wpacked=P, scales=P, zeros=P, y=P, M=1, N=16, K=256, group=64, y_real=0), **kw})
        return tl.raw().tl_gemm_4bit(ctypes.byref(job), None)
    assert tl.raw().tl_gemm_4bit(None, None) == tl.TL_ERR_NULL
    for name in ("x", "Wpacked", "scales", "y"):
        assert status(**{name: None}) == tl.TL_ERR_NULL
    for name in ("x", "Wpacked", "scales", "zeros", "y"):
        assert status(**{name: P + 8}) == tl.TL_ERR_ALIGN
    for kw in ({"M": 0}, {"N": 0}, {"K": 0}, {"group": 0}, {"group": 48}, {"group": -32}, {"N": 1 << 24}, {"K": 1 << 20}):
        assert status(**kw) == tl.TL_ERR_SHAPE, kw
    assert status(y_real=2) == tl.TL_ERR_UNSUPPORTED


def test_codes_that_are_no_type():
    """Any int may stand where a type or a kind is wanted, negative ones too: refused, and in the build with sanitizers not an undefined load."""
    scaling, table = tl.tl_rope_scaling(0, 1.0, 1.0, 0.0, 1.0, 1.0), np.zeros(8, np.float32)
    four = tl.tl_gemm_4bit_job(P, P, P, P, P, 1, 16, 256, 64, 0)
    for code in (-1, -2 ** 31, 7, 2 ** 31 - 1):
        assert norm(real=code) == tl.TL_ERR_UNSUPPORTED
        four.y_real = scaling.kind = code
        assert tl.raw().tl_gemm_4bit(ctypes.byref(four), None) == tl.TL_ERR_UNSUPPORTED
        assert tl.raw().tl_rope_table(table.ctypes.data, 1, 8, 1e4, ctypes.byref(scaling)) == tl.TL_ERR_UNSUPPORTED
