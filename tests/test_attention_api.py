"""The attention part without a GPU: the table of rotations, the layout helpers of its tests, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest

import attention as ref
import paper_2506_23025_amd as tl

P = 0x1000                                                 # an aligned address that no refusal reads


def test_table_of_rotations():
    t = tl.tl_rope_table(50, 8, 100.0)
    assert t.shape == (50, 8) and t.dtype == np.float32
    f = 100.0 ** (-np.arange(4) / 4)
    a = np.arange(50)[:, None] * f
    assert np.array_equal(t, np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)) or np.abs(t - np.concatenate([np.cos(a), np.sin(a)], 1)).max() < 1e-7


def test_table_of_rotations_for_long_contexts():
    p = np.arange(64)[:, None]
    f = 10000.0 ** (-np.arange(16) / 16)

    def near(t, f, m=1.0):
        return np.abs(t - m * np.concatenate([np.cos(p * f), np.sin(p * f)], 1)).max() < 1e-6

    assert near(tl.tl_rope_table(64, 32, kind=tl.TL_ROPE_LINEAR, factor=4.0), f / 4)
    turns = 2048 * f / (2 * np.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    assert (keep == 0).any() and (keep == 1).any() and ((keep > 0) & (keep < 1)).any()
    assert near(tl.tl_rope_table(64, 32, kind=tl.TL_ROPE_BY_PARTS, factor=8.0, trained=2048.0, low=1.0, high=32.0, magnitude=1.2), keep * f + (1 - keep) * f / 8, 1.2)


def test_table_refusals():
    def status(table=True, positions=4, rot=8, base=10000.0, **kw):
        sc = tl.tl_rope_scaling(**{**dict(kind=0, factor=1.0, trained=1.0, low=0.0, high=1.0, magnitude=1.0), **kw})
        out = np.empty(4096, dtype=np.float32)
        return tl.raw().tl_rope_table(out.ctypes.data if table else None, positions, rot, base, ctypes.byref(sc))
    assert status() == tl.TL_OK
    assert status(table=False) == tl.TL_ERR_NULL
    for kw in ({"positions": 0}, {"rot": 0}, {"rot": 7}, {"positions": 1 << 62}):
        assert status(**kw) == tl.TL_ERR_SHAPE, kw
    for kw in ({"base": 0.0}, {"base": float("nan")}, {"kind": 1, "factor": 0.0}, {"kind": 2, "low": 2.0}, {"kind": 2, "trained": -1.0}, {"magnitude": float("inf")}):
        assert status(**kw) == tl.TL_ERR_VALUE, kw
    assert status(kind=7) == tl.TL_ERR_UNSUPPORTED
    assert tl.raw().tl_rope_table(np.empty(32, np.float32).ctypes.data, 4, 8, 10.0, None) == tl.TL_OK


def test_plain_forms():
    rng = np.random.default_rng(0)
    x = rng.integers(0, 256, (2, 16, 48)).astype(np.uint8)
    for key in (True, False):
        m = ref.to_layout(x, key)
        assert sorted(m[0]) == sorted(x[0].reshape(-1)) and np.array_equal(ref.from_layout(m, 48, key), x)
    codes = np.array([c for c in range(256) if (c & 127) != 127], dtype=np.uint8)
    back = ref.encode(ref.E4M3[codes].astype(np.float32), "fp8")
    assert np.array_equal(back[codes != 128], codes[codes != 128])
    torch = pytest.importorskip("torch")
    y = (rng.standard_normal(20000) * 10.0 ** rng.uniform(-4, 2.6, 20000)).astype(np.float32).clip(-448, 448)
    assert np.array_equal(torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), ref.encode(y, "fp8"))


def heads(**kw):
    return tl.tl_heads(**{**dict(ptr=P, token_stride=256, head_stride=128), **kw})


def cache(**kw):
    return tl.tl_kv_cache(**{**dict(k=P, v=P, k_scale=P, v_scale=P, page_table=P, pages=4, page_tokens=64, pages_per_seq=2, kv_heads=2, head_dim=128, type=0), **kw})


def batch(**kw):
    return tl.tl_batch(**{**dict(seq_start=P, cached=P, seqs=3, tokens=0), **kw})


BAD_BATCHES = [({"seqs": 0}, tl.TL_ERR_SHAPE), ({"seqs": 1 << 20}, tl.TL_ERR_SHAPE), ({"tokens": -1}, tl.TL_ERR_SHAPE), ({"tokens": 1 << 30}, tl.TL_ERR_SHAPE),
               ({"seq_start": None, "tokens": 5}, tl.TL_ERR_SHAPE), ({"seq_start": P + 2}, tl.TL_ERR_ALIGN), ({"cached": P + 1}, tl.TL_ERR_ALIGN)]
BAD_HEADS = [({"ptr": None}, tl.TL_ERR_NULL), ({"ptr": P + 8}, tl.TL_ERR_ALIGN), ({"token_stride": -8}, tl.TL_ERR_SHAPE), ({"token_stride": 12}, tl.TL_ERR_ALIGN),
             ({"head_stride": 4}, tl.TL_ERR_ALIGN), ({"head_stride": -128}, tl.TL_ERR_SHAPE), ({"token_stride": 1 << 31}, tl.TL_ERR_SHAPE)]
BAD_CACHES = [({n: None}, tl.TL_ERR_NULL) for n in ("k", "v", "k_scale", "v_scale", "page_table")] + [
    ({"k": P + 8}, tl.TL_ERR_ALIGN), ({"v_scale": P + 2}, tl.TL_ERR_ALIGN), ({"page_tokens": 8}, tl.TL_ERR_SHAPE), ({"page_tokens": 48}, tl.TL_ERR_SHAPE),
    ({"page_tokens": 2048}, tl.TL_ERR_SHAPE), ({"pages": 0}, tl.TL_ERR_SHAPE), ({"pages_per_seq": 0}, tl.TL_ERR_SHAPE), ({"pages_per_seq": 1 << 30}, tl.TL_ERR_SHAPE),
    ({"kv_heads": 0}, tl.TL_ERR_SHAPE), ({"head_dim": 136}, tl.TL_ERR_SHAPE), ({"head_dim": 256}, tl.TL_ERR_SHAPE), ({"head_dim": 0}, tl.TL_ERR_SHAPE),
    ({"type": 2}, tl.TL_ERR_UNSUPPORTED), ({"type": -1}, tl.TL_ERR_UNSUPPORTED)]


def append(b=None, c=None, r=None, **kw):
    j = tl.tl_append_job(**{**dict(q=heads(), k=heads(), v=heads(), q_out=heads(), k_out=heads(), batch=b or batch(), q_heads=4, kv_heads=2, head_dim=128), **kw})
    if c is not None:
        j.cache = ctypes.pointer(c)
    if r is not None:
        j.rope = ctypes.pointer(r)
    return tl.raw().tl_kv_append(ctypes.byref(j), None)


def rope(**kw):
    return tl.tl_rope(**{**dict(table=P, positions=10, rot_dim=128, pairs=0), **kw})


def test_append_refusals():
    L = tl.raw()
    assert L.tl_kv_append(None, None) == tl.TL_ERR_NULL
    assert append(c=cache(), r=rope()) == tl.TL_OK            # no tokens: nothing to do
    for kw, e in BAD_BATCHES:
        assert append(b=batch(**kw), c=cache()) == e, kw
    for kw, e in BAD_CACHES:
        assert append(c=cache(**kw)) == e, kw
    for kw, e in BAD_HEADS:
        for name in ("q", "k", "v", "q_out", "k_out"):
            if name.endswith("out") and kw == {"ptr": None}:
                continue
            assert append(c=cache(), **{name: heads(**kw)}) == e, (name, kw)
    for kw, e in (({"table": None}, tl.TL_ERR_NULL), ({"table": P + 2}, tl.TL_ERR_ALIGN), ({"positions": 0}, tl.TL_ERR_SHAPE), ({"rot_dim": 0}, tl.TL_ERR_SHAPE),
                  ({"rot_dim": 7}, tl.TL_ERR_SHAPE), ({"rot_dim": 130}, tl.TL_ERR_SHAPE)):
        assert append(r=rope(**kw)) == e, kw
    for kw in ({"q_heads": -1}, {"kv_heads": -2}, {"q_heads": 0, "kv_heads": 0}, {"head_dim": 8}, {"head_dim": 144}, {"head_dim": 72}, {"q_heads": 5000}):
        assert append(**kw) == tl.TL_ERR_SHAPE, kw
    assert append(c=cache(), kv_heads=1) == tl.TL_ERR_SHAPE and append(c=cache(head_dim=64)) == tl.TL_ERR_SHAPE
    assert append(q=heads(ptr=None), q_out=heads(ptr=None), q_heads=0, c=cache()) == tl.TL_OK


def cached(b=None, c=None, **kw):
    j = tl.tl_cached_job(**{**dict(q=heads(), out=heads(), batch=b or batch(), q_heads=4, scale=1.0, longest=0, workspace=P, workspace_bytes=1 << 40), **kw})
    if c is not False:
        j.cache = ctypes.pointer(c or cache())
    return tl.raw().tl_attn_cached(ctypes.byref(j), None)


def test_cached_refusals():
    assert tl.raw().tl_attn_cached(None, None) == tl.TL_ERR_NULL
    assert cached() == tl.TL_OK
    assert cached(c=False) == tl.TL_ERR_NULL
    for kw, e in BAD_BATCHES:
        assert cached(b=batch(**kw)) == e, kw
    for kw, e in BAD_CACHES:
        assert cached(c=cache(**kw)) == e, kw
    for kw, e in BAD_HEADS:
        assert cached(q=heads(**kw)) == e and cached(out=heads(**kw)) == e, kw
    for kw, e in (({"q_heads": 0}, tl.TL_ERR_SHAPE), ({"q_heads": 3}, tl.TL_ERR_SHAPE), ({"q_heads": 1}, tl.TL_ERR_SHAPE), ({"longest": -1}, tl.TL_ERR_SHAPE),
                  ({"scale": float("nan")}, tl.TL_ERR_VALUE), ({"scale": float("inf")}, tl.TL_ERR_VALUE), ({"workspace": None}, tl.TL_ERR_NULL),
                  ({"workspace": P + 4}, tl.TL_ERR_ALIGN), ({"workspace_bytes": 0}, tl.TL_ERR_SHAPE)):
        assert cached(**kw) == e, kw


def test_workspace():
    size = tl.tl_attn_cached_workspace
    assert 0 < size(1, 1, 32, 8, 128) <= size(64, 64, 32, 8, 128)
    for bad in ((0, 1, 4, 2, 128), (1, -1, 4, 2, 128), (1, 1, 3, 2, 128), (1, 1, 4, 0, 128), (1, 1, 4, 2, 100), (1 << 20, 1, 4, 2, 128)):
        assert size(*bad) == 0, bad


def prompt(b=None, **kw):
    j = tl.tl_prompt_job(**{**dict(q=heads(), k=heads(), v=heads(), out=heads(), batch=b or batch(), q_heads=4, kv_heads=2, head_dim=128, scale=1.0), **kw})
    return tl.raw().tl_attn_prompt(ctypes.byref(j), None)


def test_prompt_refusals():
    assert tl.raw().tl_attn_prompt(None, None) == tl.TL_ERR_NULL
    assert prompt() == tl.TL_OK
    for kw, e in BAD_BATCHES:
        assert prompt(b=batch(**kw)) == e, kw
    for kw, e in BAD_HEADS:
        for name in ("q", "k", "v", "out"):
            assert prompt(**{name: heads(**kw)}) == e, (name, kw)
    for kw, e in (({"q_heads": 3}, tl.TL_ERR_SHAPE), ({"kv_heads": 0}, tl.TL_ERR_SHAPE), ({"head_dim": 24}, tl.TL_ERR_SHAPE), ({"head_dim": 160}, tl.TL_ERR_SHAPE),
                  ({"scale": float("-inf")}, tl.TL_ERR_VALUE)):
        assert prompt(**kw) == e, kw


def test_binding_looks_at_tensors_before_it_takes_their_addresses():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        tl.make_batch(torch.zeros(3, dtype=torch.int64), None, 2, 2)
    with pytest.raises(ValueError):
        tl.make_batch(None, torch.zeros(2, dtype=torch.int32), 2, 2)           # on the host
    with pytest.raises(tl.TlError):
        tl.tl_rope_table(4, 3)


def test_numbers_at_the_ends_of_their_ranges():
    """Sizes whose products would not fit 64 bits, and a scale that overflows on its way to powers of 2."""
    for pages in (1 << 59, (1 << 63) - 1, (1 << 31) // 64):
        assert cached(c=cache(pages_per_seq=pages)) == append(c=cache(pages_per_seq=pages)) == tl.TL_ERR_SHAPE, pages
    assert cached(c=cache(pages_per_seq=(1 << 31) // 64 - 1)) == tl.TL_OK
    assert cached(scale=3e38) == prompt(scale=-3e38) == tl.TL_ERR_VALUE
    assert cached(scale=2e38) == prompt(scale=2e38) == tl.TL_OK
    for big in (1 << 62, (1 << 63) - 1):
        assert prompt(b=batch(seqs=big)) == prompt(b=batch(tokens=big)) == tl.TL_ERR_SHAPE
        assert tl.raw().tl_attn_cached_workspace(big, 1, 4, 2, 128) == tl.raw().tl_attn_cached_workspace(1, 1, big, big, 128) == 0
