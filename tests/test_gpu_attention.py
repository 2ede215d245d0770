"""The attention part on the GPU: rotation and the way into the cache, attention over the cache, attention over prompts, against the plain forms in attention.py."""
import numpy as np
import pytest

import attention as ref
import paper_2506_23025_amd as tl
from parity import to_dev

pytestmark = pytest.mark.gpu
KINDS = {"int8": tl.TL_KV_INT8, "fp8": tl.TL_KV_FP8}


def f16(rng, *shape, scale=1.0):
    return (rng.standard_normal(shape) * scale).astype(np.float16)


def on(x, stride_extra=0):
    """numpy [T][H][D] on the device; with stride_extra, as a slice of wider rows whose other columns are NaN."""
    import torch
    T, H, D = x.shape
    wide = torch.full((T, H + stride_extra, D), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, stride_extra // 2:stride_extra // 2 + H] = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return wide[:, stride_extra // 2:stride_extra // 2 + H]


def blank(T, H, D):
    """An output between two guards."""
    import torch
    t = torch.full(((T + 2), H, D), 77.0, dtype=torch.float16, device="cuda")
    return t[1:T + 1]


def taken(t):
    """Its values, the guards looked at."""
    import torch
    torch.cuda.synchronize()
    base = t._base if t._base is not None else t
    if base.shape[0] == t.shape[0] + 2:
        assert (base[0] == 77).all() and (base[-1] == 77).all(), "written outside of the output"
    return t.cpu().numpy()


class Setup:
    """A cache with its twin on the device, sequences in pages anywhere."""

    def __init__(self, seed, new, past, heads, kv_heads, D, page, kind, more_pages=2, missing=()):
        import torch
        self.rng = rng = np.random.default_rng(seed)
        self.new, self.past, self.heads, self.kv_heads, self.D, self.page, self.kind = np.asarray(new), np.asarray(past), heads, kv_heads, D, page, kind
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T = int(self.start[-1])
        whole = np.maximum(0, self.past) + self.new
        need = -(-whole // page)
        pages = int(need.sum()) + more_pages
        self.cache = ref.Cache(rng, pages, kv_heads, page, D, kind)
        order = rng.permutation(pages)
        most = int(max(1, need.max())) + 1
        self.table = np.full((len(new), most), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        for s, i in missing:
            self.table[s, i] = -1 if (s + i) % 2 else pages + 5
        self.longest = int(whole.max())
        c = self.cache
        self.kd, self.vd = (to_dev(ref.to_layout(c.codes[n], n == "k").reshape(pages, kv_heads, -1)) for n in "kv")
        self.ksd, self.vsd = (to_dev(c.scale[n]) for n in "kv")
        self.td, self.startd, self.pastd = to_dev(self.table), to_dev(self.start), to_dev(self.past.astype(np.int32))
        self.handle = tl.make_kv_cache(self.kd, self.vd, self.ksd, self.vsd, self.td, page, D, KINDS[kind])
        self.one = bool((self.new == 1).all())
        torch.cuda.synchronize()

    def batch(self, one=None):
        return tl.make_batch(None if (self.one if one is None else one) else self.startd, self.pastd, len(self.new), self.T)

    def check_cache(self):
        import torch
        torch.cuda.synchronize()
        for n, codes, scale in (("k", self.kd, self.ksd), ("v", self.vd, self.vsd)):
            np.testing.assert_array_equal(scale.cpu().numpy(), self.cache.scale[n], err_msg=n + " scales")
            got = ref.from_layout(codes.cpu().numpy().reshape(*self.cache.codes[n].shape[:3], -1), self.D, n == "k")
            np.testing.assert_array_equal(got, self.cache.codes[n], err_msg=n + " codes")

    def append(self, q, k, v, table, rot, pairs, extra=0, in_place=False, k_out=True):
        """The call and the same by the definition; checks rotated rows and the whole cache."""
        qd, kd, vd = on(q, extra), on(k, extra), on(v, extra)
        qo, ko = (qd, kd) if in_place else (blank(*q.shape), blank(*k.shape) if k_out else None)
        rope = tl.make_rope(to_dev(table), rot, pairs) if rot else None
        tl.tl_kv_append(tl.make_append_job(qd, kd, vd, qo, ko, self.batch(), self.handle, rope))
        wq, wk = np.zeros(q.shape, np.float16), np.zeros(k.shape, np.float16)
        with np.errstate(over="ignore", invalid="ignore"):
            for s, (n, p) in enumerate(zip(self.new, self.past)):
                if p < 0 or n == 0:
                    continue
                rows = range(self.start[s], self.start[s + 1])
                x = np.stack([ref.rotate(k[r], p + i, table, rot, pairs) for i, r in enumerate(rows)])
                wk[rows] = x.astype(np.float16)
                for i, r in enumerate(rows):
                    wq[r] = ref.rotate(q[r], p + i, table, rot, pairs).astype(np.float16)
                self.cache.put("k", x, self.table, s, p)
                self.cache.put("v", v[rows].astype(np.float32), self.table, s, p)
        np.testing.assert_array_equal(taken(qo), wq)
        if ko is not None:
            np.testing.assert_array_equal(taken(ko), wk)
        self.check_cache()


def rope_table(positions, rot):
    return tl.tl_rope_table(positions, rot) if rot else None


# ---- into the cache ----------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("D,rot,pairs,page", [(128, 128, False, 64), (128, 64, True, 32), (16, 16, False, 16), (32, 32, True, 128), (64, 32, False, 16), (80, 40, False, 64),
                                               (96, 48, True, 32), (96, 96, False, 256), (112, 2, True, 1024), (48, 0, False, 64)])
def test_append(kind, D, rot, pairs, page):
    rng = np.random.default_rng(D + rot)
    new, past = ref.lengths(rng, 6, 70, empty=True), np.array([0, 5, 16, 31, -1, 100])
    st = Setup(D * 7 + rot, new, past, 4, 2, D, page, kind)
    args = f16(rng, st.T, 4, D), f16(rng, st.T, 2, D), f16(rng, st.T, 2, D, scale=3.0), rope_table(st.longest, rot), rot, pairs
    st.append(*args, extra=3)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("H,HK", [(1, 1), (6, 3), (5, 5), (32, 8)])
def test_append_one_token_each(kind, H, HK):
    rng = np.random.default_rng(H)
    past = np.array([0, 1, 15, 16, 17, 63, 64, 500, -3])
    st = Setup(H * 100 + HK, np.ones(9, int), past, H, HK, 128, 64, kind)
    st.append(f16(rng, 9, H, 128), f16(rng, 9, HK, 128, scale=2.0), f16(rng, 9, HK, 128, scale=0.01), rope_table(501, 128), 128, False, extra=2, k_out=False)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
def test_append_token_by_token_grows_scales(kind):
    rng = np.random.default_rng(4)
    st = Setup(9, [1, 1], [0, 7], 2, 2, 64, 32, kind)
    table = rope_table(200, 64)
    for step in range(40):
        size = 10.0 ** rng.uniform(-3, 2)
        st.append(f16(rng, 2, 2, 64), f16(rng, 2, 2, 64, scale=size), f16(rng, 2, 2, 64, scale=1 / size) * (step != 3), table, 64, False)
        st.past = st.past + 1
        st.pastd.copy_(to_dev(st.past.astype(np.int32)))
        if st.past.max() // 32 >= 2:
            st.past[1] = 0
            st.pastd.copy_(to_dev(st.past.astype(np.int32)))
        if st.past[0] >= 32:
            break


@pytest.mark.parametrize("kind", ["int8", "fp8"])
def test_append_zeros_infinities_and_missing_pages(kind):
    rng = np.random.default_rng(5)
    st = Setup(10, [40, 20, 33, 1], [0, 10, 3, 20], 2, 2, 64, 16, kind, missing=((0, 1), (2, 0), (3, 1)))
    k, v = f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64)
    v[:20] = 0
    k[5, 1, 7] = np.nan
    k[45, 0, 3] = np.inf
    v[70, 1, 63] = -np.inf
    k[80, 0] = 65504
    st.append(f16(rng, st.T, 2, 64), k, v, rope_table(25, 64), 64, False, in_place=True)      # and a table that is too short


def test_append_of_a_block_that_stands_for_nan_and_is_begun_again():
    rng = np.random.default_rng(6)
    st = Setup(11, [3], [0], 1, 1, 32, 16, "int8")
    bad = f16(rng, 3, 1, 32)
    bad[1, 0, 0] = np.nan
    st.append(f16(rng, 3, 1, 32), bad, f16(rng, 3, 1, 32), None, 0, False)
    st.past = st.past + 3
    st.pastd.fill_(3)
    st.append(f16(rng, 3, 1, 32), f16(rng, 3, 1, 32), f16(rng, 3, 1, 32), None, 0, False)
    assert np.isnan(st.cache.scale["k"]).any()
    st.past = st.past * 0
    st.pastd.fill_(0)
    st.append(f16(rng, 3, 1, 32), f16(rng, 3, 1, 32), f16(rng, 3, 1, 32), None, 0, False)
    assert not np.isnan(st.cache.scale["k"]).any()


@pytest.mark.parametrize("S", [1, 63, 64, 65, 200, 4100])
def test_many_sequences(S):
    rng = np.random.default_rng(S)
    new = rng.integers(0, 3, S)
    new[-1] = 1
    st = Setup(S, new, rng.integers(-1, 40, S), 1, 1, 16, 16, "int8")
    st.append(f16(rng, st.T, 1, 16), f16(rng, st.T, 1, 16), f16(rng, st.T, 1, 16), rope_table(64, 16), 16, True)


def test_rotation_alone():
    import torch
    rng = np.random.default_rng(7)
    st = Setup(12, [3, 0, 20], [4, 0, 90], 3, 1, 80, 16, "int8")
    q, k = f16(rng, 23, 3, 80), f16(rng, 23, 1, 80)
    table = rope_table(128, 80)
    rope = tl.make_rope(to_dev(table), 80, True)
    pos = np.concatenate([4 + np.arange(3), 90 + np.arange(20)])
    for with_q, with_k in ((True, True), (True, False), (False, True)):
        qd, kd = on(q) if with_q else None, on(k) if with_k else None
        qo, ko = blank(23, 3, 80), blank(23, 1, 80)
        tl.tl_kv_append(tl.make_append_job(qd, kd, None, qo if with_q else None, ko if with_k else None, st.batch(), None, rope))
        for got, x, there in ((qo, q, with_q), (ko, k, with_k)):
            want = np.stack([ref.rotate(x[i], p, table, 80, True).astype(np.float16) for i, p in enumerate(pos)]) if there else np.full(x.shape, 77, np.float16)
            np.testing.assert_array_equal(taken(got), want)
    st.check_cache()
    torch.cuda.synchronize()


# ---- attention over the cache ------------------------------------------------------------------------

def cached(st, q, scale, one=None, longest=None, stream=None, out=None, extra=0):
    import torch
    qd = on(q, extra)
    out = blank(*q.shape) if out is None else out
    size = tl.tl_attn_cached_workspace(len(st.new), st.T, st.heads, st.kv_heads, st.D)
    space = torch.full((size,), 255, dtype=torch.uint8, device="cuda")          # NaN wherever it is read before it is written
    tl.tl_attn_cached(tl.make_cached_job(qd, out, st.batch(one), st.handle, scale, st.longest if longest is None else longest, space), stream)
    return taken(out)


def check_cached(st, q, got, scale, rows=None):
    G = st.heads // st.kv_heads
    for s, (n, p) in enumerate(zip(st.new, st.past)):
        if n == 0:
            continue
        L = max(0, int(p) + int(n)) if p >= 0 else 0
        (k, there), (v, _) = st.cache.read("k", st.table, s, L), st.cache.read("v", st.table, s, L)
        for i in range(n):
            r = st.start[s] + i
            if rows is not None and r not in rows:
                continue
            for h in range(st.heads):
                seen = there & (np.arange(L) <= p + i)
                if L and (np.isnan(k[seen, h // G]).any() or np.isnan(v[seen, h // G]).any()):
                    assert np.isnan(got[r, h]).all(), (s, i, h)
                    continue
                y, tol = ref.attend(q[r, h].astype(np.float64), k[:, h // G], v[:, h // G], seen, float(np.float32(scale))) if L else (np.zeros(st.D), np.zeros(st.D))
                off = np.abs(got[r, h].astype(np.float64) - y)
                assert (off <= tol).all(), (s, i, h, off.max(), tol[off.argmax()])


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("H,HK,D,page", [(1, 1, 128, 64), (4, 4, 128, 16), (8, 2, 128, 64), (24, 3, 64, 32), (16, 1, 96, 128), (6, 2, 80, 64), (32, 1, 128, 64), (17, 1, 32, 16),
                                          (40, 1, 16, 64), (2, 1, 112, 256), (4, 2, 48, 16)])
def test_cached_one_token(kind, H, HK, D, page):
    rng = np.random.default_rng(H * 1000 + D)
    past = np.array([0, 1, 14, 15, 16, 47, 62, 63, 64, 65, 200, 1023, -1, 127])
    st = Setup(H * 13 + D, np.ones(len(past), int), past, H, HK, D, page, kind)
    q = f16(rng, st.T, H, D)
    got = cached(st, q, D ** -0.5, extra=2)
    check_cached(st, q, got, D ** -0.5)
    assert np.array_equal(got, cached(st, q, D ** -0.5, one=False))
    got = cached(st, q, D ** -0.5, longest=0)             # the way of long caches: sums meet in another order
    check_cached(st, q, got, D ** -0.5)
    assert np.array_equal(got, cached(st, q, D ** -0.5, longest=0))


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("H,HK,D", [(1, 1, 128), (8, 2, 64), (4, 1, 128), (3, 3, 80), (32, 1, 32)])
def test_cached_several_tokens(kind, H, HK, D):
    rng = np.random.default_rng(H + D)
    st = Setup(H * 17 + D, [5, 0, 1, 37, 70, 2, 3], [0, 3, 100, 61, 250, -1, 15], H, HK, D, 32, kind)
    q = f16(rng, st.T, H, D)
    check_cached(st, q, cached(st, q, D ** -0.5, extra=1), D ** -0.5)
    check_cached(st, q, cached(st, q, D ** -0.5, longest=0), D ** -0.5)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("past,H,HK", [([20000], 4, 1), ([9000, 3, 700, 30], 2, 2), ([5000, 5001, 1], 16, 2)])
def test_cached_long(kind, past, H, HK):
    rng = np.random.default_rng(len(past))
    st = Setup(H * 19 + past[0], np.ones(len(past), int), past, H, HK, 128, 64, kind)
    q = f16(rng, st.T, H, 128, scale=2.0)
    got = cached(st, q, 128 ** -0.5)
    check_cached(st, q, got, 128 ** -0.5)
    for longest in (0, 1):                             # not known, and exceeded
        check_cached(st, q, cached(st, q, 128 ** -0.5, longest=longest), 128 ** -0.5)
    assert np.array_equal(got, cached(st, q, 128 ** -0.5))


def some_of(rng, st, count):
    return set(rng.integers(0, st.T, count)) | {int(x) for x in st.start[:-1] if x < st.T} | {int(x) - 1 for x in st.start[1:]}


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("D,past", [(64, 2500), (128, 1700), (80, 1700), (64, 4000), (128, 2600)])
def test_cached_several_tokens_and_many_heads(kind, D, past):
    rng = np.random.default_rng(past + D)
    st = Setup(past, [45, 1, 20, 0, 33], [past, 5, past // 3, 9, 70], 16, 8, D, 32, kind)
    q = f16(rng, st.T, 16, D)
    rows = some_of(rng, st, 8)
    got = cached(st, q, D ** -0.5)
    check_cached(st, q, got, D ** -0.5, rows)
    assert np.array_equal(got, cached(st, q, D ** -0.5))
    check_cached(st, q, cached(st, q, D ** -0.5, longest=0), D ** -0.5, rows)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("most", [1, 2, 17])
@pytest.mark.parametrize("D", [64, 128, 96])
def test_cached_many_short_sequences(kind, most, D):
    rng = np.random.default_rng(most + D)
    n = np.ones(75, int) if most == 1 else rng.integers(0, most + 1, 75)
    past = rng.integers(0, 120, 75)
    past[[3, 70]] = -1
    st = Setup(most * D, n, past, 32, 16, D, 16, kind)
    q = f16(rng, st.T, 32, D)
    rows = some_of(rng, st, 30)
    got = cached(st, q, D ** -0.5, extra=1)
    check_cached(st, q, got, D ** -0.5, rows)
    assert np.array_equal(got, cached(st, q, D ** -0.5))
    check_cached(st, q, cached(st, q, D ** -0.5, longest=0), D ** -0.5, rows)


def test_cached_sharp_and_flat_scores():
    rng = np.random.default_rng(8)
    st = Setup(21, [1, 1, 1, 3], [700, 65, 300, 90], 4, 2, 128, 64, "int8")
    for scale in (0.0, 30.0, -1.0, 1e-4):
        q = f16(rng, st.T, 4, 128)
        check_cached(st, q, cached(st, q, scale), scale)


def test_cached_blocks_of_very_different_scales():
    rng = np.random.default_rng(9)
    st = Setup(22, [1, 1, 2], [400, 900, 250], 4, 2, 64, 64, "int8")
    for n, d in (("k", st.ksd), ("v", st.vsd)):
        st.cache.scale[n] *= (2.0 ** rng.integers(-20, 5, st.cache.scale[n].shape)).astype(np.float32)
        st.cache.scale[n][rng.random(st.cache.scale[n].shape) < 0.2] = 0
        d.copy_(to_dev(st.cache.scale[n]))
    q = f16(rng, st.T, 4, 64)
    check_cached(st, q, cached(st, q, 0.02), 0.02)
    st.cache.scale["v"][:] = 0
    st.vsd.zero_()
    assert (cached(st, q, 0.02) == 0).all()


@pytest.mark.parametrize("fill", [np.nan, np.inf])
def test_cached_what_lies_behind_a_sequence_does_not_show(fill):
    rng = np.random.default_rng(10)
    st = Setup(23, [1, 1, 2, 4], [15, 5, 62, 300], 4, 2, 128, 64, "fp8", more_pages=3)
    used = np.zeros(st.cache.scale["k"].shape, bool)
    for s, (n, p) in enumerate(zip(st.new, st.past)):
        for b in range((p + n - 1) // 16 + 1):
            used[st.table[s, 16 * b // 64], :, 16 * b % 64 // 16] = True
    for d in (st.ksd, st.vsd):
        x = d.cpu().numpy()
        x[~used] = fill
        d.copy_(to_dev(x))
    q = f16(rng, st.T, 4, 128)
    got = cached(st, q, 0.09)
    assert np.isfinite(got).all()
    check_cached(st, q, got, 0.09)


def test_cached_nan_block_missing_pages_and_rows_that_see_nothing():
    rng = np.random.default_rng(11)
    st = Setup(24, [40, 1, 1, 1, 5], [0, 200, 100, 31, 60], 4, 2, 64, 16, "int8", missing=((1, 3), (1, 7), (3, 0), (3, 1), (4, 4)))
    for n, d in (("k", st.ksd), ("v", st.vsd)):
        st.cache.scale[n][st.table[0, 1], 1, 0] = np.nan
        st.cache.scale[n][st.table[2, 2 if n == "k" else 5], 0, 0] = np.nan
        d.copy_(to_dev(st.cache.scale[n]))
    q = f16(rng, st.T, 4, 64)
    got = cached(st, q, 0.125)
    check_cached(st, q, got, 0.125)
    check_cached(st, q, cached(st, q, 0.125, longest=0), 0.125)
    assert (got[42] == 0).all() and np.isfinite(got[:16]).all() and np.isfinite(got[:40, :2]).all() and np.isnan(got[16:40, 2:]).all()


def test_cached_codes_beyond_32_bits():
    import torch
    rng = np.random.default_rng(12)
    st = Setup(25, [1, 1], [100, 60], 2, 1, 128, 64, "int8")
    far = (5 << 30) // (64 * 128)                          # pages of 8 KB whose bytes begin beyond 4 GB
    st.td.add_(far)
    big = {n: torch.zeros((far + st.cache.pages, 1, 64 * 128), dtype=torch.uint8, device="cuda") for n in "kv"}
    scale = {n: torch.ones((far + st.cache.pages, 1, 4), dtype=torch.float32, device="cuda") for n in "kv"}
    for n, c, s in (("k", st.kd, st.ksd), ("v", st.vd, st.vsd)):
        big[n][far:], scale[n][far:] = c, s
    st.handle = tl.make_kv_cache(big["k"], big["v"], scale["k"], scale["v"], st.td, 64, 128, tl.TL_KV_INT8)
    q = f16(rng, 2, 2, 128)
    check_cached(st, q, cached(st, q, 0.1), 0.1)
    k, v = f16(rng, 2, 1, 128), f16(rng, 2, 1, 128)
    tl.tl_kv_append(tl.make_append_job(None, on(k), on(v), None, None, st.batch(), st.handle, None))
    for s in range(2):
        st.cache.put("k", k[s:s + 1].astype(np.float32), st.table, s, int(st.past[s]))
        st.cache.put("v", v[s:s + 1].astype(np.float32), st.table, s, int(st.past[s]))
    st.kd, st.vd, st.ksd, st.vsd = big["k"][far:], big["v"][far:], scale["k"][far:], scale["v"][far:]
    st.check_cache()


def test_cached_on_a_stream_and_in_a_graph():
    import torch
    rng = np.random.default_rng(13)
    st = Setup(26, [1] * 5, [4000, 3, 100, -1, 2500], 8, 2, 128, 64, "int8")
    q, k, v = f16(rng, 5, 8, 128), f16(rng, 5, 2, 128), f16(rng, 5, 2, 128)
    qd, kd, vd, out = on(q), on(k), on(v), blank(5, 8, 128)
    qo = blank(5, 8, 128)
    rope = tl.make_rope(to_dev(rope_table(5000, 128)), 128)
    space = torch.empty(tl.tl_attn_cached_workspace(5, 5, 8, 2, 128), dtype=torch.uint8, device="cuda")
    put = tl.make_append_job(qd, kd, vd, qo, None, st.batch(), st.handle, rope)
    att = tl.make_cached_job(qo, out, st.batch(), st.handle, 0.09, 5000, space)
    saved = [t.clone() for t in (st.kd, st.vd, st.ksd, st.vsd)]

    def step(stream=None):
        tl.tl_kv_append(put, stream)
        tl.tl_attn_cached(att, stream)

    def eager(steps):
        for t, w in zip((st.kd, st.vd, st.ksd, st.vsd), saved):
            t.copy_(w)
        got = []
        for i in range(steps):
            st.pastd.copy_(to_dev((st.past + i * (st.past >= 0)).astype(np.int32)))
            step()
            got.append(taken(out).copy())
        return got

    want = eager(4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for t, w in zip((st.kd, st.vd, st.ksd, st.vsd), saved):
        t.copy_(w)
    for i in range(4):                                   # lengths are read by the kernels: one graph serves every step
        st.pastd.copy_(to_dev((st.past + i * (st.past >= 0)).astype(np.int32)))
        out.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        assert np.array_equal(taken(out), want[i]), i
    for t, w in zip((st.kd, st.vd, st.ksd, st.vsd), saved):
        t.copy_(w)
    st.pastd.copy_(to_dev(st.past.astype(np.int32)))
    torch.cuda.synchronize()
    step(side)
    side.synchronize()
    assert np.array_equal(taken(out), want[0])


# ---- attention over prompts ------------------------------------------------------------------------------

def prompt(q, k, v, start, scale, extra=0, stream=None, views=None):
    import torch
    T = len(q)
    qd, kd, vd = views if views else (on(q, extra), on(k, extra), on(v, extra))
    out = blank(*q.shape)
    sd = None if start is None else to_dev(np.asarray(start, dtype=np.int32))
    tl.tl_attn_prompt(tl.make_prompt_job(qd, kd, vd, out, tl.make_batch(sd, None, T if start is None else len(start) - 1, T), scale), stream)
    torch.cuda.synchronize()
    return taken(out)


def check_prompt(q, k, v, start, got, scale, rows=None):
    H, G, D = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    scale = float(np.float32(scale))
    for a, b in zip(start[:-1], start[1:]):
        for h in range(H):
            kh, vh = k[a:b, h // G].astype(np.float64), v[a:b, h // G].astype(np.float64)
            for i in range(b - a):
                if rows is not None and a + i not in rows:
                    continue
                y, tol = ref.attend(q[a + i, h].astype(np.float64), kh, vh, np.arange(b - a) <= i, scale)
                off = np.abs(got[a + i, h].astype(np.float64) - y)
                assert (off <= tol).all(), (a, i, h, off.max(), tol[off.argmax()])


def starts(*n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


@pytest.mark.parametrize("H,HK,D", [(1, 1, 128), (2, 2, 64), (4, 1, 128), (6, 2, 80), (3, 3, 16), (8, 1, 32), (2, 1, 96), (2, 2, 112), (5, 5, 48)])
def test_prompt(H, HK, D):
    rng = np.random.default_rng(H * 100 + D)
    st = starts(1, 0, 77, 2, 130, 0, 31, 33, 64, 257)
    q, k, v = f16(rng, st[-1], H, D), f16(rng, st[-1], HK, D), f16(rng, st[-1], HK, D)
    got = prompt(q, k, v, st, D ** -0.5, extra=3)
    check_prompt(q, k, v, st, got, D ** -0.5)
    assert np.array_equal(got, prompt(q, k, v, st, D ** -0.5))


@pytest.mark.parametrize("n", [1, 15, 16, 17, 32, 63, 64, 65, 127, 128, 129, 191, 192, 255, 256, 257, 511, 513])
def test_prompt_lengths(n):
    rng = np.random.default_rng(n)
    q, k, v = f16(rng, n, 2, 128), f16(rng, n, 1, 128), f16(rng, n, 1, 128)
    check_prompt(q, k, v, [0, n], prompt(q, k, v, [0, n], 0.1), 0.1)


@pytest.mark.parametrize("n,H,HK,D", [(2048, 4, 2, 128), (4097, 2, 1, 64), (6000, 8, 8, 128)])
def test_prompt_long(n, H, HK, D):
    rng = np.random.default_rng(n)
    q, k, v = f16(rng, n, H, D, scale=2.0), f16(rng, n, HK, D), f16(rng, n, HK, D)
    got = prompt(q, k, v, [0, n], D ** -0.5)
    rows = set(rng.integers(0, n, 40)) | {0, 1, 127, 128, n - 2, n - 1}
    check_prompt(q, k, v, [0, n], got, D ** -0.5, rows)
    assert np.array_equal(got, prompt(q, k, v, [0, n], D ** -0.5))


@pytest.mark.parametrize("n,H,HK,D", [((4200,), 6, 3, 128), ((3900, 0, 1000, 130), 12, 12, 64), ((4200,), 6, 6, 80), ((2500, 2500, 1), 5, 1, 112)])
def test_prompt_long_with_few_heads(n, H, HK, D):
    rng = np.random.default_rng(n[0] + D)
    st = starts(*n)
    q, k, v = f16(rng, st[-1], H, D, scale=2.0), f16(rng, st[-1], HK, D), f16(rng, st[-1], HK, D)
    got = prompt(q, k, v, st, D ** -0.5)
    check_prompt(q, k, v, st, got, D ** -0.5, some_rows(rng, st, 30))
    assert np.array_equal(got, prompt(q, k, v, st, D ** -0.5))


def test_prompt_of_one_token_each_gives_the_values():
    rng = np.random.default_rng(14)
    q, k, v = f16(rng, 70, 4, 128), f16(rng, 70, 2, 128), f16(rng, 70, 2, 128)
    got = prompt(q, k, v, None, 0.1)
    assert np.array_equal(got, np.repeat(v, 2, axis=1))


def test_prompt_sharp_and_flat_scores():
    rng = np.random.default_rng(15)
    st = starts(150, 90)
    q, k, v = f16(rng, 240, 2, 64), f16(rng, 240, 1, 64), f16(rng, 240, 1, 64)
    for scale in (0.0, 40.0, -2.0, 1e-5):
        check_prompt(q, k, v, st, prompt(q, k, v, st, scale), scale)
    k = np.sort(np.abs(k), axis=0)                         # scores that grow along the sequence: the reference moves in every tile
    q = np.abs(q)
    check_prompt(q, k, v, st, prompt(q, k, v, st, 3.0), 3.0)


@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
def test_prompt_what_a_token_does_not_see_does_not_show(what):
    rng = np.random.default_rng(16)
    st = starts(40, 300, 70)
    T = st[-1]
    q, k, v = f16(rng, T, 2, 128), f16(rng, T, 2, 128), f16(rng, T, 2, 128)
    clean = prompt(q, k, v, st, 0.1)
    for at in (45, 100, 200, 339):
        for bad_key in (False, True):
            k2, v2 = k.copy(), v.copy()
            (k2 if bad_key else v2)[at, 1, 17] = what
            got = prompt(q, k2, v2, st, 0.1)
            touched = np.zeros(got.shape, bool)
            touched[at:340, 1] = True
            assert np.array_equal(got[~touched], clean[~touched]), (at, bad_key)
            rest = got[at:340, 1]
            if bad_key:
                # a score that is an infinity or NaN makes NaN of the row, or takes it out where it is -inf
                with np.errstate(invalid="ignore", over="ignore"):
                    s = q[at:340, 1, 17].astype(np.float64) * what
                assert np.isnan(rest[~(s == -np.inf)]).all() and np.isfinite(rest[s == -np.inf][1:]).all()
            else:
                others = np.delete(rest, 17, axis=1)
                assert np.array_equal(others, np.delete(clean[at:340, 1], 17, axis=1))
                assert (np.isnan(rest[:, 17]).all() if np.isnan(what) else (rest[:, 17] == what).all())


def test_prompt_strides_streams_and_rows_of_no_sequence():
    import torch
    rng = np.random.default_rng(17)
    T, H, D = 200, 3, 64
    q, k, v = f16(rng, T, H, D), f16(rng, T, H, D), f16(rng, T, H, D)
    st = np.array([5, 100, 100, 190], dtype=np.int32)
    by_head = [torch.from_numpy(np.ascontiguousarray(x.transpose(1, 0, 2))).cuda().transpose(0, 1) for x in (q, k, v)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = prompt(q, k, v, st, 0.2, views=by_head, stream=side)
    check_prompt(q, k, v, st, got, 0.2)
    assert (got[:5] == 77).all() and (got[190:] == 77).all()
    # one key and value for all tokens: a stride of 0
    one = torch.from_numpy(k[:1]).cuda().expand(T, H, D)
    k0 = np.repeat(k[:1], T, axis=0)
    check_prompt(q, k0, v, st, prompt(q, k0, v, st, 0.2, views=(by_head[0], one, by_head[2])), 0.2)


# Few rows, whose keys are dealt to several waves; many rows; many sequences of a few tokens; more than 64 sequences.
KINDS_OF_CALL = {"few": ((0, 300, 77, 2, 130, 1, 257), 3), "many": ((0, 300, 77, 2, 130, 1, 257, 400), 24),
                 "short": ((1, 2, 64, 0, 33, 32, 31, 65, 150, 3, 63, 7, 0) * 3, 32), "sequences": (tuple(range(60, 95)) * 2, 8)}


def some_rows(rng, st, count):
    return set(rng.integers(0, st[-1], count)) | set(np.maximum(st - 1, 0)) | set(np.minimum(st, st[-1] - 1)) | {x + o for x in st[:-1] for o in (31, 32, 63, 64, 127, 128)}


@pytest.mark.parametrize("call", KINDS_OF_CALL)
@pytest.mark.parametrize("D", [128, 64, 80, 16])
def test_prompt_kinds_of_calls(call, D):
    n, H = KINDS_OF_CALL[call]
    rng = np.random.default_rng(D)
    st = starts(*n)
    HK = H if H == 3 else H // 8
    q, k, v = f16(rng, st[-1], H, D, scale=2.0), f16(rng, st[-1], HK, D), f16(rng, st[-1], HK, D)
    got = prompt(q, k, v, st, D ** -0.5, extra=3)
    check_prompt(q, k, v, st, got, D ** -0.5, some_rows(rng, st, 40))
    assert np.array_equal(got, prompt(q, k, v, st, D ** -0.5))
    check_prompt(q, k, v, st, prompt(q, k, v, st, -3.0), -3.0, some_rows(rng, st, 5))


@pytest.mark.parametrize("call", KINDS_OF_CALL)
@pytest.mark.parametrize("D", [128, 64, 80])
@pytest.mark.parametrize("group", [2, 3, 4, 12])
def test_prompt_heads_that_share_keys(call, D, group):
    n, H = KINDS_OF_CALL[call]
    rng = np.random.default_rng(D + group)
    st = starts(*n)
    H = 24 if H == 3 else H // 24 * 24 + 24                 # from 24 heads on a call of few rows has many
    q, k, v = f16(rng, st[-1], H, D, scale=2.0), f16(rng, st[-1], H // group, D), f16(rng, st[-1], H // group, D)
    got = prompt(q, k, v, st, D ** -0.5, extra=3)
    check_prompt(q, k, v, st, got, D ** -0.5, some_rows(rng, st, 10))
    assert np.array_equal(got, prompt(q, k, v, st, D ** -0.5))


@pytest.mark.parametrize("call", KINDS_OF_CALL)
@pytest.mark.parametrize("group", [2, 4])
def test_prompt_heads_that_share_keys_show_nothing_unseen(call, group):
    n, H = KINDS_OF_CALL[call]
    rng = np.random.default_rng(33)
    st = starts(*n)
    H = 24 if H == 3 else H // 24 * 24 + 24
    q, k, v = f16(rng, st[-1], H, 64), f16(rng, st[-1], H // group, 64), f16(rng, st[-1], H // group, 64)
    clean = prompt(q, k, v, st, 0.1)
    longest = int(np.argmax(np.diff(st)))
    first, end = int(st[longest]), int(st[longest + 1])
    for at in (first, (first + end) // 2, end - 1):
        touched = np.zeros(clean.shape, bool)
        touched[at:end, group:2 * group, 17] = True
        for what in (np.nan, np.inf):
            v2 = v.copy()
            v2[at, 1, 17] = what
            got = prompt(q, k, v2, st, 0.1)
            assert np.array_equal(got[~touched], clean[~touched]), at
            assert (np.isnan(got[touched]) if np.isnan(what) else got[touched] == what).all(), at


@pytest.mark.parametrize("call", KINDS_OF_CALL)
@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
def test_prompt_kinds_of_calls_show_nothing_unseen(call, what):
    n, H = KINDS_OF_CALL[call]
    rng = np.random.default_rng(31)
    st = starts(*n)
    q, k, v = f16(rng, st[-1], H, 64), f16(rng, st[-1], H, 64), f16(rng, st[-1], H, 64)
    clean = prompt(q, k, v, st, 0.1)
    longest = int(np.argmax(np.diff(st)))
    first, end = int(st[longest]), int(st[longest + 1])
    for at in (first, first + 40, end - 1):
        v2 = v.copy()
        v2[at, 1, 17] = what
        got = prompt(q, k, v2, st, 0.1)
        touched = np.zeros(got.shape, bool)
        touched[at:end, 1, 17] = True
        assert np.array_equal(got[~touched], clean[~touched]), at
        assert (np.isnan(got[touched]) if np.isnan(what) else got[touched] == what).all(), at
        k2 = k.copy()
        k2[at, 1, 17] = np.nan
        got = prompt(q, k2, v, st, 0.1)
        touched[at:end, 1] = True
        assert np.array_equal(got[~touched], clean[~touched]) and np.isnan(got[touched]).all(), at


@pytest.mark.parametrize("call", KINDS_OF_CALL)
def test_prompt_kinds_of_calls_take_strides_and_streams(call):
    import torch
    n, H = KINDS_OF_CALL[call]
    rng = np.random.default_rng(32)
    st = starts(*n) + 5
    T = int(st[-1]) + 6
    q, k, v = f16(rng, T, H, 64), f16(rng, T, H, 64), f16(rng, T, H, 64)
    by_head = [torch.from_numpy(np.ascontiguousarray(x.transpose(1, 0, 2))).cuda().transpose(0, 1) for x in (q, k, v)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = prompt(q, k, v, st, 0.2, views=by_head, stream=side)
    check_prompt(q, k, v, st, got, 0.2, some_rows(rng, st, 5))
    assert (got[:5] == 77).all() and (got[T - 6:] == 77).all()


def test_outputs_may_take_the_place_of_queries():
    import torch
    rng = np.random.default_rng(18)
    q, k, v = f16(rng, 300, 4, 128), f16(rng, 300, 2, 128), f16(rng, 300, 2, 128)
    want = prompt(q, k, v, [0, 300], 0.1)
    qd = on(q)
    tl.tl_attn_prompt(tl.make_prompt_job(qd, on(k), on(v), qd, tl.make_batch(to_dev(np.array([0, 300], np.int32)), None, 1, 300), 0.1))
    assert np.array_equal(taken(qd), want)
    st = Setup(27, [1, 1, 1], [6000, 3, 64], 4, 2, 128, 64, "int8")
    q = f16(rng, 3, 4, 128)
    want = cached(st, q, 0.1)
    qd = on(q)
    space = torch.empty(tl.tl_attn_cached_workspace(3, 3, 4, 2, 128), dtype=torch.uint8, device="cuda")
    tl.tl_attn_cached(tl.make_cached_job(qd, qd, st.batch(), st.handle, 0.1, st.longest, space))
    assert np.array_equal(taken(qd), want)


def test_prompt_and_cache_agree():
    """A prompt, and the same put into the cache and read from there token by token: as near as the codes allow."""
    rng = np.random.default_rng(19)
    n, H, HK, D = 100, 4, 2, 64
    st = Setup(28, [n], [0], H, HK, D, 32, "int8")
    q, k, v = f16(rng, n, H, D), f16(rng, n, HK, D), f16(rng, n, HK, D)
    whole = prompt(q, k, v, [0, n], D ** -0.5)
    tl.tl_kv_append(tl.make_append_job(None, on(k), on(v), None, None, st.batch(), st.handle, None))
    again = cached(st, q, D ** -0.5)
    off = np.abs(whole.astype(np.float64) - again)
    assert off.max() < 0.1 and off.mean() < 0.01


# ---- beyond 32 bits ------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 3, 1]])
def test_a_cache_of_more_than_4_gigabytes(kind, new):
    """The same calls with pages at the beginning of a small cache and near the end of a large one: the same codes and outputs."""
    import torch
    rng = np.random.default_rng(41)
    H, HK, D, page, past = 16, 8, 128, 64, [900, 17, 300]
    pages, each = 75000, 16                                   # 64 KiB a page
    T = sum(new)
    q, k, v = f16(rng, T, H, D), f16(rng, T, HK, D), f16(rng, T, HK, D)
    start, pastd = to_dev(starts(*new)), to_dev(np.array(past, np.int32))
    rope = tl.make_rope(to_dev(tl.tl_rope_table(1000, D)), D)
    codes = torch.from_numpy(rng.integers(0, 100, (2, 3 * each, HK, page * D), dtype=np.uint8)).cuda()
    scales = torch.from_numpy(rng.uniform(0.01, 0.02, (2, 3 * each, HK, page // 16)).astype(np.float32)).cuda()
    got = []
    for count in (3 * each, pages):
        at = torch.from_numpy(rng.permutation(3 * each)).cuda() + (count - 3 * each)
        kv, sc = [], []
        for i in range(2):
            kv.append(torch.empty((count, HK, page * D), dtype=torch.uint8, device="cuda"))
            sc.append(torch.empty((count, HK, page // 16), dtype=torch.float32, device="cuda"))
            kv[i][at], sc[i][at] = codes[i], scales[i]
        table = at.to(torch.int32).view(3, each)
        cache = tl.make_kv_cache(*kv, *sc, table, page, D, KINDS[kind])
        batch = tl.make_batch(None if T == 3 else start, pastd, 3, T)
        qd, out = on(q), blank(T, H, D)
        tl.tl_kv_append(tl.make_append_job(qd, on(k), on(v), qd, None, batch, cache, rope))
        outs = []
        for longest in (0, 1000):
            space = torch.empty(tl.tl_attn_cached_workspace(3, T, H, HK, D), dtype=torch.uint8, device="cuda")
            tl.tl_attn_cached(tl.make_cached_job(qd, out, batch, cache, 0.1, longest, space))
            outs.append(taken(out).copy())
        assert np.isfinite(outs[0]).all()
        got.append([x[at].cpu().numpy() for x in kv + sc] + outs)
        del kv, sc, cache
    for a, b in zip(*got):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("T,H", [(300, 2), (300, 64), (100, 64)])
def test_rows_further_apart_than_32_bits_reach(T, H):
    """Tokens 2^23 + 8 numbers apart: the whole is 5 GB; the same bits as side by side."""
    import torch
    rng = np.random.default_rng(42)
    stride, D = 2 ** 23 + 8, 64
    flat = torch.empty(T * stride, dtype=torch.float16, device="cuda")
    q, k, v = f16(rng, T, H, D), f16(rng, T, H, D), f16(rng, T, H, D)
    wide = [torch.as_strided(flat, (T, H, D), (stride, D, 1), i * H * D) for i in range(4)]
    for t, x in zip(wide, (q, k, v)):
        t.copy_(torch.from_numpy(x))
    st = starts(T) if T > 100 else starts(*[2] * (T // 2))
    batch = tl.make_batch(to_dev(st), None, len(st) - 1, T)
    tl.tl_attn_prompt(tl.make_prompt_job(*wide, batch, 0.1))
    torch.cuda.synchronize()
    assert np.array_equal(wide[3].cpu().numpy(), prompt(q, k, v, st, 0.1))
    rope = tl.make_rope(to_dev(tl.tl_rope_table(T, D)), D)
    near = [blank(T, H, D) for _ in range(2)]
    tl.tl_kv_append(tl.make_append_job(on(q), on(k), None, *near, batch, None, rope))
    tl.tl_kv_append(tl.make_append_job(wide[0], wide[1], None, wide[0], wide[1], batch, None, rope))
    for a, b in zip(near, wide):
        assert np.array_equal(taken(a), b.cpu().numpy())
