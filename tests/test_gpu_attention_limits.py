"""The attention part where its promises end: memory that nobody wrote, numbers at the ends of their ranges, lengths beyond the pages, calls of no tokens."""
import numpy as np
import pytest

import attention as ref
import paper_2506_23025_amd as tl
from parity import to_dev
from test_gpu_attention import KINDS, KINDS_OF_CALL, Setup, blank, cached, check_cached, f16, on, prompt, rope_table, some_of, starts, taken

pytestmark = pytest.mark.gpu


# ---- memory that nobody wrote ------------------------------------------------------------------

def fill(st):
    """Brings the device's codes and scales in line with the twin's."""
    for n, codes, scale in (("k", st.kd, st.ksd), ("v", st.vd, st.vsd)):
        codes.copy_(to_dev(ref.to_layout(st.cache.codes[n], n == "k").reshape(tuple(codes.shape))))
        scale.copy_(to_dev(st.cache.scale[n]))


def leave_page_0(st):
    """Page 0, which stands in for pages that are missing, belongs to no sequence."""
    free = next(p for p in range(st.cache.pages) if not (st.table == p).any())
    for d in (st.cache.codes, st.cache.scale):
        for n in "kv":
            d[n][free] = d[n][0]
    st.table[st.table == 0] = free
    st.td.copy_(to_dev(st.table))


def spoil(st, byte):
    """Every code that no token of a sequence was written to."""
    written = np.zeros((st.cache.pages, st.cache.page), bool)
    for s, (n, p) in enumerate(zip(st.new, st.past)):
        for at in range(int(p + n) if p >= 0 else 0):
            page = st.cache.page_of(st.table, s, at)
            if page >= 0:
                written[page, at % st.cache.page] = True
    w = written.reshape(st.cache.pages, 1, st.cache.page // 16, 16)
    for n in "kv":
        c = st.cache.codes[n]
        c[np.broadcast_to(~w, c.shape[:-1])] = byte
    fill(st)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("call", ["one", "several", "many", "many of several"])
def test_cached_codes_that_nobody_wrote_do_not_show(kind, D, call):
    """Ends inside a block, a tile and a page, pages that are missing, every kernel: the bits are those of a cache of zeros."""
    rng = np.random.default_rng(51)
    new, past, H, HK = {"one": (np.ones(8, int), np.array([0, 5, 15, 16, 62, 200, 700, -1]), 8, 2), "several": (np.array([5, 1, 70, 0, 33, 3]), np.array([0, 3, 61, 9, 250, -1]), 8, 2),
                        "many": (np.ones(75, int), rng.integers(0, 120, 75), 32, 16), "many of several": (rng.integers(1, 18, 75), rng.integers(0, 120, 75), 32, 16)}[call]
    st = Setup(52, new, past, H, HK, D, 32, kind, more_pages=3, missing=((2, 0), (4, 1), (5, 0)))
    leave_page_0(st)
    q = f16(rng, st.T, H, D)
    rows = some_of(rng, st, 20)
    spoil(st, 0)
    clean = {longest: cached(st, q, D ** -0.5, longest=longest) for longest in (None, 0)}
    for byte in (0x7f, 0xff):
        spoil(st, byte)
        for longest, want in clean.items():
            got = cached(st, q, D ** -0.5, longest=longest)
            assert np.isfinite(got).all(), (byte, longest)
            assert np.array_equal(got, want), (byte, longest)
    check_cached(st, q, got, D ** -0.5, rows)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [1, 17, 30, 65]])
def test_a_cache_of_unset_memory(kind, new):
    """First tokens into pages of any bytes and scales, then attention over them: as with pages of zeros."""
    import torch
    rng = np.random.default_rng(53)
    H, HK, D, page = 4, 2, 64, 32
    T, S = sum(new), len(new)
    q, k, v = f16(rng, T, H, D), f16(rng, T, HK, D), f16(rng, T, HK, D)
    start, none = to_dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)), to_dev(np.zeros(S, np.int32))
    table = to_dev(np.concatenate([[[-1, -1, -1]], 1 + np.arange(3 * S - 3).reshape(-1, 3)]).astype(np.int32))       # the first has no pages
    outs = []
    for byte, scale in ((0, 0.0), (0x7f, np.nan), (0xff, np.inf)):
        kd, vd = (torch.full((3 * S, HK, page * D), byte, dtype=torch.uint8, device="cuda") for _ in range(2))
        ks, vs = (torch.full((3 * S, HK, page // 16), scale, dtype=torch.float32, device="cuda") for _ in range(2))
        handle = tl.make_kv_cache(kd, vd, ks, vs, table, page, D, KINDS[kind])
        batch = tl.make_batch(None if T == S else start, none, S, T)
        tl.tl_kv_append(tl.make_append_job(None, on(k), on(v), None, None, batch, handle))
        for longest in (65, 0):
            out = blank(T, H, D)
            space = torch.empty(tl.tl_attn_cached_workspace(S, T, H, HK, D), dtype=torch.uint8, device="cuda")
            tl.tl_attn_cached(tl.make_cached_job(on(q), out, batch, handle, 0.125, longest, space))
            outs.append(taken(out).copy())
    for got, want in zip(outs, outs[:2] * 3):
        assert np.isfinite(got).all() and np.array_equal(got, want)
    assert (outs[0][0] == 0).all() and (outs[0][1:] != 0).any()


# ---- lengths beyond the pages --------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("new", [[1, 1, 1], [5, 1, 40]])
def test_lengths_beyond_the_pages(kind, new):
    """What is seen is what the pages hold, and no time goes into places that they cannot hold, however far beyond them a length is."""
    rng = np.random.default_rng(64)
    st = Setup(65, new, [150, 40, 300], 4, 2, 64, 32, kind)
    st.table = np.ascontiguousarray(st.table[:, :3])       # of 96 positions
    st.td = to_dev(st.table)
    st.handle = tl.make_kv_cache(st.kd, st.vd, st.ksd, st.vsd, st.td, 32, 64, KINDS[kind])
    q = f16(rng, st.T, 4, 64)
    want = {longest: cached(st, q, 0.125, longest=longest) for longest in (96, 0)}
    check_cached(st, q, want[96], 0.125)
    for far in (1 << 20, (1 << 31) - 1):
        st.pastd.copy_(to_dev(np.array([far, 40, far], np.int32)))
        for longest in (96, 0):
            assert np.array_equal(cached(st, q, 0.125, longest=longest), want[longest]), (far, longest)
    k, v = f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64)
    st.past = np.array([(1 << 31) - 1, 40, 1 << 20])
    st.pastd.copy_(to_dev(st.past.astype(np.int32)))
    st.append(q, k, v, tl.tl_rope_table(200, 64), 64, False)      # dropped there, and beyond the table


# ---- numbers at the ends of their ranges ---------------------------------------------------------

class Bounded(ref.Cache):
    """Scales below 2^-80 become 0: what the block held stays as it is, and the new codes are 0."""

    def put(self, name, x, table, s, past):
        was = self.codes[name].copy()
        super().put(name, x, table, s, past)
        for b in range(past // 16, (past + len(x) - 1) // 16 + 1):
            lo, hi = max(past, 16 * b), min(past + len(x), 16 * b + 16)
            page, blk = self.page_of(table, s, lo), 16 * b % self.page // 16
            for h in range(self.heads):
                if self.scale[name][page, h, blk] < 2.0 ** -80:
                    self.scale[name][page, h, blk] = 0
                    self.codes[name][page, h, blk] = was[page, h, blk]
                    self.codes[name][page, h, blk, lo % 16:lo % 16 + hi - lo] = 0


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("new,past", [([1, 1, 1], [0, 5, 31]), ([3, 20, 40], [0, 5, 31])])
def test_append_scales_at_the_ends_of_their_range(kind, new, past):
    """Rotated keys are coded from 32 bits, so a table of tiny or large numbers reaches scales whose reciprocals are no numbers."""
    rng = np.random.default_rng(54)
    for i, magnitude in enumerate((1e-20, 1e-22, 1e-23, 1e-25, 1e-33, 1e-36, 1e-38, 1e-40, 1e-43, 1e-38, 1e30, 3e37)):
        st = Setup(55 + i, new, past, 2, 2, 64, 32, kind)
        st.cache.__class__ = Bounded
        st.cache.scale["k"] *= np.float32(magnitude * 0.01)
        fill(st)
        table = tl.tl_rope_table(80, 64, magnitude=magnitude)
        st.append(f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64), table, 64, i % 2 == 0)


@pytest.mark.parametrize("call", KINDS_OF_CALL)
@pytest.mark.parametrize("D,group", [(64, 1), (128, 1), (128, 4)])
def test_prompt_rows_whose_scores_are_all_lost(call, D, group):
    """Scores of -infinity at all that a row sees: their softmax is 0 / 0.  A row that sees one more is an ordinary one."""
    n, H = KINDS_OF_CALL[call]
    H = 24 if H == 3 else H
    rng = np.random.default_rng(56)
    st = starts(*n)
    q, k, v = f16(rng, st[-1], H, D), f16(rng, st[-1], H // group, D), f16(rng, st[-1], H // group, D)
    q[:, :, 5] = 1
    for s in st[:-1]:
        if s < st[-1]:
            k[s:s + 3, 0, 5] = -np.inf
    got = prompt(q, k, v, st, 0.1)
    for a, b in zip(st[:-1], st[1:]):
        lost = min(3, b - a)
        assert np.isnan(got[a:a + lost, :group]).all(), a
        assert np.isfinite(got[a + lost:b]).all() and np.isfinite(got[a:b, group:]).all(), a
        if b - a > 3 and b - a < 100:
            k0, v0 = k[a + 3:b, 0].astype(np.float64), v[a + 3:b, 0].astype(np.float64)
            y, tol = ref.attend(q[b - 1, 0].astype(np.float64), k0, v0, np.ones(b - a - 3, bool), float(np.float32(0.1)))
            assert (np.abs(got[b - 1, 0] - y) <= tol).all()


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [5, 1, 40, 3]])
def test_cached_queries_that_are_no_numbers(kind, new):
    """An infinity in a query makes infinities of all its scores, and NaN of its softmax whatever their signs; a row that sees nothing is 0 all the same."""
    rng = np.random.default_rng(57)
    st = Setup(58, new, [700, 5, 90, 20], 4, 2, 64, 32, kind, missing=((3, 0),))
    c = st.cache.codes["k"]
    c[..., 7] = 40                                         # of one sign
    fill(st)
    q = f16(rng, st.T, 4, 64)
    bad = q.copy()
    rows = [0, int(st.start[2]), st.T - 1]
    for what in (np.inf, -np.inf, np.nan):
        for r in rows:
            bad[r, 1, 7] = what
        for scale in (0.125, -0.125, 0.0):
            for longest in (None, 0):
                clean, got = (cached(st, x, scale, longest=longest) for x in (q, bad))
                for r in rows[:2]:
                    assert np.isnan(got[r, 1]).all(), (what, scale, longest, r)
                    got[r, 1] = clean[r, 1]
                assert np.array_equal(got, clean), (what, scale, longest)
                if new[3] == 1:
                    assert (got[-1] == 0).all()


@pytest.mark.parametrize("call", KINDS_OF_CALL)
@pytest.mark.parametrize("D", [64, 128])
def test_prompt_queries_that_are_no_numbers(call, D):
    """Also with a scale of 0, which takes no infinity and no NaN away."""
    n, H = KINDS_OF_CALL[call]
    rng = np.random.default_rng(59)
    st = starts(*n)
    q, k, v = f16(rng, st[-1], H, D), f16(rng, st[-1], H, D), f16(rng, st[-1], H, D)
    longest = int(np.argmax(np.diff(st)))
    rows = [int(st[longest]), int(st[longest]) + 20, int(st[longest + 1]) - 1]
    for scale in (0.1, -0.1, 0.0):
        clean = prompt(q, k, v, st, scale)
        for what in (np.inf, -np.inf, np.nan):
            bad = q.copy()
            for r in rows:
                bad[r, 1, 7] = what
            got = prompt(bad, k, v, st, scale)
            for r in rows:
                assert np.isnan(got[r, 1]).all(), (what, scale, r)
                got[r, 1] = clean[r, 1]
            assert np.array_equal(got, clean), (what, scale)


SHARES = [0.7 * 2.0 ** -24, 1.3 * 2.0 ** -27, 0.9 * 2.0 ** -21, 2.0 ** -16]


def tail(n, share, value):
    """What n weights of `share` each beside one of 1 make of `value` beside 0, and what that may be off by.

    A weight is held in fp16 as 2^7 times what it is relative to the row's first and largest score, so that it is off by 2^-11 of itself or 2^-25 / 2^7; scores
    of a few units, products with whole numbers, make it off by 2^-20 of itself; sums of a tile's weights of n in 32 bits by 2^-23 of the sum each; the output by 2^-11 of itself or by half of fp16's smallest step."""
    y = n * share / (1 + n * share)
    return value * y, value * (y * (2.0 ** -10 + 2.0 ** -20 + n / 64 * 2.0 ** -23) + n * 2.0 ** -32) + 2.0 ** -25


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("share", SHARES)
@pytest.mark.parametrize("call", ["one", "several", "many"])
def test_cached_many_small_weights_beside_a_large_one(kind, share, call):
    """The first token takes nearly all of the weight, as first tokens do; hundreds of others share the rest."""
    new, n, H, HK = {"one": ([1, 1], 1400, 2, 1), "several": ([1, 20], 1000, 2, 1), "many": ([1] * 75, 500, 32, 16)}[call]
    D = 64
    st = Setup(60, new, [n] * len(new), H, HK, D, 64, kind)
    one = ref.encode(np.float32([4.0]), kind)[0]
    first = st.table[:, 0]
    for s in "kv":
        st.cache.codes[s][:] = 0 if s == "k" else one
        st.cache.scale[s][:] = 0.25 if s == "k" else 64
    st.cache.codes["k"][first, :, 0, 0, 3] = one           # 1
    st.cache.codes["v"][first, :, 0, 0] = 0                # and 256 elsewhere
    fill(st)
    q = np.zeros((st.T, H, D), np.float16)
    q[:, :, 3] = 16.0
    scale = -np.log(share) / 16.0
    share = np.exp(-16.0 * float(np.float32(scale)))
    for longest in (None, 0):
        got = cached(st, q, scale, longest=longest).astype(np.float64)
        for s in range(len(new)):
            for i in range(new[s]):
                y, tol = tail(n + i, share, 256.0)
                off = np.abs(got[st.start[s] + i] - y).max()
                assert off <= tol, (s, i, longest, off, y, tol)


@pytest.mark.parametrize("H,HK,D,n", [(1, 1, 64, 20000), (4, 1, 128, 9000), (12, 12, 64, 9000), (16, 4, 128, 9000)])
@pytest.mark.parametrize("share", SHARES)
def test_prompt_many_small_weights_beside_a_large_one(H, HK, D, n, share):
    q, k, v = np.zeros((n, H, D), np.float16), np.zeros((n, HK, D), np.float16), np.full((n, HK, D), 256, np.float16)
    q[:, :, 3], k[0, :, 3], v[0] = 16.0, 1.0, 0.0
    scale = -np.log(share) / 16.0
    share = np.exp(-16.0 * float(np.float32(scale)))
    got = prompt(q, k, v, [0, n], scale).astype(np.float64)
    for r in (0, 1, 100, 1000, n // 2, n - 1):
        y, tol = tail(r, share, 256.0)
        off = np.abs(got[r] - y).max()
        assert off <= tol, (r, off, y, tol)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("tokens", [1, 5])
def test_cached_scores_of_queries_with_a_large_common_part(kind, D, tokens):
    """Queries of 16 to 17 in steps of 2^-6 and keys of small whole numbers: products and sums are exact in 32 bits, in any order.  Two keys that differ in two places by 1 share the weight
    by a difference of scores below 1, which is what is left of sums of hundreds.

    A score in powers of 2 is off by 2^-23 of itself twice (the scale, its product), a weight and the output by 2^-11 each."""
    rng = np.random.default_rng(66)
    S, H, HK = 6, 8, 2
    st = Setup(67, [tokens] * S, [64] * S, H, HK, D, 64, kind)
    for n in "kv":
        st.cache.codes[n][:] = 0
        st.cache.scale[n][:] = 1
    unit = ref.encode(np.arange(-15, 16).astype(np.float32), kind)
    want = np.zeros((st.T, H))
    off = np.zeros((st.T, H))
    q = (16 + rng.integers(0, 64, (st.T, H, D)) / 64).astype(np.float16)
    for s in range(S):
        page, later = st.table[s, 0], st.table[s, 1]
        for g in range(HK):
            a = rng.integers(-14, 15, D)
            while a.sum() != 0:
                i = rng.integers(0, D)
                a[i] = np.clip(a[i] - np.sign(a.sum()), -14, 14)
            b = a.copy()
            i, j = rng.permutation(D)[:2]
            b[i], b[j] = b[i] + 1, b[j] - 1
            ahead = np.sign(a)                             # what the other tokens are is far behind
            st.cache.codes["k"][page, g], st.cache.codes["k"][later, g] = (unit[-a + 15] for _ in range(2))
            st.cache.codes["k"][page, g, 0, 3], st.cache.codes["k"][page, g, 2, 9] = unit[a + 15], unit[b + 15]
            st.cache.codes["v"][page, g, 2, 9] = unit[1 + 15]
            for r in range(st.start[s], st.start[s + 1]):
                for h in range(g * H // HK, (g + 1) * H // HK):
                    # the signs of the deviations are the key's, so that its score is large
                    q[r, h] = (16.5 + ahead * (np.abs(q[r, h].astype(np.float64) - 16.5))).astype(np.float16)
                    x = q[r, h].astype(np.float64)
                    scores = x @ a, x @ b
                    assert min(scores) > 60 and x @ -a < 0
                    want[r, h] = 1 / (1 + np.exp(scores[0] - scores[1]))
                    off[r, h] = want[r, h] * (2 * 2.0 ** -11 + 2 * max(scores) * 1.45 * 2.0 ** -23) + 2.0 ** -24
    fill(st)
    for longest in (None, 0):
        got = cached(st, q, 1.0, longest=longest).astype(np.float64)
        worst = np.abs(got - want[:, :, None]).max(2)
        assert (worst <= off).all(), (longest, (worst / off).max())


# ---- calls of no tokens ---------------------------------------------------------------------------

def test_calls_of_no_tokens_do_nothing():
    import torch
    st = Setup(61, [0, 0], [5, 70], 4, 2, 64, 32, "int8")
    q, k = (torch.empty((0, h, 64), dtype=torch.float16, device="cuda") for h in (4, 2))
    rope = tl.make_rope(to_dev(tl.tl_rope_table(100, 64)), 64)
    batch = tl.make_batch(st.startd, st.pastd, 2, 0)
    tl.tl_kv_append(tl.make_append_job(q, k, k.clone(), q, k, batch, st.handle, rope))
    space = torch.empty(tl.tl_attn_cached_workspace(2, 0, 4, 2, 64), dtype=torch.uint8, device="cuda")
    tl.tl_attn_cached(tl.make_cached_job(q, q.clone(), batch, st.handle, 0.1, 0, space))
    tl.tl_attn_prompt(tl.make_prompt_job(q, k, k.clone(), q.clone(), batch, 0.1))
    st.check_cache()


# ---- single tokens -------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("D,rot,pairs,page", [(128, 128, False, 64), (128, 64, True, 32), (128, 64, False, 16), (16, 16, False, 16), (32, 32, True, 128), (64, 32, False, 16), (80, 40, False, 64),
                                               (80, 40, True, 16), (96, 48, True, 32), (96, 96, False, 256), (112, 2, True, 1024), (112, 22, False, 32), (48, 0, False, 64)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_one_token_each_of_any_head(kind, D, rot, pairs, page, in_place):
    rng = np.random.default_rng(D + rot)
    past = np.array([0, 1, 9, 15, 16, 17, 30, 31, -1, 100, 127])
    st = Setup(D * 11 + rot, np.ones(len(past), int), past, 5, 5, D, page, kind)
    for size in (1.0, 30.0):                               # the second call codes what the blocks hold anew
        st.append(f16(rng, st.T, 5, D), f16(rng, st.T, 5, D, scale=size), f16(rng, st.T, 5, D, scale=3 * size), rope_table(128, rot), rot, pairs, extra=3, in_place=in_place)


@pytest.mark.parametrize("kind", ["int8", "fp8"])
@pytest.mark.parametrize("rot,pairs", [(64, False), (64, True), (36, False), (0, False)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_one_token_each_of_zeros_infinities_and_missing_pages(kind, rot, pairs, in_place):
    rng = np.random.default_rng(62)
    past = np.array([0, 7, 15, 16, 40, 3, 20, 33, -2, 64, 90])
    st = Setup(63, np.ones(len(past), int), past, 2, 2, 64, 16, kind, missing=((2, 0), (6, 1)))
    q, k, v = f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64)
    k[0] = v[1] = v[0, 1] = 0
    k[3, 1, 7], k[4, 0, 3], v[5, 1, 63], v[2, 0, 1], v[7, 0] = np.nan, np.inf, -np.inf, np.nan, 65504
    st.append(q, k, v, rope_table(60, rot), rot, pairs, in_place=in_place)      # the last two are beyond the table
    for n in "kv":                                        # and a block that stands for NaN takes another token, as does one that is begun again
        st.cache.scale[n][st.table[1, 0]] = np.nan
        st.cache.scale[n][st.table[0, 0]] = np.nan
    fill(st)
    st.append(f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64), f16(rng, st.T, 2, 64), rope_table(128, rot), rot, pairs, in_place=in_place)
    assert not np.isnan(st.cache.scale["k"][st.table[0, 0]]).any() and np.isnan(st.cache.scale["k"][st.table[1, 0]]).all()
