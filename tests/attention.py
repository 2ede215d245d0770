"""Plain forms of the attention part for its tests: loops over sequences, blocks and heads, in 64 bits where numbers are compared with a
tolerance and in single roundings of 32 bits where codes are compared bit for bit."""
import numpy as np

TOP = {"int8": 127.0, "fp8": 448.0}


def decode_table():
    """The value of every 8-bit code with 4 exponent and 3 mantissa bits, bias 7, no infinities."""
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[b] = np.nan if (b & 127) == 127 else (-x if b & 128 else x)
    return v


E4M3 = decode_table()
_ORDER = np.argsort(E4M3[:127], kind="stable")
assert np.array_equal(_ORDER, np.arange(127))


def encode(x, kind):
    """float32 within the top's rounding -> codes as bytes, to the nearest, ties to even."""
    x = np.clip(x, np.float32(-TOP[kind]), np.float32(TOP[kind]))
    if kind == "int8":
        return np.rint(x).astype(np.int8).view(np.uint8)
    a = np.abs(x.astype(np.float64))
    hi = np.clip(np.searchsorted(E4M3[:127], a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (pick | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(codes, kind):
    codes = np.asarray(codes, dtype=np.uint8)
    return codes.view(np.int8).astype(np.float64) if kind == "int8" else E4M3[codes]


def to_layout(blocks, key):
    """codes [..., 16 tokens, dim] -> [..., 16 * dim] as they stand in memory."""
    *lead, _, D = blocks.shape
    out = np.empty((*lead, 16 * D), dtype=blocks.dtype)
    for t in range(16):
        for d in range(D):
            out[..., ((t // 4) * (D // 16) + d // 16) * 64 + (t % 4) * 16 + d % 16 if key else (d // 16) * 256 + (d % 16) * 16 + t] = blocks[..., t, d]
    return out


def from_layout(memory, D, key):
    out = np.empty((*memory.shape[:-1], 16, D), dtype=memory.dtype)
    for t in range(16):
        for d in range(D):
            out[..., t, d] = memory[..., ((t // 4) * (D // 16) + d // 16) * 64 + (t % 4) * 16 + d % 16 if key else (d // 16) * 256 + (d % 16) * 16 + t]
    return out


def rotate(x, pos, table, rot, pairs):
    """fp16 [heads][D] at one position -> float32, products and sums rounded one by one."""
    x = x.astype(np.float32)
    y = x.copy()
    if rot:
        half = rot // 2
        j = np.arange(half)
        a, b = (2 * j, 2 * j + 1) if pairs else (j, half + j)
        if pos < len(table):
            c, s = table[pos, :half], table[pos, half:]
            y[:, a] = x[:, a] * c - x[:, b] * s
            y[:, b] = x[:, b] * c + x[:, a] * s
        else:
            y[:, :rot] = np.nan
    return y


class Cache:
    """codes [pages][heads][blocks][16][D] and scales [pages][heads][blocks], as the definition has them."""

    def __init__(self, rng, pages, heads, page, D, kind):
        self.kind, self.page, self.D, self.heads, self.pages = kind, page, D, heads, pages
        shape = (pages, heads, page // 16, 16, D)
        self.codes = {}
        self.scale = {}
        for n in "kv":
            c = rng.integers(0, 256, shape).astype(np.uint8)
            c[(c & 127) == (127 if kind == "fp8" else 128)] = 3
            if kind == "int8":
                c[c == 128] = 3
            self.codes[n] = c
            self.scale[n] = rng.uniform(0.5, 2.0, shape[:3]).astype(np.float32) * np.float32(3 / TOP[kind])

    def page_of(self, table, s, p):
        i = p // self.page
        return int(table[s, i]) if i < table.shape[1] and 0 <= table[s, i] < self.pages else -1

    def put(self, name, x, table, s, past):
        """x float32 [n][heads][D]: the call's tokens of sequence s."""
        n = len(x)
        with np.errstate(invalid="ignore", over="ignore"):
            for b in range(past // 16, (past + n - 1) // 16 + 1):
                lo, hi = max(past, 16 * b), min(past + n, 16 * b + 16)
                page, blk, slot = self.page_of(table, s, lo), 16 * b % self.page // 16, lo % 16
                if page < 0:
                    continue
                for h in range(self.heads):
                    new = x[lo - past:hi - past, h]
                    was = self.scale[name][page, h, blk] if slot else np.float32(0)
                    now = np.maximum(was, np.abs(new).max() / np.float32(TOP[self.kind]))
                    if not np.isfinite(new).all() or np.isnan(was):
                        now = np.float32(np.nan)
                    c = self.codes[name][page, h, blk]
                    if slot and now > was:
                        old = decode(c[:slot], self.kind).astype(np.float32)
                        c[:slot] = encode(old * (was / now), self.kind)
                    c[slot:slot + hi - lo] = encode(new / now, self.kind) if now > 0 else 0
                    self.scale[name][page, h, blk] = now

    def read(self, name, table, s, length):
        """float64 [length][heads][D], and which positions have a page."""
        x, there = np.zeros((length, self.heads, self.D)), np.zeros(length, dtype=bool)
        for b in range(-(-length // 16)):
            page, blk = self.page_of(table, s, 16 * b), 16 * b % self.page // 16
            if page < 0:
                continue
            m = min(16, length - 16 * b)
            v = decode(self.codes[name][page, :, blk], self.kind) * self.scale[name][page, :, blk, None, None].astype(np.float64)
            x[16 * b:16 * b + m] = v[:, :m].transpose(1, 0, 2)
            there[16 * b:16 * b + m] = True
        return x, there


def attend(q, k, v, seen, scale):
    """q [D], k, v [n][D] in 64 bits, seen [n]: the output and what it may be off by.

    The kernels sum in 32 bits, round the weights p = exp(s - reference) to fp16 before they meet the values and the result once more: a weight is off by 2^-11 of itself
    and what a score's own sum leaves (dim * 2^-23 of the sum of its terms' magnitudes, and the products and the exponential 2^-21 of the score's), or by 2^-25 where it is
    below fp16's normal numbers (the reference is the row's largest or less, so their sum is 1 at least); the sum of n weights by n * 2^-24.
    """
    k, v = k[seen], v[seen]
    if not len(k):
        return np.zeros(len(q)), np.zeros(len(q))
    s = (k @ q) * scale
    p = np.exp(s - s.max())
    total = p.sum()
    y = p @ v / total
    terms = (np.abs(k) @ np.abs(q)).max() * abs(scale)
    delta = 2.0 ** -11 + 2 * len(q) * 2.0 ** -23 * terms + 2.0 ** -20 * (1 + np.abs(s).max()) + len(k) * 2.0 ** -23
    return y, 2.0 ** -11 * np.abs(y) + delta * (p @ np.abs(v)) / total + 2.0 ** -25 * np.abs(v).sum(0) / total + 2.0 ** -24


def lengths(rng, seqs, most, empty=False):
    n = rng.integers(0 if empty else 1, most + 1, seqs)
    n[rng.integers(0, seqs)] = most
    return n
