"""A small ternary decoder on the library's kernels, from prompts to generated tokens.

Its weights are random, so what it says means nothing; what it does is what a served model does:

* the linear layers are ternary, 2 bits a weight (tl_ternary_gemm), the rest of a block is a few torch operations;
* prompts of different lengths come packed, one behind the other: tl_kv_append rotates queries and keys and puts keys and values into a paged 8-bit cache,
  tl_attn_prompt attends over what is at hand in fp16;
* a further turn of a conversation, several tokens of each sequence, attends over the cache (tl_attn_cached);
* generation takes one token of each sequence at a time, as one captured graph: lengths are read on the device, so it serves every step;
* with --rows8 what goes into the products is in 8 bits, made by the norm with the residual's addition (tl_norm) and by the gate (tl_gate), the products are sums of whole
  numbers (tl_ternary_gemm_rows8), and the head has 4 bits a weight (tl_gemm_4bit); no torch operation is left between them.

    python examples/generate.py --layers 8 --width 2048 --heads 16 --kv-heads 4 --new 64
"""
import argparse
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_23025_amd as tl


class Linear:
    """y = gamma * (x @ W.T) for W in {-1, 0, 1}, from random weights."""

    def __init__(self, rng, n, k):
        what, _, self.gamma = tl.tl_quantize(rng.standard_normal((n, k), dtype=np.float32) / math.sqrt(k))
        self.n, self.k = n, k
        self.words = torch.from_numpy(tl.tl_pack_2bit(what).view(np.int32)).cuda()

    def __call__(self, x):
        eight = isinstance(x, tl.tl_rows8)
        y = torch.empty((x.rows if eight else x.shape[0], self.n), dtype=torch.float16, device="cuda")
        if eight:
            tl.tl_ternary_gemm_rows8(x, self.words, self.gamma, y)
        else:
            tl.tl_ternary_gemm(x, self.words, self.gamma, y, x.shape[0], self.n, self.k)
        return y


class Head:
    """Logits in 32 bits, from 4-bit weights with a scale for every 64 of them."""

    def __init__(self, w):
        codes, scales, _ = tl.tl_quantize_4bit(w, 64)
        self.n, self.words, self.scales = w.shape[0], torch.from_numpy(tl.tl_pack_4bit(codes).view(np.int32)).cuda(), torch.from_numpy(scales).cuda()

    def __call__(self, x):
        y = torch.empty((x.shape[0], self.n), dtype=torch.float32, device="cuda")
        tl.tl_gemm_4bit(tl.make_4bit_job(x, self.words, self.scales, None, 64, y))
        return y


def norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).half()


class Flow16:
    """What stands between the products, in torch and fp16: the residual, its norms, the gate."""

    def __init__(self, x):
        self.x = x

    def norm(self):
        return norm(self.x)

    last = norm

    def add(self, y):
        self.x = self.x + y

    def rows(self, y):
        return y

    def gate(self, both):
        gate, up = both.split(both.shape[1] // 2, dim=1)
        return (torch.nn.functional.silu(gate.float()) * up.float()).half()


class Flow8:
    """The same into rows of 8 bits, the residual in 32: what is added waits for the norm that follows."""

    def __init__(self, x):
        self.y, self.residual = x, torch.zeros(x.shape, dtype=torch.float32, device="cuda")

    def eight(self, t, n):
        return tl.make_rows8(torch.empty((t, (n + 15) // 16 * 16), dtype=torch.int8, device="cuda"), torch.empty(t, device="cuda"), n)

    def norm(self):
        out = self.eight(*self.y.shape)
        tl.tl_norm(tl.make_norm_job(self.y, self.residual, self.residual, out=out))
        return out

    def last(self):
        out = torch.empty_like(self.y)
        tl.tl_norm(tl.make_norm_job(self.y, self.residual, self.residual, y=out))
        return out

    def add(self, y):
        self.y = y

    def rows(self, y, gate=None):
        out = self.eight(*y.shape)
        tl.tl_gate(tl.make_gate_job(gate, y, None, out))
        return out

    def gate(self, both):
        gate, up = both.split(both.shape[1] // 2, dim=1)
        return self.rows(up, gate)


class Decoder:
    def __init__(self, layers=4, width=1024, heads=8, kv_heads=2, dim=128, hidden=2816, vocab=1000, seqs=4, room=2048, page_tokens=64, kind=tl.TL_KV_INT8, seed=0, rows8=False):
        """seqs sequences of up to `room` tokens each."""
        rng = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.dim, self.seqs, self.kind, self.page_tokens = heads, kv_heads, dim, seqs, kind, page_tokens
        self.embedding = torch.from_numpy(rng.standard_normal((vocab, width), dtype=np.float32)).cuda().half()
        head = rng.standard_normal((width, vocab), dtype=np.float32)
        self.head = Head(head.T / math.sqrt(width)) if rows8 else torch.from_numpy(head).cuda() / math.sqrt(width)
        self.flow = Flow8 if rows8 else Flow16
        self.layers = [{"qkv": Linear(rng, (heads + 2 * kv_heads) * dim, width), "o": Linear(rng, width, heads * dim),
                        "up": Linear(rng, 2 * hidden, width), "down": Linear(rng, width, hidden)} for _ in range(layers)]
        self.rope = tl.make_rope(torch.from_numpy(tl.tl_rope_table(room, dim)).cuda(), dim)
        # A cache for each layer; all share one page table.  Pages are dealt out at random, as those of a server that has run for a while.
        each = (room + page_tokens - 1) // page_tokens
        pages = each * seqs
        self.table = torch.from_numpy(rng.permutation(pages).astype(np.int32).reshape(seqs, each)).cuda()
        self.cache = []
        for _ in range(layers):
            codes = [torch.zeros((pages, kv_heads, page_tokens * dim), dtype=torch.uint8, device="cuda") for _ in range(2)]
            scales = [torch.zeros((pages, kv_heads, page_tokens // 16), dtype=torch.float32, device="cuda") for _ in range(2)]
            self.cache.append(tl.make_kv_cache(*codes, *scales, self.table, page_tokens, dim, kind))
        self.room = each * page_tokens
        self.cached = torch.zeros(seqs, dtype=torch.int32, device="cuda")        # tokens of each sequence that the caches hold

    def run(self, ids, start=None, longest=0, fresh=False):
        """One pass: the tokens' final states, and their keys and values in the caches.

        ids: the tokens of all sequences, one sequence behind the other from start[s] on, or (None) one of each.  fresh: the caches are empty, all that
        is attended to is in the call.  longest: a bound of the tokens cached, 0 if there is none at hand."""
        T, H, G, D = ids.shape[0], self.heads, self.kv_heads, self.dim
        batch = tl.make_batch(start, self.cached, self.seqs, T)
        flow = self.flow(self.embedding[ids])
        space = None if fresh else torch.empty(tl.tl_attn_cached_workspace(self.seqs, T, H, G, D), dtype=torch.uint8, device="cuda")
        for w, cache in zip(self.layers, self.cache):
            qkv = w["qkv"](flow.norm()).view(T, H + 2 * G, D)
            q, k, v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
            # queries and keys are rotated where they stand
            tl.tl_kv_append(tl.make_append_job(q, k, v, q, k if fresh else None, batch, cache, self.rope))
            seen = torch.empty((T, H, D), dtype=torch.float16, device="cuda")
            if fresh:
                tl.tl_attn_prompt(tl.make_prompt_job(q, k, v, seen, tl.make_batch(start, None, self.seqs, T), D ** -0.5))
            else:
                tl.tl_attn_cached(tl.make_cached_job(q, seen, batch, cache, D ** -0.5, longest, space))
            flow.add(w["o"](flow.rows(seen.view(T, H * D))))
            flow.add(w["down"](flow.gate(w["up"](flow.norm()))))
        if start is None:
            self.cached += 1
        else:
            self.cached += start[1:] - start[:-1]
        return flow.last()

    def logits(self, x):
        return self.head(x) if isinstance(self.head, Head) else x.float() @ self.head

    def feed(self, turns, fresh):
        """Takes some tokens of each sequence (lists); logits after the last of each."""
        n = [len(t) for t in turns]
        if min(n) < 1:
            raise ValueError("a turn of no tokens has no last one")
        begin = np.concatenate([[0], np.cumsum(n)])
        start = torch.from_numpy(begin.astype(np.int32)).cuda()
        x = self.run(torch.tensor([i for t in turns for i in t], device="cuda"), start, fresh=fresh)
        return self.logits(x[torch.from_numpy(begin[1:] - 1).cuda()])

    def generate(self, first, steps, longest=0):
        """The likeliest tokens from `first` (one of each sequence) on, [steps][seqs], and the seconds a step took."""
        ids = first.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        was = self.cached.clone()

        def step():
            ids.copy_(self.logits(self.run(ids, longest=longest)).argmax(-1))

        with torch.cuda.stream(side):                        # once ahead of the capture; what it wrote is written again
            step()
            ids.copy_(first)
            self.cached.copy_(was)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        out = torch.empty((steps, self.seqs), dtype=ids.dtype, device="cuda")
        torch.cuda.synchronize()
        begin = time.perf_counter()
        for i in range(steps):
            graph.replay()
            out[i] = ids
        torch.cuda.synchronize()
        return out, (time.perf_counter() - begin) / max(steps, 1)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("layers", 4), ("width", 1024), ("heads", 8), ("kv-heads", 2), ("dim", 128), ("hidden", 2816), ("seqs", 4), ("prompt", 500), ("turn", 20), ("new", 32)):
        p.add_argument("--" + name, type=int, default=value)
    p.add_argument("--cache", choices=("int8", "fp8"), default="int8")
    p.add_argument("--rows8", action="store_true", help="activations of the products in 8 bits, the head in 4")
    a = p.parse_args()
    room = a.prompt + a.turn + a.new + 1
    model = Decoder(a.layers, a.width, a.heads, a.kv_heads, a.dim, a.hidden, seqs=a.seqs, room=room, kind=tl.TL_KV_INT8 if a.cache == "int8" else tl.TL_KV_FP8, rows8=a.rows8)
    rng = np.random.default_rng(1)
    vocab = model.embedding.shape[0]

    def some(most):
        return [rng.integers(0, vocab, rng.integers(max(1, most // 4), most + 1)).tolist() for _ in range(a.seqs)]

    def timed(what, turns, fresh):
        torch.cuda.synchronize()
        begin = time.perf_counter()
        y = model.feed(turns, fresh)
        torch.cuda.synchronize()
        print("%s: %d tokens of %d sequences, %.2f ms" % (what, sum(map(len, turns)), a.seqs, (time.perf_counter() - begin) * 1e3))
        return y

    prompts = some(a.prompt)
    timed("prompts, the first time", prompts, True)
    model.cached.zero_()
    timed("prompts", prompts, True)
    y = timed("next turns", some(a.turn), False)
    out, seconds = model.generate(y.argmax(-1), a.new, room)
    print("generation: %d tokens of each, %.0f us a step" % (a.new, seconds * 1e6))
    print("first sequence:", out[:10, 0].tolist())


if __name__ == "__main__":
    main()
