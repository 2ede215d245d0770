"""The example, a small decoder from prompts to generated tokens, against itself: what the cache gives is what whole prompts give, as near as 8-bit codes allow."""
import importlib.util
import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PATH = os.path.join(ROOT, "examples", "generate.py")


def load():
    spec = importlib.util.spec_from_file_location("generate_example", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


SMALL = dict(layers=2, width=256, heads=4, kv_heads=2, dim=64, hidden=512, vocab=200, seqs=3, room=200, page_tokens=32)


def near(a, b, bits):
    """A code is half a step off at most, 3 sigma / 2^bits or so of a value; keys and values of two layers and the sums behind them give errors of about 2^-bits of the logits' spread each time,
    10 times that for the largest of some hundred."""
    a, b = a.double().cpu().numpy(), b.double().cpu().numpy()
    assert np.abs(a - b).max() <= 10 * 3 * 2.0 ** -bits * b.std(), (np.abs(a - b).max(), b.std())


@pytest.mark.gpu
@pytest.mark.parametrize("kind,bits", [("INT8", 7), ("FP8", 4)])
def test_the_cache_gives_what_whole_prompts_give(kind, bits):
    import paper_2506_23025_amd as tl
    example = load()
    rng = np.random.default_rng(0)
    turns = [[rng.integers(0, 200, n).tolist() for n in sizes] for sizes in ((70, 1, 33), (5, 40, 1), (1, 17, 90))]
    whole = example.Decoder(kind=getattr(tl, "TL_KV_" + kind), **SMALL)
    want = whole.feed([sum(t, []) for t in zip(*turns)], True)
    model = example.Decoder(kind=getattr(tl, "TL_KV_" + kind), **SMALL)
    model.feed(turns[0], True)
    model.feed(turns[1], False)
    near(model.feed(turns[2], False), want, bits)
    assert model.cached.tolist() == whole.cached.tolist() == [76, 58, 124]


@pytest.mark.gpu
def test_a_captured_step_gives_what_steps_by_hand_give():
    import torch
    example = load()
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, 200, n).tolist() for n in (60, 15, 31)]
    outs = []
    for by_hand in (False, True):
        model = example.Decoder(**SMALL)
        ids = model.feed(prompts, True).argmax(-1)
        if by_hand:
            rows = []
            for _ in range(20):
                ids = model.logits(model.run(ids, longest=200)).argmax(-1)
                rows.append(ids)
            outs.append(torch.stack(rows).tolist())
        else:
            outs.append(model.generate(ids, 20, 200)[0].tolist())
        assert model.cached.tolist() == [80, 35, 51]
    assert outs[0] == outs[1]


@pytest.mark.gpu
def test_the_command_runs():
    r = subprocess.run([sys.executable, PATH, "--layers", "2", "--width", "256", "--heads", "4", "--dim", "64", "--hidden", "512", "--new", "5", "--cache", "fp8"],
                       capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "generation: 5 tokens of each" in r.stdout


def test_the_command_tells_its_options():
    r = subprocess.run([sys.executable, PATH, "--help"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "--kv-heads" in r.stdout
