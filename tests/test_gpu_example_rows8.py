"""The example with rows of 8 bits and a head of 4: it runs, and a captured step gives what steps by hand give."""
import subprocess
import sys

import numpy as np
import pytest

from test_gpu_example import PATH, SMALL, load

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden", [512, 328])
def test_a_captured_step_gives_what_steps_by_hand_give(hidden):
    import torch
    example = load()
    rng = np.random.default_rng(2)
    prompts = [rng.integers(0, 200, n).tolist() for n in (40, 1, 97)]
    outs = []
    for by_hand in (False, True):
        model = example.Decoder(**{**SMALL, "hidden": hidden}, rows8=True)
        y = model.feed(prompts, True)
        assert y.shape == (3, 200) and torch.isfinite(y).all()
        ids = y.argmax(-1)
        if by_hand:
            rows = []
            for _ in range(12):
                ids = model.logits(model.run(ids, longest=200)).argmax(-1)
                rows.append(ids)
            outs.append(torch.stack(rows).tolist())
        else:
            outs.append(model.generate(ids, 12, 200)[0].tolist())
    assert outs[0] == outs[1]


def test_the_flows_agree_on_a_pass():
    """A pass in 16 bits and one in 8 on the same weights: each product's rows are off by half a step of 1 / 127 of their largest value at most, about 2^-8 of their size at random, and four
    products to a layer of two add up to some 2^-8 * sqrt(8) = 1 % of the states; 10 times that is asked for, over all states."""
    import torch
    example = load()
    ids = [np.random.default_rng(3).integers(0, 200, n).tolist() for n in (30, 50, 11)]
    begin = np.concatenate([[0], np.cumsum([len(i) for i in ids])]).astype(np.int32)
    states = [example.Decoder(**SMALL, rows8=eight).run(torch.tensor(sum(ids, []), device="cuda"), torch.from_numpy(begin).cuda(), fresh=True).double() for eight in (False, True)]
    assert ((states[0] - states[1]).norm() / states[0].norm()).item() <= 0.1


def test_the_command_runs():
    r = subprocess.run([sys.executable, PATH, "--layers", "2", "--width", "256", "--heads", "4", "--dim", "64", "--hidden", "512", "--new", "5", "--rows8"],
                       capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "generation: 5 tokens of each" in r.stdout
