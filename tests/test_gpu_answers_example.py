"""The serving loop that draws several answers to a prompt: plan, search of shared pages, norms, updates, append, shared attention
and sampling together."""
import importlib.util
import os

import numpy as np
import pytest

from sample_common import one_row

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("width,seed", [(5, 0), (2, 1)])
def test_answers_are_drawn_from_the_right_logits(width, seed, capsys):
    spec = importlib.util.spec_from_file_location("serve_attention", os.path.join(ROOT, "examples", "serve_attention.py"))
    loop = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(loop)
    # the error against an exact recomputation: at most twice that of one with the same roundings, which the loop's sums in 32 bits
    # and the rounded weights of its attention add to
    ratio, drawn = loop.answer(prompts=3, width=width, steps=7, seed=seed, check=True)
    assert 0.0 < ratio <= 2.0
    assert len(drawn) == 7
    unsure = 0
    for logits, how, u, token in drawn:
        for r in range(len(u)):
            want, _, others = one_row(logits[r], float(np.float32(how["temperature"][r])), int(how["top_k"][r]), float(np.float32(how["top_p"][r])),
                                      float(np.float32(how["min_p"][r])), float(u[r]))
            unsure += others is not None
            assert int(token[r]) == want if others is None else int(token[r]) in others
    assert unsure <= 2
    # the groups that the loop has found: all answers share what their prompts have in whole pages
    lines = [line for line in capsys.readouterr().out.splitlines() if line.startswith("step ")]
    assert len(lines) == 7 and all(f"{3 * width} answers, {3 * width} of them in 3 groups" in line for line in lines)
