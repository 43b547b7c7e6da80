"""The serving example: append, attention, experts and sampling in one loop."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import __graft_entry__
    __graft_entry__.build()
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_steps_agree_with_one_pass(example):
    """Logits of a decoded step through the cache equal those of one prefill of the same tokens, up to bf16: keys, values,
    queries and outputs are the same numbers, attention's paths differ by their rounding of p (2^-8 of an output of
    some tenths, through projections of unit gain), so by some hundredths in logits of unit size; a wrong line, page or angle
    changes them by their size."""
    prompts = [[(7 * i + 13 * s) % example.VOCAB for i in range(n)] for s, n in enumerate((5, 40, 1, 23))]
    tokens, logits, again = example.serve(prompts, 9)
    assert [len(t) for t in tokens] == [9] * 4 and all(0 <= t < example.VOCAB for row in tokens for t in row)
    assert float(logits.std()) > 0.5
    assert float((logits - again).abs().max()) < 0.1


def test_same_tokens_again(example):
    prompts = [[1, 2, 3], [4]]
    assert example.serve(prompts, 6, seed=3)[0] == example.serve(prompts, 6, seed=3)[0]
