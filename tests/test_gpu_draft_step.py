"""The drafting example: append with norms, attention over shared lines, experts and verification in one loop."""
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
    spec = importlib.util.spec_from_file_location("draft_step", os.path.join(ROOT, "examples", "draft_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("system", [0, 15, 48, 150])
def test_steps_agree_with_one_pass(example, system):
    """The verified rows' logits, through the shared pages and the lines that refused drafts left behind, equal those of one prefill of the same
    tokens up to bf16 (some hundredths in logits of unit size, as for the serving example: attention's paths differ by their
    rounding of p); a wrong line, page, angle or norm changes them by their size."""
    prompt = [(11 * i) % 97 for i in range(system)]
    questions = [[(7 * i + 13 * s) % example.base.VOCAB for i in range(n)] for s, n in enumerate((5, 40, 1, 23))]
    said, (taken, offered), last, again = example.serve(prompt, questions, 9)
    assert all(9 <= len(t) <= 9 * (example.DRAFTS + 1) and all(0 <= x < example.base.VOCAB for x in t) for t in said)
    assert sum(map(len, said)) == 4 * 9 + taken <= 4 * 9 + offered
    assert float(last.std()) > 0.5 and float((last - again).abs().max()) < 0.1


def test_same_tokens_again(example):
    prompt, questions = list(range(40)), [[1, 2, 3], [4]]
    assert example.serve(prompt, questions, 6, seed=3)[:2] == example.serve(prompt, questions, 6, seed=3)[:2]


def test_greedy_drafts(example):
    """Without temperature a draft is taken exactly while it is the target's first choice, and the token after the drafts is that."""
    prompt, questions = [(5 * i) % 31 for i in range(70)], [[3, 1, 4], [1, 5], [9, 2, 6, 5]]
    said, (taken, offered), last, _ = example.serve(prompt, questions, 8, temperature=0.0)
    best = last.argmax(-1)
    rows = len(best)
    assert rows >= 3 and all(s[-1] in best.tolist() for s in said)


@pytest.mark.parametrize("system", [16, 48, 150])
@pytest.mark.parametrize("temperature", [0.8, 0.0])
def test_steps_through_the_shared_kernels(example, monkeypatch, system, temperature):
    """With page tables as wide as a server keeps them the streams' shared lines are read for the group (what narrow tables can hold, each
    stream reads itself): the logits still equal those of one prefill, and the tokens are the same again."""
    plain, widths = example.Server, []

    class Wide(plain):
        def __init__(self, streams, max_tokens, max_len, seed=0):
            super().__init__(streams, max_tokens, max_len, seed)
            line = streams * example.base.KV_HEADS * example.base.DIM * 4
            more = int(128e6 / (line * example.base.PAGE)) + 2
            self.pages = torch.nn.functional.pad(self.pages, (0, more)).contiguous()
            widths.append(self.pages.shape[1] * example.base.PAGE * line)

    monkeypatch.setattr(example, "Server", Wide)
    prompt = [(11 * i) % 97 for i in range(system)]
    questions = [[(7 * i + 13 * s) % example.base.VOCAB for i in range(n)] for s, n in enumerate((5, 40, 1, 23))]
    said, (taken, offered), last, again = example.serve(prompt, questions, 9, temperature=temperature)
    assert widths and min(widths) > 128e6
    assert sum(map(len, said)) == 4 * 9 + taken <= 4 * 9 + offered
    assert float(last.std()) > 0.5 and float((last - again).abs().max()) < 0.1
    assert example.serve(prompt, questions, 9, temperature=temperature)[0] == said
