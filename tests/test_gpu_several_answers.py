"""The example of several answers about an image: all operators together, against the same model on plain 64-bit operators."""
import importlib.util
import os

import pytest
import torch

from lm_util import to_np
from more_lm_util import cross_reference, rotate_reference, sample_reference
from paper_1901_06887_b200 import binding as mt
from test_gpu_language_tenants import Plain

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "several_answers.py")


def load():
    spec = importlib.util.spec_from_file_location("several_answers", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class MorePlain(Plain):
    @staticmethod
    def mt_rotate(x, positions, frequencies, out, sections):
        out.copy_(torch.from_numpy(rotate_reference(x, positions, frequencies, sections, False, False)[0]))

    @staticmethod
    def mt_cross_attention(q, k, v, offsets, ranges, out):
        out.copy_(torch.from_numpy(cross_reference(q, k, v, offsets.tolist(), ranges.tolist(), q.shape[-1] ** -0.5)[0]))

    mt_token_sample = staticmethod(mt.mt_token_sample)    # (its tokens are checked below)


@pytest.mark.parametrize("prompts,each,steps,page", [(3, 4, 4, 16), (5, 2, 9, 32)])
def test_the_example_agrees_with_plain_operators(prompts, each, steps, page):
    """Both models round at the same places, so they part only where a rounding falls the other way: 2^-8 of an activation of size 1, some thirty-two times on
    the way to logits of size 1.  sqrt(32) 2^-8 = 0.022; five times that is allowed, and the cache's codes, which may flip by a level of some 0.3 in one of
    64 channels, add 0.09."""
    ex = load()
    mt.mt_init(0, 64, 0)
    mt.mt_get_async_status()
    text, images, at, tenants, uniform = ex.inputs(prompts, each, steps)
    logits, tokens, logprobs, book = ex.answer(ex.SeveralAnswers(), text, images, at, tenants, each, steps, uniform, page)
    assert mt.mt_get_async_status() == (0, -1)
    for step in range(2 * steps):
        u = uniform[step] if step < steps else uniform[step][::2]
        for i in range(len(u)):
            want, lp, near = sample_reference(to_np(logits[step][i]), u[i].item(), torch.tensor(0.9).item(), 50, torch.tensor(0.9).item())
            assert near or (tokens[step][i] == want and abs(logprobs[step][i].item() - lp) < 1e-5)
    plain = ex.answer(ex.SeveralAnswers(ops=MorePlain), text, images, at, tenants, each, steps, uniform, page, forced=tokens)
    for a, b in zip(logits, plain[0]):
        assert (a - b).abs().max() < 0.2
    # the book at the end: only the answers that went on hold pages, all in front
    used = int((book.refs > 0).sum())
    held = sum(-(-n // page) for n in book.lengths.tolist())
    assert bool((book.refs[:used] > 0).all()) and int(book.refs.sum()) == held
    assert sum(n > 0 for n in book.lengths.tolist()) == -(-prompts * each // 2)
    assert book.refs.tolist() == plain[3].refs.tolist()


def test_answers_of_one_prompt_start_alike_and_part():
    ex = load()
    mt.mt_init(0, 64, 0)
    text, images, at, tenants, uniform = ex.inputs(2, 6, 3)
    logits, tokens, _, _ = ex.answer(ex.SeveralAnswers(), text, images, at, tenants, 6, 3, uniform)
    first = logits[0].view(2, 6, -1)
    assert (first == first[:, :1]).all() and len(set(tokens[0].tolist())) > 2


def test_the_example_runs_as_a_program(capsys):
    load().main()
    out = capsys.readouterr().out
    assert "status: (0, -1)" in out and out.count("tenant ") == 3 and "all in front: True" in out
