"""The example of language-model tenants: all operators together, against the same model on plain 64-bit operators."""
import importlib.util
import os

import pytest
import torch

from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "language_tenants.py")


def load():
    spec = importlib.util.spec_from_file_location("language_tenants", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Plain:
    """The operators from their definitions, in 64 bits, outputs rounded as the library's are."""

    class QuantBank:
        def __init__(self, codes, scales):
            w = torch.stack([codes & 15, codes >> 4], -1).flatten(2).double() - 8
            self.w = w * scales.double().repeat_interleave(w.shape[2] // scales.shape[2], 2)
            self.out_features = w.shape[1]

    @staticmethod
    def mt_quant_linear(x, ids, bank, y):
        y.copy_(torch.einsum("nk,nok->no", x.double(), bank.w[ids.long()]))

    mt_kv_append = staticmethod(mt.mt_kv_append)          # (bytes: tested against its definition elsewhere)

    @staticmethod
    def mt_prompt_attention(q, k, v, offsets, out):
        edges, g = offsets.tolist(), q.shape[1] // k.shape[1]
        for a, b in zip(edges[:-1], edges[1:]):
            for h in range(q.shape[1]):
                s = q[a:b, h].double() @ k[a:b, h // g].double().T / q.shape[2] ** 0.5
                s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), float("-inf"))
                out[a:b, h] = (torch.softmax(s, -1) @ v[a:b, h // g].double()).to(out.dtype)

    @staticmethod
    def mt_kv_attention(cache, q, tables, lengths, out):
        kc, kp, vc, vp = cache.tensors
        g, page = q.shape[1] // cache.heads, kc.shape[2]
        for s, n in enumerate(lengths.tolist()):
            pages = tables[s, : -(-n // page)].long()
            k, v = (torch.stack([c[pages] & 15, c[pages] >> 4], -1).flatten(3).double() * p[pages][..., :1].double() + p[pages][..., 1:].double()
                    for c, p in ((kc, kp), (vc, vp)))
            for h in range(q.shape[1]):
                kk, vv = k[:, h // g].flatten(0, 1)[:n], v[:, h // g].flatten(0, 1)[:n]
                out[s, h] = (torch.softmax(kk @ q[s, h].double() / q.shape[2] ** 0.5, 0) @ vv).to(out.dtype)

    @staticmethod
    def mt_token_logprobs(logits, tokens, logprobs, entropies, top_ids, top_logprobs):
        p = torch.log_softmax(logits.double(), -1)
        got = p.gather(1, tokens.long().clamp_min(0)[:, None])[:, 0]
        logprobs.copy_(torch.where(tokens >= 0, got, float("nan")))
        entropies.copy_(-(p.exp() * p).sum(-1))
        v, i = torch.sort(p, dim=-1, descending=True, stable=True)
        top_ids.copy_(i[:, :top_ids.shape[1]])
        top_logprobs.copy_(v[:, :top_ids.shape[1]])


def test_the_example_agrees_with_plain_operators():
    """Both models round at the same places (bf16 activations, 4-bit cache), so they part only where a rounding falls the other
    way: 2^-8 of an activation of size 1, some twenty times on the way to logits of size 1.  sqrt(20) 2^-8 = 0.017; five times that is allowed, and the cache's
    codes, which may flip by a level of some 0.3 in one of 64 channels, add as much again."""
    ex = load()
    mt.mt_init(0, 64, 0)
    gen = torch.Generator().manual_seed(3)
    prompts = [torch.randint(0, 1000, (l,), generator=gen).tolist() for l in (5, 40, 1, 17, 130, 64)]
    tenants = [0, 1, 2, 1, 0, 2]
    scored, taken, logprobs = ex.generate(ex.LanguageTenants(), prompts, tenants, 6)
    assert mt.mt_get_async_status() == (0, -1)
    want = ex.generate(ex.LanguageTenants(ops=Plain), prompts, tenants, 6, forced=taken)
    last = torch.tensor([len(p) for p in prompts]).cumsum(0) - 1
    assert torch.isnan(scored[last]).all() and int(torch.isnan(scored).sum()) == len(prompts)
    given = ~torch.isnan(scored)
    assert (scored - want[0])[given].abs().max() < 0.17
    assert (logprobs - want[2]).abs().max() < 0.17
    # greedy: each token taken is the likeliest, so it has more than the mean probability
    assert (logprobs > -torch.log(torch.tensor(1000.0))).all()


def test_the_example_runs_as_a_program(capsys):
    load().main()
    out = capsys.readouterr().out
    assert "status: (0, -1)" in out and out.count("tenant ") == 5
