"""Language-model tenants on one worker: a mixed batch of prompts of several tenants, then token by token.

Every tenant has a small decoder of its own (same shape, its own 4-bit weights).  A batch holds sequences of all of them:

  prompt   all prompts packed one behind the other: mt_quant_linear (each token with its tenant's weights),
           mt_prompt_attention, mt_kv_append (keys and values go to the paged 4-bit cache)
  step     one token per sequence: mt_quant_linear, mt_kv_append, mt_kv_attention
  answer   mt_token_logprobs: the likeliest next tokens, and the log probability of the one that is taken

    python examples/language_tenants.py            # three tenants, five prompts, eight tokens each
"""
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1901_06887_b200 import binding as mt  # noqa: E402

BF16 = torch.bfloat16


class Layer:
    pass


class LanguageTenants:
    """`ops` holds the operators (the package's binding; a test puts plain implementations in its place)."""

    def __init__(self, tenants=3, layers=2, dim=256, q_heads=4, kv_heads=2, head_dim=64, hidden=512, vocab=1000, group=64, seed=0, ops=mt):
        self.ops, self.dim, self.q_heads, self.kv_heads, self.head_dim, self.vocab = ops, dim, q_heads, kv_heads, head_dim, vocab
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def bank(out, inner):
            codes = torch.randint(0, 256, (tenants, out, inner // 2), generator=gen, device="cuda", dtype=torch.uint8)
            scales = torch.full((tenants, out, inner // group), 1.0 / (4.6 * math.sqrt(inner)), device="cuda").to(BF16)
            return ops.QuantBank(codes, scales)

        self.embedding = torch.randn((tenants, vocab, dim), generator=gen, device="cuda").to(BF16)
        self.layers = []
        for _ in range(layers):
            l = Layer()
            l.qkv = bank((q_heads + 2 * kv_heads) * head_dim, dim)
            l.out = bank(dim, q_heads * head_dim)
            l.up, l.down = bank(hidden, dim), bank(dim, hidden)
            l.cache = None
            self.layers.append(l)
        self.head = bank(vocab, dim)

    def open_caches(self, pages, page_tokens):
        for l in self.layers:
            l.cache = mt.KvCache.empty(pages, page_tokens, self.kv_heads, self.head_dim)

    def _linear(self, x, ids, bank, dtype=BF16):
        y = torch.empty((x.shape[0], bank.out_features), dtype=dtype, device=x.device)
        self.ops.mt_quant_linear(x, ids, bank, y)
        return y

    @staticmethod
    def _norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(BF16)

    def _turn(self, x, at):
        """Rotates pairs of channels by the token's position."""
        half = self.head_dim // 2
        angle = at.float()[:, None, None] / 10000.0 ** (torch.arange(half, device=x.device) / half)
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1).to(BF16)

    def forward(self, tokens, ids, at, slots, attend):
        """Logits fp32 [n, vocab] of n tokens at positions `at`, their keys and values written to `slots`.  attend(layer, q, k, v)
        is the attention: over the packed prompts, or over the cache."""
        x = self.embedding[ids.long(), tokens.long()]
        for l in self.layers:
            qkv = self._linear(self._norm(x), ids, l.qkv).view(len(tokens), -1, self.head_dim)
            q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
            q, k = self._turn(q, at), self._turn(k, at)
            self.ops.mt_kv_append(l.cache, k, v, slots)
            x = x + self._linear(attend(l, q, k, v).flatten(1), ids, l.out)
            x = x + self._linear(torch.relu(self._linear(self._norm(x), ids, l.up)), ids, l.down)
        return self._linear(self._norm(x), ids, self.head, torch.float32)

    def prompt(self, tokens, ids, at, slots, offsets):
        def attend(l, q, k, v):
            out = torch.empty(q.shape, dtype=BF16, device=q.device)
            self.ops.mt_prompt_attention(q, k, v, offsets, out)
            return out
        return self.forward(tokens, ids, at, slots, attend)

    def step(self, tokens, ids, at, slots, tables):
        lengths = (at + 1).int()

        def attend(l, q, k, v):
            out = torch.empty(q.shape, dtype=BF16, device=q.device)
            self.ops.mt_kv_attention(l.cache, q, tables, lengths, out)
            return out
        return self.forward(tokens, ids, at, slots, attend)

    def answer(self, logits, tokens, top=3):
        """(logprobs of `tokens`, entropies, ids and logprobs of the `top` likeliest)."""
        n = logits.shape[0]
        out = (torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, top), dtype=torch.int32, device="cuda"),
               torch.empty((n, top), device="cuda"))
        self.ops.mt_token_logprobs(logits, tokens, *out)
        return out


def generate(model, prompts, tenant_of, steps, page_tokens=16, forced=None):
    """Greedy continuation (or the tokens of `forced` [steps][sequences]) of prompts (lists of token ids) of tenants tenant_of.
    Returns the prompts' token logprobs, the tokens taken [steps][sequences] and their logprobs [steps][sequences]."""
    n, lens = len(prompts), [len(p) for p in prompts]
    width = max(-(-(l + steps) // page_tokens) for l in lens)
    model.open_caches(n * width, page_tokens)
    tables = torch.randperm(n * width, generator=torch.Generator().manual_seed(1)).int().view(n, width).cuda()
    seq = torch.repeat_interleave(torch.arange(n), torch.tensor(lens)).cuda()
    at = torch.cat([torch.arange(l) for l in lens]).cuda()
    ids = torch.tensor(tenant_of, dtype=torch.int32, device="cuda")
    tokens = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")

    def slot_of(s, a):
        return tables[s, a // page_tokens].long() * page_tokens + a % page_tokens

    logits = model.prompt(tokens, ids[seq], at, slot_of(seq, at), offsets)
    following = torch.cat([tokens[1:], tokens[:1] * 0 - 1])
    following[offsets[1:].long() - 1] = -1                      # a prompt's last token predicts nothing that is given
    scored = model.answer(logits, following)[0]
    logits = logits[offsets[1:].long() - 1]
    taken, taken_logprobs, every = [], [], torch.arange(n, device="cuda")
    at = torch.tensor(lens, device="cuda")
    for i in range(steps):
        if forced is None:
            token = model.answer(logits, torch.zeros(n, dtype=torch.int32, device="cuda"), 1)[2][:, 0].contiguous()
        else:
            token = forced[i]
        taken.append(token)
        taken_logprobs.append(model.answer(logits, token)[0])
        logits = model.step(token, ids, at, slot_of(every, at), tables)
        at = at + 1
    return scored, torch.stack(taken), torch.stack(taken_logprobs)


def main():
    mt.mt_init(0)
    model = LanguageTenants()
    gen = torch.Generator().manual_seed(2)
    prompts = [torch.randint(0, model.vocab, (l,), generator=gen).tolist() for l in (5, 40, 1, 17, 130)]
    tenants = [0, 1, 2, 1, 0]
    scored, taken, logprobs = generate(model, prompts, tenants, 8)
    print("mean log probability of the prompts' tokens: %.3f (uniform: %.3f)" % (scored.nanmean().item(), -math.log(model.vocab)))
    for s in range(len(prompts)):
        print("tenant %d, prompt of %d tokens: %s   log probability %.2f" % (tenants[s], len(prompts[s]), taken[:, s].tolist(),
                                                                             logprobs[:, s].sum().item()))
    print("status:", mt.mt_get_async_status())


if __name__ == "__main__":
    main()
