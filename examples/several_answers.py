"""Several answers to each prompt about an image, by language-model tenants on one worker.

The model of language_tenants.py, and in every layer it also looks at its image: the states of an encoder, of another length than the text.

  image    its states, one (time, height, width) position each, as keys and values of every layer: mt_quant_linear, mt_rotate
  prompt   mt_kv_reserve hands out pages, then as there; every layer looks at the image with mt_cross_attention
  answers  mt_kv_fork makes the prompt's row several: full pages are shared, the last one is copied by mt_kv_copy
  step     mt_kv_reserve, mt_quant_linear, mt_rotate, mt_kv_append, mt_kv_attention, mt_cross_attention (answers about one image share its
           states), mt_token_sample
  end      mt_kv_release gives the pages of an answer back, mt_kv_compact and mt_kv_copy move what is left to the front

    python examples/several_answers.py            # three prompts, four answers each, eight tokens
"""
import importlib.util
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
if os.path.dirname(HERE) not in sys.path:
    sys.path.insert(0, os.path.dirname(HERE))

from paper_1901_06887_b200 import binding as mt  # noqa: E402

_spec = importlib.util.spec_from_file_location("language_tenants", os.path.join(HERE, "language_tenants.py"))
lt = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(lt)
BF16 = torch.bfloat16


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


class SeveralAnswers(lt.LanguageTenants):
    def __init__(self, tenants=3, layers=2, dim=256, q_heads=4, kv_heads=2, head_dim=64, seed=0, ops=mt, **kw):
        super().__init__(tenants, layers, dim, q_heads, kv_heads, head_dim, seed=seed, ops=ops, **kw)
        gen = torch.Generator(device="cuda").manual_seed(seed + 1)

        def bank(out, inner):
            codes = torch.randint(0, 256, (tenants, out, inner // 2), generator=gen, device="cuda", dtype=torch.uint8)
            return ops.QuantBank(codes, torch.full((tenants, out, inner // 64), 1.0 / (4.6 * inner ** 0.5), device="cuda").to(BF16))

        for l in self.layers:
            l.ask, l.states, l.seen = bank(q_heads * head_dim, dim), bank(2 * kv_heads * head_dim, dim), bank(dim, q_heads * head_dim)
        half = head_dim // 2
        self.frequencies = (10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()
        self.sections = [half // 2, half // 4, half - half // 2 - half // 4]          # time, height, width

    def _turn(self, x, at):
        """Turns heads by their positions: [n] (text, which moves along all axes together) or [n, 3]."""
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        at = (at[:, None].expand(-1, 3) if at.dim() == 1 else at).int().contiguous()
        self.ops.mt_rotate(x, at, self.frequencies, out, sections=self.sections)
        return out

    def show(self, images, at, tenant_of):
        """The images' states, bf16 [n, dim] each, their positions int32 [n, 3], one image a prompt."""
        ends = torch.tensor([len(i) for i in images]).cumsum(0)
        self.image_ranges = i32(torch.stack([ends - torch.tensor([len(i) for i in images]), ends], 1))
        ids = i32([t for t, i in zip(tenant_of, images) for _ in range(len(i))])
        x, at = torch.cat(images), torch.cat(at)
        for l in self.layers:
            kv = self._linear(x, ids, l.states).view(len(x), -1, self.head_dim)
            l.image_k, l.image_v = self._turn(kv[:, :self.kv_heads], at), kv[:, self.kv_heads:]

    def _look(self, l, x, ids):
        q = self._linear(self._norm(x), ids, l.ask).view(len(x), self.q_heads, self.head_dim)
        out = torch.empty(q.shape, dtype=BF16, device=q.device)
        self.ops.mt_cross_attention(q, l.image_k, l.image_v, self.offsets, self.ranges, out)
        return x + self._linear(out.flatten(1), ids, l.seen)

    def text(self, offsets, image_of):
        """Which tokens of a call belong together, and what they look at."""
        self.offsets, self.ranges = offsets, self.image_ranges[image_of.long()].contiguous()


class Pages:
    """Rows of a cache, its pages handed out on the device."""

    def __init__(self, model, pages, page_tokens, rows, width):
        self.book = mt.KvPages.empty(pages, page_tokens, rows, width)
        model.open_caches(pages, page_tokens)
        self.copier = mt.KvCopier([l.cache for l in model.layers])

    def reserve(self, rows, counts, total):
        slots = torch.empty(total, dtype=torch.int64, device="cuda")
        mt.mt_kv_reserve(self.book, rows, counts, slots)
        return slots

    def fork(self, parents, children):
        copies = torch.empty((len(parents), 3), dtype=torch.int32, device="cuda")
        mt.mt_kv_fork(self.book, parents, children, copies)
        mt.mt_kv_copy(self.copier, copies)

    def compact(self):
        copies = torch.empty((self.book.refs.numel() // 2, 3), dtype=torch.int32, device="cuda")
        mt.mt_kv_compact(self.book, copies)
        mt.mt_kv_copy(self.copier, copies)


def answer(model, prompts, images, image_at, tenant_of, each, steps, uniform, page_tokens=16, temperature=0.9, top_k=50, top_p=0.9, forced=None):
    """`each` answers of `steps` tokens to each prompt, drawn by uniform numbers [steps][prompts * each] (or the tokens of `forced`); then every
    second answer ends, the cache is compacted, and the others go on for `steps` more (numbers [2 steps][..]).  Returns the logits, tokens and log
    probabilities of every step, a list of [answers] each, and the book of pages."""
    n, lens = len(prompts), [len(p) for p in prompts]
    width = max(-(-(l + 2 * steps) // page_tokens) for l in lens)
    pages = Pages(model, n * (1 + each) * width, page_tokens, n * (1 + each), width)
    model.show(images, image_at, tenant_of)

    # prompts
    seq = torch.repeat_interleave(torch.arange(n), torch.tensor(lens)).cuda()
    at = torch.cat([torch.arange(l) for l in lens]).cuda()
    ids, every = i32(tenant_of), i32(range(n))
    offsets = i32([0] + torch.tensor(lens).cumsum(0).tolist())
    model.text(offsets, every)
    slots = pages.reserve(every, i32(lens), sum(lens))
    logits = model.prompt(i32([t for p in prompts for t in p]), ids[seq], at, slots, offsets)[offsets[1:].long() - 1]

    # answers: rows n, n + 1, ..
    m = n * each
    rows, parents = n + i32(range(m)), every.repeat_interleave(each)
    pages.fork(parents, rows)
    mt.mt_kv_release(pages.book, every)
    logits = logits.repeat_interleave(each, 0)
    out = [], [], []
    for step in range(2 * steps):
        if step == steps:                     # every second answer has ended
            mt.mt_kv_release(pages.book, rows[1::2].contiguous())
            pages.compact()
            rows, parents, logits = rows[::2].contiguous(), parents[::2].contiguous(), logits[::2].contiguous()
            uniform = uniform[:, ::2]
        k = len(rows)
        token, logprob = torch.empty(k, dtype=torch.int32, device="cuda"), torch.empty(k, device="cuda")
        model.ops.mt_token_sample(logits, uniform[step].contiguous(), token, logprob, temperature=torch.full((k,), temperature, device="cuda"),
                                  top_k=torch.full((k,), top_k, dtype=torch.int32, device="cuda"), top_p=torch.full((k,), top_p, device="cuda"))
        if forced is not None:
            token = forced[step]
        for kept, x in zip(out, (logits, token, logprob)):
            kept.append(x)
        model.text(i32(range(k + 1)), parents)
        position = pages.book.lengths[rows.long()]
        slots = pages.reserve(rows, torch.ones_like(rows), k)
        logits = model.step(token, ids[parents.long()], position, slots, pages.book.tables[rows.long()])
    return out + (pages.book,)


def inputs(prompts=3, each=4, steps=4, vocab=1000, dim=256, seed=2):
    """Prompts, images (states and their positions) and uniform numbers."""
    gen = torch.Generator().manual_seed(seed)
    lens = [(17 * i + 5) % 60 + 1 for i in range(prompts)]
    sides = [(1, 4 + i, 7) for i in range(prompts)]
    text = [torch.randint(0, vocab, (l,), generator=gen).tolist() for l in lens]
    images = [torch.randn((t * h * w, dim), generator=gen).to(BF16).cuda() for t, h, w in sides]
    at = [torch.cartesian_prod(torch.arange(t), torch.arange(h), torch.arange(w)).int().cuda() for t, h, w in sides]
    return text, images, at, [i % 3 for i in range(prompts)], torch.rand((2 * steps, prompts * each), generator=gen).cuda()


def main():
    mt.mt_init(0)
    model = SeveralAnswers()
    text, images, at, tenants, uniform = inputs()
    _, tokens, logprobs, book = answer(model, text, images, at, tenants, 4, 4, uniform)
    for s in range(len(text)):
        print("tenant %d, prompt of %d tokens, image of %d states:" % (tenants[s], len(text[s]), len(images[s])))
        for a in range(4):
            mine = [t[4 * s + a].item() for t in tokens[:4]] + ([t[2 * s + a // 2].item() for t in tokens[4:]] if a % 2 == 0 else [])
            print("   ", mine)
    print("pages in use: %d, all in front: %s" % ((book.refs > 0).sum().item(), bool((book.refs[:(book.refs > 0).sum()] > 0).all())))
    print("status:", mt.mt_get_async_status())


if __name__ == "__main__":
    main()
