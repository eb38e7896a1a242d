"""More operators of language-model tenants: what is measured, and their plain forms.

Four operators that a worker needs to give several answers, also about an image or a recording:

  sample   a token drawn from given uniform numbers, with temperature, top-k, top-p and min-p        mt_token_sample
  rotate   rotary positions of one to three axes                                                     mt_rotate
  fork     rows of a paged cache forked into several answers: pages shared, copied, reserved and
           given back                                                                                 mt_kv_fork, mt_kv_copy, mt_kv_reserve, mt_kv_release
  compact  a cache's pages moved to its front                                                         mt_kv_compact, mt_kv_copy
  cross    attention of packed queries, or of one token a sequence, to an encoder's states            mt_cross_attention

`run` computes them in elementary torch operations, or, with `own` set, through the package's entry points.  `exact` restates the
definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

BF16 = torch.bfloat16
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_binding = None


def _mt():
    """The package's binding, initialised once (only the framework's own runs come here)."""
    global _binding
    if _binding is None:
        from paper_1901_06887_b200 import binding
        binding.mt_init(0)
        _binding = binding
    return _binding


# ------------------------------------------------------------------------------------------------
# Cases
# ------------------------------------------------------------------------------------------------
def _sample(name, rows, vocab, dtype, filters):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "filters": filters}


def _rotate(name, tokens, heads, head_dim, rotary, axes, neighbours, dtype):
    return {"name": name, "op": "rotate", "tokens": tokens, "heads": heads, "head_dim": head_dim, "rotary": rotary, "axes": axes,
            "neighbours": neighbours, "dtype": dtype}


def _fork(name, prompts, answers, longest, shortest, layers, kv_heads, head_dim, page):
    return {"name": name, "op": "fork", "seqs": prompts, "answers": answers, "longest": longest, "shortest": shortest, "layers": layers,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page}


def _compact(name, seqs, longest, shortest, spare, layers, kv_heads, head_dim, page):
    return {"name": name, "op": "compact", "seqs": seqs, "longest": longest, "shortest": shortest, "spare": spare, "layers": layers,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page}


def _cross(name, seqs, longest, shortest, sources, most, least, q_heads, kv_heads, head_dim):
    return {"name": name, "op": "cross", "seqs": seqs, "longest": longest, "shortest": shortest, "sources": sources, "most": most, "least": least,
            "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim}


def listed():
    return [
        # the next token of one conversation: nothing but latency
        _sample("sample_single", 1, 32000, "fp32", "top_p"),
        # the next tokens of a serving batch, every row with settings of its own
        _sample("sample_batch", 64, 128000, "bf16", "mixed"),
        # many answers at once, drawn from the whole distribution
        _sample("sample_whole", 512, 128000, "fp32", "none"),
        # queries and keys of one token step
        _rotate("rotate_step", 64, 40, 128, 128, 1, False, "bf16"),
        # a batch of prompts with images: positions in time, height and width
        _rotate("rotate_images", 8191, 40, 128, 128, 3, False, "bf16"),
        # four prompts of a small model, two answers each
        _fork("fork_few", 4, 2, 500, 33, 2, 2, 64, 16),
        # a batch of prompts of a large model, several answers each
        _fork("fork_batch", 16, 4, 4000, 100, 8, 8, 128, 64),
        # half of the conversations are over: the rest moves together
        _compact("compact_half", 32, 2000, 10, 600, 8, 8, 128, 64),
        # one token of one answer about half a minute of speech
        _cross("cross_single", 1, 1, 1, 1, 1500, 1500, 32, 8, 128),
        # one token of each of 64 answers, four to a source
        _cross("cross_step", 64, 1, 1, 16, 4000, 577, 32, 8, 128),
        # prompts as they arrive, each about its own image
        _cross("cross_mixed", 16, 700, 1, 16, 2305, 49, 32, 8, 128),
        # a long text about a long recording
        _cross("cross_document", 2, 6000, 5001, 2, 6000, 4500, 16, 16, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "rotate", "fork", "compact", "cross", "cross"])
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    page = rng.choice([16, 32, 64, 128])
    if op == "sample":
        vocab = _log(rng, 300, 200000)
        c = _sample("", _log(rng, 1, min(2000, 60000000 // vocab)), vocab, rng.choice(["bf16", "fp32"]),
                    rng.choice(["none", "top_k", "top_p", "min_p", "mixed", "mixed"]))
    elif op == "rotate":
        dim = rng.choice([32, 64, 80, 128, 128, 256])
        c = _rotate("", _log(rng, 1, 1200000 // (40 * dim)), rng.randint(1, 40), dim, rng.choice([dim, dim, dim // 2 // 16 * 16]),
                    rng.choice([1, 2, 3]), rng.random() < 0.4, rng.choice(["bf16", "bf16", "fp32"]))
        c["tokens"] *= rng.choice([1, 1, 30])
    elif op == "fork":
        prompts = _log(rng, 1, 40)
        longest = _log(rng, 1, 20000 // prompts)
        c = _fork("", prompts, rng.randint(1, 6), longest, max(1, int(longest * rng.random())), rng.choice([1, 2, 5, 8]), kv_heads, head_dim, page)
    elif op == "compact":
        seqs = _log(rng, 1, 60)
        longest = _log(rng, 1, 20000 // seqs)
        c = _compact("", seqs, longest, max(0, int(longest * rng.random())), _log(rng, 1, 400), rng.choice([1, 2, 4]), kv_heads, head_dim, page)
    else:
        sources = _log(rng, 1, 24)
        most = _log(rng, 1, 24000 // sources)
        seqs = sources * rng.choice([1, 1, 2, 5])
        q_heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 5, 8) if g * kv_heads <= 32])
        longest = rng.choice([1, _log(rng, 1, max(1, min(4000, 700000000 // (seqs * q_heads * most))))])
        c = _cross("", seqs, longest, max(1, int(longest * rng.random())), sources, most, int(most * rng.random()), q_heads, kv_heads, head_dim)
    del c["name"]
    return c


def _spread(n, lo, hi):
    """n lengths spread over a range, more of them short; plain whole numbers, alike for every seed."""
    if n == 1:
        return [hi]
    at = [((i * 7919) % n) / (n - 1) for i in range(n)] if math.gcd(7919, n) == 1 else [i / (n - 1) for i in range(n)]
    return [lo + int(round((hi - lo) * a * a)) for a in at]


def _lengths(case):
    return _spread(case["seqs"], case["shortest"], case["longest"])


def _states(case):
    return _spread(case["sources"], case["least"], case["most"])


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------
def _keys(shape, gen, dev):
    """Keys or values: normal, with a few channels that run larger, as trained models have them."""
    x = torch.randn(shape, generator=gen, device=dev)
    x[..., 3::37] *= 3.0
    return x


def _caches(case, pages, gen, dev):
    """The layers' caches: codes and (scale, bias) of keys and values, pages by heads by places."""
    h, p, d = case["kv_heads"], case["page"], case["head_dim"]
    out = []
    for _ in range(case["layers"]):
        layer = {}
        for name in ("k", "v"):
            layer[name + "_codes"] = torch.randint(0, 256, (pages, h, p, d // 2), generator=gen, device=dev, dtype=torch.uint8)
            layer[name + "_params"] = torch.randn((pages, h, p, 2), generator=gen, device=dev).to(BF16)
        out.append(layer)
    return out


def _hand_out(lens, page, ids, width, dev):
    """Tables of pages `ids`, one row per length, the lengths, and how often each page is used."""
    per = torch.tensor([-(-l // page) for l in lens], device=dev)
    used = torch.arange(width, device=dev)[None] < per[:, None]
    tables = torch.zeros((len(lens), width), dtype=torch.int32, device=dev)
    tables[used] = ids[:int(per.sum())].to(torch.int32)
    refs = torch.zeros(len(ids), dtype=torch.int32, device=dev)
    refs[ids[:int(per.sum())]] = 1
    return tables, torch.tensor(lens, dtype=torch.int32, device=dev), refs


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    op = case["op"]
    s = {"case": case}
    if op == "sample":
        r, v, filters = case["rows"], case["vocab"], case["filters"]
        x = 2.5 * torch.randn((r, -(-v // 8) * 8), generator=gen, device=dev)        # rows padded to whole vectors
        sure = torch.rand(r, generator=gen, device=dev) < 0.5                        # half of the rows know what they want
        x[:, :: max(1, v // 7)] += 9.0 * sure[:, None]
        x[:, v:] = math.nan                                                           # the padding is nobody's to read
        s["logits"] = x.to(DTYPES[case["dtype"]])[:, :v]
        u = torch.rand((6, r), generator=gen, device=dev)
        some = (u[4] * 4).int() if filters == "mixed" else None                      # mixed: each row has its own kind
        on = lambda i, name: (some == i) if filters == "mixed" else torch.full((r,), filters == name, device=dev)
        s["temperature"] = 0.4 + u[0]
        if filters == "mixed":
            s["temperature"][::11] = 0.0
        s["top_k"] = torch.where(on(1, "top_k"), 1 + (u[1] * min(v, 200)).int(), 0).int()
        s["top_p"] = torch.where(on(2, "top_p") | (on(1, "") & (u[5] < 0.5)), 0.5 + 0.49 * u[2], 1.0)
        s["min_p"] = torch.where(on(3, "min_p"), 0.2 * u[3], 0.0)
        s["uniform"] = torch.rand(r, generator=gen, device=dev)
        s["ids"] = torch.empty(r, dtype=torch.int32, device=dev)
        s["logprobs"] = torch.empty(r, device=dev)
    elif op == "rotate":
        n, h, d, rot, axes = case["tokens"], case["heads"], case["head_dim"], case["rotary"], case["axes"]
        qkv = _keys((n, h + 2, d), gen, dev).to(DTYPES[case["dtype"]])               # queries and keys of one projection's output
        s["x"], s["out"] = qkv[:, :h], torch.empty((n, h, d), dtype=qkv.dtype, device=dev)
        s["sections"] = [rot // 2 * (i + 1) // axes - rot // 2 * i // axes for i in range(axes)]
        s["frequencies"] = (10000.0 ** (-torch.arange(rot // 2, device=dev, dtype=torch.float64) / (rot // 2))).float()
        far = [131072, 200, 200]
        s["positions"] = torch.stack([torch.randint(0, far[a], (n,), generator=gen, device=dev, dtype=torch.int32) for a in range(axes)], 1)
    elif op == "fork":
        lens, p, b = _lengths(case), case["page"], case["answers"]
        width = max(-(-(l + 1) // p) for l in lens)
        full = sum(-(-l // p) for l in lens)
        pages = full + 2 * b * len(lens) + 3                                          # room for a copied page and a new one an answer
        ids = torch.randperm(pages, generator=gen, device=dev)
        tables, lengths, s["refs"] = _hand_out(lens, p, ids, width, dev)
        n = len(lens) * b
        s["tables"] = torch.cat([tables, torch.zeros((n, width), dtype=torch.int32, device=dev)])
        s["lengths"] = torch.cat([lengths, torch.zeros(n, dtype=torch.int32, device=dev)])
        s["parents"] = torch.arange(len(lens), dtype=torch.int32, device=dev).repeat_interleave(b)
        s["children"] = len(lens) + torch.arange(n, dtype=torch.int32, device=dev)
        s["ones"] = torch.ones(n, dtype=torch.int32, device=dev)
        s["copies"] = torch.empty((n, 3), dtype=torch.int32, device=dev)
        s["slots"] = torch.empty(n, dtype=torch.int64, device=dev)
        s["caches"] = _caches(case, pages, gen, dev)
    elif op == "compact":
        lens, p = _lengths(case), case["page"]
        width = max(1, max(-(-l // p) for l in lens))
        pages = sum(-(-l // p) for l in lens) + case["spare"]
        ids = torch.randperm(pages, generator=gen, device=dev)
        s["was"] = _hand_out(lens, p, ids, width, dev)
        s["tables"], s["lengths"], s["refs"] = (torch.empty_like(x) for x in s["was"])
        s["copies"] = torch.empty((min(pages - case["spare"], case["spare"]), 3), dtype=torch.int32, device=dev)
        s["caches"] = _caches(case, pages, gen, dev)
    else:
        lens, states, d = _lengths(case), _states(case), case["head_dim"]
        n, m, hq, hkv = sum(lens), sum(states), case["q_heads"], case["kv_heads"]
        s["q"] = _keys((n, hq, d), gen, dev).to(BF16)
        kv = _keys((m, 2 * hkv, d), gen, dev).to(BF16)                               # one projection of the encoder's states
        s["k"], s["v"] = kv[:, :hkv], kv[:, hkv:]
        s["offsets"] = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device=dev)
        ends = torch.tensor(states).cumsum(0)
        ranges = torch.stack([ends - torch.tensor(states), ends], 1).repeat_interleave(len(lens) // len(states), 0)
        s["ranges"] = ranges.to(torch.int32).to(dev)
        s["out"] = torch.empty_like(s["q"])
    if own and op in ("fork", "compact"):
        mt = _mt()
        s["handles"] = [mt.KvCache(c["k_codes"], c["k_params"], c["v_codes"], c["v_params"]) for c in s["caches"]]
        s["pages"] = mt.KvPages(s["refs"], s["tables"], s["lengths"], case["page"])
        s["copier"] = mt.KvCopier(s["handles"])
    return s


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_sample(s):
    _mt().mt_token_sample(s["logits"], s["uniform"], s["ids"], s["logprobs"], temperature=s["temperature"], top_k=s["top_k"],
                          top_p=s["top_p"], min_p=s["min_p"])
    return s["ids"], s["logprobs"]


def _own_rotate(s):
    _mt().mt_rotate(s["x"], s["positions"], s["frequencies"], s["out"], sections=s["sections"], neighbours=s["case"]["neighbours"])
    return s["out"]


def _cache_tensors(s):
    return [c[name] for c in s["caches"] for name in ("k_codes", "k_params", "v_codes", "v_params")]


def _own_fork(s):
    mt = _mt()
    mt.mt_kv_fork(s["pages"], s["parents"], s["children"], s["copies"])
    mt.mt_kv_copy(s["copier"], s["copies"])
    mt.mt_kv_reserve(s["pages"], s["children"], s["ones"], s["slots"])
    mt.mt_kv_release(s["pages"], s["children"])                                       # the answers end, so the next pass finds the same
    return [s["copies"], s["slots"], s["tables"], s["lengths"], s["refs"]] + _cache_tensors(s)


def _own_compact(s):
    mt = _mt()
    for x, was in zip((s["tables"], s["lengths"], s["refs"]), s["was"]):
        x.copy_(was)
    mt.mt_kv_compact(s["pages"], s["copies"])
    mt.mt_kv_copy(s["copier"], s["copies"])
    return [s["copies"], s["tables"], s["lengths"], s["refs"]] + _cache_tensors(s)


def _own_cross(s):
    _mt().mt_cross_attention(s["q"], s["k"], s["v"], s["offsets"], s["ranges"], s["out"])
    return s["out"]


def _plain_sample(s):
    x = s["logits"].float() + 0.0
    n, v = x.shape
    bits = x.contiguous().view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()                                 # grows with the value; ties: the lowest index first
    key = (key << 32) | (v - 1 - torch.arange(v, device=x.device))
    order = v - 1 - (key.sort(-1, descending=True).values & 0xFFFFFFFF)
    t = s["temperature"].double()[:, None]
    x = x.double()
    w = torch.exp((x - x.amax(-1, keepdim=True)) / torch.where(t > 0, t, 1.0)).gather(1, order)
    before = w.cumsum(-1) - w
    rank = torch.arange(v, device=x.device)[None]
    k = s["top_k"].long()[:, None]
    kept = torch.where(k > 0, rank < k, True) & (w >= s["min_p"].double()[:, None])
    p = s["top_p"].double()[:, None]
    kept &= torch.where(p < 1, before < p * w.sum(-1, keepdim=True), True)
    kept = torch.where(t > 0, kept, False) | (rank == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, 0.0))
    mass = w.cumsum(-1)
    ids = (mass <= s["uniform"].double()[:, None] * mass[:, -1:]).sum(-1, keepdim=True).clamp_max(v - 1)
    return ids[:, 0].int(), torch.log(w.gather(1, ids)[:, 0] / mass[:, -1]).float()


def _plain_rotate(s):
    rot, half = s["case"]["rotary"], s["case"]["rotary"] // 2
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device=s["x"].device), torch.tensor(s["sections"], device=s["x"].device))
    angle = s["positions"].double()[:, axis] * s["frequencies"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = s["x"].float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["case"]["neighbours"] else (x[..., :half], x[..., half:rot])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if s["case"]["neighbours"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1).to(s["x"].dtype)


def _plain_copy(s, copies):
    """Pages of every layer: (from, to, tokens), tokens 0 where there is nothing to do."""
    src, dst = copies[:, 0].clamp_min(0).long(), copies[:, 1].clamp_min(0).long()
    page = s["case"]["page"]
    take = (torch.arange(page, device=copies.device)[None] < copies[:, 2:])
    i, at = take.nonzero(as_tuple=True)
    src, dst = src[i], dst[i]
    for x in _cache_tensors(s):
        x[dst, :, at] = x[src, :, at]


def _plain_fork(s):
    page, tables, lengths, refs = s["case"]["page"], s["tables"], s["lengths"], s["refs"]
    parents, children = s["parents"].long(), s["children"].long()
    rows, lens, width = tables[parents], lengths[parents], tables.shape[1]
    col = torch.arange(width, device=tables.device)[None]
    whole, part = lens // page, lens % page
    free = (refs == 0).nonzero()[:, 0]                                                # lowest first
    refs.index_add_(0, rows[col < whole[:, None]].long(), torch.ones_like(rows[col < whole[:, None]]))
    needs = part > 0
    at = needs.long().cumsum(0) - 1
    fresh = free[at.clamp_min(0)].int()
    last = rows.gather(1, whole.long().clamp_max(width - 1)[:, None])[:, 0]
    none = torch.full_like(last, -1)
    copies = torch.stack([torch.where(needs, last, none), torch.where(needs, fresh, none), torch.where(needs, part, 0)], 1).int()
    refs[fresh[needs].long()] = 1
    rows = torch.where((col == whole[:, None]) & needs[:, None], fresh[:, None], rows)
    mine = col < (whole + needs.int())[:, None]
    tables[children] = torch.where(mine, rows, tables[children])
    lengths[children] = lens
    _plain_copy(s, copies)
    # one more token for each answer: a new page where the last one is full
    needs = part == 0
    free = (refs == 0).nonzero()[:, 0]
    at = needs.long().cumsum(0) - 1
    fresh = free[at.clamp_min(0)].int()
    refs[fresh[needs].long()] = 1
    rows = tables[children]
    rows = torch.where((col == whole[:, None]) & needs[:, None], fresh[:, None], rows)
    tables[children] = rows
    slots = rows.gather(1, whole.long()[:, None])[:, 0].long() * page + part
    # the answers end
    mine = col <= whole[:, None]
    refs.index_add_(0, rows[mine].long(), -torch.ones_like(rows[mine]))
    lengths[children] = 0
    return [copies, slots, tables, lengths, refs] + _cache_tensors(s)


def _plain_compact(s):
    for x, was in zip((s["tables"], s["lengths"], s["refs"]), s["was"]):
        x.copy_(was)
    page, tables, lengths, refs, most = s["case"]["page"], s["tables"], s["lengths"], s["refs"], s["copies"].shape[0]
    used = (refs > 0).sum()
    at = torch.arange(refs.numel(), device=refs.device)
    holes, high = ((refs == 0) & (at < used)).nonzero()[:, 0], ((refs > 0) & (at >= used)).nonzero()[:, 0]
    to = at.clone()
    to[high] = holes
    copies = torch.full((most, 3), -1, dtype=torch.int32, device=refs.device)
    copies[:, 2] = 0
    copies[:len(high)] = torch.stack([high, holes, torch.full_like(high, page)], 1).int()
    refs[holes] = refs[high]
    refs[high] = 0
    mine = torch.arange(tables.shape[1], device=refs.device)[None] < ((lengths + page - 1) // page)[:, None]
    tables.copy_(torch.where(mine, to[tables.long()].int(), tables))
    _plain_copy(s, copies)
    return [copies, tables, lengths, refs] + _cache_tensors(s)


def _plain_cross(s):
    q, k, v = (s[x].float() for x in "qkv")
    n, hq, d = q.shape
    hkv = k.shape[1]
    lens, counts = _lengths(s["case"]), _states(s["case"])
    longest, most = max(lens), max(max(counts), 1)
    edges, first = s["offsets"].long(), s["ranges"][:, 0].long()
    seen = torch.arange(most, device=q.device)[None] < (s["ranges"][:, 1] - s["ranges"][:, 0])[:, None]
    at = torch.arange(longest, device=q.device)[None]
    row = (edges[:-1, None] + at).clamp_max(n - 1)                                   # [sequences][longest], padded
    state = (first[:, None] + torch.arange(most, device=q.device)[None]).clamp_max(max(k.shape[0] - 1, 0))
    if k.shape[0] == 0:
        return torch.zeros_like(s["q"])
    qq = q[row].transpose(1, 2).reshape(len(lens), hkv, hq // hkv * longest, d)
    x = torch.matmul(qq, k[state].permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(d))
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    x.div_(x.sum(-1, keepdim=True).clamp_min(1e-30))                                 # a sequence without states gives zeros
    o = torch.matmul(x, v[state].transpose(1, 2)).view(len(lens), hq, longest, d)
    return o.transpose(1, 2)[at < (edges[1:] - edges[:-1])[:, None]].to(BF16)


_run_own = {"sample": _own_sample, "rotate": _own_rotate, "fork": _own_fork, "compact": _own_compact, "cross": _own_cross}
_run_plain = {"sample": _plain_sample, "rotate": _plain_rotate, "fork": _plain_fork, "compact": _plain_compact, "cross": _plain_cross}


# ------------------------------------------------------------------------------------------------
# The work of one pass
# ------------------------------------------------------------------------------------------------
def _token_bytes(case):
    """A cached token of all layers."""
    return case["layers"] * 2.0 * case["kv_heads"] * (case["head_dim"] / 2 + 4)


def work(case):
    op = case["op"]
    if op == "sample":
        r, v = case["rows"], case["vocab"]
        return {"bytes": r * (v * (4.0 if case["dtype"] == "fp32" else 2.0) + 28), "flops": 6.0 * r * v}
    if op == "rotate":
        n, h, d = case["tokens"], case["heads"], case["head_dim"]
        return {"bytes": n * (2.0 * h * d * (4 if case["dtype"] == "fp32" else 2) + 4 * case["axes"]), "flops": 3.0 * n * h * case["rotary"]}
    if op == "fork":
        lens, p, b = _lengths(case), case["page"], case["answers"]
        whole = sum(l // p for l in lens)
        # the copied tokens once in and once out; tables read for each prompt, written for each answer, references read once, and moved up and down
        return {"bytes": 2 * _token_bytes(case) * b * sum(l % p for l in lens) + 4.0 * (whole * (1 + 5 * b) + 20 * b * len(lens)), "flops": 4.0 * b * whole + 1}
    if op == "compact":
        # what is moved is a matter of chance: the mean of used pages behind the border
        used = sum(-(-l // case["page"]) for l in _lengths(case))
        moved = used * case["spare"] / max(1, used + case["spare"])
        return {"bytes": 2 * _token_bytes(case) * moved * case["page"] + 8.0 * (used + case["spare"]) + 8.0 * used, "flops": 4.0 * used + 1}
    lens, states, hq, hkv, d = _lengths(case), _states(case), case["q_heads"], case["kv_heads"], case["head_dim"]
    each = len(lens) // len(states)
    pairs = sum(l * states[i // each] for i, l in enumerate(lens))
    return {"bytes": 2.0 * d * (2 * hq * sum(lens) + 2 * hkv * sum(states)), "flops": 4.0 * d * hq * pairs + 1}


# ------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None                                                                   # whole numbers and copies
    s = prepare(case, seed)
    return {"sample": _exact_sample, "rotate": _exact_rotate, "cross": _exact_cross}[case["op"]](s, case)


def _exact_sample(s, case):
    if case["rows"] * case["vocab"] > 70000000:
        return None
    ids, logprobs = [], []
    x = s["logits"].double().cpu().numpy()
    par = {name: s[name].double().cpu().numpy() for name in ("temperature", "top_k", "top_p", "min_p", "uniform")}
    for i, row in enumerate(x):
        if par["temperature"][i] == 0:
            ids.append(int(np.argmax(row)))
            logprobs.append(0.0)
            continue
        w = np.exp((row - row.max()) / par["temperature"][i])
        order = np.argsort(-row, kind="stable")
        m = len(row)
        if par["top_k"][i] > 0:
            m = min(m, int(par["top_k"][i]))
        if par["top_p"][i] < 1:
            m = min(m, 1 + int(np.searchsorted(np.cumsum(w[order]), par["top_p"][i] * w.sum(), side="left")))
        m = max(1, min(m, int((w >= par["min_p"][i]).sum())))
        kept = np.zeros(len(row))
        kept[order[:m]] = w[order[:m]]
        mass = np.cumsum(kept)
        token = int(np.searchsorted(mass, par["uniform"][i] * mass[-1], side="right"))
        ids.append(token)
        logprobs.append(math.log(kept[token] / mass[-1]))
    return torch.tensor(ids, dtype=torch.int32), torch.tensor(logprobs, dtype=torch.float64)


def _exact_rotate(s, case):
    x, rot = s["x"].double(), case["rotary"]
    out, c0 = x.clone(), 0
    for axis, count in enumerate(s["sections"]):
        c = torch.arange(c0, c0 + count, device=x.device)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), s["positions"][:, axis, None].double() * s["frequencies"][c].double())
        first, second = (2 * c, 2 * c + 1) if case["neighbours"] else (c, c + rot // 2)
        y = torch.complex(x[:, :, first], x[:, :, second]) * turn[:, None]
        out[:, :, first], out[:, :, second] = y.real, y.imag
        c0 += count
    return out


def _exact_cross(s, case):
    if work(case)["flops"] > 4e11:
        return None
    group = case["q_heads"] // case["kv_heads"]
    edges, ranges = s["offsets"].tolist(), s["ranges"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    for i, (lo, hi) in enumerate(ranges):
        if hi <= lo:
            continue
        q = s["q"][edges[i]:edges[i + 1]].double()
        k, v = (s[x][lo:hi].double().repeat_interleave(group, 1) for x in "kv")
        for a in range(0, len(q), 512):
            p = torch.softmax(torch.einsum("qhd,khd->hqk", q[a:a + 512], k) / math.sqrt(case["head_dim"]), -1)
            out[edges[i] + a:edges[i] + a + len(p[0])] = torch.einsum("hqk,khd->qhd", p, v)
    return out
