"""The language-model operators: what is measured, and their plain forms.

Five operators that a worker needs to answer for tenants that are language models:

  prompt   causal attention over whole prompts packed one behind the other, grouped heads     mt_prompt_attention
  append   new keys and values rounded to 4 bits into a paged cache, and read back            mt_kv_append, mt_kv_read
  decode   attention of one new token per sequence over the paged 4-bit cache                 mt_kv_attention
  linear   a batch of tokens, each multiplied with its own tenant's 4-bit weights             mt_quant_linear
  score    log probability of given tokens, entropy and the likeliest alternatives            mt_token_logprobs

`run` computes them in elementary torch operations in 32 bits, or, with `own` set, through the package's entry points.
`exact` restates the definitions in 64 bits.
"""
import math

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
def _prompt(name, seqs, longest, shortest, q_heads, kv_heads, head_dim):
    return {"name": name, "op": "prompt", "seqs": seqs, "longest": longest, "shortest": shortest, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim}


def _append(name, tokens, kv_heads, head_dim, page):
    return {"name": name, "op": "append", "tokens": tokens, "kv_heads": kv_heads, "head_dim": head_dim, "page": page}


def _decode(name, seqs, longest, shortest, q_heads, kv_heads, head_dim, page):
    return {"name": name, "op": "decode", "seqs": seqs, "longest": longest, "shortest": shortest, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page}


def _linear(name, rows, tenants, k, n, group, out):
    return {"name": name, "op": "linear", "rows": rows, "tenants": tenants, "k": k, "n": n, "group": group, "out": out}


def _score(name, rows, vocab, top, dtype, allowed):
    return {"name": name, "op": "score", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "allowed": allowed}


def listed():
    return [
        # one short question to a small model: nothing but latency
        _prompt("prompt_short", 1, 57, 57, 8, 2, 64),
        # a batch of prompts as they arrive, from a single token to a page of text
        _prompt("prompt_mixed", 16, 1500, 1, 32, 8, 128),
        # one long document
        _prompt("prompt_document", 1, 8192, 8192, 32, 8, 128),
        # one new token of each of 64 conversations goes to the cache
        _append("append_step", 64, 8, 128, 64),
        # a prefilled batch goes to the cache
        _append("append_prompt", 8191, 8, 128, 64),
        # one user alone with a worker: a single short conversation
        _decode("decode_single", 1, 1000, 1000, 32, 8, 128, 64),
        # a serving batch of conversations of very different length
        _decode("decode_batch", 64, 8000, 1, 32, 8, 128, 64),
        # a few very long contexts
        _decode("decode_long", 4, 131072, 100001, 32, 8, 128, 64),
        # one token through one projection of one tenant
        _linear("linear_single", 1, 1, 4096, 4096, 64, "bf16"),
        # a mixed step: 24 conversations of 8 tenants through the wide layer
        _linear("linear_mixed", 24, 8, 4096, 16384, 64, "bf16"),
        # the next token of 8 constrained answers, most of the vocabulary ruled out, with what else could have come
        _score("score_step", 8, 32000, 20, "fp32", 0.01),
        # a scored prompt of 2000 tokens over a large vocabulary
        _score("score_prompt", 2000, 128000, 5, "bf16", 1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "append", "decode", "linear", "score"])
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8])
    page = rng.choice([16, 32, 64, 128])
    if op == "prompt":
        seqs = _log(rng, 1, 24)
        longest = _log(rng, 2, 8192 // seqs)
        c = _prompt("", seqs, longest, max(1, int(longest * rng.random())), min(32, kv_heads * group) // kv_heads * kv_heads,
                    kv_heads, head_dim)
    elif op == "append":
        c = _append("", _log(rng, 1, 16384), kv_heads, head_dim, page)
    elif op == "decode":
        seqs = _log(rng, 1, 200)
        longest = _log(rng, 1, min(131072, 400000 // seqs))
        c = _decode("", seqs, longest, int(longest * rng.random()), kv_heads * rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), kv_heads,
                    head_dim, page)
    elif op == "linear":
        rows = _log(rng, 1, 64)
        tenants = min(_log(rng, 1, 12), rows)
        quant = rng.choice([32, 64, 128])
        c = _linear("", rows, tenants, 128 * _log(rng, 1, 64), _log(rng, 10, 16384 if tenants < 8 else 4096), quant,
                    rng.choice(["bf16", "fp32"]))
    else:
        vocab = _log(rng, 300, 200000)
        c = _score("", _log(rng, 1, min(4000, 200000000 // vocab)), vocab, rng.randint(1, 32), rng.choice(["bf16", "fp32"]),
                   rng.choice([1.0, 1.0, 0.5, 0.01, 0.0001]))
    del c["name"]
    return c


def _lengths(case):
    """The case's lengths, spread over its range; a whole number of plain values, alike for every seed."""
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    if n == 1:
        return [hi]
    at = [((i * 7919) % n) / (n - 1) for i in range(n)] if math.gcd(7919, n) == 1 else [i / (n - 1) for i in range(n)]
    return [lo + int(round((hi - lo) * a * a)) for a in at]


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------
def _quantise(x):
    """Rows of the last axis as 4-bit codes with a bf16 scale and bias: value = code * scale + bias."""
    x = x.float()
    lo, hi = x.amin(-1), x.amax(-1)
    bias = lo.to(BF16)
    scale = ((hi - lo) / 15.0).to(BF16)
    step = scale.float().unsqueeze(-1)
    code = torch.where(step > 0, torch.round((x - bias.float().unsqueeze(-1)) / step), torch.zeros_like(x)).clamp(0, 15)
    return code.to(torch.uint8), torch.stack([scale, bias], -1)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(packed):
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2)


def _keys(shape, gen, dev):
    """Keys or values: normal, with a few channels that run larger, as trained models have them."""
    x = torch.randn(shape, generator=gen, device=dev)
    x[..., 3::37] *= 3.0
    return x


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    op = case["op"]
    s = {"case": case}
    if op == "prompt":
        lens = _lengths(case)
        n, hq, hkv, d = sum(lens), case["q_heads"], case["kv_heads"], case["head_dim"]
        qkv = _keys((n, hq + 2 * hkv, d), gen, dev).to(BF16)        # one projection's output, split in place
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["offsets"] = torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device=dev)
        s["out"] = torch.empty((n, hq, d), dtype=BF16, device=dev)
    elif op == "append":
        n, h, d, p = case["tokens"], case["kv_heads"], case["head_dim"], case["page"]
        kv = _keys((n, 2 * h, d), gen, dev).to(BF16)
        s["k"], s["v"] = kv[:, :h], kv[:, h:]
        pages = -(-n * 2 // p)
        s["slots"] = torch.randperm(pages * p, generator=gen, device=dev)[:n].contiguous()
        s["cache"] = _empty_cache(pages, h, p, d, dev)
        s["k_out"], s["v_out"] = (torch.empty((n, h, d), dtype=BF16, device=dev) for _ in range(2))
    elif op == "decode":
        lens, h, d, p = _lengths(case), case["kv_heads"], case["head_dim"], case["page"]
        per = [-(-l // p) for l in lens]
        pages, width = max(1, sum(per)), max(1, max(per))
        s["cache"] = c = _empty_cache(pages, h, p, d, dev)
        for name in ("k", "v"):
            for a in range(0, pages, 1 + (1 << 28) // (h * p * d)):
                b = min(pages, a + 1 + (1 << 28) // (h * p * d))
                codes, params = _quantise(_keys((b - a, h, p, d), gen, dev))
                c[name + "_codes"][a:b] = _pack(codes)
                c[name + "_params"][a:b] = params
        ids = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)
        used = torch.arange(width, device=dev)[None] < torch.tensor(per, device=dev)[:, None]
        s["tables"] = torch.zeros((len(lens), width), dtype=torch.int32, device=dev)
        s["tables"][used] = ids[:sum(per)]
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        s["q"] = (1.5 * torch.randn((len(lens), case["q_heads"], d), generator=gen, device=dev)).to(BF16)
        s["out"] = torch.empty_like(s["q"])
    elif op == "linear":
        r, t, k, n, g = case["rows"], case["tenants"], case["k"], case["n"], case["group"]
        codes = torch.randint(0, 256, (t, n, k // 2), generator=gen, device=dev, dtype=torch.uint8)
        scales = ((0.5 + torch.rand((t, n, k // g), generator=gen, device=dev)) / (5.0 * math.sqrt(k))).to(BF16)
        bias = 0.01 * torch.randn((t, n), generator=gen, device=dev)
        s["codes"], s["scales"], s["bias"] = codes, scales, bias
        s["x"] = torch.randn((r, k), generator=gen, device=dev).to(BF16)
        s["ids"] = (torch.randperm(r, generator=gen, device=dev) % t).to(torch.int32)
        s["y"] = torch.empty((r, n), dtype=DTYPES[case["out"]], device=dev)
        if own:     # the weights in the kernel's order, laid out once
            s["bank"] = _mt().QuantBank(codes, scales, bias)
    else:
        r, v, top = case["rows"], case["vocab"], case["top"]
        x = 3.0 * torch.randn((r, -(-v // 8) * 8), generator=gen, device=dev)    # rows padded to whole vectors
        if case["allowed"] < 1.0:
            x.masked_fill_(torch.rand(x.shape, generator=gen, device=dev) >= case["allowed"], -math.inf)
            x[:, :1] = 0.0
        x[:, v:] = math.nan                                       # the padding is nobody's to read
        s["logits"] = x.to(DTYPES[case["dtype"]])[:, :v]
        s["tokens"] = torch.randint(0, v, (r,), generator=gen, device=dev, dtype=torch.int32)
        s["tokens"][::3] = 0
        s["logprobs"], s["entropies"] = (torch.empty(r, device=dev) for _ in range(2))
        s["top_ids"] = torch.empty((r, top), dtype=torch.int32, device=dev)
        s["top_logprobs"] = torch.empty((r, top), device=dev)
    if op in ("append", "decode") and own:
        c = s["cache"]
        s["handle"] = _mt().KvCache(c["k_codes"], c["k_params"], c["v_codes"], c["v_params"])
    return s


def _empty_cache(pages, h, p, d, dev):
    out = {}
    for name in ("k", "v"):
        out[name + "_codes"] = torch.zeros((pages, h, p, d // 2), dtype=torch.uint8, device=dev)
        out[name + "_params"] = torch.zeros((pages, h, p, 2), dtype=BF16, device=dev)
    return out


# ------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_prompt(s):
    _mt().mt_prompt_attention(s["q"], s["k"], s["v"], s["offsets"], s["out"])
    return s["out"]


def _own_append(s):
    _mt().mt_kv_append(s["handle"], s["k"], s["v"], s["slots"])
    _mt().mt_kv_read(s["handle"], s["slots"], s["k_out"], s["v_out"])
    return s["k_out"], s["v_out"]


def _own_decode(s):
    _mt().mt_kv_attention(s["handle"], s["q"], s["tables"], s["lengths"], s["out"])
    return s["out"]


def _own_linear(s):
    _mt().mt_quant_linear(s["x"], s["ids"], s["bank"], s["y"])
    return s["y"]


def _own_score(s):
    _mt().mt_token_logprobs(s["logits"], s["tokens"], s["logprobs"], s["entropies"], s["top_ids"], s["top_logprobs"])
    return s["logprobs"], s["entropies"], s["top_ids"], s["top_logprobs"]


def _plain_prompt(s):
    edges, longest = s["offsets"].long(), s["case"]["longest"]
    n, hq, d = s["q"].shape
    hkv, lens = s["k"].shape[1], edges[1:] - edges[:-1]
    at = torch.arange(longest, device=edges.device)
    row = (edges[:-1, None] + at).clamp_max(n - 1)                        # [sequences][longest], padded
    q, k, v = (s[x].float()[row].transpose(1, 2) for x in "qkv")          # [sequences][heads][longest][dim]
    x = torch.matmul(q.reshape(-1, hkv, hq // hkv * longest, d), k.transpose(2, 3)).mul_(1.0 / math.sqrt(d))
    x = x.view(-1, hkv, hq // hkv, longest, longest)
    x.masked_fill_(at[:, None] < at[None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    x.div_(x.sum(-1, keepdim=True))
    o = torch.matmul(x.view(-1, hkv, hq // hkv * longest, longest), v).view(-1, hq, longest, d)
    return o.transpose(1, 2)[at[None] < lens[:, None]].to(BF16)


def _plain_values(codes, params):
    p = params.float()
    return _unpack(codes).float() * p[..., :1] + p[..., 1:]


def _plain_append(s):
    c, p = s["cache"], s["case"]["page"]
    page, at = s["slots"] // p, s["slots"] % p
    for name in ("k", "v"):
        codes, params = _quantise(s[name])
        c[name + "_codes"][page, :, at] = _pack(codes)
        c[name + "_params"][page, :, at] = params
    return tuple(_plain_values(c[name + "_codes"][page, :, at], c[name + "_params"][page, :, at]).to(BF16) for name in ("k", "v"))


def _plain_decode(s):
    c, q = s["cache"], s["q"].float()
    b, hq, d = q.shape
    hkv = c["k_codes"].shape[1]
    table = s["tables"].long()
    k, v = (_plain_values(c[x + "_codes"][table], c[x + "_params"][table]).transpose(1, 2).reshape(b, hkv, -1, d) for x in ("k", "v"))
    x = torch.matmul(q.view(b, hkv, -1, d), k.transpose(2, 3)) / math.sqrt(d)
    seen = (torch.arange(k.shape[2], device=q.device)[None] < s["lengths"][:, None])[:, None, None]
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(x - torch.where(top > -math.inf, top, 0.0)), 0.0)
    e = e / e.sum(-1, keepdim=True).clamp_min(1e-30)                      # a sequence without tokens gives zeros
    return torch.matmul(e, v).view(b, hq, d).to(BF16)


def _plain_linear(s):
    w = (_unpack(s["codes"]).float() - 8.0).view(*s["scales"].shape, -1) * s["scales"].float().unsqueeze(-1)
    y = torch.matmul(s["x"].float(), w.flatten(2).transpose(1, 2)) + s["bias"][:, None]
    return y[s["ids"].long(), torch.arange(len(s["ids"]), device=y.device)].to(s["y"].dtype)


def _plain_score(s):
    x, top = s["logits"].float() + 0.0, s["case"]["top"]
    v = x.shape[1]
    most = x.amax(-1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(-1, keepdim=True)
    lse = most + torch.log(total)
    entropy = (lse - (torch.where(e > 0, e * x, 0.0)).sum(-1, keepdim=True) / total)[:, 0]
    logprob = (x.gather(1, s["tokens"].long()[:, None]) - lse)[:, 0]
    bits = x.view(torch.int32) if x.is_contiguous() else x.contiguous().view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()                   # grows with the value; ties: the lowest index first
    key = (order << 32) | (v - 1 - torch.arange(v, device=x.device))
    ids = v - 1 - (key.topk(min(top, v), dim=-1).values & 0xFFFFFFFF)
    value = x.gather(1, ids)
    there = value > -math.inf                                             # what has no probability is no alternative
    ids, value = torch.where(there, ids, -1).int(), torch.where(there, value - lse, -math.inf)
    return logprob, entropy, ids, value


_run_own = {"prompt": _own_prompt, "append": _own_append, "decode": _own_decode, "linear": _own_linear, "score": _own_score}
_run_plain = {"prompt": _plain_prompt, "append": _plain_append, "decode": _plain_decode, "linear": _plain_linear, "score": _plain_score}


# ------------------------------------------------------------------------------------------------
# The work of one pass
# ------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "prompt":
        lens, hq, hkv, d = _lengths(case), case["q_heads"], case["kv_heads"], case["head_dim"]
        return {"bytes": 2.0 * sum(lens) * d * (2 * hq + 2 * hkv), "flops": 4.0 * d * hq * sum(l * (l + 1) / 2 for l in lens)}
    if op == "append":
        n, h, d = case["tokens"], case["kv_heads"], case["head_dim"]
        rows = 2.0 * n * h                                                # in, codes and parameters out and in again, values out
        return {"bytes": rows * (2 * d + 2 * (d / 2 + 4) + 2 * d), "flops": rows * d * 6}
    if op == "decode":
        lens, hq, hkv, d = _lengths(case), case["q_heads"], case["kv_heads"], case["head_dim"]
        return {"bytes": sum(lens) * hkv * (d + 8.0) + 4.0 * len(lens) * hq * d, "flops": 4.0 * d * hq * sum(lens)}
    if op == "linear":
        r, t, k, n, g = case["rows"], case["tenants"], case["k"], case["n"], case["group"]
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": t * n * (k / 2 + 2.0 * k / g + 4) + r * (2.0 * k + out * n), "flops": 2.0 * r * k * n}
    r, v = case["rows"], case["vocab"]
    return {"bytes": r * (v * (4.0 if case["dtype"] == "fp32" else 2.0) + 12 + 8 * case["top"]), "flops": 6.0 * r * v}


# ------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"prompt": _exact_prompt, "append": _exact_append, "decode": _exact_decode, "linear": _exact_linear,
            "score": _exact_score}[case["op"]](s, case)


def _exact_prompt(s, case):
    group = case["q_heads"] // case["kv_heads"]
    edges = s["offsets"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for a, b in zip(edges[:-1], edges[1:]):
        for h in range(case["q_heads"]):
            z = s["q"][a:b, h].double() @ s["k"][a:b, h // group].double().T / case["head_dim"] ** 0.5
            z = torch.softmax(z + torch.full_like(z, -math.inf).triu(1), -1)
            out[a:b, h] = z @ s["v"][a:b, h // group].double()
    return out


def _exact_append(s, case):
    """Nearest of the sixteen levels that the rounded scale and bias allow."""
    both = []
    for name in ("k", "v"):
        x = s[name].double()
        lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
        scale = ((hi - lo).float() / 15).to(BF16).double()                # held in bf16 by definition
        code = ((x - lo) / scale.clamp_min(1e-300)).round().clamp(0, 15)
        both.append(code * scale + lo)
    return tuple(both)


def _exact_decode(s, case):
    c, p = s["cache"], case["page"]
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for i, l in enumerate(s["lengths"].tolist()):
        pages = s["tables"][i, :-(-l // p)].long()
        for h in range(case["kv_heads"] if l else 0):
            k, v = (torch.stack([(c[x + "_codes"][pages, h] & 15), (c[x + "_codes"][pages, h] >> 4)], -1).flatten(2).double()
                    .mul(c[x + "_params"][pages, h, :, :1].double()).add(c[x + "_params"][pages, h, :, 1:].double()).flatten(0, 1)[:l]
                    for x in ("k", "v"))
            z = s["q"][i, h * group:(h + 1) * group].double() @ k.T / case["head_dim"] ** 0.5
            out[i, h * group:(h + 1) * group] = torch.softmax(z, -1) @ v
    return out


def _exact_linear(s, case):
    y = torch.zeros((case["rows"], case["n"]), dtype=torch.float64, device="cuda")
    for t in range(case["tenants"]):
        low, high = (s["codes"][t] & 15).double() - 8, (s["codes"][t] >> 4).double() - 8
        scale = s["scales"][t].double().repeat_interleave(case["group"] // 2, 1)
        rows = s["ids"] == t
        x = s["x"][rows].double()
        y[rows] = x[:, 0::2] @ (low * scale).T + x[:, 1::2] @ (high * scale).T + s["bias"][t].double()
    return y


def _exact_score(s, case):
    parts = []
    for x, t in zip(s["logits"].split(64), s["tokens"].split(64)):
        p = torch.log_softmax(x.double(), -1)
        entropy = -torch.where(p > -math.inf, p * p.exp(), 0.0).sum(-1)
        value, ids = (y[:, :case["top"]] for y in torch.sort(x.double(), dim=-1, descending=True, stable=True))
        there = value > -math.inf
        parts.append((p.gather(1, t.long()[:, None])[:, 0], entropy, torch.where(there, ids, -1).int(),
                      torch.where(there, p.gather(1, ids), -math.inf)))
    return tuple(torch.cat(y) for y in zip(*parts))
