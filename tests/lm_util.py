"""Plain 64-bit implementations of the language-model operators and the bounds their tests hold them to (imported by test
files; not a test module).  numpy on the host; nothing here uses the library."""
import numpy as np
import torch

from paper_1901_06887_b200 import binding as mt

U = 2.0 ** -8          # unit roundoff of bf16: 8 significant bits, so half a unit in the last place is at most 2^-8 relative
F = 2.0 ** -24         # of fp32


def init():
    mt.mt_init(0, 64, 0)
    mt.mt_get_async_status()


def code_of(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except mt.MtError as e:
        return e.code
    return 0


def to_np(t):
    return t.detach().double().cpu().numpy()


# ---- prompt attention ---------------------------------------------------------------------------
def prompt_reference(q, k, v, offsets, scale):
    """(o, a): outputs, and sum p |v|, the size that rounding the probabilities is relative to.  NaN where no sequence writes."""
    q, k, v = to_np(q), to_np(k), to_np(v)
    g = q.shape[1] // k.shape[1]
    o, a = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        n = hi - lo
        if n <= 0:
            continue
        future = np.triu(np.ones((n, n), bool), 1)
        for h in range(q.shape[1]):
            s = q[lo:hi, h] @ k[lo:hi, h // g].T * scale
            s[future] = -np.inf
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[lo:hi, h] = p @ v[lo:hi, h // g]
            a[lo:hi, h] = p @ np.abs(v[lo:hi, h // g])
    return o, a


def attention_bound(o, a):
    """The output's own rounding; the probabilities' (bf16) relative to sum p |v|; and 2^-12 of that for the fp32 scores and
    exponentials (scores of size 10 err by at most some 2^-14 absolute, which is relative in p) and the sums."""
    return U * np.abs(o) + (1.01 * U + 2.0 ** -12) * a + 1e-30


# ---- 4-bit cache --------------------------------------------------------------------------------
def bf16_round(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def quantise(x):
    """fp32 restatement of the definition, operation by operation (IEEE): codes, scale, bias."""
    x = np.ascontiguousarray(x, np.float32)
    lo, hi = x.min(-1), x.max(-1)
    with np.errstate(all="ignore"):
        scale = bf16_round((hi - lo) / np.float32(15))
        code = np.where(scale[..., None] > 0, np.rint((x - lo[..., None]) / scale[..., None]), 0)
    return np.clip(code, 0, 15).astype(np.uint8), scale, lo


def unpack(codes):
    return np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)


def cache_values(codes, params):
    """64-bit values of packed codes and (scale, bias)."""
    p = to_np(params)
    return unpack(codes.cpu().numpy()).astype(np.float64) * p[..., :1] + p[..., 1:]


def random_cache(pages, page, heads, dim, gen, spread=1.0):
    c = mt.KvCache.empty(pages, page, heads, dim)
    for codes, params in (c.tensors[:2], c.tensors[2:]):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=gen, device="cuda", dtype=torch.uint8))
        params[..., 0] = (0.1 + 0.3 * torch.rand(params.shape[:-1], generator=gen, device="cuda")).to(torch.bfloat16) * spread
        params[..., 1] = (-2.5 + torch.rand(params.shape[:-1], generator=gen, device="cuda")).to(torch.bfloat16) * spread
    return c


def decode_reference(cache, q, tables, lengths, scale):
    """(o, a): outputs, and sum p (|v| + value scale * 8), the size that rounding p * scale before the centred codes is relative to."""
    q, page = to_np(q), cache.tensors[0].shape[2]
    o, a = np.zeros(q.shape), np.zeros(q.shape)
    g = q.shape[1] // cache.heads
    for s, n in enumerate(lengths):
        pages = torch.tensor(tables[s][: -(-n // page)], dtype=torch.long, device="cuda")
        if n == 0:
            continue
        k, v = (cache_values(x[pages], p[pages]) for x, p in (cache.tensors[:2], cache.tensors[2:]))
        vs = to_np(cache.tensors[3][pages])[..., :1]
        for h in range(cache.heads):
            kk, vv, ss = (x[:, h].reshape(-1, x.shape[-1])[:n] for x in (k, v, vs))
            z = q[s, h * g:(h + 1) * g] @ kk.T * scale
            p = np.exp(z - z.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[s, h * g:(h + 1) * g] = p @ vv
            a[s, h * g:(h + 1) * g] = p @ (np.abs(vv) + 8 * ss)
    return o, a


# ---- 4-bit linear -------------------------------------------------------------------------------
def linear_reference(x, ids, codes, scales, bias):
    """(y, a): outputs and sum |x w| + |bias|."""
    x, w = to_np(x), unpack(codes.cpu().numpy()).astype(np.float64) - 8
    s = to_np(scales)
    w *= np.repeat(s, w.shape[2] // s.shape[2], 2)
    b = to_np(bias) if bias is not None else np.zeros(w.shape[:2])
    y = np.stack([w[t] @ x[i] + b[t] for i, t in enumerate(ids)])
    a = np.stack([np.abs(w[t]) @ np.abs(x[i]) + np.abs(b[t]) for i, t in enumerate(ids)])
    return y, a


def linear_bound(y, a, k, bf16):
    """fp32 accumulation over k products: 16 of them join the sum at a time and each step may lose two units (the matrix unit
    truncates), besides the joining of at most 64 partial sums; and the output's rounding."""
    return (k / 16 + 64) * 2 * F * a + (U * np.abs(y) if bf16 else 0)


# ---- log probabilities --------------------------------------------------------------------------
def logprob_reference(logits, tokens, top):
    x = to_np(logits)
    n, v = x.shape
    lp, ent = np.full(n, np.nan), np.full(n, np.nan)
    ids, tlp = np.full((n, top), -1), np.full((n, top), np.nan)
    for i in range(n):
        if np.isnan(x[i]).any() or x[i].max() in (np.inf, -np.inf):
            continue
        m = x[i].max()
        e = np.exp(x[i] - m)
        p = x[i] - m - np.log(e.sum())
        if 0 <= tokens[i] < v:
            lp[i] = p[tokens[i]]
        live = np.where(x[i] > -np.inf)[0]
        ent[i] = -(np.exp(p[live]) * p[live]).sum()
        best = live[np.argsort(-x[i][live], kind="stable")][:top]
        ids[i, :len(best)] = best
        tlp[i] = -np.inf
        tlp[i, :len(best)] = p[best]
    return lp, ent, ids, tlp


def logprob_bound(vocab, size):
    """Sums of vocab / 256 fp32 terms a thread and 64 joins, exponentials good to 2^-21 beside their argument's rounding, and the
    final subtraction relative to its operands (`size`)."""
    return (vocab / 256 + 64) * F + 2.0 ** -21 + 4 * F * size
