"""mt_token_sample against a 64-bit implementation: every limit, ties, masks, odd sizes and strides, rows that are none."""
import math

import numpy as np
import pytest
import torch

from lm_util import init, to_np
from more_lm_util import sample_bound, sample_reference
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def f32(x):
    return torch.tensor(x, dtype=F32, device="cuda")


def draw(logits, u, **kw):
    n = logits.shape[0]
    ids, logprobs = torch.full((n,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), 7.0, device="cuda")
    mt.mt_token_sample(logits, u, ids, logprobs, **kw)
    return ids.cpu().numpy(), to_np(logprobs)


def check(logits, u, most_near=0.02, **kw):
    init()
    ids, logprobs = draw(logits, u, **kw)
    x, uu = to_np(logits), to_np(u)
    near = 0
    for i in range(len(x)):
        par = {k: to_np(v)[i] for k, v in kw.items()}
        if "top_k" in par:
            par["top_k"] = int(par["top_k"])
        want, lp, close = sample_reference(x[i], uu[i], **par)
        near += close
        if close:
            continue
        assert ids[i] == want, (i, ids[i], want, par)
        assert (np.isnan(lp) and np.isnan(logprobs[i])) or abs(logprobs[i] - lp) <= sample_bound(lp), (i, logprobs[i], lp)
    assert near <= max(1, most_near * len(x))
    return ids


def random_logits(n, v, dtype, seed, spread=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (spread * torch.randn((n, v), generator=g, device="cuda")).to(dtype)
    return x, torch.rand(n, generator=g, device="cuda"), g


LIMITS = {
    "none": {}, "warm": dict(temperature=1.7), "cold": dict(temperature=0.2), "greedy": dict(temperature=0.0),
    "k1": dict(top_k=1), "k7": dict(top_k=7), "k50": dict(top_k=50), "k_over": dict(top_k=1 << 30), "k_none": dict(top_k=-3),
    "p": dict(top_p=0.9), "p_low": dict(top_p=0.05), "p_high": dict(top_p=0.9999), "p_zero": dict(top_p=0.0), "p_minus": dict(top_p=-1.0), "p_over": dict(top_p=2.0),
    "m": dict(min_p=0.1), "m_one": dict(min_p=1.0), "m_over": dict(min_p=1.5), "m_tiny": dict(min_p=1e-30),
    "all": dict(temperature=0.8, top_k=40, top_p=0.8, min_p=0.02), "k_then_p": dict(top_k=500, top_p=0.3),
}


def arrays(n, kw):
    return {k: torch.full((n,), v, dtype=torch.int32 if k == "top_k" else F32, device="cuda") for k, v in kw.items()}


@pytest.mark.parametrize("limits", LIMITS)
@pytest.mark.parametrize("v,dtype", [(1000, F32), (1000, BF16), (40000, F32), (40000, BF16)])
def test_limits(limits, v, dtype):
    n = 24 if v < 10000 else 9
    x, u, _ = random_logits(n, v, dtype, 1)
    check(x, u, **arrays(n, LIMITS[limits]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [1, 2, 3, 7, 8, 9, 31, 255, 511, 513, 4095, 8193, 32001, 65537, 200001])
def test_sizes(v, dtype):
    n = 6
    x, u, g = random_logits(n, v, dtype, v)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    check(x, u, **arrays(n, LIMITS["none"]))
    kw = arrays(n, LIMITS["all"])
    kw["top_p"] = torch.rand(n, generator=g, device="cuda")
    check(x, u, **kw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 17, 40, 80, 200, 700])
def test_rows(n, dtype):
    """From one row cut into eight parts to more rows than fit at once."""
    x, u, g = random_logits(n, 33000, dtype, n)
    kw = arrays(n, LIMITS["none"])
    kw["temperature"] = 0.3 + torch.rand(n, generator=g, device="cuda")
    kw["top_p"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.6, torch.rand(n, generator=g, device="cuda"), 1.0)
    kw["top_k"] = (torch.rand(n, generator=g, device="cuda") * 300).int()
    kw["min_p"] = 0.01 * torch.rand(n, generator=g, device="cuda")
    ids, logprobs = draw(x, u, **kw)
    first = check(x[:60], u[:60], **{k: w[:60].contiguous() for k, w in kw.items()})
    assert (ids[:60] == first).all()
    # a row does not depend on how many there are
    last = draw(x[-5:], u[-5:].contiguous(), **{k: w[-5:].contiguous() for k, w in kw.items()})
    assert (ids[-5:] == last[0]).all() and (logprobs[-5:] == last[1]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [9000, 40000, 130001])
@pytest.mark.parametrize("n", [13, 16, 33, 38, 74, 76, 148, 150, 298])
def test_a_row_does_not_depend_on_the_others(n, v, dtype):
    """Rows in more or fewer parts, held or not, one CTA an SM or two: the same tokens."""
    x, u, g = random_logits(n, v, dtype, n + v)
    kw = arrays(n, dict(temperature=0.9, min_p=0.0))
    kw["top_p"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.6, torch.rand(n, generator=g, device="cuda"), 1.0)
    kw["top_k"] = (torch.rand(n, generator=g, device="cuda") * 300).int()
    init()
    ids, logprobs = draw(x, u, **kw)
    check(x[:3], u[:3].contiguous(), **{k: w[:3].contiguous() for k, w in kw.items()})
    for i in range(0, n, 7):
        some = draw(x[i:i + 7], u[i:i + 7].contiguous(), **{k: w[i:i + 7].contiguous() for k, w in kw.items()})
        assert (ids[i:i + 7] == some[0]).all() and (logprobs[i:i + 7] == some[1]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [90, 97, 400, 512, 513, 1000, 1024, 1025, 2000])
def test_many_near_the_cut(m, dtype):
    """m logits that differ by little (bf16: not at all) and the cut among them."""
    n, v = 5, 20000
    x, u, g = random_logits(n, v, dtype, m, spread=0.5)
    for i in range(n):
        at = torch.randperm(v, generator=g, device="cuda")[:m]
        x[i, at] = (9.0 + 1e-4 * torch.rand(m, generator=g, device="cuda")).to(dtype)
    check(x, u, **arrays(n, dict(top_k=m // 3)))
    kw = arrays(n, dict(temperature=0.9, top_k=m - 1))
    kw["top_p"] = torch.rand(n, generator=g, device="cuda")
    check(x, u, **kw)


def test_rows_of_half_a_billion():
    """Sizes in bytes pass 32 bits; many rows that are one (row stride 0)."""
    v, n = (1 << 29) + 3, 300
    x = torch.full((1, v), -float("inf"), device="cuda")
    at = [0, 5, 1 << 28, v - 1]
    x[0, at] = 0.0
    u = f32([0.0, 0.2, 0.25, 0.49, 0.5, 0.7, 0.75, 1.0 - 2.0 ** -24] * 38)[:n]
    init()
    ids, logprobs = draw(x.expand(n, v), u)
    assert (ids == np.array([at[int(4 * w)] for w in u.tolist()])).all()
    assert np.abs(logprobs + math.log(4)).max() <= sample_bound(-math.log(4))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [5, 1001, 30011])
def test_strides_and_alignment(v, dtype):
    """Rows at any element, and neighbours that must not be read as logits."""
    wide = torch.full((8, v + 13), math.nan, dtype=dtype, device="cuda")
    x, u, _ = random_logits(8, v, dtype, 3)
    for at in (0, 1, 3, 7):
        wide.fill_(math.nan)
        wide[:, at:at + v] = x
        check(wide[:, at:at + v], u, **arrays(8, LIMITS["all"]))
        check(wide[:, at:at + v], u)
    same = x[:1].expand(8, v)                                   # one row for all: a stride of zero
    check(same, u, **arrays(8, LIMITS["p"]))


@pytest.mark.parametrize("v", [64, 3000, 70000])
@pytest.mark.parametrize("kind", ["equal", "two", "few", "one_high"])
def test_ties(kind, v):
    """Equal logits are kept from the front of the row, also where a limit cuts through them."""
    n = 12
    g = torch.Generator(device="cuda").manual_seed(v)
    if kind == "equal":
        x = torch.full((n, v), 1.25, device="cuda")
    elif kind == "two":
        x = (torch.rand((n, v), generator=g, device="cuda") < 0.5).float() * 2 - 3
    elif kind == "few":
        x = torch.randint(-3, 4, (n, v), generator=g, device="cuda").float()
    else:
        x = torch.zeros((n, v), device="cuda")
        x[:, v // 2] = 3.0
    u = (torch.arange(n, device="cuda") + 0.5) / n
    for dtype in (F32, BF16):
        y = x.to(dtype)
        check(y, u)
        for k in (1, 2, v // 3 + 1, v - 1):
            check(y, u, top_k=torch.full((n,), k, dtype=torch.int32, device="cuda"))
        for p in (0.001, 0.25, 0.5, 0.777, 0.999):
            check(y, u, most_near=1.0 if kind != "equal" else 0.0, top_p=torch.full((n,), p, device="cuda"))
        check(y, u, **arrays(n, LIMITS["all"]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hole", ["inf", "lowest", "far"])
def test_masks(hole, dtype):
    """Tokens that are ruled out, by minus infinity, by the type's lowest value, or by a large number."""
    n, v = 10, 20000
    x, u, g = random_logits(n, v, dtype, 7)
    value = {"inf": -math.inf, "lowest": torch.finfo(dtype).min, "far": -1e4}[hole]
    for share in (0.5, 0.99, 0.9999):
        out = torch.rand((n, v), generator=g, device="cuda") < share
        out[:, 11] = False
        y = x.masked_fill(out, value)
        for name in ("none", "k50", "p", "m", "all", "k_then_p", "greedy"):
            ids = check(y, u, **arrays(n, LIMITS[name]))
            assert not out.cpu().numpy()[np.arange(n), ids].any()
    one = torch.full((n, v), value, dtype=dtype, device="cuda")
    one[torch.arange(n), torch.arange(n) * 1999] = -5.0
    for name in ("none", "k50", "p", "m", "all", "greedy"):
        assert (check(one, u, **arrays(n, LIMITS[name])) == np.arange(n) * 1999).all()


def test_odd_ranges():
    """Values that spread over the whole of fp32, are tiny, or all but equal."""
    n, v = 8, 5000
    _, u, g = random_logits(n, v, F32, 9)
    normal = torch.randn((n, v), generator=g, device="cuda")
    wide = torch.sign(normal) * 10.0 ** (60 * torch.rand((n, v), generator=g, device="cuda") - 30)
    near = 1e6 + torch.round(normal * 3) / 8
    for x in (wide, normal * 1e-30, near, normal * 3e37, -normal.abs() * 1e-3):
        for name in ("none", "k7", "k50", "p", "p_high", "m", "all"):
            check(x, u, **arrays(n, LIMITS[name]))
    for t in (1e-40, 1e-6, 1e30, 3e38):
        for x in (normal, wide):
            for name in ("k50", "p"):
                kw = arrays(n, LIMITS[name])
                check(x, u, most_near=1.0 if t > 1 else 0.02, temperature=torch.full((n,), t, device="cuda"), **kw)


def test_rows_that_are_none():
    x, u, _ = random_logits(14, 9000, F32, 5)
    x[0] = -math.inf
    x[1, 8999] = math.nan
    x[2, 0] = math.inf
    x[3, 5] = math.nan
    x[3, 6] = math.inf
    kw = arrays(14, dict(temperature=1.0, top_k=0, top_p=0.9, min_p=0.0))
    ids = check(x, u, **kw)
    assert (ids[:4] == -1).all() and (ids[4:] >= 0).all()
    assert mt.mt_get_async_status() == (0, -1)                  # the logits' own business
    kw["temperature"][6], kw["temperature"][7], kw["temperature"][8] = -1.0, math.nan, math.inf
    kw["top_p"][9], kw["min_p"][10] = math.nan, math.nan
    u[5], u[11], u[12] = 1.0, -0.25, math.nan
    init()
    ids, lp = draw(x, u, **kw)
    none = [i for i in range(14) if i not in (4, 13)]
    assert (ids[none] == -1).all() and np.isnan(lp[none]).all() and ids[4] >= 0 and ids[13] >= 0
    assert mt.mt_get_async_status() == (1, 5)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_token_gets_its_share(dtype):
    """Evenly spaced uniform numbers: each token is drawn as often as its probability says, to one draw."""
    init()
    n, v = 4000, 40
    x = random_logits(1, v, dtype, 2, 1.5)[0].expand(n, v)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    for kw in ({}, dict(top_k=9), dict(top_p=0.7), dict(min_p=0.05), dict(temperature=0.5, top_p=0.95)):
        ids, _ = draw(x, u, **arrays(n, kw))
        z = to_np(x[0]) / kw.get("temperature", 1.0)
        w = np.exp(z - z.max())
        order = np.argsort(-z, kind="stable")
        m = min(kw.get("top_k", v), 1 + int(np.searchsorted(np.cumsum(w[order]), kw.get("top_p", 1.0) * w.sum())), int((w >= kw.get("min_p", 0)).sum()))
        p = np.zeros(v)
        p[order[:m]] = w[order[:m]] / w[order[:m]].sum()
        assert np.abs(np.bincount(ids, minlength=v) - n * p).max() <= 1
        assert (np.diff(ids) >= 0).all()                        # in the order of the vocabulary


def test_captured_and_replayed():
    init()
    n, v = 20, 50000
    x, u, g = random_logits(n, v, BF16, 4)
    kw = arrays(n, LIMITS["all"])
    ids, lp = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.mt_token_sample(x, u, ids, lp, stream=torch.cuda.current_stream(), **kw)
    for _ in range(3):
        x.copy_(2.5 * torch.randn((n, v), generator=g, device="cuda"))
        u.copy_(torch.rand(n, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = draw(x, u, **kw)
        assert (ids.cpu().numpy() == want[0]).all() and (to_np(lp) == want[1]).all()
        check(x, u, **kw)


def test_without_logprobs_and_nothing_to_do():
    init()
    x, u, _ = random_logits(3, 100, F32, 6)
    ids = torch.empty(3, dtype=torch.int32, device="cuda")
    mt.mt_token_sample(x, u, ids)
    assert (ids.cpu().numpy() == draw(x, u)[0]).all()
    mt.mt_token_sample(x[:0], u[:0], ids[:0])
