"""mt_kv_append, mt_kv_read and mt_kv_attention against 64-bit implementations: rounding to 4 bits, slots, pages that end
inside a tile, lengths of zero and one, grouped heads, refusals."""
import numpy as np
import pytest
import torch

from lm_util import F, U, attention_bound, cache_values, code_of, decode_reference, init, quantise, random_cache, to_np
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu


def gen(seed=0):
    init()
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,heads", [(1, 1), (3, 2), (33, 5), (257, 1)])
def test_append_and_read(page, dim, n, heads):
    g = gen(n)
    kv = torch.randn((n, 2 * heads, dim), generator=g, device="cuda")
    kv[n // 2] *= 1e4
    kv[n // 3, 0] = 0.37                                        # a constant row: scale zero
    kv = kv.to(torch.bfloat16)
    k, v = kv[:, :heads], kv[:, heads:]
    pages = n // page + 2
    cache = mt.KvCache.empty(pages, page, heads, dim)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n]
    before = [t.clone() for t in cache.tensors]
    mt.mt_kv_append(cache, k, v, slots)
    assert mt.mt_get_async_status() == (0, -1)
    at = (slots // page, slice(None), slots % page)
    for x, codes, params in ((k, *cache.tensors[:2]), (v, *cache.tensors[2:])):
        want, scale, bias = quantise(x.float().cpu().numpy())
        got = codes[at].cpu().numpy()
        assert np.array_equal(np.stack([got & 15, got >> 4], -1).reshape(want.shape), want)
        assert np.array_equal(to_np(params[at]), np.stack([scale, bias], -1).astype(np.float64))
        value = cache_values(codes[at], params[at])
        # half a step, and what the scale's rounding takes off the far end
        assert (np.abs(value - to_np(x)) <= (0.5 + 15 * U) * scale[..., None] * (1 + 1e-6) + 1e-30).all()
    rest = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    rest[slots] = False
    rest = torch.nonzero(rest)[:, 0]
    for t, b in zip(cache.tensors, before):                      # no other slot is touched
        assert torch.equal(t[rest // page, :, rest % page], b[rest // page, :, rest % page])
    out = [torch.empty((n, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    mt.mt_kv_read(cache, slots, *out)
    for o, codes, params in ((out[0], *cache.tensors[:2]), (out[1], *cache.tensors[2:])):
        value = cache_values(codes[at], params[at])
        size = np.abs(value) + np.abs(to_np(params[at])[..., 1:])
        assert (np.abs(to_np(o) - value) <= U * np.abs(value) + 4 * F * size).all()


def test_append_strides_and_padding_slots():
    g = gen(1)
    base = torch.randn((2, 7, 3, 72), generator=g, device="cuda").to(torch.bfloat16)
    k = base[0, :, :, :64]
    v = base[1].transpose(0, 1)[:, :, :64].transpose(0, 1)[:, :3]
    cache = mt.KvCache.empty(2, 16, 3, 64)
    slots = torch.tensor([5, -1, 31, 0, 32, 7, -2], device="cuda")        # -1: left out; 32 and -2: outside
    mt.mt_kv_append(cache, k, v, slots)
    assert mt.mt_get_async_status() == (1, 4)
    out = [torch.empty((7, 3, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    mt.mt_kv_read(cache, slots, *out)
    assert mt.mt_get_async_status() == (1, 4)
    for o, x in zip(out, (k, v)):
        for i in (0, 2, 3, 5):
            code, scale, bias = quantise(x[i].float().cpu().numpy())
            want = torch.from_numpy(code.astype(np.float32) * scale[:, None] + bias[:, None]).to(torch.bfloat16)
            assert torch.equal(o[i].cpu(), want)
        assert (o[1] == 0).all() and torch.isnan(o[4]).all() and torch.isnan(o[6]).all()
    written = sum(int((t != 0).any(-1).sum()) for t in cache.tensors[1::2])
    assert written == 4 * 3 * 2


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_rows_that_are_not_finite_read_back_as_nan(bad):
    g = gen(2)
    k = torch.randn((4, 2, 64), generator=g, device="cuda").to(torch.bfloat16)
    k[1, 1, 63] = bad
    cache = mt.KvCache.empty(1, 16, 2, 64)
    slots = torch.arange(4, device="cuda")
    mt.mt_kv_append(cache, k, k, slots)
    out = [torch.empty_like(k) for _ in range(2)]
    mt.mt_kv_read(cache, slots, *out)
    for o in out:
        assert torch.isnan(o[1, 1]).all() and int(torch.isnan(o).sum()) == 64


def test_rows_of_extreme_values():
    gen()
    k = torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    k[0, 0, 0] = 1e-40                                           # a spread whose fifteenth part is no bf16 number but zero or one step
    k[1, 0, :32] = 1e38
    k[1, 0, 32:] = -1e38
    k[2, 0, 0], k[2, 0, 1] = 3.3e38, -3.3e38                     # the spread passes fp32
    cache = mt.KvCache.empty(1, 16, 1, 64)
    slots = torch.arange(3, device="cuda")
    out = [torch.empty_like(k) for _ in range(2)]
    mt.mt_kv_append(cache, k, k, slots)
    mt.mt_kv_read(cache, slots, *out)
    assert (out[0][0].abs() <= 2e-40).all()
    assert (out[0][1].float() - k[1].float()).abs().max() <= 2e38 * 2 * U
    assert torch.isnan(out[0][2]).all()


def decode(cache, q, tables, lengths, scale=None, stream=None):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    mt.mt_kv_attention(cache, q, torch.tensor(tables, dtype=torch.int32, device="cuda").reshape(len(lengths), -1),
                       torch.tensor(lengths, dtype=torch.int32, device="cuda"), out, scale=scale, stream=stream)
    return out


def check_decode(cache, q, tables, lengths, scale=None):
    out = decode(cache, q, tables, lengths, scale)
    assert mt.mt_get_async_status() == (0, -1)
    o, a = decode_reference(cache, q, tables, lengths, q.shape[2] ** -0.5 if scale is None else scale)
    err = np.abs(to_np(out) - o)
    assert (err <= attention_bound(o, a)).all(), float(np.max(err / attention_bound(o, a)))
    return out


def make(lengths, page, heads, group, dim, seed=0, extra=0):
    g = gen(seed)
    per = [-(-n // page) for n in lengths]
    width = max(1, max(per)) + extra
    pages = sum(per) + 3
    cache = random_cache(pages, page, heads, dim, g)
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    tables, k = [], 0
    for p in per:
        tables.append(order[k:k + p] + [-5] * (width - p))       # what lies past the last page is not read
        k += p
    q = torch.randn((len(lengths), heads * group, dim), generator=g, device="cuda").to(torch.bfloat16)
    return cache, q, tables, list(lengths)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dim", [64, 128])
def test_decode_lengths(page, dim):
    check_decode(*make([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1030], page, 2, 4, dim, seed=page))


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 9, 12, 16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [1, 3])
def test_decode_head_groups(group, dim, heads):
    check_decode(*make([77, 0, 300], 32, heads, group, dim, seed=group, extra=2))


@pytest.mark.parametrize("lengths", [[1], [5000], [0], [0, 0, 0], [20000, 3], [1] * 300, [40] * 1100])
def test_decode_batches(lengths):
    check_decode(*make(lengths, 64, 1, 4, 64, seed=1))


def test_decode_long_and_many_heads():
    check_decode(*make([9000, 100, 4097], 128, 8, 4, 128, seed=2))


def test_decode_scales_and_strides():
    cache, q, tables, lengths = make([200, 31], 16, 2, 3, 128, seed=3)
    check_decode(cache, q, tables, lengths, scale=0.0)
    check_decode(cache, q, tables, lengths, scale=-0.05)
    wide = torch.zeros((2, 8, 136), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:7, :128] = q
    got = check_decode(cache, wide[:, 1:7, :128], tables, lengths)
    assert torch.equal(got, decode(cache, q, tables, lengths))


def test_decode_ignores_what_lies_past_the_length():
    cache, q, tables, lengths = make([100, 20], 64, 2, 4, 128, seed=4)
    want = check_decode(cache, q, tables, lengths)
    for s, n in enumerate(lengths):
        page = tables[s][n // 64]
        for codes, params in (cache.tensors[:2], cache.tensors[2:]):
            codes[page, :, n % 64:] = 255
            params[page, :, n % 64:] = float("nan")
    assert torch.equal(decode(cache, q, tables, lengths), want)
    for params in cache.tensors[1::2]:
        params[tables[0][1], :, 36:] = float("inf")
    assert torch.equal(decode(cache, q, tables, lengths), want)


def test_decode_of_a_nan_row_is_nan_for_its_sequence_alone():
    cache, q, tables, lengths = make([100, 20], 64, 2, 4, 128, seed=4)
    want = check_decode(cache, q, tables, lengths)
    cache.tensors[3][tables[0][0], 1, 3] = float("nan")           # one value row of head 1
    got = decode(cache, q, tables, lengths)
    assert torch.isnan(got[0, 4:]).all()
    assert torch.equal(got[0, :4], want[0, :4]) and torch.equal(got[1], want[1])


def test_decode_far_scores():
    """One token far above the rest, first or last: the others' weight underflows, no overflow on the way."""
    for at in (0, 299):
        cache, q, tables, lengths = make([300], 64, 1, 2, 64, seed=5)
        page = tables[0][at // 64]
        cache.tensors[1][page, 0, at % 64] = torch.tensor([0.0, 40.0], dtype=torch.bfloat16, device="cuda")
        q = q.abs()
        check_decode(cache, q, tables, lengths, scale=1.0)


def test_decode_bad_sequences():
    cache, q, tables, lengths = make([100, 40, 64, 30], 64, 2, 2, 64, seed=6)
    want = check_decode(cache, q, tables, lengths)
    bad = [row[:] for row in tables]
    bad[1][0] = cache.tensors[0].shape[0]                         # a page outside the cache
    got = decode(cache, q, bad, lengths)
    assert mt.mt_get_async_status() == (1, 1)
    assert torch.isnan(got[1]).all() and torch.equal(got[[0, 2, 3]], want[[0, 2, 3]])
    for n in (-1, 129, 2 ** 31 - 1):                              # lengths that the table does not hold
        got = decode(cache, q, tables, lengths[:2] + [n, 30])
        assert mt.mt_get_async_status() == (1, 2)
        assert torch.isnan(got[2]).all() and torch.equal(got[[0, 1, 3]], want[[0, 1, 3]])
    got = decode(cache, q, tables, lengths)
    assert mt.mt_get_async_status() == (0, -1) and torch.equal(got, want)


def test_decode_is_repeatable_and_streams_do_not_mix():
    """Two streams at once, different sizes, many times: each call's outputs are its own and the same every time."""
    a, b = make([3000, 2, 700], 64, 4, 4, 128, seed=7), make([900] * 9, 32, 2, 8, 64, seed=8)
    want = [check_decode(*a), check_decode(*b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    torch.cuda.synchronize()
    args = [(c, q, torch.tensor(t, dtype=torch.int32, device="cuda"), torch.tensor(n, dtype=torch.int32, device="cuda"))
            for c, q, t, n in (a, b)]
    results = [[torch.empty_like(w) for _ in range(20)] for w in want]
    torch.cuda.synchronize()
    for i in range(20):
        for j in (0, 1):
            mt.mt_kv_attention(*args[j], results[j][i], stream=streams[j])
    torch.cuda.synchronize()
    for w, rs in zip(want, results):
        assert all(torch.equal(w, r) for r in rs)


def test_decode_in_a_graph():
    cache, q, tables, lengths = make([300, 5], 64, 2, 4, 128, seed=9)
    want = check_decode(cache, q, tables, lengths)
    d_tables = torch.tensor(tables, dtype=torch.int32, device="cuda")
    d_len = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mt.mt_kv_attention(cache, q, d_tables, d_len, out)         # this stream's scratch exists before the capture
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        mt.mt_kv_attention(cache, q, d_tables, d_len, out)
    for n in ([300, 5], [17, 0]):
        d_len.copy_(torch.tensor(n, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, decode(cache, q, tables, n))


def test_offsets_beyond_two_gigabytes():
    """Pages whose byte offset passes 32 bits."""
    g = gen(10)
    heads, page, dim = 8, 256, 128
    pages = (5 << 30) // (heads * page * dim // 2)
    cache = mt.KvCache.empty(pages, page, heads, dim)
    k = torch.randn((300, heads, dim), generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn((300, heads, dim), generator=g, device="cuda").to(torch.bfloat16)
    tables = [[pages - 1, pages - 9]]
    slots = torch.tensor([tables[0][i // page] * page + i % page for i in range(300)], device="cuda")
    mt.mt_kv_append(cache, k, v, slots)
    q = torch.randn((1, 8, dim), generator=g, device="cuda").to(torch.bfloat16)
    check_decode(cache, q, tables, [300])
    out = [torch.empty_like(k) for _ in range(2)]
    mt.mt_kv_read(cache, slots, *out)
    assert (out[0].float() - k.float()).abs().max() < 0.5 and (out[1].float() - v.float()).abs().max() < 0.5


def test_refusals():
    cache, q, tables, lengths = make([20, 3], 16, 2, 2, 64)
    t, n = torch.tensor(tables, dtype=torch.int32, device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    f = mt.mt_kv_attention
    assert code_of(f, cache, q.float(), t, n, out) == 1
    assert code_of(f, cache, q, t.long(), n, out) == 1
    assert code_of(f, cache, q, t, n[:1], out) == 1
    assert code_of(f, cache, q[:, :3], t, n, out[:, :3].contiguous()) == 4
    big = torch.zeros((2, 34, 64), dtype=torch.bfloat16, device="cuda")
    assert code_of(f, cache, big, t, n, torch.empty_like(big)) == 4               # 17 heads a group
    odd = torch.zeros((2, 4, 65), dtype=torch.bfloat16, device="cuda")[:, :, :64]
    assert code_of(f, cache, odd, t, n, out) == 4
    f(cache, q[:0], t[:0], n[:0], out[:0])
    for page, dim, code in ((24, 64, 4), (8, 64, 4), (512, 64, 4), (16, 96, 4)):
        c = mt.KvCache.empty(2, page, 2, dim)
        x = torch.zeros((2, 2, dim), dtype=torch.bfloat16, device="cuda")
        s = torch.zeros(2, dtype=torch.int64, device="cuda")
        assert code_of(mt.mt_kv_append, c, x, x, s) == code
        assert code_of(mt.mt_kv_read, c, s, x, x.clone()) == code
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    s = torch.zeros(2, dtype=torch.int64, device="cuda")
    assert code_of(mt.mt_kv_append, cache, x, x, s.int()) == 1
    assert code_of(mt.mt_kv_append, cache, x, x[:1], s) == 1
    assert code_of(mt.mt_kv_append, cache, x.float(), x, s) == 1
    assert code_of(mt.mt_kv_read, cache, s, x[:1], x) == 1
    mt.mt_kv_append(cache, x[:0], x[:0], s[:0])
    mt.mt_kv_read(cache, s[:0], x[:0], x[:0])
    assert mt.mt_get_async_status() == (0, -1)
