"""Arguments that token sampling, rotary positions, the book of a cache's pages and cross attention refuse on the host, tensor by tensor."""
import pytest
import torch

from lm_util import code_of, init, random_cache
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def z(*shape, dtype=F32, device="cuda"):
    return torch.zeros(shape, dtype=dtype, device=device)


def test_sample():
    init()
    good = dict(logits=z(3, 10), uniform=z(3), ids=z(3, dtype=I32), logprobs=z(3), temperature=z(3) + 1, top_k=z(3, dtype=I32), top_p=z(3) + 1, min_p=z(3))
    assert code_of(mt.mt_token_sample, **good) == 0
    for name, bad in (("logits", z(3, 10, dtype=torch.float16)), ("logits", z(30)), ("logits", z(3, 10, device="cpu")), ("logits", z(3, 20)[:, ::2]),
                      ("uniform", z(4)), ("uniform", z(3, dtype=torch.float64)), ("uniform", z(3, 1)), ("uniform", z(6)[::2]), ("uniform", z(3, device="cpu")),
                      ("ids", z(3, dtype=torch.int64)), ("ids", z(2, dtype=I32)), ("logprobs", z(3, dtype=BF16)), ("temperature", z(1)),
                      ("top_k", z(3)), ("top_k", z(4, dtype=I32)), ("top_p", z(3, dtype=I32)), ("min_p", z(2))):
        assert code_of(mt.mt_token_sample, **{**good, name: bad}) == 1, name
    assert code_of(mt.mt_token_sample, **{**good, "logits": z(3, 0)}) == 1


def test_rotate():
    init()
    x, pos, f = z(4, 2, 64, dtype=BF16), z(4, 2, dtype=I32), z(32)
    assert code_of(mt.mt_rotate, x, pos, f, x, sections=[10, 22]) == 0
    for args, kw in (((z(4, 128, dtype=BF16), pos, f, x), {}), ((z(4, 2, 64, dtype=torch.float16), pos, f, x), {}), ((x, pos, f, z(4, 2, 64)), {}),
                     ((x, pos, f, z(4, 3, 64, dtype=BF16)), {}), ((x, z(4, 2), f, x), {}), ((x, z(5, 2, dtype=I32), f, x), {}), ((x, z(2, 4, dtype=I32).t(), f, x), {}),
                     ((x, pos, z(32, dtype=BF16), x), {}), ((x, pos, z(64)[::2], x), {}), ((x, pos, f, x), dict(sections=[32])), ((x, pos, f, x), dict(sections=[10, 10])),
                     ((x, pos, f, x), dict(sections=[40, -8])), ((x, pos, f, x), dict(sections=None)), ((x, pos, z(40), x), dict(sections=[20, 20])),
                     ((z(4, 2, 128, dtype=BF16)[..., ::2], pos, f, x), {}), ((x, pos, f, z(1, 2, 64, dtype=BF16).expand(4, 2, 64)), {}),
                     ((x.cpu(), pos, f, x), {}), ((x, z(4, 5, dtype=I32), f, x), dict(sections=[8, 8, 8, 4, 4]))):
        assert code_of(mt.mt_rotate, *args, **{"sections": [10, 22], **kw}) == 1
    assert code_of(mt.mt_rotate, x[..., :60], pos, z(16), z(4, 2, 60, dtype=BF16), sections=[8, 8]) == 4
    assert code_of(mt.mt_rotate, x, pos, z(12), x, sections=[6, 6]) == 4
    flat = z(4 * 2 * 64 + 8, dtype=BF16)
    assert code_of(mt.mt_rotate, flat[1:513].view(4, 2, 64), pos, f, x, sections=[10, 22]) == 1
    assert code_of(mt.mt_rotate, flat[:4 * 130].as_strided((3, 2, 64), (130, 64, 1)), pos[:3], f, x[:3], sections=[10, 22]) == 4


def test_cross():
    init()
    q, k, o, r = z(5, 4, 64, dtype=BF16), z(9, 2, 64, dtype=BF16), torch.tensor([0, 2, 5], dtype=I32, device="cuda"), torch.tensor([[0, 4], [4, 9]], dtype=I32, device="cuda")
    out = torch.empty_like(q)
    assert code_of(mt.mt_cross_attention, q, k, k, o, r, out) == 0
    for args in ((q[0], k, k, o, r, out), (q.float(), k, k, o, r, out), (q, k.float(), k, o, r, out), (q, k, k[:8], o, r, out), (q, z(9, 2, 128, dtype=BF16), k, o, r, out),
                 (q, k, k, o.long(), r, out), (q, k, k, o[:2], r, out), (q, k, k, o, r.view(4), out), (q, k, k, o, z(2, 3, dtype=I32), out), (q, k, k, o, r.t(), out),
                 (q, k, k, o, r, out[:4]), (q, k, k, o, r, out.float()), (q, k, k, o, r, z(5, 64, 4, dtype=BF16).transpose(1, 2)), (q, k.cpu(), k, o, r, out),
                 (z(5, 4, 128, dtype=BF16)[..., ::2], k, k, o, r, out)):
        assert code_of(mt.mt_cross_attention, *args) == 1
    assert code_of(mt.mt_cross_attention, z(5, 3, 64, dtype=BF16), k, k, o, r, z(5, 3, 64, dtype=BF16)) == 4
    assert code_of(mt.mt_cross_attention, q, k, k, o, r, out, float("nan")) == 1
    h = z(5, 4, 96, dtype=BF16)
    assert code_of(mt.mt_cross_attention, h, z(9, 2, 96, dtype=BF16), z(9, 2, 96, dtype=BF16), o, r, h.clone()) == 4


def test_pages():
    init()
    book = mt.KvPages.empty(8, 16, 3, 4)
    rows, c, s = z(2, dtype=I32), z(2, 3, dtype=I32), z(4, dtype=torch.int64)
    for bad in (z(2), z(2, dtype=torch.int64), z(2, 1, dtype=I32), z(4, dtype=I32)[::2], z(2, dtype=I32, device="cpu")):
        assert code_of(mt.mt_kv_release, book, bad) == 1
        assert code_of(mt.mt_kv_fork, book, bad, rows, c) == 1 and code_of(mt.mt_kv_fork, book, rows, bad, c) == 1
        assert code_of(mt.mt_kv_reserve, book, bad, rows, s) == 1 and code_of(mt.mt_kv_reserve, book, rows, bad, s) == 1
    for bad in (z(2, 2, dtype=I32), z(2, 3), z(3, 3, dtype=I32), z(6, dtype=I32), z(2, 3, dtype=I32, device="cpu")):
        assert code_of(mt.mt_kv_fork, book, rows, rows, bad) == 1
    copier = mt.KvCopier([random_cache(8, 16, 1, 64, torch.Generator(device="cuda").manual_seed(0))])
    for bad in (z(2, 2, dtype=I32), z(2, 3), z(6, dtype=I32), z(4, 3, dtype=I32)[::2]):
        assert code_of(mt.mt_kv_compact, book, bad) == 1 and code_of(mt.mt_kv_copy, copier, bad) == 1
    for bad in (z(4), z(2, 2, dtype=torch.int64), z(8, dtype=torch.int64)[::2], z(4, dtype=torch.int64, device="cpu")):
        assert code_of(mt.mt_kv_reserve, book, rows, rows, bad) == 1
    for args in ((z(8), book.tables, book.lengths), (book.refs, book.tables, z(4, dtype=I32)), (book.refs, z(12, dtype=I32), book.lengths),
                 (book.refs, z(4, 3, dtype=I32).t(), book.lengths), (book.refs.cpu(), book.tables, book.lengths)):
        assert code_of(mt.KvPages, *args, 16) == 1
    assert code_of(mt.mt_kv_release, mt.KvPages(book.refs, book.tables, book.lengths, 20), rows) == 4
    assert code_of(mt.mt_kv_release, mt.KvPages(z(9, dtype=I32)[1:], book.tables, book.lengths, 16), rows) == 1
    other = random_cache(9, 16, 1, 64, torch.Generator(device="cuda").manual_seed(0))
    assert code_of(mt.mt_kv_copy, mt.KvCopier(copier.caches + [other]), c) == 1
    assert mt.mt_get_async_status()[0] in (0, 1)


def test_without_a_context():
    mt.mt_shutdown()
    try:
        assert code_of(mt.mt_token_sample, z(3, 10), z(3), z(3, dtype=I32)) == 9
        assert code_of(mt.mt_rotate, z(4, 2, 64), z(4, dtype=I32), z(32), z(4, 2, 64)) == 9
        assert code_of(mt.mt_kv_copy, mt.KvCopier([]), z(2, 3, dtype=I32)) == 9
    finally:
        init()
