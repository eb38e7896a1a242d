"""The sticky status of calls in which places are left out for different reasons: the first place concerned, and its reason."""
import pytest

from paper_1901_06887_b200 import binding as mt
from test_gpu_kv_pages import Both

pytestmark = pytest.mark.gpu
INVALID, OOM = 1, 5


class First(Both):
    def same(self, errors):
        b, k = self.book, self.pages
        assert mt.mt_get_async_status() == (min(errors, key=lambda e: e[1]) if errors else (0, -1))
        assert k.lengths.tolist() == b.lengths and k.refs.tolist() == b.refs and k.tables.tolist() == b.tables


def test_no_page_before_a_bad_row():
    k = First(3, 16, 12, 4)
    k.reserve([0], [33])                                        # all pages
    assert k.reserve([1, 0, 2, 99], [0, 1, 1, 1]) == [(OOM, 2), (INVALID, 3)]
    assert k.fork([0, 0, -1], [4, 5, 6]) == [(OOM, 0), (OOM, 1), (INVALID, 2)]
    assert k.reserve([7, 7, 8], [1, 1, 1]) == [(OOM, 0), (INVALID, 1), (OOM, 2)]


def test_a_bad_row_before_no_page():
    k = First(3, 16, 12, 4)
    k.reserve([0], [33])
    assert k.reserve([99, 1], [1, 1]) == [(INVALID, 0), (OOM, 1)]
    assert k.fork([0, 0], [12, 5]) == [(INVALID, 0), (OOM, 1)]


def test_the_first_of_two_calls():
    k = First(3, 16, 12, 4)
    k.reserve([0], [33])
    one = First.reserve
    k.same = lambda errors: None                                # both calls first
    one(k, [1, 2], [0, 5])
    k.release([50])
    assert mt.mt_get_async_status() == (OOM, 1)
    assert mt.mt_get_async_status() == (0, -1)


@pytest.mark.parametrize("n", [40, 5000])
def test_large_indexes(n):
    k = First(2, 16, 2 * n, 4)
    k.reserve([0], [30])
    assert k.reserve(list(range(1, n)) + [-1], [0] * (n - 2) + [3, 1]) == [(OOM, n - 2), (INVALID, n - 1)]
