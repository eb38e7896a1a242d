"""What is written over an evicted block waits for the batch that may have read it last (host code of the library; no GPU)."""
import pytest

from paper_1901_06887_b200 import binding as mt

KB = 1024


class Worker:
    """The steps of a worker on the cache: blocks of 4 KB, room for two."""

    def __init__(self):
        self.sim, self.tick = mt.mt_cache_sim_create(8 * KB), 0

    def prepare(self, *ids, size=4 * KB):
        """A batch's (or a prefetch's) blocks are made resident.  Returns what each was and whom it displaced."""
        self.tick += 1
        out = []
        for i in ids:
            r, _, evicted = mt.mt_cache_sim_access(self.sim, i, size, self.tick)
            out.append((r, evicted))
            if r < 0:
                break
            mt.mt_cache_sim_read(self.sim, i)
        return out

    def batch(self, *ids):
        out = self.prepare(*ids)
        mt.mt_cache_sim_batch(self.sim)
        return out

    def wait(self):
        return mt.mt_cache_sim_wait(self.sim)


@pytest.fixture
def w():
    worker = Worker()
    yield worker
    mt.mt_cache_sim_destroy(worker.sim)


def test_a_load_waits_for_the_last_reader_of_what_it_displaces(w):
    w.batch(0, 1)                                    # batch 1
    assert w.wait() == 0                             # nothing was displaced
    w.batch(1)                                       # batch 2
    assert w.prepare(2) == [(1, [0])] and w.wait() == 1
    assert w.prepare(3) == [(1, [1])] and w.wait() == 2


def test_a_block_that_was_made_ready_for_a_batch_that_never_came(w):
    w.batch(0, 1)                                    # batch 1 reads block 0
    w.prepare(0)                                     # a prefetch: no batch follows
    w.prepare(1)
    assert w.prepare(2) == [(1, [0])]
    assert w.wait() == 1                             # not batch 2, which does not exist


def test_a_block_that_was_never_read(w):
    w.prepare(0, 1)
    assert w.prepare(2) == [(1, [0])] and w.wait() == 0
    w.batch(2)                                       # batch 1
    assert w.prepare(3) == [(1, [1])] and w.wait() == 1     # (block 1 was made ready for the batch that came next: it may have read it)


def test_nothing_to_wait_for_once_all_have_finished(w):
    w.batch(0, 1)
    mt.mt_cache_sim_batch(w.sim, finished=True)
    assert w.prepare(2) == [(1, [0])] and w.wait() == 0
    w.batch(2)                                       # batch 2
    w.batch(1)                                       # batch 3
    assert w.prepare(4) == [(1, [2])] and w.wait() == 2


def test_what_is_not_resident_is_not_read(w):
    with pytest.raises(mt.MtError) as e:
        mt.mt_cache_sim_read(w.sim, 7)
    assert e.value.code == 1
