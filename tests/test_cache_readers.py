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


def test_a_wait_is_owed_until_something_is_written(w):
    """A call displaces a block, then finds no room after all and writes nothing; the bytes go to a later call, which displaces nobody."""
    w.batch(0, 1)                                    # batch 1
    w.batch(1)                                       # batch 2
    assert w.prepare(1, 2, 3) == [(0, []), (1, [0]), (-1, [])]
    mt.mt_cache_sim_release(w.sim, 2)                # (its copy never began)
    assert w.prepare(4) == [(1, [])]
    assert w.wait() == 1
    assert w.wait() == 0                             # what has been waited for is not waited for again


def test_a_block_too_large_after_all(w):
    """Everything is displaced on the way, and still no room: no load of that call, but of the next ones."""
    w.batch(0)
    w.batch(1)                                       # batch 2
    assert w.prepare(1) == [(0, [])]
    w.tick += 1
    mt.mt_cache_sim_access(w.sim, 1, 4 * KB, w.tick)                                     # block 1 is of the call that is prepared
    assert mt.mt_cache_sim_access(w.sim, 2, 8 * KB, w.tick)[::2] == (-1, [0])
    assert w.prepare(3) == [(1, [])] and w.wait() == 1
    assert w.prepare(4)[0][1] == [1] and w.wait() == 2


def test_a_victim_that_comes_back_in_the_same_call(w):
    w.batch(0, 1)                                    # batch 1
    w.batch(1)                                       # batch 2: block 0 is the oldest
    assert w.prepare(2, 0) == [(1, [0]), (1, [1])]   # 0 goes, and comes back over 1
    assert w.wait() == 2
