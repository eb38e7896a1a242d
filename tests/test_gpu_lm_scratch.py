"""Scratch of mt_kv_attention: calls that may run at the same time never share it - streams by the dozen, the per-thread
default stream, graphs replayed away from the stream they were captured on."""
import ctypes
import threading

import pytest
import torch

from lm_util import init, random_cache
from paper_1901_06887_b200 import binding as mt

pytestmark = pytest.mark.gpu
PER_THREAD = 2                                                   # the handle of CUDA's per-thread default stream


class Job:
    """One call whose sequences are cut into parts (several warps share each), with its result when nothing else runs."""

    def __init__(self, seed, lengths=(3000, 2, 700), heads=4):
        init()
        g = torch.Generator(device="cuda").manual_seed(seed)
        per = [-(-n // 64) for n in lengths]
        self.cache = random_cache(sum(per), 64, heads, 128, g)
        ids, k = torch.randperm(sum(per), generator=g, device="cuda").int(), 0
        self.tables = torch.zeros((len(lengths), max(per)), dtype=torch.int32, device="cuda")
        for s, p in enumerate(per):
            self.tables[s, :p] = ids[k:k + p]
            k += p
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.q = torch.randn((len(lengths), 4 * heads, 128), generator=g, device="cuda").to(torch.bfloat16)
        self.want = self.out()
        self.call(self.want)
        torch.cuda.synchronize()

    def out(self):
        return torch.full_like(self.q, 7.0)

    def call(self, out, stream=None):
        mt.mt_kv_attention(self.cache, self.q, self.tables, self.lengths, out, stream=stream)


class Streams:
    """Streams of their own, not out of torch's pool of 32."""

    def __init__(self, n):
        self.handles = []
        for _ in range(n):
            h = ctypes.c_void_p()
            assert int(torch.cuda.cudart().cudaStreamCreate(ctypes.addressof(h))) == 0
            self.handles.append(h.value)

    def destroy(self):
        for h in self.handles:
            assert int(torch.cuda.cudart().cudaStreamDestroy(h)) == 0


def test_more_streams_than_blocks():
    job = Job(1)
    for _ in range(2):                                           # a second lot after the first has gone
        streams = Streams(80)
        outs = [job.out() for _ in range(240)]
        torch.cuda.synchronize()
        for i, o in enumerate(outs):
            job.call(o, streams.handles[i % 80])
        torch.cuda.synchronize()
        assert all(torch.equal(o, job.want) for o in outs)
        streams.destroy()


def test_streams_destroyed_with_work_pending():
    jobs = [Job(2), Job(3, (900,) * 9, 2)]
    outs = [(jobs[i % 2], jobs[i % 2].out()) for i in range(40)]
    torch.cuda.synchronize()
    for job, o in outs:                                          # the next stream may get the last one's handle
        s = Streams(1)
        job.call(o, s.handles[0])
        s.destroy()
    torch.cuda.synchronize()
    assert all(torch.equal(o, job.want) for job, o in outs)


def test_the_per_thread_default_stream():
    jobs = [Job(4 + i, (2000 + 100 * i, 50)) for i in range(4)]
    outs = [[job.out() for _ in range(50)] for job in jobs]
    torch.cuda.synchronize()
    errors, start = [], threading.Barrier(len(jobs))

    def work(i):
        try:
            start.wait()
            for o in outs[i]:
                jobs[i].call(o, PER_THREAD)
        except Exception as e:                                   # noqa: BLE001 (reported below)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for job, os in zip(jobs, outs):
        assert all(torch.equal(o, job.want) for o in os)


def capture(job, stream, out, times=1):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(times):
            job.call(out)
    return graph


def test_graphs_away_from_the_stream_they_were_captured_on():
    """Two graphs captured on one stream are replayed on two others while calls run on it; nothing was called there before."""
    jobs = [Job(10), Job(11, (900,) * 9, 2), Job(12, (5000,))]
    home, others = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)]
    outs = [jobs[0].out(), jobs[1].out()]
    graphs = [capture(jobs[i], home, outs[i], times=3) for i in range(2)]
    eager = [jobs[2].out() for _ in range(60)]
    for o in outs:
        o.fill_(7.0)
    torch.cuda.synchronize()
    for o in eager:
        for g, s in zip(graphs, others):
            with torch.cuda.stream(s):
                g.replay()
        jobs[2].call(o, home)
    torch.cuda.synchronize()
    assert all(torch.equal(o, j.want) for o, j in zip(outs, jobs))
    assert all(torch.equal(o, jobs[2].want) for o in eager)


def test_scratch_of_graphs_that_are_gone_is_used_again():
    job, out = Job(13), None
    stream = torch.cuda.Stream()
    free = []
    for _ in range(30):
        out = job.out()
        g = capture(job, stream, out)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, job.want)
        g.reset()
        del g
        free.append(torch.cuda.mem_get_info()[0])
    assert free[2] - free[-1] < 64 << 20                         # one block is some 20 MB
