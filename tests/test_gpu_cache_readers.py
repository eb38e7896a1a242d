"""Blocks that are displaced while a batch in flight reads them: the copies over them wait, so every batch's outputs are those of the all-resident context."""
import numpy as np
import pytest
import torch

from paper_1901_06887_b200 import binding as mt, harness, synth

from gpu_util import fresh
from test_gpu_cache import BLOCK, WIDTHS, block_bytes, host_run

pytestmark = pytest.mark.gpu


def two_halves(n=6000):
    """Six tenants, and batches that ask for the first three or the last three of them."""
    models = [synth.make_mlp(12, t, WIDTHS) for t in range(6)]
    rng = np.random.default_rng(8)
    batches = []
    for b in range(2):
        ids = (3 * b + rng.integers(0, 3, n)).astype(np.int32)
        batches.append((ids, synth.f32_to_bf16_bits(rng.standard_normal((n, WIDTHS[0])).astype(np.float32))))
    fresh()
    harness.register_models(models)
    return models, batches, [harness.run_batch(ids, x, 64) for ids, x in batches]


def test_a_prefetch_between_a_batch_and_the_one_that_displaces_its_tenants():
    models, batches, want = two_halves()
    fresh()
    mt.mt_set_cache_bytes(int(3.2 * BLOCK))
    harness.register_models(models)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(4):
        outs, keep = [], []
        for k in range(10):
            if k:
                mt.mt_prefetch([3 * ((k - 1) & 1) + t for t in range(3)], streams[(k - 1) % 2])      # what the batch before reads
            o, bufs = host_run(*batches[k & 1], 64, streams[k % 2], asynchronous=True)
            outs.append(o)
            keep.append(bufs)
        torch.cuda.synchronize()
        assert mt.mt_get_async_status() == (0, -1)
        for k, o in enumerate(outs):
            assert np.array_equal(o.numpy(), want[k & 1]), (rep, k)
    mt.mt_shutdown()


def test_displaced_by_a_call_that_finds_no_room():
    """A prefetch displaces two tenants that a batch in flight reads and then finds no room; the next batch's tenants take the bytes and displace nobody."""
    big = (256, 1024, 768, 64)
    assert 2.2 * BLOCK < block_bytes(big) < 3.0 * BLOCK
    models = [synth.make_mlp(12, t, WIDTHS) for t in range(5)] + [synth.make_mlp(12, 5, big)]
    rng = np.random.default_rng(9)
    n, sets, batches = 6000, [(0, 1, 2), (0, 3, 4)], []
    for live in sets:
        ids = np.array(live)[rng.integers(0, 3, n)].astype(np.int32)
        batches.append((ids, synth.f32_to_bf16_bits(rng.standard_normal((n, WIDTHS[0])).astype(np.float32))))
    fresh()
    harness.register_models(models)
    want = [harness.run_batch(ids, x, 64) for ids, x in batches]
    fresh()
    mt.mt_set_cache_bytes(int(3.2 * BLOCK))
    harness.register_models(models)
    stream = torch.cuda.Stream()
    for rep in range(12):
        outs, keep = [], []
        for k in range(2):
            o, bufs = host_run(*batches[k], 64, stream, asynchronous=True)
            outs.append(o)
            keep.append(bufs)
            with pytest.raises(mt.MtError) as e:
                mt.mt_prefetch([0, 5], stream)
            assert e.value.code == 5
        torch.cuda.synchronize()
        assert mt.mt_get_async_status() == (0, -1)
        for k, o in enumerate(outs):
            assert np.array_equal(o.numpy(), want[k]), (rep, k)
    mt.mt_shutdown()
