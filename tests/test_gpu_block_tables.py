"""Block tables and slot maps built on the GPU against the oracle."""
import numpy as np
import pytest

import workloads as W
from oracle import block_tables
from paper_2606_12688_amd import attn, cache
from tests.helpers import plan_for
from tests.test_gpu_random_batches import random_batch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
C = W.SEG_CAUSAL


def _check(b, seed=0, bad=(), with_slots=True):
    import torch

    rng = np.random.default_rng(seed)
    pl = plan_for(b)
    need = cache.block_tables_pages(pl)
    free = (rng.permutation(max(need, 1) + 5) + 0).astype(np.int32) % b.num_pages
    for i, page in bad:
        free[i] = page
    table = np.full(b.block_table.shape, -5, dtype=np.int32)
    for r in range(b.num_seqs):  # the cached positions' pages are the caller's, everything else is noise
        held = (int(b.seqs[r, 1]) - int(b.seqs[r, 0]) + 15) // 16
        table[r, :held] = b.block_table[r, :held]
    want, slots, taken = block_tables(b.seqs, free, table, b.num_pages)
    assert taken == need
    bt = torch.from_numpy(table).to(DEV)
    got = torch.full((b.total_q,), -9, dtype=torch.int64, device=DEV)
    cache.block_tables(pl, torch.from_numpy(free).to(DEV), bt, got if with_slots else None)
    bits = attn.check(pl)
    pl.destroy()
    assert np.array_equal(bt.cpu().numpy(), want)
    assert got.tolist() == [slots.get(i, -9) if with_slots else -9 for i in range(b.total_q)]
    return bits


@pytest.mark.parametrize("name", ["tiny_causal_f32", "decode_bf16", "rollout_bf16", "stream_window_bf16", "mixed"])
def test_workloads(name):
    assert _check(W.reduced(name)) == 0


@pytest.mark.parametrize("seed", range(20))
def test_random_batches(seed):
    assert _check(random_batch(seed)[0], seed, with_slots=seed % 4 != 3) == 0


def test_many_requests_with_and_without_rows():
    rng = np.random.default_rng(0)
    kv = rng.integers(0, 70, 3000)
    q = np.minimum(rng.integers(0, 40, 3000), kv)
    segs = [[(0, int(n), C, 0)] if n else [] for n in kv]
    b = W.custom("many", 2, 1, 64, q.tolist(), kv.tolist(), segs, [0] * 3000, seed=1)
    b.seqs[:, 2] += np.arange(3000, dtype=np.int32)  # a gap behind every request
    assert _check(b) == 0


def test_pages_outside_the_pool_are_reported():
    b = W.custom("bad", 2, 1, 64, [40, 1, 17], [40, 33, 50], [[(0, n, C, 0)] for n in (40, 33, 50)], [0] * 3, seed=1)
    assert _check(b) == 0
    assert _check(b, bad=[(1, b.num_pages)]) == attn.DEVERR_PAGE_RANGE
    assert _check(b, bad=[(0, -1), (3, 2 ** 31 - 1)]) == attn.DEVERR_PAGE_RANGE
    b.block_table[1, 2] = -1  # the page of a cached position
    b.seqs[1] = [1, 34, 40]
    b.segments[1, 1] = 34
    assert _check(b) == attn.DEVERR_PAGE_RANGE
