"""Attention over a 4-bit cache where the few-row kernel runs on the plan's side
stream beside the tiles: units of 33-64 rows (D = 64), and key groups.  The call
ends with the wait for that stream (nothing is merged), so the mark that its plan
is in use stands behind the join; and the fork and join are captured in a graph."""
import numpy as np
import pytest

import workloads as W
from paper_2606_12688_amd import attn, cache
from tests.helpers import plan_for
from tests.kv4_helpers import DEV, compare4, queries, random_pools, reference, run_kv4

pytestmark = pytest.mark.gpu
# heads, head_dim, query rows, keys, and the keys of another batch of the same kind
KINDS = {"wide_units": (4, 4, 64, [40, 200, 50, 150, 36], [400, 200, 333, 150, 90], [390, 200, 320, 150, 80]),
         "key_groups_d64": (4, 2, 64, [900, 1, 1], [900, 300, 77], [900, 200, 99]),
         "key_groups_d128": (4, 2, 128, [900, 1, 1], [900, 300, 77], [900, 200, 99])}


def _batch(kind, other=False):
    hq, hkv, d, q, kv, kv_other = KINDS[kind]
    kv = kv_other if other else kv
    b = W.custom(kind, hq, hkv, d, q, kv, [[(0, n, W.SEG_CAUSAL, 0)] for n in kv], [0] * len(q), seed=d)
    pl = plan_for(b, attn.FLAG_NO_SPLIT | attn.FLAG_HOST_ONLY)
    tiles, few, merged = (pl.items(k) for k in (0, 1, 3))
    wgs, small = len(pl.tile_order()), pl.stats()["device_bytes"] <= 64 << 10
    pl.destroy()
    # tiles and few-row items, and what keeps the latter out of the tiles' launch
    assert len(tiles) and len(few) and not len(merged) and small
    if kind == "wide_units":
        assert few[:, 3].max() > 32
    else:
        assert wgs <= 256 and (tiles[:, 5] - tiles[:, 4]).max() >= 640
    return b, few


def _state(b, seed=5):
    import torch

    pools = random_pools(b, seed, poison=False)
    return queries(b, seed + 1), pools, [torch.from_numpy(x).to(DEV) for x in pools], \
        torch.from_numpy(np.ascontiguousarray(b.block_table)).to(DEV)


@pytest.mark.parametrize("kind", list(KINDS))
def test_next_plan_waits_for_both_streams(kind):
    import torch

    b, few = _batch(kind)
    other, few_other = _batch(kind, other=True)
    assert not np.array_equal(few, few_other)  # the list that the side stream's kernel reads
    q, pools, pages, bt = _state(b)
    want = run_kv4(b, q, *pages, attn.FLAG_NO_SPLIT)
    compare4(b, *want, reference(b, q, *pools), kind)
    upload = torch.cuda.Stream()
    pl = plan_for(b, attn.FLAG_NO_SPLIT)
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)  # holds the stream up, some 10 ms
    cache.kv4_fwd(pl, q, *pages, bt, out, lse)
    pl.destroy()
    nxt = plan_for(other, attn.FLAG_NO_SPLIT, upload)  # takes the buffer of `pl`
    torch.cuda.synchronize()
    nxt.destroy()
    assert torch.equal(out.view(torch.int16), want[0].view(torch.int16))
    assert torch.equal(lse.view(torch.int32), want[1].view(torch.int32))


@pytest.mark.parametrize("kind", list(KINDS))
def test_serial_and_forked_are_equal(kind):
    import torch

    b, _ = _batch(kind)
    q, _, pages, _ = _state(b)
    (o1, l1), (o2, l2) = (run_kv4(b, q, *pages, attn.FLAG_NO_SPLIT | f) for f in (0, attn.FLAG_SERIAL))
    assert torch.equal(o1.view(torch.int16), o2.view(torch.int16)) and torch.equal(l1, l2)


@pytest.mark.parametrize("kind", list(KINDS))
def test_fork_and_join_captured_in_a_graph(kind):
    import torch

    b, _ = _batch(kind)
    q, _, pages, bt = _state(b)
    want = run_kv4(b, q, *pages, attn.FLAG_NO_SPLIT)
    pl = plan_for(b, attn.FLAG_NO_SPLIT)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    after = torch.empty_like(q)
    cache.kv4_fwd(pl, q, *pages, bt, out, lse)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            cache.kv4_fwd(pl, q, *pages, bt, out, lse)
            after.copy_(out)  # behind the join
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        after.fill_(float("nan"))
        graph.replay()
        run_kv4(b, q, *pages, attn.FLAG_NO_SPLIT)  # eager work between the replays
        torch.cuda.synchronize()
        for got, ref in ((out, want[0]), (after, want[0]), (lse, want[1])):
            assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8)), f"replay {rep}"
    assert attn.check(pl) == 0
    del graph
    pl.destroy()
