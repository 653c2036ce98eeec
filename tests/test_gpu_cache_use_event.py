"""The calls on paged caches mark their plan's device buffer as in use until
their last kernel is done (as ``test_gpu_use_event.py`` checks for the 16-bit
ones): behind a stream that is held up, a plan is used and destroyed at once,
and another plan that takes its buffer is uploaded on another stream meanwhile."""
import numpy as np
import pytest

import workloads as W
from paper_2606_12688_amd import attn, cache
from tests.helpers import plan_for
from tests.kv4_helpers import DEV, compare4, queries, random_pools, reference, run_kv4
from tests.test_gpu_use_event import _other

pytestmark = pytest.mark.gpu
KINDS = {"tiles": ("text_latent_bf16", attn.FLAG_NO_SPLIT, False), "few": ("decode_bf16", attn.FLAG_NO_SPLIT, False),
         "merge": ("decode_bf16", attn.FLAG_FORCE_SPLIT, False), "cascade": ("shared_prefix_decode_bf16", 0, True),
         "forked": ("mixed", attn.FLAG_NO_SPLIT, False), "append": ("decode_bf16", attn.FLAG_NO_SPLIT, False),
         "tables": ("decode_bf16", attn.FLAG_NO_SPLIT, False)}


@pytest.mark.parametrize("kind", list(KINDS))
def test_next_plan_waits_for_the_last_kernel(kind):
    import torch

    name, flags, cascade = KINDS[kind]
    b, other = W.reduced(name), _other(name)
    k0, v0 = random_pools(b, 5, poison=False)
    q = queries(b, 6)
    ref = reference(b, q, k0, v0)
    new = [torch.randn((b.total_q, b.num_kv_heads, b.head_dim), device=DEV).bfloat16() for _ in range(2)]
    bt = torch.from_numpy(np.ascontiguousarray(b.block_table)).to(DEV)
    free = torch.zeros(4096, dtype=torch.int32, device=DEV)

    def call(pl, k4, v4, out, lse, table, slots, ws):
        if kind == "append":
            cache.kv4_append(pl, *new, bt, k4, v4)
        elif kind == "tables":
            cache.block_tables(pl, free, table, slots)
        else:
            cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, ws)

    def state(pl):
        return [torch.from_numpy(k0).to(DEV), torch.from_numpy(v0).to(DEV), torch.full_like(q, float("nan")),
                torch.full(q.shape[:2], float("nan"), device=DEV), bt.clone(),
                torch.full((b.total_q,), -1, dtype=torch.int64, device=DEV), attn.workspace(pl, DEV)]

    pl = plan_for(b, flags, cascade=cascade)
    want = state(pl)
    call(pl, *want)
    assert attn.check(pl) == 0
    got = state(pl)
    torch.cuda.synchronize()
    hold = torch.randn((4096, 4096), device=DEV)
    side = torch.cuda.Stream()
    for _ in range(8):  # holds the current stream up for milliseconds
        hold = hold @ hold * 1e-3
    call(pl, *got)
    pl.destroy()
    nxt = plan_for(other, flags, side, cascade=cascade)  # takes the buffer of `pl`
    torch.cuda.synchronize()
    nxt.destroy()
    for x, y in zip(got[:6], want[:6]):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    if kind not in ("append", "tables"):
        compare4(b, got[2], got[3], ref, kind)


def test_another_stream_than_the_current_one():
    import torch

    b = W.reduced("mixed")
    k0, v0 = random_pools(b, 5)
    q = queries(b, 6)
    want = run_kv4(b, q, k0, v0)
    side = torch.cuda.Stream()
    pl = plan_for(b, 0, side)
    k4, v4 = torch.from_numpy(k0).to(DEV), torch.from_numpy(v0).to(DEV)
    bt = torch.from_numpy(np.ascontiguousarray(b.block_table)).to(DEV)
    out, lse, ws = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV), attn.workspace(pl, DEV)
    side.wait_stream(torch.cuda.current_stream())
    cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, ws, side)
    side.synchronize()
    assert attn.check(pl, side) == 0
    pl.destroy()
    assert torch.equal(out.view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse, want[1])
