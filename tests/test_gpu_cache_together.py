"""The operators on paged caches as a serving loop uses them: random cascades,
plans from the async planner, two calls at once on two streams, pages freed
behind a sliding window, and steps that grow a cache token by token."""
import numpy as np
import pytest

import workloads as W
from oracle import block_tables, kv4_append, kv4_read, kv4_values
from paper_2606_12688_amd import attn, cache
from tests.helpers import host64, plan_for
from tests.kv4_helpers import DEV, compare4, queries, random_pools, reference, run_kv4
from tests.test_gpu_random_cascades import random_cascade

pytestmark = pytest.mark.gpu
FLAGS = (0, attn.FLAG_FORCE_SPLIT, attn.FLAG_NO_SPLIT)
C = W.SEG_CAUSAL


def _device(b, k4, v4, table=None):
    import torch

    return (torch.from_numpy(k4).to(DEV), torch.from_numpy(v4).to(DEV),
            torch.from_numpy(np.ascontiguousarray(b.block_table if table is None else table)).to(DEV))


@pytest.mark.parametrize("seed", range(16))
def test_random_cascades(seed):
    b = random_cascade(seed)
    k4, v4 = random_pools(b, seed, poison=False)
    q = queries(b, seed)
    ref = reference(b, q, k4, v4)
    for policy in (0, attn.FLAG_CASCADE_ALL):
        for flag in FLAGS:
            compare4(b, *run_kv4(b, q, k4, v4, flag | policy, cascade=True), ref, f"cascade {seed} {flag | policy}")


@pytest.mark.parametrize("name", ["mixed", "decode_bf16", "shared_prefix_decode_bf16"])
def test_plans_of_the_async_planner(name):
    import torch

    b = W.reduced(name)
    k4, v4 = random_pools(b, 5)
    q = queries(b, 6)
    cascade = b.prefix_groups is not None
    want = run_kv4(b, q, k4, v4, cascade=cascade)
    k4, v4, bt = _device(b, k4, v4)
    planner = attn.AsyncPlanner(depth=2)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        planner.submit(b.num_qo_heads, b.num_kv_heads, b.head_dim, b.dtype, b.seqs, b.masks, b.segments,
                       b.block_table.shape[1], b.num_pages, b.sm_scale, prefix_groups=b.prefix_groups)
        pl = planner.take(stream)
        out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
        stream.wait_stream(torch.cuda.current_stream())
        cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, attn.workspace(pl, DEV), stream)
        assert attn.check(pl, stream) == 0
        pl.destroy()
        assert torch.equal(out.view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse, want[1])
    planner.close()


def test_two_calls_at_once():
    """Plans and workspaces of their own, on two streams, among them a plan that forks."""
    import torch

    kv = [400, 200, 333, 150, 90]
    wide = W.custom("wide", 4, 4, 64, [40, 200, 50, 150, 36], kv, [[(0, n, C, 0)] for n in kv], [0] * 5, seed=1)
    jobs = []
    for b, cascade in ((W.reduced("mixed"), False), (W.reduced("shared_prefix_decode_bf16"), True), (wide, False)):
        k4, v4 = random_pools(b, 5)
        q = queries(b, 6)
        want = run_kv4(b, q, k4, v4, cascade=cascade)
        pl = plan_for(b, cascade=cascade)
        jobs.append((pl, q, *_device(b, k4, v4), want, attn.workspace(pl, DEV)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        outs = []
        for (pl, q, k4, v4, bt, want, ws), s in zip(jobs, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
                for _ in range(4):
                    cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, ws)
            outs.append((out, lse))
        torch.cuda.synchronize()
        for (out, lse), job in zip(outs, jobs):
            assert torch.equal(out.view(torch.int16), job[5][0].view(torch.int16)) and torch.equal(lse, job[5][1])
    for job in jobs:
        assert attn.check(job[0]) == 0
        job[0].destroy()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [1, 16, 100, 257])
def test_pages_freed_behind_a_window(d, window):
    """Entries of pages that no row sees any more may hold anything: they are neither read nor reported."""
    import torch

    q_lens, kv = [1, 16, 200, 130, 3], [700, 500, 900, 130, 333]
    b = W.custom("freed", 8, 2, d, q_lens, kv, [[(0, n, C, 0)] for n in kv], [window] * 5, seed=d)
    k4, v4 = random_pools(b, window)
    q = queries(b, window)
    ref = reference(b, q, k4, v4)
    table = b.block_table.copy()
    for r, (n, total, _) in enumerate(b.seqs.tolist()):
        table[r, :max(0, total - n - window + 1) // 16] = (-1, b.num_pages, 2 ** 31 - 1)[r % 3]
    k4, v4, bt = _device(b, k4, v4, table)
    for flag in FLAGS:
        pl = plan_for(b, flag)
        out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
        cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, attn.workspace(pl, DEV))
        assert attn.check(pl) == 0
        pl.destroy()
        compare4(b, out, lse, ref, f"window {window} d{d} flags {flag}")


@pytest.mark.parametrize("d,hq,hkv", [(64, 6, 3), (128, 8, 2)])
def test_a_cache_that_grows_step_by_step(d, hq, hkv):
    """Prompts, then decode steps and a chunk: each step takes its pages from the
    front of one free list, stores its rows and attends over all that came before."""
    import torch

    n, width, pool = 3, 20, 70
    rng = np.random.default_rng(d)
    free, at = rng.permutation(pool).astype(np.int32), 0
    table = np.full((n, width), -1, np.int32)
    k4, v4 = (np.zeros((pool, hkv, cache.record_bytes(d)), np.uint8) for _ in range(2))
    dk, dv, bt = (torch.from_numpy(x).to(DEV) for x in (k4.copy(), v4.copy(), table.copy()))
    have = np.zeros(n, int)
    for step, new in enumerate([(30, 0, 150), (1, 17, 1), (1, 1, 1), (2, 1, 0), (1, 40, 15), (1, 1, 1)]):
        have += new
        starts = np.cumsum([0, *new[:-1]])
        b = W.custom("grow", hq, hkv, d, list(new), have.tolist(), [[(0, int(x), C, 0)] if x else [] for x in have],
                     [0] * n, seed=1)
        b.seqs[:, 2] = starts
        table, slots, taken = block_tables(b.seqs, free[at:], table, pool)
        b.block_table, b.num_pages = table, pool
        pl = plan_for(b)
        got = torch.full((b.total_q,), -9, dtype=torch.int64, device=DEV)
        cache.block_tables(pl, torch.from_numpy(free[at:].copy()).to(DEV), bt, got)
        assert cache.block_tables_pages(pl) == taken
        at += taken
        kn, vn = (torch.randn((b.total_q, hkv, d), device=DEV).bfloat16() for _ in range(2))
        q = queries(b, step)
        out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
        cache.kv4_append(pl, kn, vn, bt, dk, dv)
        cache.kv4_fwd(pl, q, dk, dv, bt, out, lse, attn.workspace(pl, DEV))
        assert attn.check(pl) == 0
        pl.destroy()
        assert np.array_equal(bt.cpu().numpy(), table) and got.tolist() == [slots.get(i, -9) for i in range(b.total_q)]
        k4, v4 = kv4_append(b, host64(kn), host64(vn), k4, v4)
        assert np.array_equal(dk.cpu().numpy(), k4) and np.array_equal(dv.cpu().numpy(), v4)
        compare4(b, out, lse, reference(b, q, k4, v4), f"step {step} d{d}")


@pytest.mark.parametrize("d", [64, 128])
def test_two_rows_for_one_slot_leave_finite_values_and_other_slots_alone(d):
    import torch

    b = W.custom("twice", 2, 2, d, [3, 3], [20, 20], [[(0, 20, C, 0)]] * 2, [0, 0], seed=1)
    b.block_table[1] = b.block_table[0]  # both requests' rows go to slots 1-3 of one page
    k4, v4 = random_pools(b, 1, poison=False)
    g = torch.Generator(DEV).manual_seed(d)
    kn, vn = ((torch.randn((6, 2, d), generator=g, device=DEV) * 2.0 ** 100).bfloat16() for _ in range(2))
    kn[3:], vn[3:] = kn[3:] * 2.0 ** -180, vn[3:] * 2.0 ** -180
    dk, dv, bt = _device(b, k4, v4)
    pl = plan_for(b)
    cache.kv4_append(pl, kn, vn, bt, dk, dv)
    assert attn.check(pl) == 0
    pl.destroy()
    page, slots = b.block_table[0, 1], [1, 2, 3]
    for which, got, old in (("k", dk, k4), ("v", dv, v4)):
        now, before = (kv4_read(which, x, d) for x in (got.cpu().numpy(), old))
        assert np.isfinite(kv4_values(*now)).all()
        for x, y in zip(now, before):
            x, y = x.copy(), y.copy()
            x[page, slots] = y[page, slots] = 0
            assert np.array_equal(x, y)
