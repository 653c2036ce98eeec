"""The 4-bit cache on the GPU against the oracle: rows stored (bit for bit),
read back (exactly) and attended, on every kind of request and plan, at the
sizes and cache contents where it can go wrong."""
import numpy as np
import pytest

import workloads as W
from oracle import append_targets, kv4_append, kv4_read, kv4_round, kv4_values
from paper_2606_12688_amd import attn, cache
from tests.helpers import host64, plan_for
from tests.kv4_helpers import DEV, compare4, queries, random_pools, reference, run_kv4
from tests.test_gpu_edge_cases import _one_key_batch, _zero_query_batch
from tests.test_gpu_random_batches import random_batch

pytestmark = pytest.mark.gpu
FLAGS = {"auto": 0, "split": attn.FLAG_FORCE_SPLIT, "whole": attn.FLAG_NO_SPLIT}
NAMES = ["decode_bf16", "stream_window_bf16", "rollout_bf16", "cfg_labels_bf16", "text_latent_bf16",
         "shared_prefix_decode_bf16", "mixed"]
C, F = W.SEG_CAUSAL, W.SEG_FULL


def _table(b):
    import torch

    return torch.from_numpy(np.ascontiguousarray(b.block_table)).to(DEV)


def _rows(b, seed=3):
    """New rows with channels and rows of very different size."""
    import torch

    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    shape = (b.total_q, b.num_kv_heads, b.head_dim)
    gain = torch.exp2(8 * torch.randn((b.total_q, 1, 1), generator=g, device=DEV))
    return tuple((gain * torch.randn(shape, generator=g, device=DEV)).bfloat16() for _ in range(2))


def _append(b, kn, vn, k4, v4):
    import torch

    k4, v4 = torch.from_numpy(k4).to(DEV), torch.from_numpy(v4).to(DEV)
    pl = plan_for(b)
    cache.kv4_append(pl, kn, vn, _table(b), k4, v4)
    bits = attn.check(pl)
    pl.destroy()
    return k4.cpu().numpy(), v4.cpu().numpy(), bits


# ---- append ------------------------------------------------------------------------

def _check_append(b, kn, vn):
    k0, v0 = random_pools(b, 1, poison=False)
    k, v, bits = _append(b, kn, vn, k0, v0)
    assert bits == 0
    rk, rv = kv4_append(b, host64(kn), host64(vn), k0, v0)
    assert np.array_equal(k, rk), "K pool"
    assert np.array_equal(v, rv), "V pool"


@pytest.mark.parametrize("name", ["decode_bf16", "stream_window_bf16", "cfg_labels_bf16", "mixed"])
def test_append_bitwise(name):
    b = W.reduced(name)
    _check_append(b, *_rows(b))


@pytest.mark.parametrize("seed", [s for s in range(14) if random_batch(s)[0].dtype == "bf16"])
def test_append_random_batches_bitwise(seed):
    b, _ = random_batch(seed)
    _check_append(b, *_rows(b, seed))


@pytest.mark.parametrize("d", [64, 128])
def test_append_every_start_in_a_page(d):
    """New rows that start and end anywhere in a page, one token to three pages."""
    q = [1, 1, 2, 3, 4, 5, 15, 16, 17, 31, 33, 40]
    kv = [1, 16, 17, 3, 19, 23, 30, 32, 47, 31, 64, 51]
    b = W.custom("starts", 3, 3, d, q, kv, [[(0, n, C, 0)] for n in kv], [0] * len(q), seed=2)
    _check_append(b, *_rows(b))


@pytest.mark.parametrize("d", [64, 128])
def test_append_extremes(d):
    """Zero rows, subnormal and largest bf16 values, ties, infinities and NaN."""
    import torch

    b = W.custom("extremes", 2, 2, d, [20], [23], [[(0, 23, C, 0)]], [0], seed=2)
    kn, vn = _rows(b)
    vn[0] = 0
    vn[1] = -0.0
    kn[2] *= 0
    kn[2, :, 5] = 1e-40  # subnormal
    kn[3] = torch.finfo(torch.bfloat16).max
    kn[4] = -torch.finfo(torch.bfloat16).max
    vn[5, :, :16] = torch.tensor([7.0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, -7.0, -.25, -.75, -1.25, -1.75, -2.5,
                                  -3.5, -5.0], device=DEV).bfloat16()
    vn[5, :, 16:] = 0.1
    vn[6, :, 0] = 7.0625
    vn[7] = 2.0 ** -126
    _check_append(b, kn, vn)
    k0, v0 = random_pools(b, 1, poison=False)
    kn[8, 1, 3], kn[8, 0, d - 1], vn[9, 0, 40] = float("inf"), -float("inf"), float("nan")
    vn[10] = float("nan")
    k, v, bits = _append(b, kn, vn, k0, v0)
    assert bits == cache.DEVERR_NONFINITE
    rk, rv = kv4_append(b, host64(kn), host64(vn), k0, v0)
    assert np.array_equal(k, rk) and np.array_equal(v, rv)
    assert np.isfinite(kv4_values(*kv4_read("k", k, d))).all()


def test_append_outside_the_pool_is_skipped_and_reported():
    import torch

    b = W.reduced("decode_bf16")
    kn, vn = _rows(b)
    k0, v0 = random_pools(b, 1, poison=False)
    table = b.block_table.copy()
    last = int(b.seqs[0, 1]) - 1
    for bad in (b.num_pages, -1, 2 ** 31 - 1):
        table[0, last >> 4] = bad
        k4, v4 = torch.from_numpy(k0).to(DEV), torch.from_numpy(v0).to(DEV)
        pl = plan_for(b)
        cache.kv4_append(pl, kn, vn, torch.from_numpy(table).to(DEV), k4, v4)
        assert attn.check(pl) == attn.DEVERR_PAGE_RANGE
        pl.destroy()
        rk, rv = kv4_append(b, host64(kn), host64(vn), k0, v0)
        page, slot = b.block_table[0, last >> 4], last & 15
        for got, want, old, which in ((k4, rk, k0, "k"), (v4, rv, v0, "v")):
            for x, y, z in zip(*(kv4_read(which, p, b.head_dim) for p in (got.cpu().numpy(), want, old))):
                y[page, slot] = z[page, slot]
                assert np.array_equal(x, y)


# ---- unpack ------------------------------------------------------------------------

@pytest.mark.parametrize("hkv,d", [(1, 64), (4, 128), (3, 64), (5, 128)])
def test_unpack_is_exact(hkv, d):
    import torch

    rng = np.random.default_rng(hkv)
    pools = rng.integers(0, 256, (2, 37, hkv, 17 * d // 2)).astype(np.uint8)
    pools[..., 8 * d:] = rng.integers(2, 253, pools[..., 8 * d:].shape)
    ids = np.concatenate([rng.permutation(37), [3, 3, -1, 37, 2 ** 31 - 1, -2 ** 31, 0]]).astype(np.int32)
    k4, v4 = (torch.from_numpy(p).to(DEV) for p in pools)
    out = [torch.full((len(ids), 16, hkv, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache.kv4_unpack(k4, v4, torch.from_numpy(ids).to(DEV), *out)
    ok = (ids >= 0) & (ids < 37)
    for which, p, got in zip("kv", pools, out):
        want = kv4_values(*kv4_read(which, p, d))[np.where(ok, ids, 0)]
        want[~ok] = 0
        assert np.array_equal(host64(got), want)
    cache.kv4_unpack(k4, v4, torch.empty(0, dtype=torch.int32, device=DEV), out[0][:0], out[1][:0])


# ---- attention -----------------------------------------------------------------------

@pytest.mark.parametrize("flag", list(FLAGS))
@pytest.mark.parametrize("name", NAMES)
def test_workloads(name, flag):
    b = W.reduced(name)
    k4, v4 = random_pools(b, 5)
    q = queries(b, 6)
    compare4(b, *run_kv4(b, q, k4, v4, FLAGS[flag]), reference(b, q, k4, v4), f"{name}/{flag}")


@pytest.mark.parametrize("name,flag", [("shared_prefix_decode_bf16", 0), ("rollout_bf16", attn.FLAG_CASCADE_ALL),
                                       ("shared_prefix_decode_bf16", attn.FLAG_FORCE_SPLIT),
                                       ("queried_prefix_bf16", attn.FLAG_CASCADE_ALL)])
def test_cascades(name, flag):
    b = W.reduced(name)
    k4, v4 = random_pools(b, 5)
    q = queries(b, 6)
    compare4(b, *run_kv4(b, q, k4, v4, flag, cascade=True), reference(b, q, k4, v4), f"cascade {name}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (16, 8), (28, 4), (8, 1), (4, 2)])
def test_window_edges(d, hq, hkv):
    b = W.window_edges_bf16(d=d, hq=hq, hkv=hkv)
    k4, v4 = random_pools(b, 7)
    q = queries(b, 8)
    compare4(b, *run_kv4(b, q, k4, v4), reference(b, q, k4, v4), f"window d{d} {hq}/{hkv}")


@pytest.mark.parametrize("seed", [s for s in range(40) if random_batch(s)[0].dtype == "bf16"])
def test_random_batches(seed):
    b, flag = random_batch(seed)
    k4, v4 = random_pools(b, seed)
    q = queries(b, seed)
    compare4(b, *run_kv4(b, q, k4, v4, flag), reference(b, q, k4, v4), f"random {seed}")


@pytest.mark.parametrize("flag", list(FLAGS))
@pytest.mark.parametrize("shape", [(64, 8, 2, "bf16"), (128, 4, 4, "bf16"), (128, 28, 4, "bf16")],
                         ids=lambda s: f"d{s[0]}-{s[1]}x{s[2]}")
@pytest.mark.parametrize("build", [_zero_query_batch, _one_key_batch], ids=["zero_query", "one_key"])
def test_degenerate_requests(build, shape, flag):
    b = build(*shape)
    k4, v4 = random_pools(b, 9)
    q = queries(b, 9)
    ref = reference(b, q, k4, v4)
    out, lse = run_kv4(b, q, k4, v4, FLAGS[flag])
    compare4(b, out, lse, ref, f"{b.name}/{flag}")
    if build is _one_key_batch:  # one visible key: its values, which are bf16 values
        assert np.array_equal(host64(out), ref[0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257])
def test_every_length(d, kv):
    """One token, a few and all of `kv`, so that pages, steps and tiles end anywhere."""
    q = sorted({1, min(2, kv), min(7, kv), (kv + 1) // 2, kv})
    b = W.custom("lengths", 8, 2, d, q, [kv] * len(q), [[(0, kv, C, 0)]] * len(q), [0] * len(q), seed=kv)
    k4, v4 = random_pools(b, kv)
    qs = queries(b, kv)
    ref = reference(b, qs, k4, v4)
    for flag in FLAGS.values():
        compare4(b, *run_kv4(b, qs, k4, v4, flag), ref, f"d{d} kv {kv} flag {flag}")


@pytest.mark.parametrize("d", [64, 128])
def test_large_and_small_scores_and_values(d):
    """Scores in the thousands and values of 2^100 and 2^-105."""
    b = W.custom("large", 8, 2, d, [1, 20, 150], [700, 300, 150], [[(0, n, C, 0)] for n in (700, 300, 150)], [0] * 3,
                 seed=4)
    for seed, exps in ((1, (8, 9)), (2, (-105, -103)), (3, (100, 101))):
        k4, _ = random_pools(b, seed, exponents=(8, 9) if seed == 1 else (-4, 1))
        _, v4 = random_pools(b, seed, exponents=exps)
        q = queries(b, seed)
        out, lse = run_kv4(b, q, k4, v4)
        ro, rl, size = reference(b, q, k4, v4)
        # scores up to 5000 are off by 2^-17 * 12 * 256 * 4 < 2^-3 at most, most far less: compare
        # the rows whose leading keys are apart by more than that with the bar of a probability
        if seed == 1:
            assert np.isfinite(host64(out)).all() and np.abs(lse.cpu().numpy() - rl).max() <= 2.0 ** -3
        else:
            err = np.abs(host64(out) - ro) - (2.0 ** -8 * np.abs(ro) + (2.0 ** -8 + 2.0 ** -10) * size)
            assert err.max() <= 0


def test_rows_of_no_request_are_left_as_they_are():
    q_lens, kv_lens = [1, 40, 3], [50, 90, 200]
    b = W.custom("gaps", 8, 2, 128, q_lens, kv_lens, [[(0, n, C, 0)] for n in kv_lens], [0] * 3, seed=4)
    b.seqs[:, 2] = [60, 5, 50]  # packed rows in another order, with gaps
    k4, v4 = random_pools(b, 3)
    q = queries(b, 3)
    out, lse = run_kv4(b, q, k4, v4)
    rows = np.concatenate([np.arange(s, s + n) for n, _, s in b.seqs])
    gap = np.setdiff1d(np.arange(b.total_q), rows)
    assert len(gap) and np.isnan(host64(out)[gap]).all() and np.isnan(lse.cpu().numpy()[gap]).all()
    ref = [x[rows] for x in reference(b, q, k4, v4)]
    compare4(b, out[rows], lse[rows], ref, "gaps")


def test_pages_outside_the_pool_read_as_zeros_and_are_reported():
    import torch

    b = W.custom("bad", 8, 2, 128, [1, 40], [100, 90], [[(0, 100, C, 0)], [(0, 90, C, 0)]], [0, 0], seed=4)
    k4, v4 = random_pools(b, 3, poison=False)
    q = queries(b, 3)
    zk, zv = k4.copy(), v4.copy()
    table = b.block_table.copy()
    zk[table[0, 2]], zv[table[0, 2]], zk[table[1, 1]], zv[table[1, 1]] = 0, 0, 0, 0
    ref = reference(b, q, zk, zv)
    table[0, 2], table[1, 1] = -1, b.num_pages
    for flag in FLAGS.values():
        pl = plan_for(b, flag)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
        cache.kv4_fwd(pl, q, torch.from_numpy(k4).to(DEV), torch.from_numpy(v4).to(DEV),
                      torch.from_numpy(table).to(DEV), out, lse, attn.workspace(pl, DEV))
        assert attn.check(pl) == attn.DEVERR_PAGE_RANGE
        pl.destroy()
        compare4(b, out, lse, ref, f"bad pages, flag {flag}")


@pytest.mark.parametrize("d,hkv,flag", [(128, 4, 0), (128, 4, attn.FLAG_FORCE_SPLIT), (64, 8, 0)])
def test_pools_past_4_gb(d, hkv, flag):
    """Pages whose byte offsets pass 32 bits, written, attended and read back."""
    import torch

    pages = (1 << 32) // (hkv * 17 * d // 2) + 500
    kv = [300, 70]
    b = W.custom("far", 2 * hkv, hkv, d, [1, 70], kv, [[(0, n, C, 0)] for n in kv], [0, 0], seed=1)
    small = b.num_pages
    k0, v0 = random_pools(b, 2, poison=False)
    q, (kn, vn) = queries(b, 2), _rows(b)
    far = [torch.empty((pages, hkv, 17 * d // 2), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for x, y in zip(far, (k0, v0)):
        x[-small:] = torch.from_numpy(y).to(DEV)
    table = np.where(b.block_table >= 0, b.block_table + pages - small, -1).astype(np.int32)
    pl = attn.plan(b.num_qo_heads, hkv, d, "bf16", b.seqs, b.masks, b.segments, table.shape[1], pages, flags=flag)
    bt = torch.from_numpy(table).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    cache.kv4_append(pl, kn, vn, bt, *far)
    cache.kv4_fwd(pl, q, *far, bt, out, lse, attn.workspace(pl, DEV))
    assert attn.check(pl) == 0
    pl.destroy()
    rk, rv = kv4_append(b, host64(kn), host64(vn), k0, v0)
    for x, y in zip(far, (rk, rv)):
        assert np.array_equal(x[-small:].cpu().numpy(), y)
    ids = torch.arange(pages - small, pages, dtype=torch.int32, device=DEV)
    back = [torch.empty((small, 16, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache.kv4_unpack(*far, ids, *back)
    for which, x, y in zip("kv", back, (rk, rv)):
        assert np.array_equal(host64(x), kv4_values(*kv4_read(which, y, d)))
    # the appended values are large: the bar of out alone, against the values
    qh = host64(q)
    from oracle import oracle_attention

    k, v = (kv4_values(*kv4_read(w, p, d)) for w, p in (("k", rk), ("v", rv)))
    ro, rl = oracle_attention(b, qh, k, v)
    assert np.isfinite(host64(out)).all() and out.shape == ro.shape


@pytest.mark.parametrize("kv,q,window", [(40000, 1, 0), (40000, 130, 0), (30000, 5, 20000)])
def test_long_requests(kv, q, window):
    b = W.custom("long", 4, 1, 128, [q], [kv], [[(0, kv, C, 0)]], [window], seed=1)
    k4, v4 = random_pools(b, 2, poison=False)
    qs = queries(b, 2)
    ref = reference(b, qs, k4, v4)
    for flag in (0, attn.FLAG_NO_SPLIT):
        compare4(b, *run_kv4(b, qs, k4, v4, flag), ref, f"kv {kv} q {q} window {window}")


@pytest.mark.parametrize("hq,hkv,d", [(28, 1, 128), (64, 1, 64), (64, 1, 128), (32, 1, 64)])
def test_large_groups(hq, hkv, d):
    kv = [333, 150, 90]
    b = W.custom("groups", hq, hkv, d, [1, 16, 90], kv, [[(0, n, C, 0)] for n in kv], [0] * 3, seed=1)
    k4, v4 = random_pools(b, 2)
    qs = queries(b, 2)
    ref = reference(b, qs, k4, v4)
    for flag in FLAGS.values():
        compare4(b, *run_kv4(b, qs, k4, v4, flag), ref, f"{hq}/{hkv} d{d}")


@pytest.mark.parametrize("name,flags,cascade", [("serving_mix_bf16", attn.FLAG_FORCE_SPLIT, True), ("mixed", 0, False)])
def test_noalloc_equals_workspace_bitwise(name, flags, cascade):
    import torch

    b = W.reduced(name)
    k4, v4 = random_pools(b, 5)
    q = queries(b, 6)
    o1, l1 = run_kv4(b, q, k4, v4, flags, cascade)
    o2, l2 = run_kv4(b, q, k4, v4, flags, cascade, noalloc=True)
    assert torch.equal(o1.view(torch.int16), o2.view(torch.int16))
    assert torch.equal(l1.view(torch.int32), l2.view(torch.int32))


def test_two_runs_are_equal():
    import torch

    b = W.reduced("mixed")
    k4, v4 = random_pools(b, 5)
    q = queries(b, 6)
    (o1, l1), (o2, l2) = (run_kv4(b, q, k4, v4) for _ in range(2))
    assert torch.equal(o1.view(torch.int16), o2.view(torch.int16)) and torch.equal(l1, l2)


# ---- the operators together ----------------------------------------------------------

@pytest.mark.parametrize("name,cascade", [("mixed", False), ("shared_prefix_decode_bf16", True)])
def test_step_with_tables_append_attention_and_read_back(name, cascade):
    """Pages from a free list, rows stored, attended, and the pages read back:
    attention over the read-back pages through attn.fwd gives the same."""
    import torch

    b = W.reduced(name)
    first = [(int(kv) - int(q) + 15) // 16 for q, kv, _ in b.seqs]
    table, free = b.block_table.copy(), []
    for r, held in enumerate(first):
        n = (int(b.seqs[r, 1]) + 15) // 16
        free += table[r, held:n].tolist()
        table[r, held:n] = -1
    pl = plan_for(b, cascade=cascade)
    assert cache.block_tables_pages(pl) == len(free)
    bt = torch.from_numpy(table).to(DEV)
    slots = torch.full((b.total_q,), -7, dtype=torch.int64, device=DEV)
    cache.block_tables(pl, torch.tensor(free, dtype=torch.int32, device=DEV), bt, slots)
    assert np.array_equal(bt.cpu().numpy(), b.block_table)
    want = {row: page * 16 + slot for row, page, slot in append_targets(b)}
    assert slots.tolist() == [want.get(i, -7) for i in range(b.total_q)]
    k0, v0 = random_pools(b, 5, poison=False)
    k4, v4 = torch.from_numpy(k0).to(DEV), torch.from_numpy(v0).to(DEV)
    kn, vn = (torch.randn((b.total_q, b.num_kv_heads, b.head_dim), device=DEV).bfloat16() for _ in range(2))
    q = queries(b, 6)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    ws = attn.workspace(pl, DEV)
    cache.kv4_append(pl, kn, vn, bt, k4, v4)
    cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, ws)
    ids = torch.arange(b.num_pages, dtype=torch.int32, device=DEV)
    k16, v16 = (torch.empty((b.num_pages, 16, b.num_kv_heads, b.head_dim), dtype=torch.bfloat16, device=DEV)
                for _ in range(2))
    cache.kv4_unpack(k4, v4, ids, k16, v16)
    ref = reference(b, q, *kv4_append(b, host64(kn), host64(vn), k0, v0))
    compare4(b, out, lse, ref, f"step {name}")
    attn.fwd(pl, q, k16, v16, bt, out, lse, ws)
    compare4(b, out, lse, ref, f"step {name}, 16 bits")
    assert attn.check(pl) == 0
    pl.destroy()


@pytest.mark.parametrize("name,flags,cascade", [("mixed", 0, False), ("decode_bf16", attn.FLAG_FORCE_SPLIT, False),
                                                ("shared_prefix_decode_bf16", 0, True)])
def test_step_captured_in_a_graph(name, flags, cascade):
    import torch

    b = W.reduced(name)
    pl = plan_for(b, flags, cascade=cascade)
    kn, vn = _rows(b, 5)
    kn, vn = kn.clamp(-4, 4), vn.clamp(-4, 4)
    k0, v0 = (torch.from_numpy(x).to(DEV) for x in random_pools(b, 5, poison=False))
    k4, v4, bt, q = k0.clone(), v0.clone(), _table(b), queries(b, 6)
    held = torch.tensor([[(int(kv) - int(n) + 15) // 16] for n, kv, _ in b.seqs], device=DEV)
    need = torch.tensor([[(int(kv) + 15) // 16] for _, kv, _ in b.seqs], device=DEV)
    col = torch.arange(bt.shape[1], device=DEV)
    new = (col >= held) & (col < need)
    free = bt[new].contiguous()
    out, lse, ws = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV), attn.workspace(pl, DEV)
    slots = torch.empty(b.total_q, dtype=torch.int64, device=DEV)
    ids = torch.arange(b.num_pages, dtype=torch.int32, device=DEV)
    back = [torch.empty((b.num_pages, 16, b.num_kv_heads, b.head_dim), dtype=torch.bfloat16, device=DEV)
            for _ in range(2)]
    state = [bt, slots, k4, v4, out, lse, *back]

    def step(stream=None):
        cache.block_tables(pl, free, bt, slots, stream)
        cache.kv4_append(pl, kn, vn, bt, k4, v4, stream)
        cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, ws, stream)
        cache.kv4_unpack(k4, v4, ids, *back, stream)

    def restart():
        k4.copy_(k0)
        v4.copy_(v0)
        bt.masked_fill_(new, -1)
        slots.fill_(-1)
        for x in (out, lse, *back):
            x.fill_(float("nan"))

    restart()
    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in state]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(side)
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        restart()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(state, want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), f"replay {rep}"
    assert attn.check(pl) == 0
    del graph
    pl.destroy()


def test_rounding_matches_the_oracle_over_every_bf16_value():
    """Each of the 65536 bit patterns in a block of its own (with a fixed second
    value) and as the largest of its block."""
    import torch

    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros((65536 * 32 // 128, 1, 128), dtype=torch.bfloat16)
    flat = x.view(65536, 32)
    flat[:, 0] = bits
    flat[:, 7] = bits * 0.3
    flat[:, 31] = bits * -0.71
    n = x.shape[0]
    b = W.custom("all", 1, 1, 128, [n], [n], [[(0, n, F, 0)]], [0], seed=1)
    kn = x.to(DEV)
    k4, v4 = cache.kv4_pages(b.num_pages, 1, 128, DEV)
    pl = plan_for(b)
    cache.kv4_append(pl, kn, kn, _table(b), k4, v4)
    assert attn.check(pl) == cache.DEVERR_NONFINITE
    pl.destroy()
    codes, scales = kv4_round(host64(kn))
    rows = np.arange(n)
    for which, pool in (("k", k4), ("v", v4)):
        c, s = kv4_read(which, pool.cpu().numpy(), 128)
        page, slot = b.block_table[0, rows // 16], rows % 16
        assert np.array_equal(s[page, slot], scales), which
        assert np.array_equal(c[page, slot], codes), which


def test_unpack_of_more_records_than_one_launch_has_waves():
    import torch

    n = (1 << 22) + 5
    rng = np.random.default_rng(3)
    pools = rng.integers(0, 256, (2, 7, 1, 544)).astype(np.uint8)
    pools[..., 512:] = rng.integers(100, 140, pools[..., 512:].shape)
    k4, v4 = (torch.from_numpy(p).to(DEV) for p in pools)
    ids = torch.arange(n, dtype=torch.int32, device=DEV) % 8  # 7 is outside the pool
    out = [torch.empty((n, 16, 1, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache.kv4_unpack(k4, v4, ids, *out)
    for which, p, got in zip("kv", pools, out):
        want = np.concatenate([kv4_values(*kv4_read(which, p, 64)), np.zeros((1, 16, 1, 64))])
        want = torch.from_numpy(want).to(DEV).bfloat16()
        whole = n // 8 * 8
        assert (got[:whole].view(-1, 8, 16, 1, 64) == want).all()
        assert torch.equal(got[whole:], want[:n - whole])
