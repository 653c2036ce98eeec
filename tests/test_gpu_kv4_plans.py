"""Attention over a 4-bit cache on the plans that decide how it is launched: key
groups, few-row items behind the tiles or the cascade, beside them on the side
stream, or on their own, and references that keep moving."""
import pytest

import workloads as W
from paper_2606_12688_amd import attn
from tests.helpers import plan_for
from tests.kv4_helpers import compare4, queries, random_pools, reference, run_kv4
from tests.test_gpu_key_groups import _batch

pytestmark = pytest.mark.gpu
C, F = W.SEG_CAUSAL, W.SEG_FULL


def _check(b, flags, label, seed=3, cascade=False):
    k4, v4 = random_pools(b, seed)
    q = queries(b, seed)
    ref = reference(b, q, k4, v4)
    for flag in flags:
        compare4(b, *run_kv4(b, q, k4, v4, flag, cascade), ref, f"{label} flags {flag}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (7, 1), (6, 2)])
def test_key_groups(hq, hkv, d):
    _check(_batch(hq, hkv, d), (0, attn.FLAG_NO_SPLIT), f"key groups {hq}/{hkv} d{d}")


@pytest.mark.parametrize("d", [64, 128])
def test_key_groups_beside_few_row_items(d):
    kv = [900, 300, 77]
    b = W.custom("groups_few", 4, 2, d, [900, 1, 1], kv, [[(0, n, C, 0)] for n in kv], [0] * 3, seed=d)
    _check(b, (0, attn.FLAG_SERIAL), f"key groups beside few rows d{d}")


def _mixed(hq, hkv, d, q, kv):
    return W.custom("mixed_plan", hq, hkv, d, q, kv, [[(0, n, C, 0)] for n in kv], [0] * len(q), seed=d + hq)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,rows", [(8, 2, 1), (4, 4, 1), (8, 2, 6), (4, 4, 20), (16, 2, 7), (28, 4, 1)])
def test_few_row_items_behind_the_tiles(hq, hkv, rows, d):
    """Units of up to 16, 32 and 64 rows (the last go on their own stream at D = 64)."""
    q = [1, 200, rows, 333, rows, 0, 150]
    kv = [500, 200, 90, 600, 1000, 30, 150]
    b = _mixed(hq, hkv, d, q, kv)
    pl = plan_for(b, attn.FLAG_HOST_ONLY)
    assert pl.stats()["decode_items"] > 0 and pl.stats()["prefill_items"] > 0
    pl.destroy()
    _check(b, (0, attn.FLAG_SERIAL, attn.FLAG_FORCE_SPLIT, attn.FLAG_NO_SPLIT), f"mixed {hq}/{hkv} {rows} rows d{d}")


@pytest.mark.parametrize("d", [64, 128])
def test_more_tiles_than_the_gpu_holds(d):
    q = [1] * 9 + [900] * 12
    kv = [1000 + 37 * i for i in range(9)] + [900] * 12
    _check(_mixed(16, 8, d, q, kv), (0,), f"many tiles d{d}")


@pytest.mark.parametrize("d", [64, 128])
def test_cascade_with_tiles_and_few_row_items(d):
    """Members of a prefix group, a prompt and decode steps in one plan."""
    b = W.reduced("shared_prefix_decode_bf16")
    for flags in (0, attn.FLAG_FORCE_SPLIT, attn.FLAG_CASCADE_ALL, attn.FLAG_SERIAL):
        _check(b, (flags,), "cascade", cascade=True)
    q, kv = [1, 1, 3, 150, 1], [400, 333, 350, 400, 700]
    b = _mixed(8, 2, d, q, kv)
    b.block_table[1, :20] = b.block_table[2, :20] = b.block_table[0, :20]
    b.prefix_groups = [([0, 1, 2], 320)]
    for flags in (0, attn.FLAG_FORCE_SPLIT, attn.FLAG_NO_SPLIT, attn.FLAG_SERIAL):
        _check(b, (flags,), f"cascade and tiles d{d}", cascade=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("up", [1, -1])
def test_growing_and_falling_scores(d, up):
    """Key scales that double (or halve) every ten pages: references that move all
    along, tiles redone exactly, pieces and key groups that end far apart."""
    kv = [700, 900, 640, 333]
    b = W.custom("growing", 4, 2, d, [700, 1, 90, 8], kv, [[(0, n, C, 0)] for n in kv], [0] * 4, seed=d)
    k4, v4 = random_pools(b, 1)
    for r in range(b.num_seqs):
        for p in range((kv[r] + 15) // 16):
            live = min(16, kv[r] - 16 * p)
            scales = k4[b.block_table[r, p], :, 8 * d:].reshape(b.num_kv_heads, d // 32, 16)
            scales[:, :, :live] += p // 10 if up > 0 else 6 - p // 10
            k4[b.block_table[r, p], :, 8 * d:] = scales.reshape(b.num_kv_heads, -1)
    q = queries(b, 2, scale=2.0 ** -6)  # the largest keys make scores as large as the bars assume
    ref = reference(b, q, k4, v4)
    for flag in (0, attn.FLAG_FORCE_SPLIT, attn.FLAG_NO_SPLIT):
        compare4(b, *run_kv4(b, q, k4, v4, flag), ref, f"scores d{d} up {up} flags {flag}")
    q = queries(b, 2, scale=4.0)  # and far apart
    out, lse = run_kv4(b, q, k4, v4)
    ro, rl, _ = reference(b, q, k4, v4)
    assert abs(lse.cpu().numpy() - rl).max() <= 2.0 ** -3  # scores 256 times as large: 2^-11 * 2^8


# how many requests of how many query rows: units of up to 16, 32 and 64 rows (the last at D = 64 only)
@pytest.mark.parametrize("few", [True, False], ids=["few_items", "many_items"])
@pytest.mark.parametrize("d,hq,hkv,rows", [(64, 16, 8, 1), (128, 28, 4, 1), (64, 12, 12, 5), (128, 8, 8, 16),
                                           (64, 16, 8, 12), (128, 28, 4, 4), (64, 28, 4, 8), (64, 8, 8, 50)])
def test_few_row_items_on_their_own(d, hq, hkv, rows, few):
    """Launches that leave a CU one workgroup at most, and more than it holds of two: both sizes of a workgroup."""
    n = 2 if few else 520 // hkv + 1
    kv = [rows + (37 * i) % 230 for i in range(n - 1)] + [1100]
    b = W.custom("few_alone", hq, hkv, d, [rows] * n, kv, [[(0, x, C, 0)] for x in kv], [0] * n, seed=rows)
    pl = plan_for(b, attn.FLAG_HOST_ONLY | attn.FLAG_NO_SPLIT)
    s = pl.stats()
    pl.destroy()
    assert s["prefill_items"] == 0 and (0 < s["decode_items"] <= 256 if few else s["decode_items"] > 512), s
    _check(b, (attn.FLAG_NO_SPLIT, 0), f"few alone {hq}/{hkv} {rows} rows d{d} x {n}")


@pytest.mark.parametrize("few", [True, False], ids=["few_tiles", "many_tiles"])
@pytest.mark.parametrize("d,hq,hkv", [(64, 8, 8), (128, 8, 8), (64, 28, 4), (128, 28, 4), (128, 12, 12)])
def test_tiles_on_their_own(d, hq, hkv, few):
    """Tiles without key groups that leave a CU two workgroups at most, and more."""
    lens = [170, 333] if few else [170 + 17 * i for i in range(12)] * (1 if hq == 28 else 3)
    b = W.custom("tiles_alone", hq, hkv, d, lens, lens, [[(0, x, C, 0)] for x in lens], [0] * len(lens), seed=d)
    pl = plan_for(b, attn.FLAG_HOST_ONLY)
    s, wgs = pl.stats(), len(pl.tile_order())
    pl.destroy()
    assert s["decode_items"] == 0 and (0 < wgs <= 512 if few else wgs > 512), (s, wgs)
    _check(b, (0,), f"tiles alone {hq}/{hkv} d{d} x {len(lens)}")


@pytest.mark.parametrize("few", [True, False], ids=["few_items", "many_items"])
@pytest.mark.parametrize("cascade", [False, True], ids=["tiles", "cascade"])
@pytest.mark.parametrize("d,hq,hkv,rows", [(128, 8, 2, 1), (128, 8, 8, 1), (128, 8, 2, 6), (128, 8, 8, 20), (64, 8, 4, 1)])
def test_mixed_launches_of_few_and_of_many_items(d, hq, hkv, rows, cascade, few):
    """Few-row items behind tiles, or behind a cascade (of one prefix for all of
    them), on both sides of three workgroups a CU."""
    n = 5 if few else 780 // hkv + 1
    kv = [352 + rows + (29 * i) % 120 for i in range(n)]
    q = [rows] * n
    if not cascade:
        q, kv = q + [200, 333], kv + [450, 333]
    b = _mixed(hq, hkv, d, q, kv)
    if cascade:
        b.block_table[:, :20] = b.block_table[0, :20]
        b.prefix_groups = [(list(range(n)), 320)]
    pl = plan_for(b, attn.FLAG_HOST_ONLY | attn.FLAG_NO_SPLIT, cascade=cascade)
    s, wgs = pl.stats(), len(pl.tile_order(cascade))
    pl.destroy()
    assert s["decode_items"] > 0 and 0 < wgs <= 512, (s, wgs)
    assert (wgs + s["decode_items"] <= 768) == few, (s, wgs)
    _check(b, (attn.FLAG_NO_SPLIT, 0), f"mixed {hq}/{hkv} {rows} rows d{d} x {n} cascade {cascade}", cascade=cascade)


def test_a_cascade_of_more_keys_than_items():
    """A launch of many items whose cascade item is longer still."""
    n, prefix = 800, 1600
    kv = [prefix + 1 + (7 * i) % 40 for i in range(n)]
    b = _mixed(2, 1, 128, [1] * n, kv)
    b.block_table[:, :prefix // 16] = b.block_table[0, :prefix // 16]
    b.prefix_groups = [(list(range(n)), prefix)]
    pl = plan_for(b, attn.FLAG_HOST_ONLY | attn.FLAG_NO_SPLIT, cascade=True)
    s, wgs = pl.stats(), len(pl.tile_order(True))
    pl.destroy()
    assert s["decode_items"] == n and 0 < wgs <= 512, (s, wgs)
    _check(b, (attn.FLAG_NO_SPLIT, 0), f"cascade of {prefix} keys, {n} items", cascade=True)
