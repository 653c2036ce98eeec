"""Outputs (not only lse) of attention over a 4-bit cache whose scores are large,
far apart and moving, so that references move by large steps and tiles are redone
exactly, and under the largest values that attention takes.

Bars.  With u = 2^-24, a score is a sum of d fp32 products (each exact: 8 by 2
significant bits) taken in fp32, so off by at most 2 d u A, where A is the sum of
the products' magnitudes times the scale; scaling, the difference from the
reference and a partial's lse add at most 2^-21 of the largest |score|, exp2, the
sums and the merge less than 2^-17 in all.  E, per row, is the sum of these for
its largest A and |score|.  Weights are then right to a factor within exp(+-2 E)
and rounded to bf16 (2^-8 of each), and out is rounded to bf16 (2^-8 of it):
  |out - ref| <= 2^-8 |ref| + 2^-8 sum p |V| + (exp(2 E) - 1) sum p |V - ref| + n 2^-126 (1 + max |V|)
where that sum is small for a row whose leading key leads by far, and the last
term is fp32's smallest normal number: of n keys, a weight below it counts as 0
(against the row's largest, which is at least 1), and so may a product with a
value below 1.  lse is off by at most E, and 2^-22 of itself for its own rounding."""
import numpy as np
import pytest

import workloads as W
from oracle import kv4_read, kv4_values
from oracle.kv4 import nibble_at, scale_at
from paper_2606_12688_amd import attn
from tests.helpers import host64
from tests.kv4_helpers import queries, random_pools, run_kv4

pytestmark = pytest.mark.gpu
FLAGS = (0, attn.FLAG_NO_SPLIT, attn.FLAG_FORCE_SPLIT)


def _causal(b, q, k4, v4):
    """out, lse and the bars of both, in 64 bits, of a batch of causal requests."""
    d, group = b.head_dim, b.num_qo_heads // b.num_kv_heads
    k, v = (kv4_values(*kv4_read(w, p, d)) for w, p in (("k", k4), ("v", v4)))
    q = host64(q)
    out, bar = np.zeros_like(q), np.zeros_like(q)
    lse, lbar = np.zeros(q.shape[:2]), np.zeros(q.shape[:2])
    for r, (n, kv, at) in enumerate(b.seqs.tolist()):
        pages = b.block_table[r, :(kv + 15) // 16]
        kr, vr = (x[pages].reshape(-1, *x.shape[2:])[:kv] for x in (k, v))
        hidden = np.arange(kv)[None, :] > np.arange(kv - n, kv)[:, None]
        for h in range(b.num_qo_heads):
            qh, kh, vh = q[at:at + n, h], kr[:, h // group], vr[:, h // group]
            s = qh @ kh.T * b.sm_scale
            size = np.where(hidden, 0, np.abs(qh) @ np.abs(kh).T * b.sm_scale).max(1)
            err = 2 * d * 2.0 ** -24 * size + 2.0 ** -21 * np.where(hidden, 0, np.abs(s)).max(1) + 2.0 ** -17
            s = np.where(hidden, -np.inf, s)
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            total = p.sum(1, keepdims=True)
            p /= total
            o = p @ vh
            spread = np.stack([p[i] @ np.abs(vh - o[i]) for i in range(n)])
            out[at:at + n, h] = o
            bar[at:at + n, h] = 2.0 ** -8 * (np.abs(o) + p @ np.abs(vh)) + np.expm1(2 * err)[:, None] * spread \
                + kv * 2.0 ** -126 * (1 + np.where(hidden, 0, np.abs(vh).max(1)).max(1))[:, None]
            lse[at:at + n, h] = (top + np.log(total))[:, 0]
            lbar[at:at + n, h] = err + 2.0 ** -22 * np.abs(lse[at:at + n, h])
    return out, bar, lse, lbar


def _check(b, q, k4, v4, label, flags=FLAGS):
    ro, bar, rl, lbar = _causal(b, q, k4, v4)
    tight = (bar <= 2.0 ** -4 * np.abs(ro)).mean()
    for flag in flags:
        out, lse = run_kv4(b, q, k4, v4, flag)
        o, l = host64(out), host64(lse)
        assert np.isfinite(o).all() and np.isfinite(l).all(), f"{label} flags {flag}: not finite"
        assert (np.abs(o - ro) <= bar).all() and (np.abs(l - rl) <= lbar).all(), f"{label} flags {flag}"
        worst, worst_l = (np.abs(o - ro) / bar).max(), (np.abs(l - rl) / lbar).max()
        print(f"{label} flags {flag}: out {worst:.3f} and lse {worst_l:.3f} of their bars ({tight:.2f} of outputs "
              "to a sixteenth or better)", flush=True)
    return tight


def _batch(d, kv=(700, 900, 640, 333), q=(700, 1, 90, 8), hq=4, hkv=2):
    return W.custom("scores", hq, hkv, d, list(q), list(kv), [[(0, n, W.SEG_CAUSAL, 0)] for n in kv], [0] * len(q),
                    seed=d)


def _ramp(b, pool, up, every):
    """Key scales doubled (or halved) every so many pages."""
    d = b.head_dim
    for r in range(b.num_seqs):
        kv = int(b.seqs[r, 1])
        for p in range((kv + 15) // 16):
            scales = pool[b.block_table[r, p], :, 8 * d:].reshape(b.num_kv_heads, d // 32, 16)
            scales[:, :, :min(16, kv - 16 * p)] += p // every if up else 60 // every - p // every
            pool[b.block_table[r, p], :, 8 * d:] = scales.reshape(b.num_kv_heads, -1)


@pytest.mark.parametrize("d", [64, 128])
def test_scores_in_the_thousands(d):
    b = _batch(d, kv=(700, 300, 150), q=(1, 20, 150), hq=8)
    k4, v4 = random_pools(b, 1, exponents=(8, 9))
    _, v4 = random_pools(b, 2)
    _check(b, queries(b, 1), k4, v4, f"thousands d{d}")


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_growing_and_falling_scores(d, up):
    b = _batch(d)
    k4, v4 = random_pools(b, 1)
    _ramp(b, k4, up, 10)
    tight = _check(b, queries(b, 2, scale=4.0), k4, v4, f"moving d{d} up {up}")
    assert tight > 0.5  # the bars say something


@pytest.mark.parametrize("d", [64, 128])
def test_growing_scores_in_mixed_launches_and_cascades(d):
    """The same where few-row items ride behind tiles, or behind a cascade."""
    b = _batch(d, kv=(500, 200, 400, 333, 450), q=(1, 200, 3, 150, 1), hq=8)
    k4, v4 = random_pools(b, 1)
    _ramp(b, k4, True, 8)
    _check(b, queries(b, 2, scale=4.0), k4, v4, f"mixed d{d}")


@pytest.mark.parametrize("d", [64, 128])
def test_values_up_to_2_64(d):
    """Values of up to 6 * 2^61 under scores that grow past a row's reference."""
    b = _batch(d)
    k4, v4 = random_pools(b, 1)
    _ramp(b, k4, True, 20)
    _, v4 = random_pools(b, 2, exponents=(61, 62))
    for scale in (0.25, 1.0, 4.0):
        _check(b, queries(b, 2, scale=scale), k4, v4, f"values of 2^61 d{d} scale {scale}")


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_do_not_see_the_largest_values(d):
    """A key whose values are of the largest magnitude (a stored infinity): rows before it are as without it."""
    b = _batch(d, kv=(333, 150), q=(333, 20), hq=8)
    k4, v4 = random_pools(b, 1)
    far = {0: 200, 1: 140}  # of each request, the key
    rows = np.concatenate([np.arange(far[0]), 333 + np.arange(far[1] - 130)])
    ro, bar, rl, lbar = (x[rows] for x in _causal(b, queries(b, 2), k4, v4))
    for r, key in far.items():
        page, slot = b.block_table[r, key // 16], key % 16
        v4[page][:, scale_at(d)[slot]] = 252
        v4[page][:, np.unique(nibble_at("v", d)[slot] // 2)] = 0x7F
    for flag in FLAGS:
        out, lse = run_kv4(b, queries(b, 2), k4, v4, flag)
        o, l = host64(out)[rows], host64(lse)[rows]
        assert (np.abs(o - ro) <= bar).all() and (np.abs(l - rl) <= lbar).all(), f"d{d} flags {flag}"
