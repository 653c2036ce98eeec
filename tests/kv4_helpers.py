"""Shared by the tests of the 4-bit cache: pools of random codes, the oracle's
attention over them with the bars of its outputs, and calls of the HIP path."""
import numpy as np

from oracle import kv4_read, kv4_values, oracle_attention
from oracle.kv4 import nibble_at, scale_at
from paper_2606_12688_amd import attn, cache
from tests.helpers import host64, plan_for

DEV = "cuda:0"


def random_pools(b, seed, poison=True, exponents=(-4, 1)):
    """K and V pools (numpy) of random codes and of scales 2^e, e drawn from
    ``exponents``.  With ``poison`` every slot that holds no key of a request,
    and every key that no row of its only request may see, has all its code bits
    set and the scale byte 255, which a row never holds."""
    rng = np.random.default_rng([seed, 4])
    d = b.head_dim
    used = visible_slots(b) if poison else None
    out = []
    for _ in range(2):
        p = rng.integers(0, 256, (b.num_pages, b.num_kv_heads, 17 * d // 2)).astype(np.uint8)
        p[:, :, 8 * d:] = rng.integers(127 + exponents[0], 127 + exponents[1], p[:, :, 8 * d:].shape)
        out.append(p)
    if poison:
        for slot in range(16):
            pages, heads = np.nonzero(~used[:, slot])[0], np.arange(b.num_kv_heads)
            for which, p in zip("kv", out):  # a key's codes fill whole bytes of a record
                where = np.unique(np.concatenate([nibble_at(which, d)[slot] // 2, scale_at(d)[slot]]))
                p[np.ix_(pages, heads, where)] = 255
    return out


def visible_slots(b):
    """``[pages, 16]``: slots whose key some row may see (of a request without queries, all of its keys)."""
    used = np.zeros((b.num_pages, 16), dtype=bool)
    for r in range(b.num_seqs):
        q_len, kv_len, _ = (int(x) for x in b.seqs[r])
        w = int(b.masks[r, 2])
        lo = max(0, kv_len - q_len - w + 1) if w else 0
        for t in range(lo, kv_len):
            used[b.block_table[r, t // 16], t % 16] = True
    return used


def queries(b, seed, scale=1.0):
    import torch

    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (scale * torch.randn((b.total_q, b.num_qo_heads, b.head_dim), generator=g, device=DEV)).bfloat16()


def run_kv4(b, q, k4, v4, flags=0, cascade=False, noalloc=False, fill=float("nan")):
    """Plan and attention over pools (numpy or device tensors); (out, lse) on the device."""
    import torch

    k4, v4 = (torch.from_numpy(x).to(DEV) if isinstance(x, np.ndarray) else x for x in (k4, v4))
    pl = plan_for(b, flags, cascade=cascade)
    out = torch.full_like(q, fill)
    lse = torch.full(q.shape[:2], fill, dtype=torch.float32, device=DEV)
    bt = torch.from_numpy(np.ascontiguousarray(b.block_table)).to(DEV)
    if noalloc:
        cache.kv4_fwd_noalloc(pl, q, k4, v4, bt, out, lse)
    else:
        cache.kv4_fwd(pl, q, k4, v4, bt, out, lse, attn.workspace(pl, DEV))
    assert attn.check(pl) == 0
    pl.destroy()
    return out, lse


def reference(b, q, k4, v4):
    """The oracle's out and lse over the pools' values, and the attention over
    |V|, which bounds what rounded probabilities can move."""
    d, qh = b.head_dim, host64(q)
    k, v = (kv4_values(*kv4_read(which, p, d)) for which, p in (("k", k4), ("v", v4)))
    out, lse = oracle_attention(b, qh, k, v)
    size, _ = oracle_attention(b, qh, k, np.abs(v))
    return out, lse, size


def compare4(b, out, lse, ref, label=""):
    """Bars.  out is rounded to bf16 (half a step: 2^-8 of it) and every
    probability is (2^-8 of the values' weighted magnitude, ``size``); partials
    and sums are fp32.  A score is a sum of d <= 128 products in fp32, off by at
    most 128 * 2^-24 of the products' magnitudes; |q| <= 5 and |k| <= 6 with
    scale d^-1/2 >= 1/11.4 bound those by 128 * 30 / 11.4 = 340, unit-variance
    queries (mean |q| 0.8, mean |k| below 1.3) keep them near 12, so the error of
    a score and with it of lse below 2^-17 * 12 * 4 < 2^-11, and that of a
    probability below 2^-11, of out twice that (numerator and sum): 2^-10."""
    ro, rl, size = ref
    o, l = host64(out), lse.cpu().numpy().astype(np.float64)
    assert o.shape == ro.shape and np.isfinite(o).all(), f"{label}: shape or non-finite output"
    if not o.size:
        return
    eo = np.abs(o - ro) - (2.0 ** -8 * np.abs(ro) + (2.0 ** -8 + 2.0 ** -10) * size)
    el = np.abs(l - rl)
    fine = np.isfinite(rl)
    assert np.array_equal(np.isneginf(l), ~fine), f"{label}: empty rows"
    worst = float(el[fine].max()) if fine.any() else 0.0
    print(f"{label}: max|dout|={np.abs(o - ro).max():.3e} (slack {eo.max():.2e}) max|dlse|={worst:.3e}", flush=True)
    assert eo.max() <= 0, f"{label}: out is {eo.max()} past its bar"
    assert worst <= 2.0 ** -11, f"{label}: lse error {worst}"
