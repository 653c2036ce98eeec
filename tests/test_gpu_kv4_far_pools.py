"""Attention over 4-bit pages whose byte offsets pass 32 bits, by value, on every
kind of launch: a page address cut to 32 bits would read the pool's first pages,
which hold other finite values."""
import numpy as np
import pytest

import workloads as W
from oracle import kv4_append
from paper_2606_12688_amd import attn, cache
from tests.helpers import host64, plan_for
from tests.kv4_helpers import DEV, compare4, queries, random_pools, reference

pytestmark = pytest.mark.gpu
# query rows, keys, length of a prefix that all requests share (0: none)
KINDS = {"few": ([1, 1, 2], [300, 70, 33], 0), "tiles": ([333, 170], [333, 400], 0), "mixed": ([1, 90, 200], [300, 90, 333], 0),
         "key_groups": ([700, 150], [700, 666], 0), "cascade": ([1] * 6, [355, 370, 401, 352, 380, 360], 320)}


@pytest.fixture(scope="module", autouse=True)
def _free():
    yield
    import torch

    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 4), (64, 8, 8)])
def test_append_and_attention_past_4_gb(d, hq, hkv, kind):
    import torch

    q_lens, kv, prefix = KINDS[kind]
    b = W.custom("far", hq, hkv, d, q_lens, kv, [[(0, n, W.SEG_CAUSAL, 0)] for n in kv], [0] * len(kv), seed=1)
    if prefix:
        b.block_table[:, :prefix // 16] = b.block_table[0, :prefix // 16]
        b.prefix_groups = [(list(range(len(kv))), prefix)]
    small = b.num_pages
    pages = (1 << 32) // (hkv * cache.record_bytes(d)) + small  # every used page starts at 4 GB or behind
    k0, v0 = random_pools(b, 2, poison=False)
    q = queries(b, 2)
    kn, vn = (torch.randn((b.total_q, hkv, d), generator=torch.Generator(DEV).manual_seed(s), device=DEV).bfloat16()
              for s in (3, 4))
    far = [torch.empty((pages + 1, hkv, cache.record_bytes(d)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for x, y in zip(far, (k0, v0)):
        x.fill_(119)  # elsewhere: codes 7 under the scale 2^-8
        x[-small:] = torch.from_numpy(y).to(DEV)
    first = pages + 1 - small
    assert first * hkv * cache.record_bytes(d) >= 1 << 32
    table = np.where(b.block_table >= 0, b.block_table + first, -1).astype(np.int32)
    bt = torch.from_numpy(table).to(DEV)
    ref = reference(b, q, *kv4_append(b, host64(kn), host64(vn), k0, v0))
    b.num_pages = pages + 1
    pl = plan_for(b, attn.FLAG_NO_SPLIT | attn.FLAG_HOST_ONLY, cascade=bool(prefix))
    tiles, few, casc = (pl.items(k) for k in (0, 1, 4))
    assert (len(tiles) > 0, len(few) > 0, len(casc) > 0) == (kind in ("tiles", "mixed", "key_groups"),
                                                             kind in ("few", "mixed", "cascade"), kind == "cascade")
    if kind == "key_groups":
        assert len(pl.tile_order()) <= 256 and (tiles[:, 5] - tiles[:, 4]).max() >= 640
    pl.destroy()
    for flag in (0, attn.FLAG_NO_SPLIT, attn.FLAG_FORCE_SPLIT):
        pl = plan_for(b, flag, cascade=bool(prefix))
        out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=DEV)
        cache.kv4_append(pl, kn, vn, bt, *far)
        cache.kv4_fwd(pl, q, *far, bt, out, lse, attn.workspace(pl, DEV))
        assert attn.check(pl) == 0
        pl.destroy()
        compare4(b, out, lse, ref, f"far {kind} d{d} flags {flag}")
