"""Host side of the operators on paged caches (no GPU): exported symbols, pages
that a plan takes, and every refusal of the C entry points that needs no device."""
import os
import re

import numpy as np
import pytest

import workloads as W
from oracle import block_tables
from paper_2606_12688_amd import attn, cache
from tests.helpers import plan_for

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    hdr = open(os.path.join(ROOT, "include", "mstar_cache.h")).read()
    declared = set(re.findall(r"^\s*(?:int|int64_t|size_t|void|const char\*)\s+(mstar_\w+)\s*\(", hdr, re.M))
    assert declared == set(cache.EXPORTS)
    for name in declared:
        assert hasattr(cache.lib(), name), name
    assert int(re.search(r"MSTAR_DEVERR_NONFINITE (\d+)", hdr).group(1)) == cache.DEVERR_NONFINITE
    assert cache.record_bytes(128) == 1088 and cache.record_bytes(64) == 544


@pytest.mark.parametrize("name", ["tiny_causal_f32", "decode_bf16", "stream_window_bf16", "rollout_bf16", "mixed"])
def test_pages_taken(name):
    b = W.reduced(name)
    pl = plan_for(b, attn.FLAG_HOST_ONLY)
    _, _, taken = block_tables(b.seqs, np.zeros(10000, int), b.block_table, b.num_pages)
    assert cache.block_tables_pages(pl) == taken
    pl.destroy()


def test_pages_taken_after_another_plan_on_the_same_host_lists():
    for kv, q, pages in ((33, 33, 3), (33, 1, 1), (32, 1, 0), (0, 0, 0), (16, 16, 1)):
        pl = attn.plan(2, 1, 64, "bf16", [[q, kv, 0]], [[0, 1 if kv else 0, 0]], [[0, kv, 0, 0]] if kv else [], 4, 8,
                       flags=attn.FLAG_HOST_ONLY)
        assert cache.block_tables_pages(pl) == pages
        pl.destroy()


def test_refusals():
    L = cache.lib()
    pl = plan_for(W.reduced("decode_bf16"), attn.FLAG_HOST_ONLY)
    p = 0x10000  # never read: every call below is refused first
    assert L.mstar_block_tables_pages(None) == 0
    for h in (None, pl.handle):  # no plan, and a host-only one
        assert L.mstar_kv4_append(h, p, p, p, p, p, None) == attn.ERR_INVALID_ARG
        assert L.mstar_kv4_fwd(h, p, p, p, p, p, p, p, 1 << 30, None) == attn.ERR_INVALID_ARG
        assert L.mstar_kv4_fwd_noalloc(h, p, p, p, p, p, p, None) == attn.ERR_INVALID_ARG
        assert L.mstar_block_tables(h, p, 1 << 30, p, p, None) == attn.ERR_INVALID_ARG
        assert attn.last_error()
    pl.destroy()
    unpack = L.mstar_kv4_unpack
    assert unpack(4, 128, 10, p, p, p, 0, p, p, None) == attn.OK  # nothing to do
    for bad in ((0, 128, 10, p, p, p, 1, p, p), (4, 128, 0, p, p, p, 1, p, p), (4, 128, 10, p, p, p, -1, p, p),
                (-1, 128, 10, p, p, p, 1, p, p), (4, 128, 10, None, p, p, 1, p, p), (4, 128, 10, p, None, p, 1, p, p),
                (4, 128, 10, p, p, None, 1, p, p), (4, 128, 10, p, p, p, 1, None, p),
                (4, 128, 10, p, p, p, 1, p, None), (4, 128, 10, p + 8, p, p, 1, p, p),
                (4, 128, 10, p, p + 1, p, 1, p, p), (4, 128, 10, p, p, p + 2, 1, p, p),
                (4, 128, 10, p, p, p, 1, p + 4, p), (4, 128, 10, p, p, p, 1, p, p + 15)):
        assert unpack(*bad, None) == attn.ERR_INVALID_ARG, bad
    for d in (0, 32, 96, 256, -64):
        assert unpack(4, d, 10, p, p, p, 1, p, p, None) == attn.ERR_UNSUPPORTED
