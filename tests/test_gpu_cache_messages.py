"""mstar_attn_check names every error that the plan's error word holds."""
import numpy as np
import pytest

import workloads as W
from paper_2606_12688_amd import attn, cache
from tests.helpers import plan_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("page,value", [(False, False), (True, False), (False, True), (True, True)])
def test_message_names_every_bit(page, value):
    import torch

    b = W.custom("messages", 4, 2, 64, [3, 20], [30, 40], [[(0, n, W.SEG_CAUSAL, 0)] for n in (30, 40)], [0, 0], seed=1)
    pl = plan_for(b)
    new = torch.zeros((b.total_q, 2, 64), dtype=torch.bfloat16, device=DEV)
    table = np.array(b.block_table)
    if page:
        table[0, 1] = b.num_pages
    if value:
        new[10, 1, 5] = float("inf")
    cache.kv4_append(pl, new, new, torch.from_numpy(table).to(DEV), *cache.kv4_pages(b.num_pages, 2, 64, DEV))
    bits = attn.check(pl)
    assert bits == attn.DEVERR_PAGE_RANGE * page + cache.DEVERR_NONFINITE * value
    if bits:
        assert ("block-table entry" in attn.last_error()) == page
        assert ("infinite" in attn.last_error()) == value
    assert attn.check(pl) == 0  # cleared
    pl.destroy()
