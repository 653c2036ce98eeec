"""The calls on paged caches refuse what does not match the plan, whichever
argument it is, and take what does."""
import numpy as np
import pytest

import workloads as W
from paper_2606_12688_amd import attn, cache
from tests.helpers import plan_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CALLS = {"kv4_append": ["k_new", "v_new", "block_table", "k_pages", "v_pages"],
         "kv4_fwd": ["q", "k_pages", "v_pages", "block_table", "out", "lse"],
         "kv4_fwd_noalloc": ["q", "k_pages", "v_pages", "block_table", "out", "lse"],
         "block_tables": ["free_pages", "block_table", "slots"],
         "kv4_unpack": ["k_pages", "v_pages", "page_ids", "k_out", "v_out"]}


def _batch():
    kv = [300, 90, 17]
    return W.custom("checks", 8, 2, 128, [1, 40, 17], kv, [[(0, n, W.SEG_CAUSAL, 0)] for n in kv], [0] * 3, seed=1)


def _wrong(t, lists):
    import torch

    yield "device", t.cpu()
    if not lists:
        yield "shape", torch.cat([t, t])
    yield "dims", t[None]
    yield "strides", torch.stack([t, t], -1)[..., 0]
    yield "dtype", t.to(torch.float16 if t.is_floating_point() else torch.int16)


def _good(b, pl):
    import torch

    d = b.head_dim
    new = torch.zeros((b.total_q, b.num_kv_heads, d), dtype=torch.bfloat16, device=DEV)
    k4, v4 = cache.kv4_pages(b.num_pages, b.num_kv_heads, d, DEV)
    q = torch.zeros((b.total_q, b.num_qo_heads, d), dtype=torch.bfloat16, device=DEV)
    pages = torch.zeros((4, 16, b.num_kv_heads, d), dtype=torch.bfloat16, device=DEV)
    return dict(k_new=new, v_new=new.clone(), q=q, out=torch.empty_like(q), lse=torch.empty(q.shape[:2], device=DEV),
                k_pages=k4, v_pages=v4, block_table=torch.from_numpy(np.ascontiguousarray(b.block_table)).to(DEV),
                free_pages=torch.arange(cache.block_tables_pages(pl) + 3, dtype=torch.int32, device=DEV),
                slots=torch.empty(b.total_q, dtype=torch.int64, device=DEV),
                page_ids=torch.arange(4, dtype=torch.int32, device=DEV), k_out=pages, v_out=pages.clone())


@pytest.mark.parametrize("call", list(CALLS))
def test_every_mismatch_is_refused(call):
    b = _batch()
    pl = plan_for(b)
    good, names, fn = _good(b, pl), CALLS[call], getattr(cache, call)
    plan_arg = () if call == "kv4_unpack" else (pl,)
    extra = (attn.workspace(pl, DEV),) if call == "kv4_fwd" else ()
    fn(*plan_arg, *(good[n] for n in names), *extra)
    for n in names:
        for what, bad in _wrong(good[n], n in ("free_pages", "page_ids")):
            if n == "k_pages" and call == "kv4_unpack" and what == "shape":
                continue  # a longer K pool says how long both are: v_pages is refused below
            with pytest.raises(ValueError):
                fn(*plan_arg, *(bad if m == n else good[m] for m in names), *extra)
                pytest.fail(f"{call}: {n} with the wrong {what} was taken")
    assert attn.check(pl) == 0
    pl.destroy()
    if plan_arg:
        with pytest.raises(ValueError):
            fn(*plan_arg, *(good[n] for n in names), *extra)


def test_other_refusals():
    b = _batch()
    pl = plan_for(b, attn.FLAG_FORCE_SPLIT)
    g = _good(b, pl)
    fwd = [g[n] for n in CALLS["kv4_fwd"]]
    ws = attn.workspace(pl, DEV)
    for bad in (None, ws[:-256]):
        with pytest.raises(attn.MStarError) as e:
            cache.kv4_fwd(pl, *fwd, bad)
        assert e.value.code == attn.ERR_WORKSPACE
    with pytest.raises(attn.MStarError) as e:  # one page short
        cache.block_tables(pl, g["free_pages"][:-4], g["block_table"], g["slots"])
    assert e.value.code == attn.ERR_INVALID_ARG
    pl.destroy()
    f = W.reduced("tiny_causal_f32")
    pl = plan_for(f)
    g = _good(f, pl)
    for call in ("kv4_append", "kv4_fwd", "kv4_fwd_noalloc"):
        with pytest.raises(attn.MStarError) as e:
            getattr(cache, call)(pl, *(g[n] for n in CALLS[call]))
        assert e.value.code == attn.ERR_UNSUPPORTED
    L, p = cache.lib(), 0x10000  # never read: refused first
    pl.destroy()
    pl = plan_for(b)
    for bad in ((None, p, p, p, p), (p, None, p, p, p), (p, p, None, p, p), (p, p, p, None, p), (p, p, p, p, None),
                (p + 8, p, p, p, p), (p, p, p + 2, p, p), (p, p, p, p + 8, p)):
        assert L.mstar_kv4_append(pl.handle, *bad, None) == attn.ERR_INVALID_ARG
    for bad in ((None, p, p, p, p, p), (p, p + 8, p, p, p, p), (p, p, p, p, None, p), (p, p, p, p, p, p + 2)):
        assert L.mstar_kv4_fwd(pl.handle, *bad, None, 0, None) == attn.ERR_INVALID_ARG
        assert L.mstar_kv4_fwd_noalloc(pl.handle, *bad, None) == attn.ERR_INVALID_ARG
    n = cache.block_tables_pages(pl)
    for bad in ((p, n, None, p), (p, n, p + 2, p), (p, n, p, p + 4), (p + 1, n, p, p), (p, n - 1, p, p)):
        assert L.mstar_block_tables(pl.handle, *bad, None) == attn.ERR_INVALID_ARG
    pl.destroy()


def test_a_batch_without_rows():
    import torch

    b = W.custom("none", 4, 2, 128, [0, 0], [40, 0], [[(0, 40, 0, 0)], []], [0, 0], seed=1)
    pl = plan_for(b)
    g = _good(b, pl)
    for call in ("kv4_append", "kv4_fwd", "kv4_fwd_noalloc", "block_tables"):
        getattr(cache, call)(pl, *(g[n] for n in CALLS[call]))
    assert attn.check(pl) == 0
    torch.cuda.synchronize()
    pl.destroy()
