"""Operators on paged caches: a cache held in 4 bits (rows stored, attended and
read back) and block tables built on the GPU.

The 4-bit cache.  K and V are ``uint8 [pages, Hkv, 17 d / 2]`` pools; a record
holds the 16 keys of one page and KV head.  32 consecutive dims of a key share
a scale byte b; a value is a 4-bit code (sign in bit 3, magnitude 0, .5, 1,
1.5, 2, 3, 4, 6 in bits 0-2) times 2^(b - 127).  A K record is ``[4][16 keys]
[d / 8]`` bytes (piece g: dims g d/4 .. of each key), a V record ``[4 key
groups][16][4 keys][d / 32]`` (piece n: dims n d/16 .. of the group's keys),
two codes a byte, the lower dim in the low half; the scale bytes follow as
``[d / 32][16 keys]``.  Stored rows take the smallest scale under which no
magnitude exceeds 7, and the nearest code (ties to the even code).

Kinds of cases:

* attend: one layer's attention over the 4-bit cache.  ``decode`` one new
  token per request; ``chunk`` a few tokens, causal, under a window;
  ``prompt`` a whole causal prompt; ``latent`` causal text followed by image
  tokens that see each other; ``roll`` frames, block causal, over one prefix
  that every request shares; ``shared`` one token over a shared prefix and own
  tokens, planned as a cascade;
* store: a step's new rows go into the cache, and the pages they touch are
  read back in 16 bits, as when finished pages move to a 16-bit pool;
* tables: the pages of a step's new tokens are taken from the free list.

``lens`` seeds the drawn lengths, so that a case always has the same ones;
values and page orders come from the seed of ``prepare``.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
PAGE = 16


def listed():
    return [
        # one conversation decoding alone: the smallest attention call, all latency
        {"name": "decode_1", "op": "attend", "kind": "decode", "hq": 28, "hkv": 4, "d": 128, "lens": 1,
         "n": 1, "ctx_min": 1500, "ctx_max": 1500},
        # sixteen speech streams decoding together, head_dim 64, without a workspace
        {"name": "decode_16_d64", "op": "attend", "kind": "decode", "hq": 16, "hkv": 8, "d": 64, "lens": 2,
         "n": 16, "ctx_min": 300, "ctx_max": 4000, "noalloc": True},
        # a full decode batch over long contexts (the repository's decode configuration)
        {"name": "decode_64", "op": "attend", "kind": "decode", "hq": 28, "hkv": 4, "d": 128, "lens": 3,
         "n": 64, "ctx_min": 512, "ctx_max": 8192},
        # candidates continued from one context, as a shared-prefix cascade
        {"name": "shared_decode_128", "op": "attend", "kind": "shared", "hq": 28, "hkv": 4, "d": 128, "lens": 9,
         "n": 128, "prefix": 4096, "ctx_min": 256, "ctx_max": 1024},
        # streaming speech chunks under a sliding window (the repository's chunk configuration)
        {"name": "chunks_256", "op": "attend", "kind": "chunk", "hq": 16, "hkv": 8, "d": 128, "lens": 7,
         "n": 256, "chunk": 16, "ctx_min": 1024, "ctx_max": 16384, "window": 1024},
        # a few ragged text prompts entering an empty cache
        {"name": "prompt_4", "op": "attend", "kind": "prompt", "hq": 28, "hkv": 4, "d": 128, "lens": 4,
         "n": 4, "ctx_min": 200, "ctx_max": 2000},
        # world-model rollouts of three frames over one context, head_dim 64
        {"name": "rollout_64", "op": "attend", "kind": "roll", "hq": 16, "hkv": 16, "d": 64, "lens": 8,
         "n": 64, "prefix": 2048, "frames": 3, "frame": 256},
        # image-generation prefill of eight requests (the repository's prefill configuration)
        {"name": "text_latent_8", "op": "attend", "kind": "latent", "hq": 28, "hkv": 4, "d": 128, "lens": 6,
         "n": 8, "text": 256, "image": 4096},
        # one decoded token of one conversation stored: all latency
        {"name": "store_1", "op": "store", "kind": "decode", "hq": 28, "hkv": 4, "d": 128, "lens": 21,
         "n": 1, "ctx_min": 1500, "ctx_max": 1500},
        # the rows of eight image-generation prefills stored
        {"name": "store_8_prefills", "op": "store", "kind": "prompt", "hq": 28, "hkv": 4, "d": 128, "lens": 22,
         "n": 8, "ctx_min": 4352, "ctx_max": 4352},
        # a decode step's pages: every request has one new token, every sixteenth a new page
        {"name": "tables_64", "op": "tables", "kind": "decode", "hq": 28, "hkv": 4, "d": 128, "lens": 31,
         "n": 64, "ctx_min": 512, "ctx_max": 8192},
        # the pages of 300 requests' rollouts behind their contexts
        {"name": "tables_300", "op": "tables", "kind": "chunk", "hq": 16, "hkv": 16, "d": 64, "lens": 32,
         "n": 300, "chunk": 1024, "ctx_min": 100, "ctx_max": 4000, "window": 0},
    ]


def draw(rng):
    def log(a, b):
        return max(a, min(b, round(math.exp(rng.uniform(math.log(a), math.log(b))))))

    def span(a, b):  # a range of lengths inside [a, b]
        x, y = sorted((log(a, b), log(a, b)))
        return {"ctx_min": x, "ctx_max": y}

    what = rng.choice(["decode", "decode", "decode", "shared", "chunk", "chunk", "prompt", "prompt", "roll", "latent",
                       "store", "store", "tables", "tables"])
    hq, hkv, d = rng.choice([(28, 4, 128), (16, 8, 128), (8, 2, 128), (8, 1, 128), (16, 16, 64), (16, 8, 64),
                             (28, 4, 64), (12, 12, 128)])
    case = {"op": "attend", "kind": what, "hq": hq, "hkv": hkv, "d": d, "lens": rng.randrange(1 << 30)}
    if what == "decode":
        case.update(n=log(1, 96), noalloc=rng.random() < 0.3, **span(1, 12000))
    elif what == "shared":
        case.update(n=log(4, 160), prefix=PAGE * log(16, 320), **span(20, 1500))
    elif what == "chunk":
        case.update(n=log(1, 200), chunk=rng.randint(2, 40), window=rng.choice([0, log(50, 4000)]), **span(30, 8000))
    elif what == "prompt":
        case.update(n=log(1, 16), **span(2, 4000))
    elif what == "roll":
        case.update(n=log(2, 60), prefix=PAGE * log(8, 128), frames=rng.randint(1, 3), frame=log(50, 256))
    elif what == "latent":
        case.update(n=log(1, 8), text=log(10, 400), image=log(200, 4096))
    else:  # store and tables: decoded tokens, chunks or prompts
        kind = rng.choice(["decode", "chunk", "prompt"])
        case.update(op=what, kind=kind)
        if kind == "decode":
            case.update(n=log(1, 300), **span(1, 8000))
        elif kind == "chunk":
            case.update(n=log(1, 200), chunk=log(2, 170), window=0, **span(1, 4000))
        else:
            case.update(n=log(1, 16), **span(1, 2100))
    if case["op"] == "attend" and "noalloc" not in case:
        case["noalloc"] = False
    return case


def _requests(case):
    """(new tokens, tokens with them) of every request."""
    rng, kind = random.Random(case["lens"]), case["kind"]
    drawn = [rng.randint(case.get("ctx_min", 0), case.get("ctx_max", 0)) for _ in range(case["n"])]
    if kind == "decode":
        return [(1, n) for n in drawn]
    if kind == "shared":
        return [(1, case["prefix"] + n) for n in drawn]
    if kind == "chunk":
        return [(case["chunk"], n + case["chunk"]) for n in drawn]
    if kind == "prompt":
        return [(n, n) for n in drawn]
    if kind == "latent":
        return [(case["text"] + case["image"],) * 2 for _ in drawn]
    new = case["frames"] * case["frame"]
    return [(new, case["prefix"] + new) for _ in drawn]


def _tables(case, reqs, rng):
    """Block table over a permuted pool with an eighth of its pages unused,
    and the unused pages."""
    shared = case.get("prefix", 0) // PAGE
    need = [-(-kv // PAGE) for _, kv in reqs]
    used = sum(need) - shared * (len(need) - 1)
    pool = used + used // 8 + 1
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((len(reqs), max(need)), -1, dtype=np.int32)
    at = shared
    for r, n in enumerate(need):
        table[r, :shared] = perm[:shared]
        table[r, shared:n] = perm[at:at + n - shared]
        at += n - shared
    return table, pool, perm[at:]


def _plan(case, reqs, width, pool):
    """The framework's plan of the step: its descriptors and mask segments."""
    from paper_2606_12688_amd import attn

    kind = case["kind"]
    seqs, masks, segs, at = [], [], [], 0
    for q, kv in reqs:
        if kind == "latent":
            own_segs = [(0, case["text"], attn.SEG_CAUSAL, 0), (case["text"], case["image"], attn.SEG_FULL, 0)]
        elif kind == "roll":
            own_segs = [(0, kv - q, attn.SEG_FULL, 0), (kv - q, q, attn.SEG_BLOCKS, case["frame"])]
        else:
            own_segs = [(0, kv, attn.SEG_CAUSAL, 0)]
        seqs.append((q, kv, at))
        masks.append((len(segs), len(own_segs), case.get("window", 0)))
        segs.extend(own_segs)
        at += q
    groups = [(list(range(len(reqs))), case["prefix"])] if kind == "shared" else None
    return attn.plan(case["hq"], case["hkv"], case["d"], "bf16", np.array(seqs, np.int32), np.array(masks, np.int32),
                     np.array(segs, np.int32), width, pool, prefix_groups=groups)


def _inputs(case, seed):
    reqs = _requests(case)
    table, pool, spare = _tables(case, reqs, np.random.default_rng(seed))
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    total = sum(q for q, _ in reqs)
    # some channels of keys and values are larger than others, the same ones in every token
    gain = torch.exp(0.5 * torch.randn((2, hkv, d), generator=g, device=DEV))

    def rows(n, which):
        return (torch.randn((n, hkv, d), generator=g, device=DEV) * gain[which]).bfloat16()

    lens = np.array(reqs, np.int32)
    s = {"case": case, "reqs": reqs, "table": table, "pool": pool, "total": total,
         "q_len": torch.from_numpy(lens[:, 0].copy()).to(DEV), "kv_len": torch.from_numpy(lens[:, 1].copy()).to(DEV),
         "block_table": torch.from_numpy(table).to(DEV)}
    if case["op"] == "tables":
        # pages of the cached tokens are there; the rest is on the free list, spare pages behind
        held = np.array([-(-(kv - q) // PAGE) for q, kv in reqs])
        col = np.arange(table.shape[1])
        new = (col >= held[:, None]) & (table >= 0)
        s["free_pages"] = torch.from_numpy(np.concatenate([table[new], spare])).to(DEV)
        s["block_table"] = torch.from_numpy(np.where(new, -1, table)).to(DEV)
        s["slots"] = torch.full((total,), -1, dtype=torch.int64, device=DEV)
        return s
    shape = (pool, hkv, 17 * d // 2)
    s["k_pages"], s["v_pages"] = (torch.empty(shape, dtype=torch.uint8, device=DEV) for _ in range(2))
    where = torch.arange(pool, device=DEV).repeat_interleave(PAGE)
    slot = torch.arange(PAGE, device=DEV).repeat(pool)
    _store(s["k_pages"], s["v_pages"], rows(pool * PAGE, 0), rows(pool * PAGE, 1), where, slot)
    if case["op"] == "store":
        s["k_new"], s["v_new"] = rows(total, 0), rows(total, 1)
        pages = [table[r, (kv - q) // PAGE:-(-kv // PAGE)] for r, (q, kv) in enumerate(reqs)]
        s["pages"] = torch.from_numpy(np.concatenate(pages)).to(DEV)
        s["k_out"], s["v_out"] = (torch.empty((len(s["pages"]), PAGE, hkv, d), dtype=torch.bfloat16, device=DEV)
                                  for _ in range(2))
        return s
    s["q"] = torch.randn((total, hq, d), generator=g, device=DEV).bfloat16()
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((total, hq), dtype=torch.float32, device=DEV)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2606_12688_amd import attn

        s["plan"] = _plan(case, s["reqs"], s["table"].shape[1], s["pool"])
        s["workspace"] = None if case.get("noalloc") else attn.workspace(s["plan"], DEV)
    return s


# ---- the plain form --------------------------------------------------------------

def _k_view(pages, d):
    """A K pool's codes as [pages, hkv, 4, 16 keys, d / 8] bytes."""
    p, h, _ = pages.shape
    return pages[:, :, :8 * d].view(p, h, 4, PAGE, d // 8)


def _v_view(pages, d):
    """A V pool's codes as [pages, hkv, 4, 16, 4 keys, d / 32] bytes."""
    p, h, _ = pages.shape
    return pages[:, :, :8 * d].view(p, h, 4, 16, 4, d // 32)


def _scale_view(pages, d):
    p, h, _ = pages.shape
    return pages[:, :, 8 * d:].view(p, h, d // 32, PAGE)


def _quantise(x):
    """bf16 rows [n, hkv, d] -> codes, two a byte, [n, hkv, d / 2], and scale bytes [n, hkv, d / 32]."""
    n, h, d = x.shape
    b = (((x.view(torch.int16) & 0x7fff).view(n, h, d // 32, 32).amax(-1).int() + 31) >> 7) - 2
    b = b.clamp(2, 252)
    y = x.float().abs().view(n, h, d // 32, 32) * torch.exp2(127.0 - b.double()).float()[..., None]
    code = ((y > 0.25).byte() + (y >= 0.75).byte() + (y > 1.25).byte() + (y >= 1.75).byte() + (y > 2.5).byte()
            + (y >= 3.5).byte() + (y > 5.0).byte())
    code = code.view(n, h, d) + 8 * torch.signbit(x).byte()
    return code[..., 0::2] + 16 * code[..., 1::2], b.byte()


def _store(k_pages, v_pages, k_new, v_new, page, slot):
    n, h, d = k_new.shape
    code, scale = _quantise(k_new)
    _k_view(k_pages, d)[page, :, :, slot] = code.view(n, h, 4, d // 8)
    _scale_view(k_pages, d)[page, :, :, slot] = scale
    code, scale = _quantise(v_new)
    _v_view(v_pages, d)[page, :, slot // 4, :, slot % 4] = code.view(n, h, 16, d // 32)
    _scale_view(v_pages, d)[page, :, :, slot] = scale


def _values(code, scale):
    """Codes [..., d / 2] and scale bytes [..., d / 32] as fp32 values [..., d]."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    table = torch.cat([table, -table])
    power = torch.exp2(torch.arange(256, device=DEV).double() - 127.0).float()
    x = torch.stack([table[(code & 15).int()], table[(code >> 4).int()]], -1)
    lead = code.shape[:-1]
    return (x.view(*lead, -1, 32) * power[scale.int()][..., None]).view(*lead, -1)


def _read(k_pages, v_pages, d, page, slot):
    """Cached keys and values at (page, slot), fp32 [..., hkv, d]."""
    k = _k_view(k_pages, d)[page, :, :, slot].flatten(-2)
    v = _v_view(v_pages, d)[page, :, slot // 4, :, slot % 4].flatten(-2)
    return (_values(k, _scale_view(k_pages, d)[page, :, :, slot]),
            _values(v, _scale_view(v_pages, d)[page, :, :, slot]))


def _row_of(s):
    """Request and index within it of every packed row."""
    first = torch.cumsum(s["q_len"], 0) - s["q_len"]
    n = s["q_len"].shape[0]
    req = torch.repeat_interleave(torch.arange(n, device=DEV), s["q_len"].long(), output_size=s["total"])
    return req, torch.arange(s["total"], device=DEV) - first[req]


def _interval(case, pos, kv):
    """Visible keys [lo, hi) of the row at position `pos` of a request of `kv` tokens."""
    if case["kind"] == "latent":
        hi = torch.where(pos < case["text"], pos + 1, kv)
    elif case["kind"] == "roll":
        p, f = case["prefix"], case["frame"]
        hi = torch.minimum(p + ((pos - p) // f + 1) * f, kv)
    else:
        hi = pos + 1
    w = case.get("window", 0)
    return ((pos - w + 1).clamp(min=0) if w else torch.zeros_like(pos)), hi


def _attend(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    n, group = len(s["reqs"]), hq // hkv
    q_len, kv_len, w = s["q_len"].long(), s["kv_len"].long(), case.get("window", 0)
    first = (kv_len - q_len - w + 1).clamp(min=0) if w else torch.zeros_like(kv_len)
    keys = max(kv - max(0, kv - q - w + 1) if w else kv for q, kv in s["reqs"])
    rows = max(q for q, _ in s["reqs"])
    # keys and values of every request, padded to the longest
    at = first[:, None] + torch.arange(keys, device=DEV)
    live = at < kv_len[:, None]
    at = torch.minimum(at, kv_len[:, None] - 1)
    page = s["block_table"].long().gather(1, at // PAGE)
    k, v = _read(s["k_pages"], s["v_pages"], d, page, at % PAGE)
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()
    # queries [n, hkv, group * rows, d]
    req, i = _row_of(s)
    q = torch.zeros((n, rows, hq, d), device=DEV)
    q[req, i] = s["q"].float()
    q = q.view(n, rows, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, group * rows, d)
    pos = (kv_len - q_len)[:, None] + torch.arange(rows, device=DEV)
    lo, hi = _interval(case, pos, kv_len[:, None])
    hidden = (at[:, None, :] < lo[:, :, None]) | (at[:, None, :] >= hi[:, :, None]) | ~live[:, None, :]
    x = torch.matmul(q, k).mul_(1.0 / math.sqrt(d)).view(n, hkv, group, rows, keys)
    x.masked_fill_(hidden[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top.masked_fill_(top == -math.inf, 0.0)  # rows of the padding
    x.sub_(top).exp_()
    total = x.sum(-1)
    out = torch.matmul(x.view(n, hkv, group * rows, keys), v).view(n, hkv, group, rows, d) / total[..., None]
    lse = top[..., 0] + total.log()
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(n, rows, hq, d)[req, i])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(n, rows, hq)[req, i])


def _targets(s):
    """Page and slot of every packed row."""
    req, i = _row_of(s)
    pos = (s["kv_len"] - s["q_len"])[req] + i
    return s["block_table"][req, pos // PAGE].long(), pos % PAGE


def _build_tables(s):
    held = (s["kv_len"] - s["q_len"] + PAGE - 1) // PAGE
    need = (s["kv_len"] + PAGE - 1) // PAGE
    off = torch.cumsum(need - held, 0) - (need - held)
    col = torch.arange(s["block_table"].shape[1], device=DEV)
    new = (col >= held[:, None]) & (col < need[:, None])
    pick = torch.where(new, off[:, None] + col - held[:, None], 0)
    s["block_table"].copy_(torch.where(new, s["free_pages"][pick], s["block_table"]))
    page, slot = _targets(s)
    s["slots"].copy_(torch.where(page >= 0, page * PAGE + slot, -1))


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2606_12688_amd import cache

        if op == "tables":
            cache.block_tables(s["plan"], s["free_pages"], s["block_table"], s["slots"])
        elif op == "store":
            cache.kv4_append(s["plan"], s["k_new"], s["v_new"], s["block_table"], s["k_pages"], s["v_pages"])
            cache.kv4_unpack(s["k_pages"], s["v_pages"], s["pages"], s["k_out"], s["v_out"])
        elif s["case"].get("noalloc"):
            cache.kv4_fwd_noalloc(s["plan"], s["q"], s["k_pages"], s["v_pages"], s["block_table"], s["out"], s["lse"])
        else:
            cache.kv4_fwd(s["plan"], s["q"], s["k_pages"], s["v_pages"], s["block_table"], s["out"], s["lse"],
                          s["workspace"])
    elif op == "tables":
        _build_tables(s)
    elif op == "store":
        _store(s["k_pages"], s["v_pages"], s["k_new"], s["v_new"], *_targets(s))
        slot = torch.arange(PAGE, device=DEV).expand(len(s["pages"]), PAGE)
        page = s["pages"].long()[:, None].expand(-1, PAGE)
        k, v = _read(s["k_pages"], s["v_pages"], s["case"]["d"], page, slot)
        s["k_out"].copy_(k)
        s["v_out"].copy_(v)
    else:
        _attend(s)
    if op == "tables":
        return {"block_table": s["block_table"], "slots": s["slots"]}
    if op == "store":
        return {"k": s["k_out"], "v": s["v_out"]}
    return {"out": s["out"], "lse": s["lse"]}


def _visible(case, q, kv):
    """Visible keys [lo, hi) of a request's rows, on the host."""
    lo, hi = _interval(case, torch.arange(kv - q, kv), torch.tensor(kv))
    return lo, hi


def work(case):
    reqs = _requests(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    new = sum(q for q, _ in reqs)
    if case["op"] == "tables":
        taken = sum(-(-kv // PAGE) - -(-(kv - q) // PAGE) for q, kv in reqs)
        return {"bytes": 8 * len(reqs) + 8 * taken + 8 * new, "flops": 0}
    record = 17 * d // 2  # bytes of a page and KV head, K or V
    if case["op"] == "store":
        pages = sum(-(-kv // PAGE) - (kv - q) // PAGE for q, kv in reqs)
        return {"bytes": 2 * hkv * (new * 2 * d + new * record // PAGE + pages * (record + 32 * d)), "flops": 0}
    pairs, cached = 0, 0
    for r, (q, kv) in enumerate(reqs):
        lo, hi = _visible(case, q, kv)
        pairs += int((hi - lo).sum())
        cached += int(hi[-1]) - max(int(lo[0]), case.get("prefix", 0) if r else 0)
    return {"bytes": new * hq * (4 * d + 4) + 2 * hkv * (cached * record // PAGE), "flops": 4 * d * hq * pairs}


# ---- the definition in 64 bits -----------------------------------------------------

def _decode64(pool, d, where_code):
    """Pool -> float64 [pages, 16, hkv, d]; ``where_code(slot, dim)`` is a code's nibble in a record."""
    slot, dim = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    nibble = torch.from_numpy(where_code(slot, dim)).to(pool.device)
    scale = torch.from_numpy(8 * d + dim // 32 * PAGE + slot).to(pool.device)
    code = (pool[:, :, nibble // 2].int() >> (4 * (nibble % 2)).int()) & 15
    e, m = (code >> 1) & 3, code & 1
    size = torch.where(e == 0, 0.5 * m.double(), (1 + 0.5 * m.double()) * 2.0 ** (e.double() - 1))
    x = torch.where(code >= 8, -size, size) * 2.0 ** (pool[:, :, scale].double() - 127)
    return x.permute(0, 2, 1, 3)


def _k_nibble(d):
    return lambda slot, dim: (dim // (d // 4) * PAGE + slot) * (d // 4) + dim % (d // 4)


def _v_nibble(d):
    return lambda slot, dim: ((slot // 4 * 16 + dim // (d // 16)) * 4 + slot % 4) * (d // 16) + dim % (d // 16)


def _rounded64(x):
    """The values that rows [n, hkv, d] stand for once stored."""
    n, h, d = x.shape
    y = x.double().view(n, h, d // 32, 32)
    mant, exp = torch.frexp(y.abs().amax(-1))  # amax = mant 2^exp, 0.5 <= mant < 1
    e = (exp - 3 + (mant > 0.875)).clamp(-125, 125)  # the smallest e with amax <= 7 * 2^e
    unit = 2.0 ** e.double()[..., None]
    size = (y / unit).abs().clamp(max=6.0)
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0)).double()
    return (torch.sign(y) * torch.round(size / step) * step * unit).view(n, h, d)


def exact(case, seed):
    s = _inputs(case, seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "tables":
        table, slots = s["block_table"].cpu().numpy(), []
        free = iter(s["free_pages"].tolist())
        for r, (q, kv) in enumerate(s["reqs"]):
            for page in range(-(-(kv - q) // PAGE), -(-kv // PAGE)):
                table[r, page] = next(free)
            pos = np.arange(kv - q, kv)
            slots.append(table[r, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE)
        return {"block_table": torch.from_numpy(table), "slots": torch.from_numpy(np.concatenate(slots))}
    if case["op"] == "store":
        got, at = {}, 0
        new = {"k": _rounded64(s["k_new"]), "v": _rounded64(s["v_new"])}
        for name, where in (("k", _k_nibble(d)), ("v", _v_nibble(d))):
            got[name] = _decode64(s[name + "_pages"][s["pages"].long()], d, where)
        first = 0  # a request's first touched page in the list
        for q, kv in s["reqs"]:
            pos = torch.arange(kv - q, kv, device=DEV)
            for name in got:
                got[name][first + pos // PAGE - (kv - q) // PAGE, pos % PAGE] = new[name][at:at + q]
            at += q
            first += -(-kv // PAGE) - (kv - q) // PAGE
        return got
    group = hq // hkv
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    at = 0
    for r, (q, kv) in enumerate(s["reqs"]):
        lo, hi = (x.to(DEV) for x in _visible(case, q, kv))
        a = int(lo[0])
        pos = torch.arange(a, int(hi[-1]), device=DEV)
        pages = s["block_table"][r, a // PAGE:-(-int(hi[-1]) // PAGE)].long()
        skip = a % PAGE
        k = _decode64(s["k_pages"][pages], d, _k_nibble(d)).flatten(0, 1)[skip:skip + len(pos)]
        v = _decode64(s["v_pages"][pages], d, _v_nibble(d)).flatten(0, 1)[skip:skip + len(pos)]
        hidden = (pos < lo[:, None]) | (pos >= hi[:, None])
        for h in range(hkv):
            heads = slice(h * group, (h + 1) * group)
            qs = s["q"][at:at + q, heads].double().transpose(0, 1).reshape(group * q, d)
            x = torch.matmul(qs, k[:, h].t().contiguous()).view(group, q, -1)
            x.div_(math.sqrt(d)).masked_fill_(hidden, -math.inf)
            ls = torch.logsumexp(x, -1)
            x.sub_(ls[..., None]).exp_()
            o = torch.matmul(x.view(group * q, -1), v[:, h].contiguous())
            out[at:at + q, heads] = o.view(group, q, d).transpose(0, 1)
            lse[at:at + q, heads] = ls.transpose(0, 1)
        at += q
    return {"out": out, "lse": lse}
