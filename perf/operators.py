"""The operators of the block-structured 8-bit KV cache, as cases that can be
timed and compared: a plain form in elementary torch operations, and the
library's calls.

The cache holds K and V as e4m3 with one fp32 scale for each block of tokens
and kv head.  Four operators work on it:

* "store": quantises new keys and values (a prompt's, or a step's single
  tokens) into the cache; a block's scale is the smallest power of two that
  holds its largest element, and only grows while the block fills.  The
  blocks' key bounds are updated with it.
* "bounds": the same key bounds (elementwise minimum and maximum of a block's
  keys) of a bf16 or fp32 cache.
* "select": the blocks of largest upper bound max_h sum_d max(q kmin, q kmax)
  (ties to the lower block), and the set sink U blocks U window.
* "dense", "sparse", "reuse": decode attention over the 8-bit cache: over all
  its tokens, over an index set, over a set and the tokens since its anchor.

Keys, queries and bounds of "select" lie on the grid j/16, |j| <= 255, on which
every score is exact in fp32, so that the chosen blocks are the same whatever
the order of the sums.
"""

import math

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
EXP_MIN = -100   # exponent of the smallest block scale


def _case(name, op, **kw):
    c = {"name": name, "op": op, "dtype": "bf16", "batch": 1, "hq": 32, "hkv": 8, "d": 128,
         "n": 4096, "ragged": False, "paged": False, "block": 16}
    if op in ("store", "bounds"):
        c["new"] = 1
    if op in ("select", "sparse", "reuse"):
        c.update(k=256, sink=4, window=64)
    if op == "reuse":
        c["tail"] = 3
    c.update(kw)
    return c


def listed():
    return [
        # the step's token of every sequence of a serving batch, one layer: a
        # latency, as every layer makes this call at every step
        _case("store-step-b64", "store", batch=64, n=16383, ragged=True, paged=True),
        # a 16k prompt of one sequence
        _case("store-prompt-16k", "store", n=16384, new=16384, paged=True),
        # chunks of three fp32 prompts, 64-dim heads, that begin and end inside
        # blocks
        _case("store-chunk-f32", "store", dtype="f32", batch=3, hq=12, hkv=4, d=64, n=2035,
              ragged=True, new=777, block=32),
        # the key bounds of a bf16 cache after one step of a serving batch
        _case("bounds-step-b64", "bounds", batch=64, n=16383, ragged=True, paged=True),
        # and after a 32k prompt, blocks of 64
        _case("bounds-prompt-32k", "bounds", n=32768, new=32768, block=64),
        # the smallest selection: one short fp32 sequence
        _case("select-1k-f32", "select", dtype="f32", hq=4, hkv=4, d=64, n=1025, k=64, window=32),
        # one paged sequence at 128k: 8 rows of 8192 blocks
        _case("select-128k-paged", "select", n=131072, k=2048, window=256, paged=True),
        # the throughput sweep's largest batch, mixed lengths up to 16k
        _case("select-b64-16k", "select", batch=64, n=16384, ragged=True, k=768, window=128),
        # the smallest attention: one short sequence with fp32 queries
        _case("dense-1k-f32", "dense", dtype="f32", hq=4, hkv=4, d=64, n=1025),
        # LLaMA-2-7B-shaped heads at 4k, blocks of 64
        _case("dense-mha-4k", "dense", batch=8, hkv=32, n=4096, block=64),
        # the throughput sweep's largest batch, mixed lengths up to 16k
        _case("dense-b64-16k", "dense", batch=64, n=16384, ragged=True, paged=True),
        # the selected blocks of a paged 128k sequence
        _case("sparse-128k-paged", "sparse", n=131072, k=2048, window=256, paged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "store", "bounds", "select", "select", "dense", "dense", "sparse",
                     "sparse", "reuse"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 8, 32])
    hq = hkv * (1 if hkv == 32 else rng.choice([1, 2, 4, 4, 5, 8, 16]))
    c = _case("drawn", op, dtype="f32" if rng.random() < 0.25 else "bf16", hq=hq, hkv=hkv, d=d,
              ragged=rng.random() < 0.6, paged=rng.random() < 0.5,
              block=rng.choice([16, 16, 32, 64, 128]))
    del c["name"]
    c["n"] = _log(rng, 1 if rng.random() < 0.2 else 200, 131072)
    c["batch"] = max(1, min(_log(rng, 1, 64), (1 << 29) // (hkv * d * c["n"])))
    if op in ("store", "bounds"):
        c["new"] = 1 if rng.random() < 0.4 else _log(rng, 1, c["n"])
        if c["batch"] * c["new"] * hkv * d > 1 << 25:
            c["new"] = max(1, (1 << 25) // (c["batch"] * hkv * d))
    if op in ("select", "sparse", "reuse"):
        c.update(k=max(1, min(4096, c["n"] // rng.choice([4, 8, 16, 64]))),
                 sink=rng.choice([0, 4, 16, 30]), window=rng.choice([0, 32, 64, 255]))
    if op == "reuse":
        c["tail"] = rng.choice([0, 1, 3, 7])
    return c


# ---- inputs ------------------------------------------------------------------

def _lens(c):
    """Lengths of the sequences: n, or with ragged between n / 2 and n."""
    n, B = c["n"], c["batch"]
    if not c["ragged"]:
        return [n] * B
    return [max(1, n - (b * 40503 % (n // 2 + 1))) for b in range(B)]


def _new_lens(c):
    """New tokens of each sequence: with ragged, some have fewer or none."""
    if not c["ragged"] or c["new"] == 1:
        return [min(c["new"], n) for n in _lens(c)]
    return [min(n, c["new"] - (b * 271 % (c["new"] + 1))) for b, n in enumerate(_lens(c))]


def _blocks(c):
    return -(-c["n"] // c["block"])


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _grid(x):
    return (x * 16).round_().clamp_(-255, 255).div_(16)


def _exponent(amax):
    """Smallest e with amax <= 448 * 2^e, at least EXP_MIN."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(amax > 0, e, EXP_MIN).clamp_(min=EXP_MIN)


def _power(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _row_shape(c):
    """Leading shape of the cache's blocks: [.., blocks ..], as the library lays them out."""
    nb = _blocks(c)
    return (c["batch"] * nb, c["hkv"]) if c["paged"] else (c["batch"], c["hkv"], nb)


def _cache_shape(c):
    nb, bs = _blocks(c), c["block"]
    if c["paged"]:
        return (c["batch"] * nb, c["hkv"], bs, c["d"])
    return (c["batch"], c["hkv"], nb * bs, c["d"])


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    B, nb, bs, d, dt = c["batch"], _blocks(c), c["block"], c["d"], _type(c)
    s = {"c": c, "scale": 1 / math.sqrt(d), "n_max": c["n"]}
    s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device=DEV)
    s["table"] = None
    if c["paged"]:
        perm = torch.randperm(B * nb, generator=g, device=DEV)
        s["table"] = perm.reshape(B, nb).to(torch.int32)
    rows = math.prod(_row_shape(c))
    outliers = 1 + 3 * (randn(d) > 1.5)   # some dimensions of the keys are large

    def quantised(wide):
        x8 = torch.empty(rows, bs, d, dtype=torch.uint8, device=DEV)
        sc = torch.empty(rows, device=DEV)
        for lo in range(0, rows, 1 << 15):   # in parts: the fp32 form is four times as large
            x = randn(min(rows, lo + (1 << 15)) - lo, bs, d) * wide
            e = _power(_exponent(x.abs().amax(dim=(1, 2))))
            x8[lo:lo + len(x)] = (x / e[:, None, None]).to(E4M3).view(torch.uint8)
            sc[lo:lo + len(x)] = e
        return x8.view(E4M3).view(_cache_shape(c)), sc.view(_row_shape(c))

    if c["op"] == "select":   # the cache whose blocks are chosen; its keys are not read
        s["k8"], s["v8"] = (torch.empty(_cache_shape(c), dtype=E4M3, device=DEV) for _ in "kv")
        s["ks"], s["vs"] = (torch.ones(_row_shape(c), device=DEV) for _ in "kv")
    elif c["op"] != "bounds":
        s["k8"], s["ks"] = quantised(outliers)
        s["v8"], s["vs"] = quantised(1.0)
    if c["op"] in ("store", "bounds", "select"):
        mid = 1.2 + 0.3 * math.log2(bs / 8)   # about the extremes of bs normal values
        x = (mid + 0.5 * randn(rows, d)) * outliers
        y = (-mid + 0.5 * randn(rows, d)) * outliers
        s["kmin"] = _grid(torch.minimum(x, y)).to(dt).view(*_row_shape(c), d)
        s["kmax"] = _grid(torch.maximum(x, y)).to(dt).view(*_row_shape(c), d)
    if c["op"] == "store":
        s["k_new"] = _grid(randn(B, c["hkv"], c["new"], d) * outliers).to(dt)
        s["v_new"] = randn(B, c["hkv"], c["new"], d).to(dt)
        s["new_lens"] = torch.tensor(_new_lens(c), dtype=torch.int32, device=DEV)
    elif c["op"] == "bounds":
        s["k"] = _grid(randn(*_cache_shape(c)) * outliers).to(dt)
        s["new_lens"] = torch.tensor(_new_lens(c), dtype=torch.int32, device=DEV)
    else:
        s["q"] = _grid(1.5 * randn(B, c["hq"], d)).to(dt)
    if c["op"] == "select":
        kb, cap = _select_caps(c)
        s["blk"] = torch.zeros(B, c["hkv"], max(1, kb), dtype=torch.int32, device=DEV)
        s["blk_len"] = torch.zeros(B, c["hkv"], dtype=torch.int32, device=DEV)
        s["set"] = torch.zeros(B, c["hkv"], max(1, cap), dtype=torch.int32, device=DEV)
        s["set_len"] = torch.zeros(B, c["hkv"], dtype=torch.int32, device=DEV)
    if c["op"] in ("sparse", "reuse"):
        s["anchor"] = (s["lens"] - c.get("tail", 0)).clamp_(min=0)
        s["set"], s["set_len"] = _block_sets(c, s["anchor"], torch.rand(B, c["hkv"], nb, generator=g, device=DEV))
    if c["op"] in ("dense", "sparse", "reuse"):
        s["out"] = torch.zeros(B, c["hq"], d, device=DEV)
        s["lse"] = torch.zeros(B, c["hq"], device=DEV)
    if own:
        _handles(s)
    return s


def _select_caps(c):
    """Most blocks a row takes, and the size of its set."""
    n, bs = c["n"], c["block"]
    se = min(c["sink"], n)
    ws = max(se, n - c["window"])
    cand = -(-ws // bs) - se // bs if ws > se else 0
    kb = min(-(-c["k"] // bs), cand)
    return kb, min(n, c["sink"] + kb * bs + c["window"])


def _block_sets(c, n, score):
    """The sets sink U best blocks U window of random scores, at lengths n."""
    bs, (kb, cap) = c["block"], _select_caps(c)
    _, chosen = _top_blocks(c, n, score)
    return _members(c, n, chosen, max(1, cap + c.get("tail", 0)))


# ---- the plain forms ---------------------------------------------------------

def _block_ids(s, j):
    """Flat ids of the blocks j [B, x] of every kv head: [B, Hkv, x]."""
    c = s["c"]
    B, Hkv, nb = c["batch"], c["hkv"], _blocks(c)
    heads = torch.arange(Hkv, device=DEV)
    if c["paged"]:
        return s["table"].long().gather(1, j)[:, None, :] * Hkv + heads[None, :, None]
    unit = torch.arange(B, device=DEV)[:, None] * Hkv + heads
    return unit[:, :, None] * nb + j[:, None, :]


def _touched(s):
    """Blocks that hold new tokens [B, x] (clamped, so that repeats are whole
    copies), their positions [B, x, bs], and which of these are new and old."""
    c, n, bs = s["c"], s["lens"].long(), s["c"]["block"]
    lo = n - s["new_lens"].long()
    last = (n - 1).clamp(min=0) // bs
    j = lo[:, None] // bs + torch.arange(-(-c["new"] // bs) + 1, device=DEV)
    j = torch.minimum(j, last[:, None])
    pos = j[:, :, None] * bs + torch.arange(bs, device=DEV)
    return j, pos, (pos >= lo[:, None, None]) & (pos < n[:, None, None]), pos < lo[:, None, None]


def _store_one(s, x8, sc, new, ids, pos, is_new, is_old):
    c, bs, d = s["c"], s["c"]["block"], s["c"]["d"]
    raw, flat = x8.view(torch.uint8).view(-1, bs, d), sc.view(-1)
    before, s_old = raw[ids], flat[ids]                       # [B, Hkv, x, bs, d], [B, Hkv, x]
    t = (pos - (s["lens"] - s["new_lens"])[:, None, None]).clamp(0, c["new"] - 1)
    x = new[torch.arange(c["batch"], device=DEV)[:, None, None], :, t]   # [B, x, bs, Hkv, d]
    x = x.permute(0, 3, 1, 2, 4).float()
    is_new, is_old = is_new[:, None, :, :, None], is_old[:, None, :, :, None]
    need = _power(_exponent((x.abs() * is_new).amax(dim=(3, 4))))
    s_new = torch.where(is_old.any(dim=3)[..., 0], torch.maximum(s_old, need), need)
    s_new = torch.where(is_new.any(dim=3)[..., 0], s_new, s_old)
    old = before.view(E4M3).float() * s_old[..., None, None]
    y = (torch.where(is_new, x, old) / s_new[..., None, None]).to(E4M3).view(torch.uint8)
    raw[ids] = torch.where(is_new | is_old, y, before)
    flat[ids] = s_new


def _store(s):
    d = s["c"]["d"]
    j, pos, is_new, is_old = _touched(s)
    ids = _block_ids(s, j)
    _store_one(s, s["k8"], s["ks"], s["k_new"], ids, pos, is_new, is_old)
    _store_one(s, s["v8"], s["vs"], s["v_new"], ids, pos, is_new, is_old)
    t = (pos - (s["lens"] - s["new_lens"])[:, None, None]).clamp(0, s["c"]["new"] - 1)
    x = s["k_new"][torch.arange(s["c"]["batch"], device=DEV)[:, None, None], :, t]
    x = x.permute(0, 3, 1, 2, 4)
    m, fresh = is_new[:, None, :, :, None], ~is_old.any(dim=2)[:, None, :, None]
    changed = is_new.any(dim=2)[:, None, :, None]
    lo, hi = s["kmin"].view(-1, d), s["kmax"].view(-1, d)
    mn, mx = x.masked_fill(~m, math.inf).amin(3), x.masked_fill(~m, -math.inf).amax(3)
    mn = torch.where(fresh, mn, torch.minimum(mn, lo[ids]))
    mx = torch.where(fresh, mx, torch.maximum(mx, hi[ids]))
    lo[ids] = torch.where(changed, mn, lo[ids])
    hi[ids] = torch.where(changed, mx, hi[ids])


def _bounds(s):
    bs, d = s["c"]["block"], s["c"]["d"]
    j, pos, is_new, is_old = _touched(s)
    ids = _block_ids(s, j)
    x = s["k"].view(-1, bs, d)[ids]
    m, changed = (is_new | is_old)[:, None, :, :, None], is_new.any(dim=2)[:, None, :, None]
    lo, hi = s["kmin"].view(-1, d), s["kmax"].view(-1, d)
    lo[ids] = torch.where(changed, x.masked_fill(~m, math.inf).amin(3), lo[ids])
    hi[ids] = torch.where(changed, x.masked_fill(~m, -math.inf).amax(3), hi[ids])


def _top_blocks(c, n, score):
    """Blocks a row may take, of scores [B, Hkv, nb]: its best first, and a
    mask of the chosen ones."""
    bs, n = c["block"], n.long()[:, None, None]
    se = n.clamp(max=c["sink"])
    ws = torch.maximum(se, n - c["window"])
    j = torch.arange(score.shape[2], device=DEV)
    cand = (j >= se // bs) & (j < (ws + bs - 1) // bs) & (ws > se)
    score = score.masked_fill(~cand, -math.inf)
    order = torch.sort(score, dim=2, descending=True, stable=True).indices
    kb = torch.minimum(cand.sum(dim=2, keepdim=True),
                       torch.full_like(se, -(-c["k"] // bs)))
    rank = torch.empty_like(order).scatter_(2, order, j.expand_as(order).contiguous())
    return kb[..., 0], rank < kb


def _compact(mask, cap):
    """Indices of the true entries of mask [.., x], ascending, in rows of cap
    (zeros behind them), and their number."""
    at = torch.cumsum(mask, dim=-1) - 1
    to = torch.where(mask & (at < cap), at, cap)
    src = torch.arange(mask.shape[-1], device=DEV, dtype=torch.int32).expand(mask.shape)
    out = torch.zeros(*mask.shape[:-1], cap + 1, dtype=torch.int32, device=DEV)
    out.scatter_(-1, to, src.contiguous())
    return out[..., :cap].contiguous(), mask.sum(dim=-1).clamp(max=cap).to(torch.int32)


def _members(c, n, chosen, cap):
    bs, n = c["block"], n.long()[:, None, None]
    se = n.clamp(max=c["sink"])
    ws = torch.maximum(se, n - c["window"])
    pos = torch.arange(chosen.shape[2] * bs, device=DEV)
    member = chosen.repeat_interleave(bs, dim=2) | (pos < se) | (pos >= ws)
    return _compact(member & (pos < n), cap)


def _select(s):
    c = s["c"]
    B, Hkv, nb, d, G = c["batch"], c["hkv"], _blocks(c), c["d"], c["hq"] // c["hkv"]
    ids = _block_ids(s, torch.arange(nb, device=DEV).expand(B, nb))
    lo, hi = s["kmin"].view(-1, d)[ids].float(), s["kmax"].view(-1, d)[ids].float()
    q = s["q"].float().view(B, Hkv, G, d)
    sc = torch.matmul(hi, q.clamp(min=0).transpose(2, 3).contiguous())
    sc = sc + torch.matmul(lo, q.clamp(max=0).transpose(2, 3).contiguous())
    _, chosen = _top_blocks(c, s["lens"], sc.amax(dim=3))
    blk, blk_len = _compact(chosen, s["blk"].shape[2])
    sets, set_len = _members(c, s["lens"], chosen, s["set"].shape[2])
    return {"blocks": blk, "blocks_len": blk_len, "set": sets, "set_len": set_len}


def _attend(s, k, v, ks, vs, valid):
    """k, v [B, Hkv, x, d] e4m3, scales and validity [B, Hkv, x]."""
    c = s["c"]
    B, Hkv, G, d = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["d"]
    q = s["q"].float().view(B, Hkv, G, d)
    k = k.float().mul_(ks[..., None])
    x = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    x = x.masked_fill(~valid[:, :, None, :], -math.inf)
    m = x.amax(dim=3, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(dim=3, keepdim=True)
    del k
    out = torch.matmul(p, v.float().mul_(vs[..., None])) / l
    return {"out": out.reshape(B, Hkv * G, d), "lse": (m + torch.log(l)).reshape(B, Hkv * G)}


def _dense(s):
    c = s["c"]
    B, Hkv, nb, bs, d = c["batch"], c["hkv"], _blocks(c), c["block"], c["d"]
    ids = _block_ids(s, torch.arange(nb, device=DEV).expand(B, nb))

    def rows(x8):
        return x8.view(torch.uint8).view(-1, bs, d)[ids].view(E4M3).view(B, Hkv, nb * bs, d)

    def scales(x):
        return x.view(-1)[ids].repeat_interleave(bs, dim=2)

    valid = (torch.arange(nb * bs, device=DEV) < s["lens"][:, None])[:, None, :].expand(B, Hkv, -1)
    return _attend(s, rows(s["k8"]), rows(s["v8"]), scales(s["ks"]), scales(s["vs"]), valid)


def _sparse(s):
    c = s["c"]
    bs, d = c["block"], c["d"]
    pos = s["set"].long()
    valid = torch.arange(pos.shape[2], device=DEV) < s["set_len"][..., None]
    if c["op"] == "reuse":
        n0 = s["anchor"].long()[:, None, None]
        tail = (n0 + torch.arange(c["tail"], device=DEV)).expand(-1, c["hkv"], -1)
        pos = torch.cat([pos, tail], dim=2)
        valid = torch.cat([valid & (s["set"] < n0), tail < s["lens"].long()[:, None, None]], dim=2)
    pos = torch.where(valid, pos, 0)
    nb, heads = _blocks(c), torch.arange(c["hkv"], device=DEV)[None, :, None]
    if c["paged"]:
        t = s["table"].long()[:, None, :].expand(-1, c["hkv"], -1)
        ids = t.gather(2, pos // bs) * c["hkv"] + heads
    else:
        ids = (torch.arange(c["batch"], device=DEV)[:, None, None] * c["hkv"] + heads) * nb + pos // bs

    def rows(x8):
        return x8.view(torch.uint8).view(-1, d)[ids * bs + pos % bs].view(E4M3)

    return _attend(s, rows(s["k8"]), rows(s["v8"]), s["ks"].view(-1)[ids], s["vs"].view(-1)[ids], valid)


def _state(s):
    if s["c"]["op"] == "bounds":
        return {"kmin": s["kmin"], "kmax": s["kmax"]}
    return {"k": s["k8"], "v": s["v8"], "k_scale": s["ks"], "v_scale": s["vs"], "kmin": s["kmin"],
            "kmax": s["kmax"]}


# ---- the library -------------------------------------------------------------

def _handles(s):
    """Descriptors, budget and workspace, as a serving loop keeps them."""
    from paper_2602_08329_amd import binding as B
    c = s["c"]
    if c["op"] == "bounds":
        s["kv"] = B.KV(s["k"], s["k"], s["lens"], s["n_max"], c["hq"], s["table"])
    else:
        s["kv"] = B.QuantKV(s["k8"], s["v8"], s["ks"], s["vs"], s["lens"], s["n_max"], c["hq"],
                            s["table"], dtype=_type(c))
    if c["op"] == "select":
        s["p"] = B.params(k=c["k"], sink=c["sink"], window=c["window"])
    if c["op"] in ("store", "bounds", "select"):
        s["bounds"] = B.BlockBounds(s["kv"], s["kmin"], s["kmax"])
    if c["op"] == "select":
        s["ws"] = B.workspace(B.prhs_block_workspace_size(s["kv"], s["bounds"]), DEV)
    if c["op"] == "dense":
        s["ws"] = B.workspace(B.prhs_workspace_size(B.PRHS_OP_QUANT_DENSE_ATTN, s["kv"]), DEV)
    if c["op"] in ("sparse", "reuse"):
        s["ws"] = B.workspace(B.prhs_workspace_size(B.PRHS_OP_QUANT_SPARSE_ATTN, s["kv"], None,
                                                    s["set"].shape[2]), DEV)


def _own(s):
    from paper_2602_08329_amd import binding as B
    op = s["c"]["op"]
    if op == "store":
        B.prhs_quant_store(s["kv"], s["k_new"], s["v_new"], s["new_lens"], s["bounds"])
        return _state(s)
    if op == "bounds":
        B.prhs_block_bounds(s["kv"], s["bounds"], s["c"]["new"], s["new_lens"])
        return _state(s)
    if op == "select":
        B.prhs_block_select(s["kv"], s["q"], s["p"], s["bounds"], s["blk"], s["blk_len"], s["set"],
                            s["set_len"], s["ws"])
        return {"blocks": s["blk"], "blocks_len": s["blk_len"], "set": s["set"],
                "set_len": s["set_len"]}
    if op == "dense":
        B.prhs_quant_dense_decode_attn(s["kv"], s["q"], s["scale"], s["out"], s["lse"], s["ws"])
    elif op == "sparse":
        B.prhs_quant_sparse_decode_attn(s["kv"], s["q"], s["set"], s["set_len"], s["scale"],
                                        s["out"], s["lse"], s["ws"])
    else:
        B.prhs_quant_reuse_decode_attn(s["kv"], s["q"], s["set"], s["set_len"], s["anchor"],
                                       s["scale"], s["out"], s["lse"], s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    op = state["c"]["op"]
    if op == "store":
        _store(state)
        return _state(state)
    if op == "bounds":
        _bounds(state)
        return _state(state)
    if op == "select":
        return _select(state)
    return _dense(state) if op == "dense" else _sparse(state)


def work(case):
    c = case
    e, d, hkv, bs = 4 if c["dtype"] == "f32" else 2, c["d"], c["hkv"], c["block"]
    lens, G = _lens(c), c["hq"] // c["hkv"]
    if c["op"] in ("store", "bounds"):
        new = _new_lens(c)
        # a block counts where it gets a token; the tokens before it in the
        # block are read for their bounds, or because its scale may grow
        blocks = sum(-(-n // bs) - (n - t) // bs for n, t in zip(lens, new) if t)
        old = sum((n - t) % bs for n, t in zip(lens, new) if t)
        if c["op"] == "bounds":
            return {"bytes": hkv * ((sum(new) + old) * d * e + 2 * blocks * d * e),
                    "flops": 2 * hkv * sum(new) * d}
        open_ = sum(1 for n, t in zip(lens, new) if t and (n - t) % bs)
        return {"bytes": hkv * (sum(new) * 2 * d * (e + 1) + 8 * (blocks + open_)
                                + 2 * (blocks + open_) * d * e),
                "flops": 6 * hkv * sum(new) * d}
    q = c["batch"] * c["hq"] * d * e
    if c["op"] == "select":
        byte, flop = q, 0
        for n in lens:
            se = min(c["sink"], n)
            ws = max(se, n - c["window"])
            cand = -(-ws // bs) - se // bs if ws > se else 0
            rows = min(n, c["sink"] + min(-(-c["k"] // bs), cand) * bs + c["window"])
            byte += hkv * (cand * 2 * d * e + rows * 4)
            flop += hkv * cand * 4 * d * G
        return {"bytes": byte, "flops": flop}
    rows = lens
    if c["op"] != "dense":
        rows = [min(n, _select_caps({**c, "n": n})[1]) for n in lens]
    listed_ = 0 if c["op"] == "dense" else 4 * sum(rows)
    return {"bytes": hkv * (sum(rows) * (2 * d + 8 / bs) + listed_) + q + c["batch"] * c["hq"] * (d + 1) * 4,
            "flops": 4 * c["hq"] * d * sum(rows)}


# ---- the definition in 64 bits -------------------------------------------------

def _id(s, b, g, j):
    """The block of the flat cache that holds block j of sequence b and head g."""
    c = s["c"]
    if c["paged"]:
        return s["table"][b, j].long() * c["hkv"] + g
    return (b * c["hkv"] + g) * _blocks(c) + j


def _exact_store(s):
    c = s["c"]
    bs, d, g = c["block"], c["d"], torch.arange(c["hkv"], device=DEV)[:, None]
    res = {k: s[n].double() for k, n in (("k_scale", "ks"), ("v_scale", "vs"), ("kmin", "kmin"),
                                         ("kmax", "kmax"))}
    res |= {"k": s["k8"].double(), "v": s["v8"].double()}
    for b, (n, t) in enumerate(zip(_lens(c), _new_lens(c))):
        if not t:
            continue
        j0, j1, lo = (n - t) // bs, -(-n // bs), n - t
        ids = _id(s, b, g, torch.arange(j0, j1, device=DEV)).reshape(-1)
        pos = torch.arange(j0 * bs, j1 * bs, device=DEV)
        blank = torch.zeros(c["hkv"], len(pos), d, dtype=torch.float64, device=DEV)
        for key, new, mn, mx in (("k", "k_new", "kmin", "kmax"), ("v", "v_new", None, None)):
            x8, sc = res[key].view(-1, bs, d), res[key + "_scale"].view(-1)
            x = blank.clone()
            x[:, (pos >= lo) & (pos < n)] = s[new][b, :, :t].double()
            fresh = (pos.view(-1, bs)[:, 0] >= lo).repeat(c["hkv"])
            top = x.view(-1, bs * d).abs().amax(1)
            # powers of two from the smallest upwards, until the block fits
            e = torch.full_like(top, EXP_MIN)
            e = torch.maximum(e, torch.ceil(torch.log2(top / 448).clamp(min=EXP_MIN)))
            e = torch.where(448 * torch.exp2(e - 1) >= top, (e - 1).clamp(min=EXP_MIN), e)
            e = torch.where(448 * torch.exp2(e) < top, e + 1, e)
            scale = torch.where(fresh, torch.exp2(e), torch.maximum(torch.exp2(e), sc[ids]))
            val = x + (pos < lo)[:, None] * (x8[ids] * sc[ids][:, None, None]).view_as(x)
            y = val.view(-1, bs, d) / scale[:, None, None]
            # nearest of 8 steps in each power of two, ties to even, smallest step 2^-9
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
            y = torch.round(y / step) * step
            keep = (pos >= n).view(-1, bs).repeat(c["hkv"], 1)
            x8[ids] = torch.where(keep[:, :, None], x8[ids], y)
            sc[ids] = scale
            if mn is not None:
                inside = ((pos >= lo) & (pos < n)).view(-1, bs).repeat(c["hkv"], 1)[:, :, None]
                xb = x.view(-1, bs, d)
                low = torch.where(inside, xb, math.inf).amin(1)
                high = torch.where(inside, xb, -math.inf).amax(1)
                f = fresh[:, None]
                a, z = res[mn].view(-1, d), res[mx].view(-1, d)
                a[ids], z[ids] = (torch.where(f, low, torch.minimum(low, a[ids])),
                                  torch.where(f, high, torch.maximum(high, z[ids])))
    return res


def _exact_bounds(s):
    c = s["c"]
    bs, d = c["block"], c["d"]
    lo, hi = s["kmin"].double(), s["kmax"].double()
    for b, (n, t) in enumerate(zip(_lens(c), _new_lens(c))):
        for g in range(c["hkv"] if t else 0):
            ids = _id(s, b, g, torch.arange((n - t) // bs, -(-n // bs), device=DEV))
            x = s["k"].view(-1, bs, d)[ids].double()
            past = torch.arange(len(ids) * bs, device=DEV) >= n - (n - t) // bs * bs
            past = past.view(-1, bs, 1)
            lo.view(-1, d)[ids] = torch.where(past, math.inf, x).amin(1)
            hi.view(-1, d)[ids] = torch.where(past, -math.inf, x).amax(1)
    return {"kmin": lo, "kmax": hi}


def _exact_select(s):
    c = s["c"]
    bs, d, G = c["block"], c["d"], c["hq"] // c["hkv"]
    res = {k: torch.zeros_like(s[n]) for k, n in (("blocks", "blk"), ("blocks_len", "blk_len"),
                                                  ("set", "set"), ("set_len", "set_len"))}
    for b, n in enumerate(_lens(c)):
        se = min(c["sink"], n)
        ws = max(se, n - c["window"])
        j = torch.arange(se // bs, -(-ws // bs) if ws > se else se // bs, device=DEV)
        for g in range(c["hkv"]):
            ids = _id(s, b, g, j)
            q = s["q"][b, g * G:(g + 1) * G].double()
            lo, hi = s["kmin"].view(-1, d)[ids].double(), s["kmax"].view(-1, d)[ids].double()
            best = torch.full((len(j),), -math.inf, dtype=torch.float64, device=DEV)
            for h in range(G):
                best = torch.maximum(best, torch.maximum(lo * q[h], hi * q[h]).sum(1))
            order = torch.argsort(best, descending=True, stable=True)
            blk = torch.sort(j[order[:-(-c["k"] // bs)]]).values
            member = torch.zeros(-(-n // bs) * bs, dtype=torch.bool, device=DEV)
            member.view(-1, bs)[blk] = True
            member[:se] = True
            member[ws:] = True
            pos = member[:n].nonzero()[:, 0]
            res["blocks"][b, g, :len(blk)] = blk.int()
            res["blocks_len"][b, g] = len(blk)
            res["set"][b, g, :len(pos)] = pos.int()
            res["set_len"][b, g] = len(pos)
    return res


def _exact_attention(s):
    c = s["c"]
    bs, d, G = c["block"], c["d"], c["hq"] // c["hkv"]
    out = torch.zeros(c["batch"], c["hq"], d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(c["batch"], c["hq"], dtype=torch.float64, device=DEV)
    lens = _lens(c)
    for b in range(c["batch"]):
        for g in range(c["hkv"]):
            if c["op"] == "dense":
                pos = torch.arange(lens[b], device=DEV)
            else:
                pos = s["set"][b, g, :int(s["set_len"][b, g])].long()
            if c["op"] == "reuse":
                n0 = int(s["anchor"][b])
                pos = torch.cat([pos[pos < n0], torch.arange(n0, lens[b], device=DEV)])
            ids = _id(s, b, g, pos // bs)
            at = ids * bs + pos % bs
            k, v = (s[x].view(torch.uint8).view(-1, d)[at].view(E4M3).double() * s[y].view(-1)[ids].double()[:, None]
                    for x, y in (("k8", "ks"), ("v8", "vs")))
            for h in range(g * G, (g + 1) * G):
                x = (k * s["q"][b, h].double()).sum(1) * s["scale"]
                w = torch.exp(x - x.max())
                out[b, h] = (v * w[:, None]).sum(0) / w.sum()
                lse[b, h] = x.max() + torch.log(w.sum())
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "store":
        return _exact_store(s)
    if case["op"] == "bounds":
        return _exact_bounds(s)
    return _exact_select(s) if case["op"] == "select" else _exact_attention(s)
