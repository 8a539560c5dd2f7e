"""Operators on a paged KV cache beside decode attention and token writes, as
cases that can be timed and compared: the append of new tokens with the
position rotation, the per-block bounds of the keys, the choice of blocks by
those bounds, decode attention over the chosen blocks, and decode attention of
a batch that shares a prefix.

A case is a dict of plain values.  ``kind`` names the operator; ``layers``,
``heads`` (KV heads of this GPU's shard), ``group`` (query heads per KV head),
``dim``, ``block`` (tokens per block) and ``dtype`` give the pool.  With ``own``
false ``run`` computes the operator from elementary torch operations, with
``own`` true through the framework's entry points.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
LAYOUT_CODES = {"NHD": 0, "HND": 1, "HCNX": 2, "HDN": 3}


def listed():
    return [
        # One layer's token of a single request: the smallest call a decode
        # step makes, all latency.
        dict(name="append_one", kind="append", layers=1, heads=8, group=4, dim=128, block=16, dtype="bf16", batch=1,
             first=700, tokens=1, rotary=128, interleaved=False, layouts="NHD/NHD"),
        # The new tokens of a decode step of a batch, all layers at once.
        dict(name="append_step", kind="append", layers=32, heads=8, group=4, dim=128, block=16, dtype="bf16", batch=61,
             first=1500, tokens=1, rotary=128, interleaved=False, layouts="NHD/NHD"),
        # Prompts of several requests enter the cache of a 7B-shaped model
        # in the paged layouts.
        dict(name="append_prompts", kind="append", layers=8, heads=32, group=1, dim=128, block=16, dtype="fp16",
             batch=5, first=0, tokens=1900, rotary=64, interleaved=True, layouts="HCNX/HDN"),
        # A decode step refreshes the bounds of the block it wrote into.
        dict(name="bounds_step", kind="bounds", layers=32, heads=8, group=4, dim=128, block=16, dtype="bf16", batch=32,
             ctx=3000, tail=1),
        # The bounds of long prompts after their prefill.
        dict(name="bounds_prompts", kind="bounds", layers=4, heads=8, group=4, dim=128, block=16, dtype="bf16", batch=3,
             ctx=32768, tail=32768),
        # One layer chooses the blocks of a few requests.
        dict(name="select_one_layer", kind="select", layers=1, heads=8, group=4, dim=128, block=16, dtype="bf16",
             batch=3, ctx=9000, count=64, keep_first=1, keep_last=2),
        # A batch of long contexts, several layers at once.
        dict(name="select_long", kind="select", layers=4, heads=8, group=8, dim=128, block=16, dtype="bf16", batch=12,
             ctx=65536, count=256, keep_first=1, keep_last=4),
        # One layer attends to the chosen blocks of a few requests.
        dict(name="blocks_one_layer", kind="blocks", layers=1, heads=8, group=4, dim=128, block=16, dtype="bf16",
             batch=3, ctx=9000, count=64),
        # A batch of long contexts on small blocks of a wide group.
        dict(name="blocks_long", kind="blocks", layers=4, heads=8, group=8, dim=128, block=16, dtype="bf16", batch=12,
             ctx=32768, count=256),
        # One layer of a few requests behind one system prompt.
        dict(name="prefix_one_layer", kind="prefix", layers=1, heads=8, group=4, dim=128, block=16, dtype="bf16",
             batch=7, prefix=125, own=90),
        # A 7B-shaped batch (a query head per KV head) behind one document.
        dict(name="prefix_mha", kind="prefix", layers=8, heads=32, group=1, dim=128, block=16, dtype="fp16", batch=40,
             prefix=256, own=300),
        # A large grouped-query batch behind a long document: the matrix
        # products outweigh the reads.
        dict(name="prefix_long", kind="prefix", layers=4, heads=8, group=8, dim=128, block=16, dtype="bf16", batch=64,
             prefix=1024, own=500),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng: random.Random) -> dict:
    """One more case: any kind, pools of shapes that models and their
    tensor-parallel shards have, sizes spread over their logarithm; none is
    costlier than the largest listed case."""
    kind = rng.choice(["append", "append", "bounds", "select", "blocks", "blocks", "prefix", "prefix"])
    c = dict(kind=kind, layers=_log_int(rng, 1, 40), heads=rng.choice([1, 2, 4, 8, 8, 13, 32, rng.randint(1, 40)]),
             group=rng.choice([1, 2, 4, 8, 8, 16]), dim=rng.choice([64, 128, 128]),
             block=rng.choice([8, 16, 16, 16, 32]), dtype=rng.choice(["fp16", "bf16"]), batch=_log_int(rng, 1, 64))
    if c["heads"] * c["group"] > 128:
        c["group"] = 1
    row = c["layers"] * c["heads"] * c["dim"] * 2             # bytes of one token's keys
    if kind == "append":
        most = max(1, min(4096, 250_000_000 // (row * (4 + 2 * c["group"])) // c["batch"]))
        c["tokens"] = rng.choice([1, 1, _log_int(rng, 1, most)])
        c["first"] = _log_int(rng, 1, 2000) - 1
        c["rotary"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, 16, 24])
        c["interleaved"] = rng.choice([False, False, True])
        c["layouts"] = rng.choice(["NHD/NHD", "NHD/NHD", "HND/HND", "HCNX/HDN"])
        blocks = c["batch"] * (-(-(c["first"] + c["tokens"]) // c["block"]) + 1)
        c["layers"] = max(1, min(c["layers"], 2_000_000_000 // (row // c["layers"] * 2 * c["block"] * blocks)))
    elif kind == "bounds":
        most = max(40, min(32768, 400_000_000 // row // c["batch"]))
        c["ctx"] = _log_int(rng, 1, most)
        c["tail"] = rng.choice([1, c["ctx"], _log_int(rng, 1, c["ctx"])])
    elif kind == "select":
        most = max(40, min(131072, 400_000_000 * c["block"] // (2 * row) // c["batch"]))
        c["ctx"] = _log_int(rng, 1, most)
        c["keep_first"], c["keep_last"] = rng.choice([(0, 0), (1, 1), (1, 2), (4, 8)])
        c["count"] = c["keep_first"] + c["keep_last"] + _log_int(rng, 1, 400)
    elif kind == "blocks":
        most = max(40, min(32768, 1_200_000_000 // (2 * row) // c["batch"]))
        c["ctx"] = _log_int(rng, 1, most)
        c["count"] = _log_int(rng, 1, 512)
    else:
        most = max(40, min(4000, 500_000_000 // (2 * row) // c["batch"]))
        c["own"] = _log_int(rng, 1, most)
        most = max(2, min(1024 * 16, 1_000_000_000 // (2 * row), 70_000_000_000 // (row * c["group"] * c["batch"])))
        c["prefix"] = _log_int(rng, 1, max(1, most // c["block"]))
    return c


# ---- what a case comes to ---------------------------------------------------

def _spread(c, most, salt):
    """One length a request: the longest is ``most``, the others spread over
    the logarithm below it, as requests of mixed age have them."""
    rng = random.Random(most * 1000003 + c["batch"] * 17 + salt)
    return [most] + [max(1, int(most * math.exp(-2.0 * rng.random()))) for _ in range(c["batch"] - 1)]


def _up(n, d):
    return -(-n // d)


def _lengths(c):
    """(tokens a request holds before the call, tokens it holds after it)."""
    if c["kind"] == "append":
        new = _spread(c, c["tokens"], 1)
        old = _spread(c, c["first"], 2) if c["first"] else [0] * c["batch"]
        return old, [a + b for a, b in zip(old, new)]
    if c["kind"] == "prefix":
        n = c["prefix"] * c["block"]
        return [n] * c["batch"], [n + x for x in _spread(c, c["own"], 3)]
    after = _spread(c, c["ctx"], 4)
    if c["kind"] == "bounds":
        return [max(0, n - c["tail"]) for n in after], after
    return after, after


def _listed_tokens(c, after):
    """Tokens behind the lists of a ``blocks`` case, one layer and KV head."""
    return sum(min(n, c["count"] * c["block"]) for n in after)


def work(c) -> dict:
    before, after = _lengths(c)
    row = c["layers"] * c["heads"] * c["dim"]                 # elements of one token's keys
    n = sum(after) - sum(before)
    queries = c["batch"] * row * c["group"]
    if c["kind"] == "append":
        return {"bytes": n * row * 2 * (4 + 2 * c["group"]) + n * c["rotary"] * 4,
                "flops": 3 * n * c["layers"] * c["heads"] * (1 + c["group"]) * c["rotary"]}
    if c["kind"] == "bounds":
        blocks = [(a // c["block"], _up(b, c["block"])) for a, b in zip(before, after)]
        read = sum(b - lo * c["block"] for (lo, _), b in zip(blocks, after))
        return {"bytes": 2 * row * (read + 2 * sum(hi - lo for lo, hi in blocks)), "flops": 2 * read * row}
    if c["kind"] == "select":
        blocks = sum(_up(x, c["block"]) for x in after)
        return {"bytes": 4 * row * blocks + 2 * queries + 4 * c["layers"] * c["heads"] * c["batch"] * c["count"],
                "flops": 4 * row * blocks}
    if c["kind"] == "blocks":
        t = _listed_tokens(c, after)
        return {"bytes": 4 * row * t + 6 * queries + 4 * c["layers"] * c["heads"] * c["batch"] * c["count"],
                "flops": 4 * row * c["group"] * t}
    t = c["prefix"] * c["block"]
    return {"bytes": 4 * row * (t + n) + 6 * queries, "flops": 4 * row * c["group"] * (t * c["batch"] + n)}


# ---- inputs -------------------------------------------------------------------

def _normal(shape, c, gen, step=1 << 28):
    t = torch.empty(shape, dtype=DTYPES[c["dtype"]], device="cuda")
    flat = t.view(-1)
    for at in range(0, flat.numel(), step):
        flat[at:at + step].normal_(generator=gen)
    return t


def _rotary_table(positions, rotary):
    """cos, then sin, of position * 10000^(-2 i / rotary), i < rotary / 2."""
    inv = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * inv
    return torch.cat([torch.cos(angle), torch.sin(angle)], dim=1).float()


def prepare(c, seed: int) -> dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    before, after = _lengths(c)
    L, H, G, D, bs, B = (c[x] for x in ("layers", "heads", "group", "dim", "block", "batch"))
    s = {"case": c, "before": before, "after": after, "scale": 1.0 / math.sqrt(D)}
    s["before_gpu"], s["after_gpu"] = (torch.tensor(x, device="cuda") for x in (before, after))
    # Block tables: every request's blocks in random order; a shared prefix
    # is the same blocks in every row.
    shared = c["prefix"] if c["kind"] == "prefix" else 0
    per = [_up(n, bs) - shared for n in after]
    nb = shared + sum(per) + (shared + sum(per)) // 8 + 3
    order = rng.permutation(nb).astype(np.int32)
    tables = np.zeros((B, shared + max(per)), np.int32)
    tables[:, :shared] = order[:shared]
    at = shared
    for b, n in enumerate(per):
        tables[b, shared:shared + n] = order[at:at + n]
        at += n
    s["tables"] = torch.from_numpy(tables).cuda()
    s["layouts"] = tuple(LAYOUT_CODES[x] for x in c.get("layouts", "NHD/NHD").split("/"))
    if c["kind"] == "append":
        n = sum(after) - sum(before)
        s["kv"] = torch.zeros((2, L, nb, bs, H, D), dtype=DTYPES[c["dtype"]], device="cuda")
        qkv = _normal((L, n, H * (G + 2), D), c, gen)        # the projection's output: q, k and v heads of a token
        s["q"], s["k"], s["v"] = qkv[:, :, :H * G], qkv[:, :, H * G:H * (G + 1)], qkv[:, :, H * (G + 1):]
        s["q_out"] = torch.empty((L, n, H * G, D), dtype=DTYPES[c["dtype"]], device="cuda")
        s["cos_sin"] = _rotary_table(max(after), c["rotary"])
        s["new"] = [a - b for a, b in zip(after, before)]
    elif c["kind"] == "select":
        a = _normal((2, L, nb, 1, H, D), c, gen)
        s["bounds"] = torch.stack([torch.minimum(a[0], a[1]), torch.maximum(a[0], a[1])])
        del a
        s["blocks"] = torch.empty((L, B, H, c["count"]), dtype=torch.int32, device="cuda")
    else:
        s["kv"] = _normal((2, L, nb, bs, H, D), c, gen)
    if c["kind"] == "bounds":
        s["bounds"] = torch.zeros((2, L, nb, 1, H, D), dtype=DTYPES[c["dtype"]], device="cuda")
    if c["kind"] == "blocks":
        # for each layer, request and KV head some of the request's blocks, ascending
        lists = np.full((L * H, B, c["count"]), -1, np.int32)
        for b, n in enumerate(_up(x, bs) for x in after):
            k = min(c["count"], n)
            pick = np.sort(np.argpartition(rng.random((L * H, n), dtype=np.float32), k - 1, axis=1)[:, :k], axis=1)
            lists[:, b, :k] = pick
        s["blocks"] = torch.from_numpy(lists.reshape(L, H, B, -1).transpose(0, 2, 1, 3).copy()).cuda()
    if c["kind"] in ("select", "blocks", "prefix"):
        s["q"] = _normal((L, B, H * G, D), c, gen)
        s["out"] = torch.empty((L, B, H * G, D), dtype=torch.float32, device="cuda")
    if own:
        from paper_2406_03243_amd import llmig
        if "kv" in s:
            s["pool"] = llmig.Pool(list(s["kv"][0].unbind(0)), list(s["kv"][1].unbind(0)), s["layouts"])
        if "bounds" in s:
            s["bounds_pool"] = llmig.Pool(list(s["bounds"][0].unbind(0)), list(s["bounds"][1].unbind(0)))
        need = {"select": lambda: llmig.select_workspace_bytes(s["bounds_pool"], bs, after),
                "blocks": lambda: llmig.decode_blocks_workspace_bytes(s["pool"], after, H * G, c["count"]),
                "prefix": lambda: llmig.decode_prefix_workspace_bytes(s["pool"], after, H * G, shared)}
        if c["kind"] in need:
            s["ws"] = torch.empty(max(16, need[c["kind"]]()), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass: the framework's calls --------------------------------------------

def _run_own(s):
    from paper_2406_03243_amd import llmig
    c = s["case"]
    if c["kind"] == "append":
        llmig.llmig_append_rotary(s["pool"], s["k"], s["v"], s["tables"], s["before"], s["new"], s["cos_sin"],
                                  q=s["q"], q_out=s["q_out"], interleaved=c["interleaved"])
        return {"kv": s["kv"], "q": s["q_out"]}
    if c["kind"] == "bounds":
        llmig.llmig_key_bounds(s["pool"], s["bounds_pool"], s["tables"], s["before"], s["after"])
        return {"bounds": s["bounds"]}
    if c["kind"] == "select":
        llmig.llmig_select_blocks(s["bounds_pool"], c["block"], s["q"], s["tables"], s["after"], c["keep_first"],
                                  c["keep_last"], s["ws"], s["blocks"])
        return {"blocks": s["blocks"]}
    if c["kind"] == "blocks":
        llmig.llmig_decode_attention_blocks(s["pool"], s["q"], s["tables"], s["after"], s["blocks"], s["scale"],
                                            s["ws"], s["out"])
        return {"out": s["out"]}
    llmig.llmig_decode_attention_prefix(s["pool"], s["q"], s["tables"], s["after"], c["prefix"], s["scale"], s["ws"],
                                        s["out"])
    return {"out": s["out"]}


# ---- one pass: elementary operations --------------------------------------------

def _tiles(t, layout):
    """A layer stack [L][blocks][...] of tiles as [L][blocks][slot][head][dim],
    whatever the order inside a tile."""
    L, nb, bs, H, D = t.shape
    if layout == 1:
        return t.view(L, nb, H, bs, D).permute(0, 1, 3, 2, 4)
    if layout == 3:
        return t.view(L, nb, H, D, bs).permute(0, 1, 4, 2, 3)
    return t


def _ragged(lo, hi):
    """(row, value) of every value in [lo[row], hi[row]), row after row."""
    n = hi - lo
    row = torch.repeat_interleave(torch.arange(len(n), device=n.device), n)
    return row, torch.arange(len(row), device=n.device) - (torch.cumsum(n, 0) - n)[row] + lo[row]


def _rotate(x, cos, sin, interleaved):
    h = cos.shape[-1]
    x = x.float()
    if interleaved:
        a, b = x[..., 0:2 * h:2], x[..., 1:2 * h:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :h], x[..., h:2 * h]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([y, x[..., 2 * h:]], dim=-1)


def _plain_append(s):
    c, t = s["case"], s["kv"]
    row, tok = _ragged(s["before_gpu"], s["after_gpu"])
    blk, slot = s["tables"].long()[row, tok // c["block"]], tok % c["block"]
    half = c["rotary"] // 2
    cos, sin = s["cos_sin"][tok, None, :half], s["cos_sin"][tok, None, half:]
    k = _rotate(s["k"], cos, sin, c["interleaved"]).to(t.dtype)
    if s["layouts"][0] == 2:
        L, nb, bs, H, D = t[0].shape
        t[0].view(L, nb, H, D // 8, bs, 8).permute(0, 1, 4, 2, 3, 5)[:, blk, slot] = k.view(L, -1, H, D // 8, 8)
    else:
        _tiles(t[0], s["layouts"][0])[:, blk, slot] = k
    _tiles(t[1], s["layouts"][1])[:, blk, slot] = s["v"]
    s["q_out"].copy_(_rotate(s["q"], cos, sin, c["interleaved"]))
    return {"kv": t, "q": s["q_out"]}


def _plain_bounds(s):
    bs = s["case"]["block"]
    row, j = _ragged(s["before_gpu"] // bs, (s["after_gpu"] + bs - 1) // bs)
    ids = s["tables"].long()[row, j]
    keys = s["kv"][0][:, ids].float()                                        # [L][n][bs][H][D]
    past = j[:, None] * bs + torch.arange(bs, device="cuda") >= s["after_gpu"][row][:, None]
    past = past[None, :, :, None, None]
    s["bounds"][0][:, ids, 0] = keys.masked_fill(past, math.inf).amin(2).to(s["bounds"].dtype)
    s["bounds"][1][:, ids, 0] = keys.masked_fill(past, -math.inf).amax(2).to(s["bounds"].dtype)
    return {"bounds": s["bounds"]}


def _plain_select(s):
    c = s["case"]
    L, H, G, D, bs, B, K = (c[x] for x in ("layers", "heads", "group", "dim", "block", "batch", "count"))
    ids = s["tables"].long()                                                 # rows past a request's end: any block
    q = s["q"].double().view(L, B, 1, H, G, D)
    # 64 bits: scores are compared with each other
    score = (q.clamp(min=0).sum(4) * s["bounds"][1][:, ids, 0].double()).sum(-1)
    score += (q.clamp(max=0).sum(4) * s["bounds"][0][:, ids, 0].double()).sum(-1)
    score = score.transpose(2, 3)                                            # [L][B][H][blocks]
    top = torch.finfo(torch.float64).max
    score = torch.nan_to_num(score, nan=top, posinf=top, neginf=-top)
    j = torch.arange(ids.shape[1], device="cuda")
    n = ((s["after_gpu"] + bs - 1) // bs)[:, None]
    kept = (j < c["keep_first"]) | (j >= n - c["keep_last"])
    score = torch.where(kept[:, None], math.inf, score)
    score = torch.where((j < n)[:, None], score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :K]
    order = torch.where(order < n[:, None], order, ids.shape[1])
    order = torch.sort(order, dim=-1)[0]
    s["blocks"].fill_(-1)
    s["blocks"][..., :order.shape[-1]] = torch.where(order < n[:, None], order, -1)
    return {"blocks": s["blocks"]}


def _plain_blocks(s):
    c, t = s["case"], s["kv"]
    L, H, G, D, bs, B, K = (c[x] for x in ("layers", "heads", "group", "dim", "block", "batch", "count"))
    j = s["blocks"].long()                                                   # [L][B][H][K]
    ids = torch.gather(s["tables"].long()[None, :, None, :].expand(L, B, H, -1), 3, j.clamp(min=0))
    layer = torch.arange(L, device="cuda")[:, None, None, None]
    head = torch.arange(H, device="cuda")[None, None, :, None]
    k, v = (x[layer, ids, :, head].float().view(L, B, H, K * bs, D) for x in (t[0], t[1]))
    seen = (j >= 0)[..., None] & (j[..., None] * bs + torch.arange(bs, device="cuda") <
                                  s["after_gpu"][None, :, None, None, None])
    score = torch.matmul(s["q"].float().view(L, B, H, G, D), k.transpose(3, 4).contiguous()) * s["scale"]
    score = score.masked_fill(~seen.view(L, B, H, 1, K * bs), -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    s["out"].copy_((torch.matmul(p, v) / p.sum(-1, keepdim=True)).view(L, B, H * G, D))
    return {"out": s["out"]}


def _plain_prefix(s):
    c, t = s["case"], s["kv"]
    L, H, G, D, bs, B, P = (c[x] for x in ("layers", "heads", "group", "dim", "block", "batch", "prefix"))
    ids = s["tables"].long()
    q = s["q"].float().view(L, B, H, G, D)
    k, v = (x[:, ids[0, :P]].float().view(L, P * bs, H, D).transpose(1, 2).contiguous() for x in (t[0], t[1]))
    rows = q.transpose(1, 2).reshape(L, H, B * G, D)
    score = torch.matmul(rows, k.transpose(2, 3).contiguous()) * s["scale"]  # [L][H][B G][prefix]
    k2, v2 = (x[:, ids[:, P:]].float().view(L, B, -1, H, D).transpose(2, 3).contiguous() for x in (t[0], t[1]))
    score2 = torch.matmul(q, k2.transpose(3, 4).contiguous()) * s["scale"]   # [L][B][H][G][own]
    past = P * bs + torch.arange(score2.shape[-1], device="cuda") >= s["after_gpu"][:, None]
    score2 = score2.masked_fill(past[None, :, None, None], -math.inf)
    score = score.view(L, H, B, G, P * bs).transpose(1, 2)
    top = torch.maximum(score.amax(-1, keepdim=True), score2.amax(-1, keepdim=True))
    p, p2 = torch.exp(score - top), torch.exp(score2 - top)
    o = torch.matmul(p.transpose(1, 2).reshape(L, H, B * G, P * bs), v).view(L, H, B, G, D).transpose(1, 2)
    o = (o + torch.matmul(p2, v2)) / (p.sum(-1, keepdim=True) + p2.sum(-1, keepdim=True))
    s["out"].copy_(o.reshape(L, B, H * G, D))
    return {"out": s["out"]}


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    plain = {"append": _plain_append, "bounds": _plain_bounds, "select": _plain_select, "blocks": _plain_blocks,
             "prefix": _plain_prefix}
    return plain[kind](s)


# ---- from the definition, in 64 bits -----------------------------------------------

def _softmax_of(scores, values):
    w = torch.softmax(scores, dim=-1)
    return torch.matmul(w, values)


def exact(c, seed: int):
    s = prepare(c, seed)
    L, H, G, D, bs, B = (c[x] for x in ("layers", "heads", "group", "dim", "block", "batch"))
    before, after, tables = s["before"], s["after"], s["tables"].cpu().numpy()
    if c["kind"] == "append":
        kv, q_out = s["kv"].double(), torch.empty(s["q_out"].shape, dtype=torch.float64, device="cuda")
        # a pool's tiles with the elements of slot, head and dim in that order
        axes = {0: (bs, H, D), 1: (H, bs, D), 2: (H, D // 8, bs, 8), 3: (H, D, bs)}
        perm = {0: (0, 1, 2, 3, 4), 1: (0, 1, 3, 2, 4), 2: (0, 1, 4, 2, 3, 5), 3: (0, 1, 4, 2, 3)}
        at = 0
        for b in range(B):
            t = np.arange(before[b], after[b])
            n = len(t)
            ids = torch.from_numpy(tables[b][t // bs].astype(np.int64)).cuda()
            slot = torch.from_numpy(t % bs).cuda()
            half = c["rotary"] // 2
            cs = s["cos_sin"][torch.from_numpy(t).cuda()].double()
            turn = torch.complex(cs[:, :half], cs[:, half:])[None, :, None, :]
            for name in ("q", "k"):
                x = s[name][:, at:at + n].double()
                if c["interleaved"]:
                    z = torch.complex(x[..., 0:2 * half:2].contiguous(), x[..., 1:2 * half:2].contiguous()) * turn
                    x[..., 0:2 * half:2], x[..., 1:2 * half:2] = z.real, z.imag
                else:
                    z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
                    x[..., :half], x[..., half:2 * half] = z.real, z.imag
                if name == "q":
                    q_out[:, at:at + n] = x
                else:
                    lay = s["layouts"][0]
                    view = kv[0].view(L, -1, *axes[lay]).permute(*perm[lay])
                    view[:, ids, slot] = x.view(L, n, *view.shape[3:])
            lay = s["layouts"][1]
            kv[1].view(L, -1, *axes[lay]).permute(*perm[lay])[:, ids, slot] = s["v"][:, at:at + n].double()
            at += n
        return {"kv": kv, "q": q_out}
    if c["kind"] == "bounds":
        out = s["bounds"].double()
        for b in range(B):
            for first in range(before[b] // bs, _up(after[b], bs), 512):
                last = min(first + 512, _up(after[b], bs))
                ids = torch.from_numpy(tables[b, first:last].astype(np.int64)).cuda()
                keys = s["kv"][0][:, ids].double()
                whole = last - first if after[b] >= last * bs else last - first - 1
                if whole:
                    out[0][:, ids[:whole], 0] = keys[:, :whole].min(2)[0]
                    out[1][:, ids[:whole], 0] = keys[:, :whole].max(2)[0]
                if whole < last - first:
                    part = keys[:, whole, :after[b] - (last - 1) * bs]
                    out[0][:, ids[whole], 0] = part.min(1)[0]
                    out[1][:, ids[whole], 0] = part.max(1)[0]
        return {"bounds": out}
    if c["kind"] == "select":
        out = np.full((L, B, H, c["count"]), -1, np.int32)
        for b in range(B):
            n = _up(after[b], bs)
            ids = s["tables"][b, :n].long()
            must = sorted(set(range(min(n, c["keep_first"]))) | set(range(max(0, n - c["keep_last"]), n)))
            for layer in range(L):
                lo, hi = (s["bounds"][k, layer, ids, 0].double() for k in (0, 1))           # [n][H][D]
                q = s["q"][layer, b].double().view(H, G, D)
                score = torch.zeros((n, H), dtype=torch.float64, device="cuda")
                for h in range(G):
                    score += torch.maximum(q[:, h] * lo, q[:, h] * hi).sum(-1)
                score = score.cpu().numpy()
                for g in range(H):
                    rank = np.lexsort((np.arange(n), -score[:, g]))
                    rest = [j for j in rank[:c["count"] + len(must)].tolist() if j not in must]
                    best = sorted(must + rest[:max(0, min(c["count"], n) - len(must))])
                    out[layer, b, g, :len(best)] = best
        return {"blocks": torch.from_numpy(out)}
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        for layer in range(L):
            q = s["q"][layer, b].double().view(H, G, D)
            if c["kind"] == "prefix":
                ids = s["tables"][b, :_up(after[b], bs)].long()
                k, v = (x[layer][ids].reshape(-1, H, D)[:after[b]].double().transpose(0, 1).contiguous()
                        for x in (s["kv"][0], s["kv"][1]))
                o = _softmax_of(torch.matmul(q, k.transpose(1, 2).contiguous()) * s["scale"], v)
                out[layer, b] = o.view(H * G, D)
                continue
            for g in range(H):
                chosen = s["blocks"][layer, b, g]
                chosen = chosen[chosen >= 0].long()
                tok = (chosen[:, None] * bs + torch.arange(bs, device="cuda")).view(-1)
                tok = tok[tok < after[b]]
                ids = s["tables"][b].long()[tok // bs]
                k, v = (x[layer, ids, tok % bs, g].double() for x in (s["kv"][0], s["kv"][1]))
                o = _softmax_of(torch.matmul(q[g], k.t().contiguous()) * s["scale"], v)
                out[layer, b, g * G:(g + 1) * G] = o
    return {"out": out}
