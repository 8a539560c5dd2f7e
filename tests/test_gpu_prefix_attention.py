"""Decode attention of a batch behind a shared prefix against attention in 64
bits (reference and bound: tests/operator_cases.py)."""
import math

import pytest
import torch

import operator_cases as oc

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2406_03243_amd.llmig import Pool, decode_prefix_workspace_bytes, llmig_decode_attention_prefix


def setup(L, H, G, D, bs, dtype, ctx, prefix, seed=1):
    gen = torch.Generator().manual_seed(seed)
    tdt, B = oc.TYPES[dtype], len(ctx)
    need = [max(0, -(-n // bs)) for n in ctx]
    longest = max(need + [prefix, 1])
    shared = min(prefix, max(need + [0]))
    nb = shared + sum(need) + 3
    order = torch.randperm(nb, generator=gen).to(torch.int32)
    tables = torch.full((B + 1, longest), -7, dtype=torch.int32)     # what no sequence reaches is no id
    at = shared
    for b, k in enumerate(need):
        first = shared if k >= prefix and ctx[b] >= prefix * bs else 0
        tables[b, :first] = order[:first]
        own = k - first
        tables[b, first:k] = order[at:at + own]
        at += own
    kv = torch.randn((2, L, nb, bs, H, D), generator=gen).to(tdt)
    q = torch.randn((L, B, H * G, D), generator=gen).to(tdt)
    return kv, q, tables


def run(kv, q, tables, ctx, prefix, dtype, scale=None, stream=None):
    L, B, HQ, D = q.shape
    scale = 1 / math.sqrt(D) if scale is None else scale
    dev = kv.cuda()
    pool = Pool(list(dev[0].unbind(0)), list(dev[1].unbind(0)))
    nbytes = decode_prefix_workspace_bytes(pool, ctx, HQ, prefix)
    ws = torch.full((nbytes + 32,), 0xFF, dtype=torch.uint8, device="cuda")     # NaN patterns
    out = torch.full((L, B + 1, HQ, D), 7.0, device="cuda")
    mine = torch.full(q.shape, 7.0, device="cuda")
    llmig_decode_attention_prefix(pool, q.cuda(), tables.cuda(), ctx, prefix, scale, ws[:nbytes], mine)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xFF).all()), "written behind the workspace"
    want, tol = oc.decode(kv, q, tables, scale, dtype, lambda l, b, g: range(ctx[b]))
    ratio = oc.worst(mine, want, tol)
    print("[case] largest error / bound", ratio, flush=True)
    assert ratio <= 1
    return mine


# layers, heads, group, dim, block, type, lengths, prefix blocks
CASES = [
    (1, 2, 4, 128, 16, "bf16", [70, 64, 65, 200], 4),
    (1, 2, 4, 128, 16, "fp16", [70, 64, 65, 200], 4),
    (2, 1, 8, 64, 16, "bf16", [333, 320, 400, 321, 700], 20),
    (1, 2, 1, 128, 8, "fp16", [100] * 40, 11),                      # 40 rows: two of the four wavefronts split them
    (1, 1, 16, 64, 32, "bf16", [1000 + i for i in range(9)], 31),   # 144 rows: two workgroups a partition
    (1, 1, 2, 128, 16, "bf16", [17, 16], 1),                        # a prefix of one block
    (1, 2, 2, 128, 12, "bf16", [130, 120, 145], 10),                # blocks that 8 does not divide
    (1, 2, 2, 64, 1, "fp16", [75, 70, 101], 70),
    (3, 2, 2, 128, 16, "bf16", [160, 0, 40, 161, 159, 160], 10),    # empty and shorter sequences share nothing
    (1, 1, 4, 128, 16, "bf16", [5000, 4800, 4801], 300),            # several partitions, ragged ends
    (1, 4, 8, 128, 16, "fp16", [2100 + 3 * i for i in range(33)], 130),   # 264 rows
    (1, 2, 2, 64, 16, "bf16", [50, 60], 0),                         # nothing shared
    (1, 2, 2, 64, 16, "bf16", [50, 60], 4),                         # no sequence reaches the prefix's end
    (1, 2, 2, 64, 16, "bf16", [90, 60, 0], 4),                      # one does
    (1, 13, 1, 64, 16, "bf16", [130] * 7, 8),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"L{c[0]}_H{c[1]}_G{c[2]}_D{c[3]}_bs{c[4]}_{c[5]}_B{len(c[6])}_p{c[7]}")
def test_matches_attention(case):
    print("[case]", case, flush=True)
    L, H, G, D, bs, dtype, ctx, prefix = case
    run(*setup(L, H, G, D, bs, dtype, ctx, prefix), ctx, prefix, dtype)


def test_full_batch():
    ctx = [48 + (i % 5) for i in range(256)]
    run(*setup(1, 1, 2, 64, 16, "bf16", ctx, 3), ctx, 3, "bf16")


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_other_scales(scale):
    """A negative scale turns the order of the scores round, a large one makes
    one weight outweigh all others, and its partition's maximum move."""
    ctx = [600, 577, 592]
    run(*setup(1, 2, 4, 128, 16, "bf16", ctx, 36), ctx, 36, "bf16", scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rising_scores(dtype):
    """Scores that rise token by token by less than, and by more than, what the
    running maximum lets pass."""
    for step in (0.5, 5.0, 30.0):
        ctx = [257, 300]
        kv, q, tables = setup(1, 1, 2, 64, 16, dtype, ctx, 16)
        q[:] = 0
        q[..., 0] = 1
        for b in range(2):
            blk, slot = oc.rows_of(tables, b, range(ctx[b]), 16)
            kv[0, 0, blk, slot, 0, 0] = (torch.arange(ctx[b]) * step / 8).to(kv.dtype)
        run(kv, q, tables, ctx, 16, dtype, scale=1.0)


@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf", "all -inf"])
def test_nonfinite_scores(where, bad):
    """A NaN or +inf score gives that row zeros and no other; -inf a weight of 0."""
    ctx = [200, 192, 210]
    kv, q, tables = setup(1, 2, 2, 128, 16, "bf16", ctx, 12)
    q[..., 0], kv[0, ..., 0] = 4.0, 0.0
    tokens = range(0, 192) if where == "prefix" else range(192, ctx[0])
    if bad != "all -inf":
        tokens = [tokens[3], tokens[5]]
    blk, slot = oc.rows_of(tables, 0, tokens, 16)
    # the value's product with q overflows in 32 bits, or does not need to
    kv[0, 0, blk, slot, 1, 0] = {"nan": float("nan"), "inf": float("inf")}.get(bad, float("-inf"))
    out = run(kv, q, tables, ctx, 12, "bf16")
    if bad in ("nan", "inf"):
        assert bool((out[0, 0, 2:] == 0).all()) and bool((out[0, 0, :2] != 0).any())


def test_what_lies_behind_a_sequence_does_not_count():
    """Slots behind the last token, and blocks of others, may hold NaN."""
    ctx = [100, 97, 96]
    kv, q, tables = setup(1, 2, 2, 128, 16, "bf16", ctx, 6)
    used = torch.zeros(kv.shape[2:4], dtype=torch.bool)
    for b, n in enumerate(ctx):
        used[oc.rows_of(tables, b, range(n), 16)] = True
    kv[:, :, ~used] = float("nan")
    run(kv, q, tables, ctx, 6, "bf16")


def test_on_a_stream_replayed_and_repeated():
    """Captured once and replayed, with eager calls between, every result has
    the same bits; the same call on two streams with workspaces of their own, too."""
    ctx, prefix = [700, 643, 640, 901], 40
    kv, q, tables = setup(2, 2, 4, 128, 16, "bf16", ctx, prefix)
    first = run(kv, q, tables, ctx, prefix, "bf16")
    dev = kv.cuda()
    pool = Pool(list(dev[0].unbind(0)), list(dev[1].unbind(0)))
    nbytes = decode_prefix_workspace_bytes(pool, ctx, q.shape[2], prefix)
    qd, tab, scale = q.cuda(), tables.cuda(), 1 / math.sqrt(128)
    ws = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in range(3)]
    outs = [torch.zeros(q.shape, device="cuda") for _ in range(3)]
    call = lambda i, s=None: llmig_decode_attention_prefix(pool, qd, tab, ctx, prefix, scale, ws[i], outs[i], stream=s)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    call(0, side)
    call(1, other)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first) and torch.equal(outs[1], first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(2)
    for k in range(4):
        outs[2].fill_(float("nan"))
        graph.replay()
        call(0)
        torch.cuda.synchronize()
        assert torch.equal(outs[2], first) and torch.equal(outs[0], first)
