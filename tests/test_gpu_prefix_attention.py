"""Decode attention of a batch behind a shared prefix against attention in 64
bits (reference and bound: tests/operator_cases.py).

Short prefixes and small batches run as plain attention.  The lengths here stay
below the 768 tokens from which plain attention would want a workspace (or the
case says so), so the workspace's size tells which way a call goes; SHARED lists
cases that read the prefix once, of every variant of that kernel."""
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


def run(kv, q, tables, ctx, prefix, dtype, scale=None, once=None):
    L, B, HQ, D = q.shape
    scale = 1 / math.sqrt(D) if scale is None else scale
    dev = kv.cuda()
    pool = Pool(list(dev[0].unbind(0)), list(dev[1].unbind(0)))
    nbytes = decode_prefix_workspace_bytes(pool, ctx, HQ, prefix)
    if once is not None:
        assert (nbytes > 0) == once
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


# Up to 64 and more rows a KV head; few partitions and more than 8; one workgroup a partition and two;
# blocks of 16 tokens or a multiple, and others; prefixes that end inside a tile.
SHARED = [
    (1, 16, 1, 128, 16, "bf16", [688 + i for i in range(30)], 43),
    (1, 16, 1, 128, 12, "fp16", [684 + 2 * i for i in range(30)], 57),
    (1, 16, 4, 128, 32, "bf16", [736 + (i % 3) for i in range(8)] + [1300] * 24, 23),
    (1, 64, 2, 64, 48, "fp16", [672 + i for i in range(16)], 14),
    (1, 32, 1, 64, 1, "bf16", [600 + i for i in range(32)], 600),
    (1, 8, 1, 128, 16, "fp16", [704 + (i % 40) for i in range(60)], 44),
    (1, 8, 1, 128, 24, "bf16", [720 + (i % 40) for i in range(60)], 30),
    (1, 8, 2, 128, 16, "bf16", [656 + (i % 7) for i in range(100)], 41),
    (1, 8, 2, 128, 20, "fp16", [660 + (i % 7) for i in range(100)], 33),
    (2, 16, 4, 64, 16, "bf16", [720 + (i % 9) for i in range(60)], 45),
    (2, 16, 4, 64, 8, "fp16", [720 + (i % 9) for i in range(60)], 90),
    (3, 4, 4, 128, 16, "bf16", [700, 0, 699, 41, 0, 688, 687] + [688] * 60, 43),     # some share nothing, some end there
    (1, 8, 8, 128, 16, "bf16", [3520 + (i % 50) for i in range(20)], 220),      # more partitions than are joined at a time
    (1, 16, 2, 128, 16, "fp16", [2400 + (i % 50) for i in range(30)], 150),
]


@pytest.mark.parametrize("case", SHARED, ids=lambda c: f"L{c[0]}_H{c[1]}_G{c[2]}_D{c[3]}_bs{c[4]}_{c[5]}_B{len(c[6])}_p{c[7]}")
def test_reads_the_prefix_once(case):
    print("[case]", case, flush=True)
    L, H, G, D, bs, dtype, ctx, prefix = case
    run(*setup(L, H, G, D, bs, dtype, ctx, prefix), ctx, prefix, dtype, once=True)


def test_long_prefix_in_several_partitions():
    ctx = [5000 + 3 * i for i in range(20)]
    run(*setup(1, 8, 4, 128, 16, "bf16", ctx, 311), ctx, 311, "bf16")


def test_full_batch():
    ctx = [304 + (i % 5) for i in range(256)]
    run(*setup(1, 8, 1, 64, 16, "bf16", ctx, 19), ctx, 19, "bf16", once=True)


# as those, with more tokens behind the prefix than one partition takes
LONG = [
    (1, 8, 4, 128, 16, "bf16", [5000 + 997 * i for i in range(12)] + [4000, 4010, 5, 0, 3999], 250),
    (8, 4, 4, 64, 8, "fp16", [700, 4000, 1500, 640, 2300] + [650 + i for i in range(60)], 80),
    (4, 16, 1, 128, 16, "fp16", [1100 + 640 * i for i in range(5)] + [700] * 20, 40),
]


@pytest.mark.parametrize("case", LONG, ids=lambda c: f"L{c[0]}_H{c[1]}_G{c[2]}_D{c[3]}_bs{c[4]}_{c[5]}")
def test_many_own_tokens(case):
    print("[case]", case, flush=True)
    L, H, G, D, bs, dtype, ctx, prefix = case
    run(*setup(L, H, G, D, bs, dtype, ctx, prefix), ctx, prefix, dtype)


# as those, with few tokens behind the prefix: a wavefront takes those of a KV head
FEW = [
    (2, 5, 1, 128, 16, "bf16", [700, 0, 41, 688, 770] + [688 + (i % 30) for i in range(110)], 43),
    (3, 4, 2, 64, 8, "fp16", [731, 640, 12, 0] + [640 + (i * i) % 90 for i in range(96)], 80),
    (5, 2, 4, 128, 24, "bf16", [480 + (i % 70) for i in range(128)], 20),
]


@pytest.mark.parametrize("case", FEW, ids=lambda c: f"L{c[0]}_H{c[1]}_G{c[2]}_D{c[3]}_bs{c[4]}_{c[5]}")
def test_few_own_tokens_of_many(case):
    print("[case]", case, flush=True)
    L, H, G, D, bs, dtype, ctx, prefix = case
    run(*setup(L, H, G, D, bs, dtype, ctx, prefix), ctx, prefix, dtype)


# the batch of the tests below, and its prefix: rows of both halves of a product's
# columns, three tiles, the last one partly filled
CTX, PREFIX = [688 + (5 * i) % 13 for i in range(30)], 43
SHAPE = (1, 16, 1, 128, 16)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_other_scales(scale):
    """A negative scale turns the order of the scores round, a large one makes
    one weight outweigh all others, and its partition's maximum move."""
    run(*setup(*SHAPE, "bf16", CTX, PREFIX), CTX, PREFIX, "bf16", scale=scale, once=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("step", [0.5, 5.0, 30.0])
def test_rising_scores(dtype, step):
    """Scores that rise token by token by less than, and by more than, what the
    running maximum lets pass."""
    kv, q, tables = setup(*SHAPE, dtype, CTX, PREFIX)
    q[:] = 0
    q[..., 0] = 1
    for b in range(len(CTX)):
        blk, slot = oc.rows_of(tables, b, range(CTX[b]), 16)
        kv[0, 0, blk, slot, :, 0] = (torch.arange(CTX[b]) * step / 8).to(kv.dtype)[:, None]
    run(kv, q, tables, CTX, PREFIX, dtype, scale=1.0, once=True)


@pytest.mark.parametrize("own", [0, 60])
def test_small_weights_beside_a_large_one(own):
    ctx = [688 + own] * 30
    kv, q, tables = setup(*SHAPE, "fp16", ctx, PREFIX)
    for b in range(30):
        want, tol = oc.small_weights(kv, q, tables, b, 688 + own)
    out = run(kv, q, tables, ctx, PREFIX, "fp16", scale=1.0, once=True)
    assert float((out.double() - want).abs().max()) <= tol


@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf", "all -inf"])
def test_nonfinite_scores(where, bad):
    """A NaN or +inf score gives its rows zeros and no others; -inf is a weight
    of 0.  Head 1 alone has such keys, in the prefix or in sequence 2's own
    tokens."""
    kv, q, tables = setup(*SHAPE, "bf16", CTX, PREFIX)
    q[..., 0], kv[0, ..., 0] = 4.0, 0.0
    tokens = range(0, 688) if where == "prefix" else range(688, CTX[2])
    if bad != "all -inf":
        tokens = [tokens[3], tokens[5]]
    blk, slot = oc.rows_of(tables, 2, tokens, 16)
    kv[0, 0, blk, slot, 1, 0] = {"nan": float("nan"), "inf": float("inf")}.get(bad, float("-inf"))
    out = run(kv, q, tables, CTX, PREFIX, "bf16", once=True)
    if bad in ("nan", "inf"):
        hit = range(len(CTX)) if where == "prefix" else [2]
        for b in range(len(CTX)):
            assert bool((out[0, b, 1] == 0).all()) == (b in hit)
        assert bool((out[0, :, 0] != 0).any(-1).all())


def test_what_lies_behind_a_sequence_does_not_count():
    """Slots behind the last token, and blocks of others, may hold NaN."""
    for shape, ctx, prefix in ((SHAPE, CTX, PREFIX), ((1, 2, 2, 128, 16), [100, 97, 96], 6)):
        kv, q, tables = setup(*shape, "bf16", ctx, prefix)
        used = torch.zeros(kv.shape[2:4], dtype=torch.bool)
        for b, n in enumerate(ctx):
            used[oc.rows_of(tables, b, range(n), 16)] = True
        kv[:, :, ~used] = float("nan")
        run(kv, q, tables, ctx, prefix, "bf16")


def test_on_a_stream_replayed_and_repeated():
    """Captured once and replayed, with eager calls between, every result has
    the same bits; the same call on two streams with workspaces of their own, too."""
    ctx, prefix = CTX, PREFIX
    kv, q, tables = setup(*SHAPE, "bf16", ctx, prefix)
    first = run(kv, q, tables, ctx, prefix, "bf16", once=True)
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
