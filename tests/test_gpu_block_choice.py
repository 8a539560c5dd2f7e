"""Bounds of the blocks' keys, the choice of blocks by them and decode attention
over listed blocks against plain references in 64 bits (tests/operator_cases.py)."""
import math

import pytest
import torch

import operator_cases as oc

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2406_03243_amd.llmig import (LlmigError, Pool, decode_blocks_workspace_bytes, llmig_append_rotary,
                                            llmig_decode_attention_blocks, llmig_decode_attention_prefix,
                                            llmig_key_bounds, llmig_select_blocks, llmig_stage, select_workspace_bytes)


def make(L, H, G, D, bs, dtype, ctx, seed=2):
    gen = torch.Generator().manual_seed(seed)
    tdt, B = oc.TYPES[dtype], len(ctx)
    need = [-(-n // bs) for n in ctx]
    nb = sum(need) + 3
    order = torch.randperm(nb, generator=gen).to(torch.int32)
    tables = torch.full((B + 1, max(need + [1]) + 1), -7, dtype=torch.int32)
    at = 0
    for b, k in enumerate(need):
        tables[b, :k] = order[at:at + k]
        at += k
    kv = torch.randn((2, L, nb, bs, H, D), generator=gen).to(tdt)
    q = torch.randn((L, B, H * G, D), generator=gen).to(tdt)
    return kv, q, tables, gen


def pool_of(t):
    return Pool(list(t[0].unbind(0)), list(t[1].unbind(0)))


# ---- bounds -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("L,H,D,bs,ctx,first", [
    (1, 2, 64, 16, [1], [0]), (2, 3, 128, 16, [33, 16, 0, 200], [32, 0, 0, 100]), (1, 1, 8, 4, [9, 4], [3, 4]),
    (2, 40, 128, 16, [50], [17]), (1, 13, 64, 1, [20, 3], [5, 0]), (1, 2, 72, 12, [100, 1], [0, 0]),
    (1, 8, 128, 32, [1000] * 3, [0, 500, 999])])
def test_bounds(dtype, L, H, D, bs, ctx, first):
    print("[case]", L, H, D, bs, ctx, first, flush=True)
    kv, _, tables, _ = make(L, H, 1, D, bs, dtype, ctx)
    kv[0, 0, tables[0, 0].long(), 0, 0, 0] = -0.0
    for b, n in enumerate(ctx):         # a slot behind the last token must not count
        if n % bs:
            kv[0, :, tables[b, n // bs].long(), n % bs:] = float("nan")
    dev = kv.cuda()
    bounds = torch.full((2, L, kv.shape[2], 1, H, D), 3.0, dtype=kv.dtype, device="cuda")
    want = bounds.cpu().clone()
    for b, n in enumerate(ctx):
        for j in range(first[b] // bs, -(-n // bs)) if first[b] < n else ():
            rows = kv[0, :, tables[b, j].long(), :min(bs, n - j * bs)]
            want[0, :, tables[b, j].long(), 0], want[1, :, tables[b, j].long(), 0] = rows.amin(1), rows.amax(1)
    llmig_key_bounds(pool_of(dev), pool_of(bounds), tables.cuda(), first, ctx)
    torch.cuda.synchronize()
    assert torch.equal(bounds.cpu(), want)


@pytest.mark.parametrize("at", [0, 1, 7, 15])
def test_bounds_of_nonfinite_keys(at):
    kv, _, tables, _ = make(1, 1, 1, 64, 16, "bf16", [16])
    b = tables[0, 0].long()
    kv[0, 0, b, at, 0, 1], kv[0, 0, b, at, 0, 2], kv[0, 0, b, at, 0, 3] = float("nan"), float("inf"), float("-inf")
    dev = kv.cuda()
    bounds = torch.zeros((2, 1, kv.shape[2], 1, 1, 64), dtype=kv.dtype, device="cuda")
    llmig_key_bounds(pool_of(dev), pool_of(bounds), tables.cuda(), [15], [16])
    torch.cuda.synchronize()
    lo, hi = bounds[0, 0, b, 0, 0].cpu(), bounds[1, 0, b, 0, 0].cpu()
    assert bool(torch.isnan(lo[1])) and bool(torch.isnan(hi[1]))
    assert lo[3] == -math.inf and hi[2] == math.inf
    rows = kv[0, 0, b, :, 0]
    rest = [0, 2] + list(range(4, 64))
    assert torch.equal(lo[rest], rows.amin(0)[rest])
    rest = [0, 3] + list(range(4, 64))
    assert torch.equal(hi[rest], rows.amax(0)[rest])


# sequences of one group share their first blocks: `common` tokens of them
@pytest.mark.parametrize("L,H,D,bs,common,ctx,first,group", [
    (1, 8, 128, 16, 32, [50, 40, 33, 32], [0] * 4, [0] * 4),              # whole blocks, then their own
    (3, 16, 128, 16, 40, [40] * 5, [39, 0, 32, 40, 17], [0] * 5),         # and a partly filled one, all as far
    (2, 40, 128, 8, 12, [12] * 3, [8, 11, 0], [0] * 3),
    (5, 2, 64, 16, 32, [35 + i % 13 for i in range(30)], [i % 33 for i in range(30)], [i % 3 for i in range(30)]),
    (2, 1, 8, 4, 7, [7] * 200, [4 + i % 3 for i in range(200)], [i % 9 for i in range(200)]),
    (1, 13, 64, 12, 24, [30, 24, 34, 26], [24, 0, 0, 25], [0, 0, 1, 1])])
def test_bounds_of_shared_blocks(L, H, D, bs, common, ctx, first, group):
    print("[case]", L, H, D, bs, ctx, first, flush=True)
    kv, _, tables, gen = make(L, H, 1, D, bs, "bf16", ctx)
    for b, g in enumerate(group):
        tables[b, :-(-common // bs)] = tables[group.index(g), :-(-common // bs)]
    held = torch.zeros(kv.shape[2:4], dtype=torch.bool)
    for b, n in enumerate(ctx):
        held[oc.rows_of(tables, b, range(n), bs)] = True
    kv[0][:, ~held] = float("nan")
    want = torch.full((2, L, kv.shape[2], 1, H, D), 3.0, dtype=kv.dtype)
    for b, n in enumerate(ctx):
        for j in range(first[b] // bs, -(-n // bs)) if first[b] < n else ():
            rows = kv[0, :, tables[b, j].long(), :min(bs, n - j * bs)]
            want[0, :, tables[b, j].long(), 0], want[1, :, tables[b, j].long(), 0] = rows.amin(1), rows.amax(1)
    dev, tab = kv.cuda(), tables.cuda()
    for _ in range(3):
        bounds = torch.full(want.shape, 3.0, dtype=kv.dtype, device="cuda")
        llmig_key_bounds(pool_of(dev), pool_of(bounds), tab, first, ctx)
        torch.cuda.synchronize()
        assert torch.equal(bounds.cpu(), want)


@pytest.mark.parametrize("L,H,D,bs,ctx", [(2, 8, 128, 16, [40, 33]), (3, 2, 64, 16, [90, 40, 70]), (1, 40, 128, 4, [9, 8])])
def test_bounds_of_ids_outside_the_pool(L, H, D, bs, ctx):
    """An id that is not a block's is never written to; other blocks get their bounds."""
    kv, _, tables, _ = make(L, H, 1, D, bs, "bf16", ctx)
    nb = kv.shape[2]
    right = tables.clone()
    bad = {(0, 0): -1, (0, 1): nb, (1, 1): 2 ** 31 - 1, (1, 0): -2 ** 31}
    for (b, j), x in bad.items():
        tables[b, j] = x
    dev = kv.cuda()
    flat = torch.full((2 * L * nb * H * D + 4096,), 3.0, dtype=kv.dtype, device="cuda")
    bounds = flat[2048:-2048].view(2, L, nb, 1, H, D)
    want = bounds.cpu().clone()
    for b, n in enumerate(ctx):
        for j in range(-(-n // bs)):
            if (b, j) not in bad:
                rows = kv[0, :, right[b, j].long(), :min(bs, n - j * bs)]
                want[0, :, right[b, j].long(), 0], want[1, :, right[b, j].long(), 0] = rows.amin(1), rows.amax(1)
    llmig_key_bounds(pool_of(dev), pool_of(bounds), tables.cuda(), [0] * len(ctx), ctx)
    torch.cuda.synchronize()
    assert torch.equal(bounds.cpu(), want) and torch.equal(dev.cpu(), kv)
    assert bool((flat[:2048] == 3).all()) and bool((flat[-2048:] == 3).all())


# ---- choice -------------------------------------------------------------------

def choose(bounds, q, tables, ctx, bs, first, last, count):
    """bounds [2][L][blocks][1][H][D] on the CPU; checks against the reference."""
    L, B, H = q.shape[0], q.shape[1], bounds.shape[4]
    dev = bounds.cuda()
    pool = pool_of(dev)
    nbytes = select_workspace_bytes(pool, bs, ctx)
    ws = torch.full((nbytes + 32,), 0xFF, dtype=torch.uint8, device="cuda")
    blocks = torch.full((L, B + 1, H, count), -9, dtype=torch.int32, device="cuda")
    got = torch.full((L, B, H, count), -9, dtype=torch.int32, device="cuda")
    llmig_select_blocks(pool, bs, q.cuda(), tables.cuda(), ctx, first, last, ws[:nbytes], got)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xFF).all()) and bool((blocks == -9).all())
    want = torch.empty(got.shape, dtype=torch.int32)
    for l in range(L):
        for b in range(B):
            n = -(-ctx[b] // bs)
            ids = tables[b, :n].long()
            want[l, b] = oc.select(bounds[0, l, ids, 0], bounds[1, l, ids, 0], q[l, b], n, first, last, count)
    assert torch.equal(got.cpu(), want)
    return want


def random_bounds(kv, gen):
    a = torch.randn((2,) + (kv.shape[1], kv.shape[2], 1) + kv.shape[4:], generator=gen).to(kv.dtype)
    return torch.stack([torch.minimum(a[0], a[1]), torch.maximum(a[0], a[1])])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("L,H,G,D,bs,ctx,first,last,count", [
    (1, 2, 4, 128, 16, [1], 0, 0, 1), (1, 2, 4, 128, 16, [600, 17, 0, 33], 1, 1, 4),
    (2, 3, 1, 64, 8, [500, 77, 400], 0, 0, 7), (1, 1, 16, 128, 4, [1500], 2, 3, 5), (1, 40, 1, 128, 16, [300], 0, 1, 3),
    (1, 13, 2, 64, 16, [900, 899], 0, 0, 56), (1, 1, 1, 64, 1, [3000, 2999, 257], 1, 2, 100),
    (1, 2, 2, 128, 16, [4000], 0, 0, 249), (1, 2, 2, 128, 16, [4000], 0, 0, 250), (1, 2, 2, 128, 16, [4000], 0, 0, 500),
    (1, 1, 2, 64, 2, [20000], 4, 4, 1000), (1, 1, 1, 64, 1, [17000, 16385, 40], 2, 3, 300)])
def test_choice(dtype, L, H, G, D, bs, ctx, first, last, count):
    print("[case]", L, H, G, D, bs, ctx, first, last, count, flush=True)
    kv, q, tables, gen = make(L, H, G, D, bs, dtype, ctx)
    choose(random_bounds(kv, gen), q, tables, ctx, bs, first, last, count)


def test_equal_scores_go_to_the_first():
    kv, q, tables, gen = make(1, 2, 2, 64, 16, "bf16", [1600])
    b = random_bounds(kv, gen)
    b[:, :, :, :, 0] = b[:, :, :1, :, 0]                        # head 0: all blocks alike
    b[:, :, :, :, 1] = b[:, :, torch.arange(b.shape[2]) % 3, :, 1]    # head 1: three kinds
    for count in (1, 10, 40, 99):
        choose(b, q, tables, [1600], 16, 0, 0, count)
        choose(b, q, tables, [1600], 16, 0, 1, count)


@pytest.mark.parametrize("blocks", [5000, 9000, 17000])
def test_equal_scores_of_long_rows(blocks):
    kv, q, tables, gen = make(1, 1, 1, 64, 1, "fp16", [blocks])
    b = random_bounds(kv, gen)
    b = b[:, :, torch.arange(b.shape[2]) % 7]
    for count in (600, 3000):
        choose(b, q, tables, [blocks], 1, 1, 2, count)


def test_scores_that_differ_by_little():
    """Sums that are equal in 32 bits but not in 64."""
    kv, q, tables, gen = make(1, 1, 1, 64, 16, "bf16", [1600])
    b = torch.zeros((2, 1, kv.shape[2], 1, 1, 64), dtype=kv.dtype)
    q[:] = 1.0
    b[..., 0] = 4096.0
    j = torch.arange(100)
    b[:, 0, tables[0, :100].long(), 0, 0, 1] = ((j * 37 % 100).float() * 2.0 ** -30).to(b.dtype)
    choose(b, q, tables, [1600], 16, 0, 0, 10)


def test_scores_that_are_not_finite():
    kv, q, tables, gen = make(1, 1, 2, 64, 16, "bf16", [640])
    b = random_bounds(kv, gen)
    ids = tables[0].long()
    b[:, 0, ids[5], 0, 0, 7] = float("nan")
    b[1, 0, ids[9], 0, 0, 8] = float("inf")
    b[0, 0, ids[11], 0, 0, 9] = float("-inf")
    q[..., 8], q[..., 9] = 1.0, 1.0
    choose(b, q, tables, [640], 16, 0, 0, 2)
    choose(b, q, tables, [640], 16, 0, 0, 3)
    b[:, 0, ids[20:30], 0, 0, 8] = float("-inf")
    choose(b, q, tables, [640], 16, 0, 0, 35)
    q[:] = 0
    choose(random_bounds(kv, gen), q, tables, [640], 16, 1, 1, 5)


# ---- attention over lists ---------------------------------------------------------

def attend(kv, q, tables, ctx, lists, dtype, scale=None):
    L, B, HQ, D = q.shape
    bs = kv.shape[3]
    scale = 1 / math.sqrt(D) if scale is None else scale
    dev = kv.cuda()
    pool = pool_of(dev)
    nbytes = decode_blocks_workspace_bytes(pool, ctx, HQ, lists.shape[3])
    ws = torch.full((nbytes + 32,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 7.0, device="cuda")
    llmig_decode_attention_blocks(pool, q.cuda(), tables.cuda(), ctx, lists.cuda(), scale, ws[:nbytes], out)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xFF).all())

    def tokens(l, b, g):
        read = lists[l, b, g, :min(lists.shape[3], -(-ctx[b] // bs))].tolist()
        return [t for j in read if j >= 0 for t in range(j * bs, min((j + 1) * bs, ctx[b]))]

    want, tol = oc.decode(kv, q, tables, scale, dtype, tokens)
    ratio = oc.worst(out, want, tol)
    print("[case] largest error / bound", ratio, flush=True)
    assert ratio <= 1
    return out


def some_lists(L, B, H, count, ctx, bs, gen, order="ascending", holes=False):
    lists = torch.full((L, B, H, count), -1, dtype=torch.int32)
    for l in range(L):
        for b in range(B):
            n = -(-ctx[b] // bs)
            for g in range(H):
                pick = torch.randperm(n, generator=gen)[:count]
                if order == "ascending":
                    pick = pick.sort()[0]
                elif order == "last":           # the partly filled last block first
                    pick = torch.cat([torch.tensor([n - 1]), pick])[:count] if n else pick
                lists[l, b, g, :len(pick)] = pick.to(torch.int32)
                if holes and n:
                    lists[l, b, g, ::3] = torch.tensor([-1, n, 1 << 30, -(1 << 31)])[(l + b + g) % 4].to(torch.int32)
    return lists


@pytest.mark.parametrize("order,holes", [("ascending", False), ("last", False), ("any", True)])
@pytest.mark.parametrize("dtype,L,H,G,D,bs,ctx,count", [
    ("bf16", 1, 2, 4, 128, 16, [1], 1), ("bf16", 2, 2, 4, 128, 16, [300, 45, 0, 17], 5),
    ("fp16", 1, 3, 1, 64, 8, [500, 77], 20), ("bf16", 1, 1, 16, 128, 4, [203], 13), ("fp16", 1, 2, 2, 64, 12, [301, 5], 9),
    ("bf16", 1, 2, 2, 128, 1, [70, 64], 33), ("bf16", 1, 1, 2, 128, 16, [9000], 200), ("fp16", 1, 1, 8, 64, 32, [5001], 100),
    ("bf16", 1, 2, 1, 128, 24, [1000, 990], 30)])
def test_attention_over_lists(order, holes, dtype, L, H, G, D, bs, ctx, count):
    print("[case]", order, dtype, L, H, G, D, bs, ctx, count, flush=True)
    kv, q, tables, gen = make(L, H, G, D, bs, dtype, ctx)
    attend(kv, q, tables, ctx, some_lists(L, len(ctx), H, count, ctx, bs, gen, order, holes), dtype)


@pytest.mark.parametrize("order,holes", [("ascending", False), ("any", True)])
@pytest.mark.parametrize("dtype,L,H,G,D,bs,B,longest", [
    ("bf16", 2, 5, 2, 128, 16, 110, 90), ("fp16", 2, 4, 1, 64, 8, 140, 93), ("bf16", 8, 2, 16, 64, 32, 70, 77),
    ("fp16", 4, 13, 1, 128, 16, 60, 260), ("bf16", 30, 3, 4, 128, 24, 75, 500)])
def test_many_short_lists(order, holes, dtype, L, H, G, D, bs, B, longest):
    """A wavefront walks the list of a KV head by itself; heads that four does not divide."""
    print("[case]", order, dtype, L, H, G, D, bs, B, longest, flush=True)
    ctx = [0, longest, 1] + [1 + (i * i * 7) % (longest if i < 20 else min(longest, 60)) for i in range(B - 3)]
    kv, q, tables, gen = make(L, H, G, D, bs, dtype, ctx)
    attend(kv, q, tables, ctx, some_lists(L, B, H, -(-longest // bs), ctx, bs, gen, order, holes), dtype)


def test_a_block_listed_twice_counts_twice():
    kv, q, tables, _ = make(1, 1, 2, 64, 16, "bf16", [100])
    attend(kv, q, tables, [100], torch.tensor([3, 0, 3, 6, 6], dtype=torch.int32).view(1, 1, 1, 5), "bf16")


@pytest.mark.parametrize("D,bs,n", [(128, 16, 700), (64, 12, 2100)])
def test_small_weights_beside_a_large_one(D, bs, n):
    kv, q, tables, _ = make(1, 2, 4, D, bs, "fp16", [n])
    want, tol = oc.small_weights(kv, q, tables, 0, n)
    lists = torch.arange(-(-n // bs), dtype=torch.int32).expand(1, 1, 2, -1).contiguous()
    out = attend(kv, q, tables, [n], lists, "fp16", scale=1.0)
    assert float((out.double() - want).abs().max()) <= tol


@pytest.mark.parametrize("bs", [16, 8, 12, 2])
def test_lists_that_name_nothing(bs):
    kv, q, tables, _ = make(1, 2, 2, 64, bs, "bf16", [100, 5])
    lists = torch.full((1, 2, 2, 7), -1, dtype=torch.int32)
    out = attend(kv, q, tables, [100, 5], lists, "bf16")
    assert bool((out == 0).all())
    lists[0, 0, 1, 3] = 2
    out = attend(kv, q, tables, [100, 5], lists, "bf16")
    assert bool((out[0, 0, :2] == 0).all()) and bool((out[0, 0, 2:] != 0).any())


@pytest.mark.parametrize("bs", [16, 8, 12, 3])
def test_what_no_list_names_does_not_count(bs):
    """Blocks that are not listed, and the slots behind the last token, hold
    NaN, the pool's first block among them; -1 entries stand between."""
    ctx = [200, 205]
    kv, q, tables, gen = make(1, 2, 2, 128, bs, "bf16", ctx)
    lists = some_lists(1, 2, 2, 9, ctx, bs, gen, "last", holes=True)
    used = torch.zeros(kv.shape[2:4] + (2,), dtype=torch.bool)
    for b in range(2):
        for g in range(2):
            for j in lists[0, b, g].tolist():
                t = [t for t in range(j * bs, j * bs + bs) if 0 <= t < ctx[b]] if 0 <= j < 1000 else []
                used[oc.rows_of(tables, b, t, bs) + (g,)] = True
    kv[:, :, ~used] = float("nan")
    attend(kv, q, tables, ctx, lists, "bf16")


def test_all_blocks_listed_is_decode_attention():
    ctx = [333, 90, 16]
    kv, q, tables, gen = make(2, 2, 4, 128, 16, "bf16", ctx)
    n = 21
    lists = torch.full((2, 3, 2, n), -1, dtype=torch.int32)
    for b, c in enumerate(ctx):
        lists[:, b, :, :-(-c // 16)] = torch.arange(-(-c // 16), dtype=torch.int32)
    attend(kv, q, tables, ctx, lists, "bf16")


# ---- all of them, one after the other -----------------------------------------------

def test_a_decode_step_of_long_contexts():
    """append, bounds, choice and attention, on one stream without a wait in
    between, then again from a graph; then the migration of cache and bounds by
    the same block map, and the same step's attention on the destination."""
    L, H, G, D, bs, ctx, count = 2, 2, 4, 128, 16, [700, 33, 260], 12
    kv, _, tables, gen = make(L, H, G, D, bs, "bf16", [n + 1 for n in ctx])
    dev, tab = kv.cuda(), tables.cuda()
    bounds = torch.zeros((2, L, kv.shape[2], 1, H, D), dtype=kv.dtype, device="cuda")
    pool, bpool = pool_of(dev), pool_of(bounds)
    inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    angle = torch.arange(1024, dtype=torch.float64)[:, None] * inv
    cs = torch.cat([angle.cos(), angle.sin()], 1).float()
    qkv = torch.randn((L, 3, H * (G + 2), D), generator=gen).to(kv.dtype)
    llmig_key_bounds(pool, bpool, tab, [0, 0, 0], ctx)
    after, scale = [n + 1 for n in ctx], 1 / math.sqrt(D)
    q_out = torch.empty((L, 3, H * G, D), dtype=kv.dtype, device="cuda")
    lists = torch.empty((L, 3, H, count), dtype=torch.int32, device="cuda")
    out = torch.empty((L, 3, H * G, D), device="cuda")
    ws = torch.empty(max(select_workspace_bytes(bpool, bs, after), decode_blocks_workspace_bytes(pool, after, H * G, count),
                         16), dtype=torch.uint8, device="cuda")
    x, csd = qkv.cuda(), cs.cuda()

    def step():
        llmig_append_rotary(pool, x[:, :, H * G:H * (G + 1)], x[:, :, H * (G + 1):], tab, ctx, [1, 1, 1], csd,
                            q=x[:, :, :H * G], q_out=q_out)
        llmig_key_bounds(pool, bpool, tab, ctx, after)
        llmig_select_blocks(bpool, bs, q_out, tab, after, 1, 1, ws, lists)
        llmig_decode_attention_blocks(pool, q_out, tab, after, lists, scale, ws, out)

    step()
    torch.cuda.synchronize()
    got, got_lists, now, b_now = out.clone(), lists.clone(), dev.cpu(), bounds.cpu()
    q = q_out.cpu()
    for b in range(3):
        n = -(-after[b] // bs)
        ids = tables[b, :n].long()
        for l in range(L):
            for j in range(n):
                rows = now[0, l, ids[j], :min(bs, after[b] - j * bs)]
                assert torch.equal(b_now[0, l, ids[j], 0], rows.amin(0)) and torch.equal(b_now[1, l, ids[j], 0], rows.amax(0))
            want = oc.select(b_now[0, l, ids, 0], b_now[1, l, ids, 0], q[l, b], n, 1, 1, count)
            assert torch.equal(got_lists[l, b].cpu(), want)
    tokens = lambda l, b, g: [t for j in got_lists[l, b, g].tolist() if j >= 0
                              for t in range(j * bs, min((j + 1) * bs, after[b]))]
    want, tol = oc.decode(now, q, tables, scale, "bf16", tokens)
    assert oc.worst(got, want, tol) <= 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        out.fill_(float("nan"))
        lists.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, got) and torch.equal(lists, got_lists)
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, got)
    # migrate: cache and bounds by one block map
    used = torch.cat([tables[b, :-(-after[b] // bs)] for b in range(3)])
    to = torch.randperm(kv.shape[2], generator=gen)[:len(used)].to(torch.int32)
    dev2, bounds2 = torch.zeros_like(dev), torch.zeros_like(bounds)
    pool2, bpool2 = pool_of(dev2), pool_of(bounds2)
    llmig_stage(pool, pool2, used.numpy(), to.numpy())
    llmig_stage(bpool, bpool2, used.numpy(), to.numpy())
    tab2, at = torch.zeros_like(tables), 0
    for b in range(3):
        n = -(-after[b] // bs)
        tab2[b, :n] = to[at:at + n]
        at += n
    lists2, out2 = torch.empty_like(lists), torch.empty_like(out)
    llmig_select_blocks(bpool2, bs, q_out, tab2.cuda(), after, 1, 1, ws, lists2)
    llmig_decode_attention_blocks(pool2, q_out, tab2.cuda(), after, lists2, scale, ws, out2)
    torch.cuda.synchronize()
    assert torch.equal(lists2, got_lists) and torch.equal(out2, got)


def test_tensors_elsewhere_are_refused():
    """A tensor on the CPU, or of another shape or type, never reaches a kernel."""
    kv, q, tables, _ = make(1, 2, 2, 64, 16, "bf16", [40])
    dev, tab, qd = kv.cuda(), tables.cuda(), q.cuda()
    pool = pool_of(dev)
    low = torch.zeros((2, 1, kv.shape[2], 1, 2, 64), dtype=kv.dtype, device="cuda")
    bounds = pool_of(low)
    lists, out = torch.zeros((1, 1, 2, 2), dtype=torch.int32, device="cuda"), torch.empty((1, 1, 4, 64), device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    k = torch.zeros((1, 1, 2, 64), dtype=kv.dtype, device="cuda")
    wide = torch.zeros((1, 1, 2, 64), dtype=torch.float32, device="cuda")
    calls = [
        (llmig_append_rotary, (pool, k, k, tab, [40], [1], None), [(1, k.cpu()), (2, wide), (3, tables), (1, k[:, :, :1])]),
        (llmig_key_bounds, (pool, bounds, tab, [0], [40]), [(2, tables), (2, tab.long()), (4, [40, 41])]),
        (llmig_select_blocks, (bounds, 16, qd, tab, [40], 0, 0, ws, lists),
         [(2, q), (3, tables), (4, [40, 3]), (7, ws.cpu()), (8, lists.cpu()), (8, lists[:, :, :1])]),
        (llmig_decode_attention_blocks, (pool, qd, tab, [40], lists, 0.1, ws, out),
         [(1, q), (2, tables), (3, []), (4, lists.cpu()), (4, lists.long()), (6, ws.cpu()), (7, out.cpu()), (7, out.half())]),
        (llmig_decode_attention_prefix, (pool, qd, tab, [40], 1, 0.1, ws, out),
         [(1, q), (2, tables), (3, [1, 2]), (6, ws.cpu()), (7, out.cpu()), (7, out[:, :, :2])])]
    for fn, args, bad in calls:
        for at, value in bad:
            with pytest.raises((ValueError, LlmigError)):
                fn(*args[:at], value, *args[at + 1:])
    torch.cuda.synchronize()


# ---- fp16 rows of 128, and what stands around the outputs -----------------------------

@pytest.mark.parametrize("order,holes", [("ascending", False), ("last", False), ("any", True)])
@pytest.mark.parametrize("L,H,G,D,bs,ctx,count", [
    (2, 2, 4, 128, 16, [300, 45, 0, 17], 5), (1, 1, 16, 128, 4, [203], 13), (1, 1, 2, 128, 16, [9000], 200),
    (1, 2, 1, 128, 24, [1000, 990], 30), (1, 8, 8, 128, 16, [3001, 2500, 40], 64), (4, 3, 2, 128, 8, [700, 650], 70)])
def test_attention_over_lists_of_fp16_rows(order, holes, L, H, G, D, bs, ctx, count):
    print("[case]", order, L, H, G, D, bs, ctx, count, flush=True)
    kv, q, tables, gen = make(L, H, G, D, bs, "fp16", ctx)
    attend(kv, q, tables, ctx, some_lists(L, len(ctx), H, count, ctx, bs, gen, order, holes), "fp16")


# rows that are listed whole, and lists of each kernel (one wavefront, four, sixteen; keys in registers or not)
@pytest.mark.parametrize("D,bs,ctx,count", [
    (64, 16, [40, 0, 17], 7), (128, 16, [600, 33], 3), (64, 16, [4000, 100], 61), (64, 4, [4097], 129), (64, 1, [5000], 77),
    (128, 1, [9001, 5], 301), (64, 1, [17000, 16385], 1000)])
def test_nothing_is_written_around_the_lists(D, bs, ctx, count):
    print("[case]", D, bs, ctx, count, flush=True)
    kv, q, tables, gen = make(2, 3, 2, D, bs, "bf16", ctx)
    b = random_bounds(kv, gen)
    dev = b.cuda()
    pool = pool_of(dev)
    ws, ws_whole = oc.guarded((select_workspace_bytes(pool, bs, ctx),), torch.uint8, 0xFF)
    blocks, whole = oc.guarded((2, len(ctx), 3, count), torch.int32, -9)
    llmig_select_blocks(pool, bs, q.cuda(), tables.cuda(), ctx, 0, 1, ws, blocks)
    torch.cuda.synchronize()
    assert whole() and ws_whole() and torch.equal(dev.cpu(), b)
    for x in range(len(ctx)):
        n = -(-ctx[x] // bs)
        ids = tables[x, :n].long()
        for l in range(2):
            assert torch.equal(blocks[l, x].cpu(), oc.select(b[0, l, ids, 0], b[1, l, ids, 0], q[l, x], n, 0, 1, count))
