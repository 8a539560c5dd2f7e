"""Attention over listed blocks and behind a shared prefix where scores are exact
and few weights count, so that the bounds are those of the parts that a weight is
taken in (operator_cases.py; test_operator_bounds.py shows that a part less does not
pass).  Outputs stand between guards."""
import pytest
import torch

import operator_cases as oc
import test_gpu_block_choice as lists_of
import test_gpu_prefix_attention as behind

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2406_03243_amd.llmig import (decode_blocks_workspace_bytes, decode_prefix_workspace_bytes,
                                            llmig_decode_attention_blocks, llmig_decode_attention_prefix)


def over_lists(kv, q, tables, ctx, lists):
    pool = lists_of.pool_of(kv.cuda())       # (holds its tensors)
    nbytes = decode_blocks_workspace_bytes(pool, ctx, q.shape[2], lists.shape[3])
    ws, ws_whole = oc.guarded((nbytes,), torch.uint8, 0xFF)
    out, out_whole = oc.guarded(q.shape, torch.float32, 7.0)
    named, named_whole = oc.guarded(lists.shape, torch.int32, -9)
    named.copy_(lists)
    llmig_decode_attention_blocks(pool, q.cuda(), tables.cuda(), ctx, named, 1.0, ws, out)
    torch.cuda.synchronize()
    assert ws_whole() and out_whole() and named_whole() and torch.equal(named.cpu(), lists)
    return out


def behind_prefix(kv, q, tables, ctx, prefix):
    pool = lists_of.pool_of(kv.cuda())       # (holds its tensors)
    nbytes = decode_prefix_workspace_bytes(pool, ctx, q.shape[2], prefix)
    ws, ws_whole = oc.guarded((nbytes,), torch.uint8, 0xFF)
    out, out_whole = oc.guarded(q.shape, torch.float32, 7.0)
    llmig_decode_attention_prefix(pool, q.cuda(), tables.cuda(), ctx, prefix, 1.0, ws, out)
    torch.cuda.synchronize()
    assert ws_whole() and out_whole()
    return out


# blocks of 8 tokens or a multiple, and others; several partitions; many short
# sequences, of which a wavefront takes a KV head
LISTS = [
    (1, 2, 16, 128, 16, [300, 45, 0, 17]), (1, 3, 16, 64, 8, [500, 77]), (1, 2, 4, 128, 12, [301, 5]), (1, 2, 4, 64, 1, [70, 64]),
    (1, 1, 8, 128, 16, [9000]), (1, 1, 8, 64, 32, [5001, 4000]), (1, 2, 2, 128, 20, [4400]),
    (8, 5, 2, 128, 16, [3 + (i * 7) % 60 for i in range(70)]), (8, 4, 4, 64, 8, [3 + (i * 7) % 60 for i in range(70)])]
NAME = lambda c: f"L{c[0]}_H{c[1]}_G{c[2]}_D{c[3]}_bs{c[4]}" if isinstance(c, tuple) else None


@pytest.mark.parametrize("dtype,parts", [("bf16", 3), ("fp16", 2)])
@pytest.mark.parametrize("case", LISTS, ids=NAME)
def test_over_lists(case, dtype, parts):
    print("[case]", case, dtype, flush=True)
    L, H, G, D, bs, ctx = case
    kv, q, tables, gen = lists_of.make(L, H, G, D, bs, dtype, ctx)
    live = [(b, t) for b, n in enumerate(ctx) if n > 2 for t in (n // 3, n - 1)]
    oc.exact_scores(kv, q, tables, live, dtype, parts)
    lists = lists_of.some_lists(L, len(ctx), H, -(-max(ctx) // bs), ctx, bs, gen, "any")
    out = over_lists(kv, q, tables, ctx, lists)
    ratio = oc.check_exact(out, q, ctx, [2 * (n > 2) for n in ctx], dtype, parts)
    print("[case] largest error / bound", ratio, flush=True)
    assert ratio <= 1


PLAIN = [(1, 2, 4, 128, 16, [70, 64, 65, 200], 4), (1, 2, 2, 64, 12, [130, 120, 145], 10), (1, 1, 8, 128, 16, [5000, 4800], 300)]
SHARED = [c[:5] + c[6:] for c in behind.SHARED + behind.LONG + behind.FEW]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", PLAIN + SHARED, ids=lambda c: f"{NAME(c)}_B{len(c[5])}_p{c[6]}")
def test_behind_a_prefix(case, dtype):
    print("[case]", case, dtype, flush=True)
    L, H, G, D, bs, ctx, prefix = case
    kv, q, tables = behind.setup(L, H, G, D, bs, dtype, ctx, prefix)
    shared = prefix * bs
    members = [b for b, n in enumerate(ctx) if n >= shared]
    live, counts = [(b, shared * 2 // 3 + 1) for b in members[:1] if shared], []
    for b, n in enumerate(ctx):
        own = ([shared + (n - shared) // 2] if n > shared else []) if b in members and shared else [n // 3, n - 1] if n > 2 else []
        live += [(b, t) for t in own]
        counts.append(len(own) + (b in members and shared > 0))
    oc.exact_scores(kv, q, tables, live, dtype, 2)
    out = behind_prefix(kv, q, tables, ctx, prefix)
    ratio = oc.check_exact(out, q, ctx, counts, dtype, 2)
    print("[case] largest error / bound", ratio, flush=True)
    assert ratio <= 1


@pytest.mark.parametrize("D,bs,n", [(128, 16, 700), (64, 12, 2100), (64, 16, 748)])
def test_tiny_weights_over_lists(D, bs, n):
    kv, q, tables, _ = lists_of.make(1, 2, 4, D, bs, "fp16", [n])
    oc.small_weights(kv, q, tables, 0, n)
    lists = torch.arange(-(-n // bs), dtype=torch.int32).expand(1, 1, 2, -1).contiguous()
    out = over_lists(kv, q, tables, [n], lists)
    want, tol = oc.tiny_weights(n)
    assert float((out.double() - want).abs().max()) <= tol


@pytest.mark.parametrize("own", [0, 60])
def test_tiny_weights_behind_a_prefix(own):
    ctx = [688 + own] * 30
    kv, q, tables = behind.setup(*behind.SHAPE, "fp16", ctx, behind.PREFIX)
    for b in range(30):
        oc.small_weights(kv, q, tables, b, 688 + own)
    out = behind_prefix(kv, q, tables, ctx, behind.PREFIX)
    want, tol = oc.tiny_weights(688 + own)
    assert float((out.double() - want).abs().max()) <= tol
