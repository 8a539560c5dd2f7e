"""The append of new tokens with the position rotation (llmig_append_rotary)
against the rotation in 64 bits, rounded once.

Bound of a rotated element x c - y s: each product and the sum round to 24 bits
(three roundings, or two where the compiler fuses), at most 2 u (|x c| + |y s|)
with u = 2^-24, then half a step of the pool's type of the result; below the
type's normal range a step is its smallest number."""
import numpy as np
import pytest
import torch

import operator_cases as oc

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2406_03243_amd.llmig import Pool, llmig_append_rotary

SMALLEST = {"fp16": 2.0 ** -24, "bf16": 2.0 ** -133}


def tiles(t, layout):
    """A stack [L][blocks][bs][H][D] as slots, heads, dims whatever its layout."""
    L, nb, bs, H, D = t.shape
    if layout == 1:
        return t.reshape(L, nb, H, bs, D).permute(0, 1, 3, 2, 4)
    if layout == 2:
        return t.reshape(L, nb, H, D // 8, bs, 8).permute(0, 1, 4, 2, 3, 5).reshape(L, nb, bs, H, D)
    if layout == 3:
        return t.reshape(L, nb, H, D, bs).permute(0, 1, 4, 2, 3)
    return t


def table_of(positions, rotary):
    inv = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))
    a = torch.arange(positions, dtype=torch.float64)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


def run(L=1, H=2, G=2, D=64, bs=16, dtype="bf16", froms=(3,), news=(1,), rotary=64, interleaved=False, layouts=(0, 0),
        with_q=True, fused=True, shift=None, table_offset=0, seed=0, values=None):
    print("[case]", L, H, G, D, bs, dtype, froms, news, rotary, interleaved, layouts, flush=True)
    gen = torch.Generator().manual_seed(seed)
    tdt, n, B = oc.TYPES[dtype], sum(news), len(news)
    need = [-(-(f + a) // bs) for f, a in zip(froms, news)]
    nb = sum(need) + 3
    order = torch.randperm(nb, generator=gen).to(torch.int32)
    tables = torch.zeros((B + 1, max(need) + 2), dtype=torch.int32)
    at = 0
    for b, k in enumerate(need):
        tables[b, :k] = order[at:at + k]
        at += k
    if fused:
        qkv = torch.randn((L, n, H * (G + 2), D), generator=gen).to(tdt)
        if values is not None:
            qkv.view(torch.int16)[:] = values(qkv.shape)
        q, k, v = qkv[:, :, :H * G], qkv[:, :, H * G:H * (G + 1)], qkv[:, :, H * (G + 1):]
        dev = qkv.cuda()
        qd, kd, vd = dev[:, :, :H * G], dev[:, :, H * G:H * (G + 1)], dev[:, :, H * (G + 1):]
    else:       # three arrays, keys with tokens in the outer order
        q, k, v = (torch.randn((L, n, h, D), generator=gen).to(tdt) for h in (H * G, H, H))
        qd, vd = q.cuda(), v.cuda()
        kd = k.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    before = torch.randn((2, L, nb, bs, H, D), generator=gen).to(tdt)
    kv = before.cuda()
    pos0 = list(froms) if shift is None else [f + s for f, s in zip(froms, shift)]
    cs = table_of(max(p + a for p, a in zip(pos0, news)) + 1, rotary) if rotary else None
    csd = None
    if rotary:
        csd = torch.empty(cs.numel() + table_offset, device="cuda")[table_offset:].view(cs.shape)
        csd.copy_(cs)
    q_out = torch.full((L, n, H * G, D), float("nan"), dtype=tdt, device="cuda")
    pool = Pool(list(kv[0].unbind(0)), list(kv[1].unbind(0)), layouts)
    llmig_append_rotary(pool, kd, vd, tables.cuda(), froms, news, csd, q=qd if with_q else None,
                        q_out=q_out if with_q else None, interleaved=interleaved,
                        first_pos=None if shift is None else pos0)
    torch.cuda.synchronize()
    got = kv.cpu()
    gk, gv = tiles(got[0], layouts[0]), tiles(got[1], layouts[1])
    bk, bv = tiles(before[0], layouts[0]).clone(), tiles(before[1], layouts[1]).clone()
    pos = torch.cat([torch.arange(p, p + a) for p, a in zip(pos0, news)])
    h = rotary // 2
    cos, sin = (cs[pos].double()[:, None, :h], cs[pos].double()[:, None, h:]) if rotary else (None, None)

    def check(x, y):
        """y (the result) against the rotation of x, both [L][n][heads][D]."""
        x, y = x.double(), y.double()
        if not rotary:
            assert torch.equal(x, y)
            return
        want = oc.rotate(x, cos, sin, interleaved)
        size = oc.rotate(x.abs(), cos.abs(), -sin.abs(), interleaved).abs()     # |x c| + |y s|, at least
        size = torch.maximum(size, oc.rotate(x.abs(), cos.abs(), sin.abs(), interleaved).abs())
        exact = 2 * 2.0 ** -24 * size
        tol = exact + oc.HALF_STEP[dtype] * (want.abs() + exact) + SMALLEST[dtype]
        assert bool(((y - want).abs() <= tol).all()), float(((y - want).abs() / tol).max())
        assert torch.equal(x[..., 2 * h:], y[..., 2 * h:])

    if values is None:
        at = 0
        for b in range(B):
            t = torch.arange(froms[b], froms[b] + news[b])
            blk, slot = oc.rows_of(tables, b, t, bs)
            bk[:, blk, slot], bv[:, blk, slot] = gk[:, blk, slot], v[:, at:at + news[b]]
            at += news[b]
        rows = [oc.rows_of(tables, b, torch.arange(froms[b], froms[b] + news[b]), bs) for b in range(B)]
        blk, slot = (torch.cat([r[i] for r in rows]) for i in (0, 1))
        check(k, gk[:, blk, slot])
        if with_q:
            check(q, q_out.cpu())
        # everything else is as it was, the values bit for bit
        assert torch.equal(gk.contiguous().view(torch.int16), bk.contiguous().view(torch.int16))
        assert torch.equal(gv.contiguous().view(torch.int16), bv.contiguous().view(torch.int16))
    return gk, gv, q_out.cpu(), k, v, q


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rotary", [(64, 64), (128, 128), (128, 64), (80, 32), (96, 24), (72, 72), (8, 8), (64, 2),
                                      (64, 16), (256, 252)])
def test_rotations(dtype, interleaved, D, rotary):
    run(L=2, H=3, G=2, D=D, dtype=dtype, froms=(5, 0, 40), news=(1, 3, 9), rotary=rotary, interleaved=interleaved)


@pytest.mark.parametrize("layouts", [(0, 0), (1, 1), (2, 3), (3, 2), (0, 3), (2, 0)])
@pytest.mark.parametrize("bs", [8, 16, 32])
def test_layouts(layouts, bs):
    run(L=2, H=2, D=64, bs=bs, froms=(0, 7, 31), news=(70, 1, 33), layouts=layouts)
    run(L=1, H=1, G=1, D=128, bs=bs, dtype="fp16", froms=(8, 1), news=(16, 8), rotary=128, layouts=layouts)


# prompts large enough to go block by block where a layout scatters their tokens
BIG = dict(L=3, H=8, G=1, D=128, froms=(0, 7, 31, 5), news=(300, 129, 150, 1), rotary=128)


@pytest.mark.parametrize("layouts", [(2, 3), (3, 2), (0, 3), (2, 0)])
@pytest.mark.parametrize("bs,interleaved,rotary", [(8, False, 128), (16, True, 128), (16, False, 64), (32, False, 24),
                                                   (16, True, 2), (64, False, 0)])
def test_prompts_block_by_block(layouts, bs, interleaved, rotary):
    run(**dict(BIG, rotary=rotary), bs=bs, interleaved=interleaved, layouts=layouts)


@pytest.mark.parametrize("bs", [4, 12, 24, 40])
def test_prompts_block_by_block_of_odd_sizes(bs):
    run(**dict(BIG, L=2, H=13, D=104, rotary=104, news=(400, 129, 150, 2)), bs=bs, dtype="fp16", layouts=(2, 3))
    run(**dict(BIG, L=30, H=1, D=80, rotary=80, news=(900, 129, 400, 2)), bs=bs, layouts=(3, 2), with_q=False, table_offset=1)


def test_many_layers_block_by_block():
    """Units enough for two layers a workgroup, an odd number of layers."""
    run(**dict(BIG, L=41, H=2, D=64, rotary=64), layouts=(2, 3))


@pytest.mark.parametrize("bs", [1, 4, 12])
def test_odd_blocks(bs):
    run(bs=bs, froms=(0, 11), news=(13, 30))
    run(bs=bs, froms=(3,), news=(30,), layouts=(1, 3), rotary=0)


def test_one_token_of_each():
    run(L=3, H=8, G=4, D=128, rotary=128, froms=tuple(range(0, 256)), news=(1,) * 256)


def test_some_sequences_append_nothing():
    run(froms=(0, 5, 9, 2), news=(0, 4, 0, 1))
    run(froms=(7, 0), news=(0, 0))


def test_without_queries_and_without_rotation():
    run(with_q=False, froms=(4,), news=(20,))
    run(rotary=0, froms=(4,), news=(20,))


def test_strides_positions_and_alignment():
    run(L=3, fused=False, froms=(4, 17), news=(20, 3))
    run(L=2, shift=(100, 3), froms=(4, 17), news=(20, 3))
    for offset in (1, 2, 3):        # a table that is not 16-byte aligned
        run(L=2, table_offset=offset, froms=(4, 17), news=(20, 3))


def test_far_positions_and_large_prompt():
    run(H=1, G=1, froms=(131000,), news=(72,), rotary=64, bs=32)
    run(L=2, H=8, G=1, D=128, rotary=128, froms=(0, 3), news=(1500, 900))


def test_values_keep_their_bits():
    """Values and dims behind the rotation are copied: every 16-bit pattern,
    NaN payloads and subnormals among them."""
    g = np.random.default_rng(3)
    bits = lambda shape: torch.from_numpy(g.integers(-32768, 32768, size=tuple(shape)).astype(np.int16))
    for layouts, H, news in (((0, 0), 2, 40), ((2, 3), 2, 40), ((1, 1), 2, 40), ((2, 3), 24, 530), ((3, 2), 24, 530)):
        gk, gv, q_out, k, v, q = run(H=H, D=128, rotary=64, froms=(0,), news=(news,), layouts=layouts, values=bits)
        tables_free = gv.reshape(1, -1, H, 128)        # slots in block order
        want = {r.numpy().tobytes() for r in v.contiguous().view(torch.int16).reshape(-1, H, 128)}
        have = {r.numpy().tobytes() for r in tables_free.contiguous().view(torch.int16)[0]}
        assert want <= have
        tail = {r.numpy().tobytes() for r in k.contiguous().view(torch.int16).reshape(-1, H, 128)[:, :, 64:].contiguous()}
        assert tail <= {r.numpy().tobytes() for r in gk.reshape(1, -1, H, 128)[0, :, :, 64:].contiguous().view(torch.int16)}
        assert torch.equal(q_out[..., 64:].contiguous().view(torch.int16), q[..., 64:].contiguous().view(torch.int16))


def test_a_nan_or_infinity_stays_in_its_pair():
    x = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16)
    x[..., 3], x[..., 5] = float("nan"), float("inf")
    kv = torch.zeros((2, 1, 1, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    pool = Pool([kv[0, 0]], [kv[1, 0]])
    q_out = torch.empty_like(x).cuda()
    llmig_append_rotary(pool, x.cuda(), x.cuda(), torch.zeros((1, 1), dtype=torch.int32, device="cuda"), [2], [1],
                        table_of(4, 64).cuda(), q=x.cuda(), q_out=q_out)
    torch.cuda.synchronize()
    for y in (kv[0, 0, 0, 2, 0].cpu(), q_out[0, 0, 0].cpu()):
        assert bool(torch.isnan(y[[3, 35]]).all()) and bool(torch.isinf(y[[5, 37]]).all())
        rest = [d for d in range(64) if d not in (3, 35, 5, 37)]
        assert bool((y[rest] == 0).all())


def test_ids_outside_the_pool_are_not_written():
    kv = torch.zeros((2, 1, 4, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    pool = Pool([kv[0, 0, 1:3]], [kv[1, 0, 1:3]])
    x = torch.ones((1, 3, 1, 64), dtype=torch.bfloat16, device="cuda")
    llmig_append_rotary(pool, x, x, torch.tensor([[2], [-1], [1]], dtype=torch.int32, device="cuda"), [0, 0, 0], [1, 1, 1],
                        None)
    torch.cuda.synchronize()
    want = torch.zeros_like(kv)
    want[:, 0, 2, 0] = 1
    assert torch.equal(kv, want)


@pytest.mark.parametrize("layouts", [(0, 0), (1, 1), (2, 3), (3, 2)])
@pytest.mark.parametrize("L,H,G,D,news", [(1, 2, 3, 64, [1, 1]), (3, 8, 1, 128, [300, 129]), (2, 13, 1, 104, [400, 2])])
def test_nothing_is_written_around_pool_and_queries(layouts, L, H, G, D, news):
    print("[case]", layouts, L, H, G, D, news, flush=True)
    bs, n, froms = 16, sum(news), [5, 0]
    need = [-(-(f + a) // bs) for f, a in zip(froms, news)]
    nb = sum(need)
    tables = torch.zeros((2, max(need)), dtype=torch.int32)
    tables[0, :need[0]], tables[1, :need[1]] = torch.arange(need[0]), torch.arange(need[0], nb)
    kv, whole = oc.guarded((2, L, nb, bs, H, D), torch.bfloat16, 3.0)
    q_out, q_whole = oc.guarded((L, n, H * G, D), torch.bfloat16, 5.0)
    x = torch.randn((L, n, H * (G + 2), D), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    llmig_append_rotary(Pool(list(kv[0].unbind(0)), list(kv[1].unbind(0)), layouts), x[:, :, H * G:H * (G + 1)],
                        x[:, :, H * (G + 1):], tables.cuda(), froms, news, table_of(512, D).cuda(), q=x[:, :, :H * G], q_out=q_out)
    torch.cuda.synchronize()
    assert whole() and q_whole()
    assert int((q_out == 5).sum()) < q_out.numel() // 1000 + 10
    written = (kv != 3).view(2, -1).sum(1)
    assert bool((written <= L * n * H * D).all()) and bool((written > L * n * H * D * 0.999 - 10).all())
