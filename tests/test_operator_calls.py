"""The operators for long contexts without a GPU: what they refuse, and which
kernels their calls launch, over a stand-in HIP runtime (operator_calls.py)."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from paper_2406_03243_amd.build import LIBRARY

TESTS = os.path.dirname(os.path.abspath(__file__))
pytestmark = pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc missing")
OK, EINVAL = 0, -1
FAR = 1 << 44


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    fake = str(tmp_path_factory.mktemp("fake") / "libfakehip.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", fake, os.path.join(TESTS, "fake_hip.c")], check=True)

    def run(calls):
        res = subprocess.run([sys.executable, os.path.join(TESTS, "operator_calls.py"), fake, LIBRARY],
                             input=json.dumps(calls), capture_output=True, text=True, timeout=300)
        assert res.returncode == 0, res.stderr[-3000:]
        return json.loads(res.stdout)
    return run


def kernels(got):
    return [x["kernel"] for x in got["launches"]]


BAD = {
    "append": [
        dict(no_pool=True), dict(dtype=2), dict(dtype=-1), dict(batch=0), dict(batch=257), dict(q_heads=-1),
        dict(table_stride=0), dict(table_stride=1), dict(tables=0), dict(tables=FAR + 2), dict(from_toks=None), dict(n_toks=None),
        dict(interleaved=2), dict(rotary_dim=-2), dict(rotary_dim=7), dict(rotary_dim=66), dict(cos_sin=0), dict(cos_sin=FAR + 2),
        dict(positions=0), dict(positions=19), dict(first_pos=[0, 81]), dict(first_pos=[-1, 0]), dict(from_toks=[-1, 0]),
        dict(n_toks=[1, -1]), dict(from_toks=[5, 2 ** 31 - 5]), dict(from_toks=[64, 0]), dict(q=0), dict(k=0), dict(v=0),
        dict(q_out=0), dict(q=FAR + 8), dict(k=2 * FAR + 8), dict(v=3 * FAR + 2), dict(q_out=4 * FAR + 4), dict(q_layer=-8),
        dict(k_token=-8), dict(v_layer=12), dict(k_token=4), dict(q_out=FAR), dict(q_out=FAR + 16), dict(q_out=2 * FAR - 32),
        dict(pool_args=dict(elem=4)), dict(pool_args=dict(dim=68)), dict(k_layer=2 ** 62), dict(v_token=2 ** 61)],
    "bounds": [
        dict(no_pool=True), dict(no_bounds=True), dict(dtype=2), dict(batch=0), dict(batch=257), dict(tables=0),
        dict(tables=FAR + 1), dict(table_stride=0), dict(table_stride=2), dict(from_toks=None), dict(ctx_lens=None),
        dict(from_toks=[-1, 0]), dict(from_toks=[7, 0]), dict(ctx_lens=[-1, 40]), dict(bounds_args=dict(bs=2)),
        dict(bounds_args=dict(blocks=63)), dict(bounds_args=dict(heads=1)), dict(bounds_args=dict(dim=128)),
        dict(bounds_args=dict(layers=2)), dict(bounds_args=dict(elem=4)), dict(bounds_args=dict(at=1)),
        dict(bounds_args=dict(layouts=(1, 0))), dict(pool_args=dict(layouts=(0, 3))), dict(pool_args=dict(elem=1))],
    "select": [
        dict(no_bounds=True), dict(dtype=3), dict(block_size=0), dict(q=0), dict(q=FAR + 8), dict(batch=0), dict(batch=257),
        dict(q_heads=0), dict(q_heads=3), dict(tables=0), dict(tables=FAR + 2), dict(table_stride=6), dict(ctx_lens=None),
        dict(ctx_lens=[-1, 0]), dict(keep_first=-1), dict(keep_last=-1), dict(keep_last=4), dict(count=0), dict(count=-4),
        dict(workspace=0), dict(workspace=FAR + 4), dict(less=1), dict(blocks=0), dict(blocks=FAR + 1),
        dict(bounds_args=dict(bs=16)), dict(bounds_args=dict(dim=96)), dict(bounds_args=dict(layouts=(0, 1))),
        dict(keep_first=2 ** 31 - 1, keep_last=2 ** 31 - 1, count=5)],
    "attend": [
        dict(no_pool=True), dict(dtype=2), dict(q=0), dict(q=FAR + 8), dict(batch=0), dict(batch=257), dict(q_heads=3),
        dict(q_heads=6), dict(tables=0), dict(table_stride=6), dict(ctx_lens=None), dict(ctx_lens=[-1, 3]), dict(blocks=0),
        dict(blocks=FAR + 2), dict(count=0), dict(count=-1), dict(out=0), dict(out=FAR + 8), dict(pool_args=dict(dim=96)),
        dict(pool_args=dict(layouts=(1, 1))), dict(pool_args=dict(elem=4)), dict(workspace=FAR + 8),
        dict(ctx_lens=[9000, 3], table_stride=600, count=600, workspace=0),
        dict(ctx_lens=[9000, 3], table_stride=600, count=600, less=1)],
    "prefix": [
        dict(no_pool=True), dict(dtype=2), dict(q=0), dict(q=FAR + 8), dict(batch=0), dict(batch=257), dict(q_heads=3),
        dict(q_heads=6), dict(tables=0), dict(table_stride=6), dict(ctx_lens=None), dict(ctx_lens=[-1, 3]),
        dict(prefix_blocks=-1), dict(prefix_blocks=9), dict(out=0), dict(out=FAR + 8), dict(pool_args=dict(dim=32)),
        dict(pool_args=dict(layouts=(0, 2))), dict(workspace=FAR + 8),
        dict(ctx_lens=[9000] * 40, table_stride=600, prefix_blocks=560, workspace=0),
        dict(ctx_lens=[9000] * 40, table_stride=600, prefix_blocks=560, less=1)],
}


@pytest.mark.parametrize("op", BAD)
def test_refusals(call, op):
    """Nothing is launched by a call that is refused; the call itself is fine."""
    good, *got = call([dict(op=op)] + [dict(op=op, **c) for c in BAD[op]])
    assert good["rc"] == OK and good["launches"]
    for c, r in zip(BAD[op], got):
        assert r["rc"] == EINVAL and not r["launches"], (op, c, r)


def test_calls_without_work_launch_nothing(call):
    got = call([dict(op="append", n_toks=[0, 0]), dict(op="append", n_toks=[0, 0], k=0, v=0, q=0, q_out=0),
                dict(op="bounds", from_toks=[6, 40])])
    assert [(r["rc"], r["launches"]) for r in got] == [(OK, [])] * 3


def test_append_goes_block_by_block_where_tokens_are_scattered(call):
    many, one = dict(n_toks=[2, 20000], positions=21000, table_stride=2600), dict(n_toks=[1, 1])
    paged = dict(layouts=(2, 3))
    for kw, want in [
            (dict(**many), ["append_rotary_rows"]), (dict(pool_args=dict(layouts=(1, 1)), **many), ["append_rotary_rows"]),
            (dict(pool_args=paged, **one), ["append_rotary_rows"]), (dict(pool_args=paged, n_toks=[2, 20]), ["append_rotary_rows"]),
            (dict(pool_args=paged, **many), ["append_rotary_rows", "append_rotary_slots", "append_rotary_dims"]),
            (dict(pool_args=paged, q_heads=0, **many), ["append_rotary_slots", "append_rotary_dims"]),
            (dict(pool_args=dict(layouts=(3, 2)), **many), ["append_rotary_rows", "append_rotary_dims", "append_rotary_slots"]),
            (dict(pool_args=dict(layouts=(3, 0)), **many), ["append_rotary_rows", "append_rotary_dims"]),
            (dict(pool_args=dict(layouts=(0, 3), bs=12), **many), ["append_rotary_rows"])]:
        got = call([dict(op="append", **kw)])[0]
        assert got["rc"] == OK and kernels(got) == want, kw


def test_select_scores_only_what_has_to_be_chosen_from(call):
    few, many, some, long, longer, longish, longest = call([
        dict(op="select", count=7, keep_first=0), dict(op="select"),
        dict(op="select", ctx_lens=[16 * 257, 3], table_stride=300),
        dict(op="select", ctx_lens=[16 * 1025, 3], table_stride=2000), dict(op="select", ctx_lens=[16 * 4097, 3], table_stride=9000),
        dict(op="select", ctx_lens=[16 * 8193, 3], table_stride=9000),
        dict(op="select", ctx_lens=[16 * 16385, 3], table_stride=20000)])
    assert kernels(few) == ["list_blocks"] and kernels(many) == ["score_blocks", "list_blocks"]
    assert [x["launches"][-1]["template"] for x in (many, some, long, longer, longish, longest)] == [
        [64, 4], [256, 4], [1024, 4], [1024, 8], [1024, 16], [1024, 0]]


def test_prefix_is_read_once_only_where_that_pays(call):
    many = dict(pool_args=dict(heads=16, dim=128), q_heads=16, table_stride=200)
    short, shared, split, lone, none, long = call([
        dict(op="prefix"), dict(op="prefix", ctx_lens=[700] * 30, prefix_blocks=43, **many),
        dict(op="prefix", ctx_lens=[3000] * 100, prefix_blocks=180, **many),
        dict(op="prefix", ctx_lens=[3000] + [40] * 29, prefix_blocks=180, **many),
        dict(op="prefix", ctx_lens=[3000] * 30, prefix_blocks=0, **many),
        dict(op="prefix", ctx_lens=[700] * 30 + [9000, 3], prefix_blocks=43, **dict(many, table_stride=600))])
    once = ["prefix_rows", "attn_partial_mfma"]
    assert kernels(long) == once + ["prefix_join"]
    assert kernels(short) == ["attn_partial_mfma"] and kernels(shared) == once and kernels(split) == once
    assert shared["launches"][0]["template"][2] == 2 and split["launches"][0]["template"][2] == 4
    for x in (lone, none):
        assert kernels(x)[0] == "attn_partial_mfma" and "prefix_rows" not in kernels(x)


def test_prefix_cases_of_the_gpu_tests_read_it_once(call):
    import test_gpu_prefix_attention as t
    joins = set()
    for L, H, G, D, bs, dtype, ctx, prefix in t.SHARED + t.LONG + t.FEW + [(*t.SHAPE, "bf16", t.CTX, t.PREFIX)]:
        got = call([dict(op="prefix", pool_args=dict(layers=L, blocks=2000, bs=bs, heads=H, dim=D), q_heads=H * G,
                         table_stride=max(ctx) // bs + 1, ctx_lens=ctx, prefix_blocks=prefix)])[0]
        assert got["rc"] == OK and kernels(got)[0] == "prefix_rows", (L, H, G, D, bs)
        if (L, H, G, D, bs, dtype, ctx, prefix) in t.LONG:
            assert kernels(got)[2] == "prefix_join"
            joins.add(tuple(got["launches"][2]["template"]))
        if (L, H, G, D, bs, dtype, ctx, prefix) in t.FEW:
            assert got["launches"][1]["template"][3] == 2, (L, H, G, D, bs)
    assert {j[1] for j in joins} == {1, 8}, joins


def test_workspaces_are_those_of_the_records(call):
    """Listed blocks: a record of head_dim + 4 floats per layer, query head and
    partition of a sequence of several.  Shared prefix: the same of the tokens behind
    it, and one per layer, query head, sequence and partition of the prefix."""
    a, b, c = call([dict(op="attend", ctx_lens=[9000, 3], table_stride=600, count=600), dict(op="attend"),
                    dict(op="select")])
    assert b["workspace"] == 0 and a["workspace"] > 0 and a["workspace"] % (4 * (64 + 4) * 4) == 0
    assert c["workspace"] == 8 * 2 * (7 + 3)
    p = call([dict(op="prefix", ctx_lens=[700] * 30, prefix_blocks=43, pool_args=dict(heads=16, dim=128), q_heads=16,
                   table_stride=60)])[0]
    records = p["workspace"] // (16 * 132 * 4)
    assert p["workspace"] % (16 * 132 * 4) == 0 and records >= 30 and records % 30 == 0


def test_short_sequences_take_a_wavefront_a_head(call):
    shape = dict(pool_args=dict(layers=2, heads=8, dim=128), q_heads=32, table_stride=80)
    many, longer = dict(batch=128, ctx_lens=[40] * 128), dict(batch=128, ctx_lens=[400] * 128)
    got = call([dict(op="attend", **shape, **dict(batch=60, ctx_lens=[40] * 60)), dict(op="attend", **shape, **many),
                dict(op="attend", count=64, **shape, **longer), dict(op="attend", **dict(shape, pool_args=dict(
                    layers=16, heads=1, dim=128), q_heads=4), **many),
                dict(op="attend", **dict(shape, pool_args=dict(layers=2, heads=8, dim=128, bs=12)), **many),
                dict(op="prefix", ctx_lens=[1000] * 128, prefix_blocks=60, **shape)])
    assert all(x["rc"] == OK for x in got)
    kind = [[l["template"][3] for l in x["launches"] if l["kernel"] == "attn_partial_mfma"] for x in got]
    assert kind == [[1], [2], [1], [1], [0], [2]]


@pytest.mark.parametrize("tokens", [2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 2048, 2 ** 31 - 2049])
@pytest.mark.parametrize("kw", [dict(op="attend"), dict(op="prefix"), dict(op="prefix", prefix_blocks=0), dict(op="bounds"),
                                dict(op="select")] + [dict(op="decode", form=f) for f in ("workspace", "noalloc", "migrate")],
                         ids=lambda c: "_".join(str(x) for x in c.values()))
def test_lengths_near_the_end_of_32_bits_need_their_blocks(call, kw, tokens):
    """A sequence whose length rounds up to blocks past 2^31 is one the table row is too short for."""
    good, bad = call([dict(kw), dict(kw, ctx_lens=[tokens, 70])])
    assert good["rc"] == OK and good["launches"]
    assert bad["rc"] == EINVAL and not bad["launches"]


def test_longest_sequences_of_decode_attention(call):
    """2^31 - 2049 tokens, a row of blocks for all of them; more are refused whatever the row holds."""
    n, row = 2 ** 31 - 2049, dict(table_stride=2 ** 31 - 1, pool_args=dict(bs=1))
    ops = [dict(op="attend", count=7), dict(op="prefix", prefix_blocks=0), dict(op="decode")]
    for c in ops:
        good, bad = call([dict(c, **row, ctx_lens=[n, 70]), dict(c, **row, ctx_lens=[n + 1, 70])])
        assert good["rc"] == OK and good["launches"], c
        assert bad["rc"] == EINVAL and not bad["launches"], c
    wide = dict(op="attend", pool_args=dict(bs=1 << 16), table_stride=1 << 15, ctx_lens=[n, 70])
    few, all_of_them = call([dict(wide, count=100), dict(wide, count=1 << 15)])
    assert few["rc"] == OK and all_of_them["rc"] == EINVAL and not all_of_them["launches"]
