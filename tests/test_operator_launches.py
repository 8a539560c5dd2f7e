"""Calls of the operators for long contexts that take more than one launch: the
launches cover every unit of work once, in order, and each fits the grid (CPU only,
over a stand-in HIP runtime)."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from paper_2406_03243_amd.build import LIBRARY

TESTS = os.path.dirname(os.path.abspath(__file__))
pytestmark = pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc missing")
MOST = 1 << 22      # workgroups of a launch


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    fake = str(tmp_path_factory.mktemp("fake") / "libfakehip.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", fake, os.path.join(TESTS, "fake_hip.c")], check=True)

    def run(call):
        res = subprocess.run([sys.executable, os.path.join(TESTS, "operator_calls.py"), fake, LIBRARY],
                             input=json.dumps([call]), capture_output=True, text=True, timeout=300)
        assert res.returncode == 0, res.stderr[-3000:]
        got = json.loads(res.stdout)[0]
        assert got["rc"] == 0
        by_kernel = {}
        for x in got["launches"]:
            by_kernel.setdefault(x["kernel"], []).append(x)
        return by_kernel
    return run


def covers(launches, first, per, units, several=True):
    """`per` workgroups a unit; `first` names the field that holds a launch's first unit."""
    at = 0
    for x in launches:
        assert x["args"][first] == at and 0 < x["grid"] <= MOST and x["grid"] % per == 0
        at += x["grid"] // per
    assert at == units and (len(launches) > 1) == several


def ceil(a, b):
    return -(-a // b)


# a prompt of 512k tokens into 80 layers of 32 heads of 128, 64 query heads
LONG = dict(op="append", n_toks=[3, 1 << 19], positions=1 << 20, table_stride=40000, q_heads=64)


@pytest.mark.parametrize("layouts", [(0, 0), (2, 3), (3, 2)])
@pytest.mark.parametrize("layers", [80, 79])
@pytest.mark.parametrize("bs", [16, 24])
def test_append(launches, layouts, layers, bs):
    got = launches(dict(LONG, pool_args=dict(layers=layers, heads=32, dim=128, bs=bs, layouts=layouts)))
    tokens, from_toks, n_toks = 3 + (1 << 19), (5, 0), (3, 1 << 19)
    blocks = sum((f + n - 1) // bs - f // bs + 1 for f, n in zip(from_toks, n_toks))
    seen = 0
    for kernel, runs in got.items():
        for tensor in sorted({x["args"]["tensor"] for x in runs}):
            part = [x for x in runs if x["args"]["tensor"] == tensor]
            a = part[0]["args"]
            slices = a["by_slice"]
            if kernel == "append_rotary_dims":
                assert a["by_layer"] == layers and slices == ceil(32 * 128 // 8, 256 // (bs // 8))     # (head, 8 dims) each
            else:
                lg = part[0]["template"][1]
                assert a["by_layer"] == ceil(layers, lg) and slices == ceil(a["lanes"], 256)
            units = (tokens if kernel == "append_rotary_rows" else blocks) * a["by_layer"]
            covers(part, "first_unit", slices, units, several=units * slices > MOST)
            seen += len(part) > 1
    assert seen == len(got), {k: len(v) for k, v in got.items()}


@pytest.mark.parametrize("heads,dim,bs", [(8, 128, 16), (40, 128, 8), (2, 64, 16)])
def test_bounds(launches, heads, dim, bs):
    blocks = 1 << 20
    got = launches(dict(op="bounds", pool_args=dict(layers=80, heads=heads, dim=dim, bs=bs), table_stride=blocks + 3,
                        bounds_args=dict(layers=80, heads=heads, dim=dim), from_toks=[5, 0], ctx_lens=[6, blocks * bs]))
    (runs,) = got.values()
    a = runs[0]["args"]
    assert a["by_slice"] == ceil(heads * dim // 8, 256) and a["by_group"] == ceil(blocks + 1, a["side"])
    covers(runs, "first_item", 1, a["by_group"] * 80 * a["by_slice"])


def test_scores(launches):
    got = launches(dict(op="select", batch=256, q_heads=16, ctx_lens=[120000 - i for i in range(256)], table_stride=8000,
                        count=64, bounds_args=dict(layers=80, heads=8, dim=128)))
    scores, lists = got["score_blocks"], got["list_blocks"]
    a = scores[0]["args"]
    assert a["slices"] == 1 and a["parts"] * 2 * a["per_row"] >= 7500
    covers(scores, "first_item", 1, 80 * 256 * a["slices"] * a["parts"])
    covers(lists, "first_item", 1, 80 * 256 * 8, several=False)


def test_lists(launches):
    got = launches(dict(op="select", batch=256, q_heads=256, ctx_lens=[700] * 256, table_stride=60, count=9,
                        bounds_args=dict(layers=80, heads=256, dim=64)))
    covers(got["list_blocks"], "first_item", 1, 80 * 256 * 256)
    a = got["score_blocks"][0]["args"]
    assert a["slices"] == 8
    covers(got["score_blocks"], "first_item", 1, 80 * 256 * 8 * a["parts"], several=80 * 256 * 8 * a["parts"] > MOST)


@pytest.mark.parametrize("op", ["attend", "prefix"])
@pytest.mark.parametrize("tokens", [100, 700])
def test_attention(launches, op, tokens):
    """Of short sequences a wavefront takes a head, of longer ones a workgroup."""
    heads, layers, batch = 1002, 80, 250
    kw = dict(count=64) if op == "attend" else dict(prefix_blocks=0)
    got = launches(dict(op=op, batch=batch, q_heads=heads, ctx_lens=[tokens] * batch, table_stride=60,
                        pool_args=dict(layers=layers, heads=heads, dim=64), **kw))
    runs = got["attn_partial_mfma"]
    alone = tokens == 100
    assert all(x["template"][3] == (2 if alone else 1) for x in runs)
    covers(runs, "item_base", (ceil(heads, 4) if alone else heads) * layers, batch)
