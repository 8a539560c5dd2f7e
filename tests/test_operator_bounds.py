"""The bounds of operator_cases.py tell weights of fewer parts (CPU only)."""
import pytest
import torch

import operator_cases as oc


def rows(dtype, parts, D=64, bs=16, n=700, G=16):
    tables = torch.arange(-(-n // bs), dtype=torch.int32)[None]
    kv = torch.empty((2, 1, tables.shape[1], bs, 1, D), dtype=oc.TYPES[dtype])
    q = torch.empty((1, 1, G, D), dtype=kv.dtype)
    oc.exact_scores(kv, q, tables, [(0, 3), (0, 400)], dtype, parts)
    return kv, q, tables, range(n)


def emulated(kv, q, tables, tokens, dtype, parts):
    """Attention whose weights, but not their sum, are taken in parts."""
    blk, slot = oc.rows_of(tables, 0, tokens, kv.shape[3])
    k, v = kv[0, 0, blk, slot, 0].double(), kv[1, 0, blk, slot, 0].double()
    w = torch.exp(q[0, 0].double() @ k.t()).float().double()
    return ((oc.split(w, dtype, parts) @ v) / w.sum(1, keepdim=True))[None, None]


@pytest.mark.parametrize("dtype,parts", list(oc.PARTS))
def test_a_part_less_exceeds_the_bound(dtype, parts):
    kv, q, tables, tokens = rows(dtype, parts)
    check = lambda p: oc.check_exact(emulated(kv, q, tables, tokens, dtype, p), q, [len(tokens)], [2], dtype, parts)
    assert check(parts) <= 1 and check(parts - 1) > 1.5, (check(parts), check(parts - 1))
    # every one of the rows, not the worst alone
    want, _ = oc.decode(kv, q, tables, 1.0, dtype, lambda l, b, g: tokens)
    assert float((oc.exact_rows(q, 64, [len(tokens)], [2]) / want - 1).abs().max()) < 1e-12
    err = ((emulated(kv, q, tables, tokens, dtype, parts - 1) - want).abs() / want).amax(-1)
    assert float(err.min()) > 1.3 * (oc.PARTS[dtype, parts] + oc.CHAIN)


@pytest.mark.parametrize("n", [688, 700, 748, 2100])
def test_small_weights_tell_their_parts(n):
    """The bound of tiny_weights() against fp16 weights of one part, and of two that are not scaled up."""
    want, tol = oc.tiny_weights(n)
    w = torch.exp(torch.tensor([-10.6], dtype=torch.float16).double())
    high = w.float().to(torch.float16)
    unscaled = high.double() + (w.float() - high.float()).to(torch.float16).double()
    for got in (oc.split(w, "fp16", 1), unscaled):
        err = abs(float((n - 1) * got / (1 + (n - 1) * w)) - want)
        assert err > 1.5 * tol, (err, tol)
    got = oc.split(w, "fp16", 2)
    assert abs(float((n - 1) * got / (1 + (n - 1) * w)) - want) <= tol

