"""Plain references in 64 bits, and error bounds, for the operators of a decode
step over long contexts.  Everything is computed on the CPU from the 16-bit
inputs as they are.

Bound of an attention output (the reasoning is that of tests/attn_cases.py),
for a row of n tokens, u = 2^-24 and lambda = 8:

    tol = A (eps_p + lambda u (2 sqrt(depth) + 4 (sqrt(D) + 2) S + 2)) + lambda sqrt(n) u_lo / W + u

A the softmax-weighted mean of |v|, eps_p = 2^-16 (bf16) or 2^-22 (fp16) the
weights' error as a 16-bit high and a 16-bit low part, depth = 64 + ceil(n / 16)
at least the longest chain of fp32 additions (a matrix product adds 32 terms, a
wavefront takes at most every 16-token group, then wavefronts and partitions
join, fewer than 32 of them), S a bound on |score| (here |k| is not bounded by
1, so it is the largest sum_d |q_d k_d|, scaled), u_lo = 2^-25 for fp16 (the
low part's absolute rounding; 0 for bf16), W the weights' sum relative to the
largest."""
from __future__ import annotations

import math

import torch

LAMBDA, U32 = 8.0, 2.0 ** -24
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
EPS_P = {"fp16": 2.0 ** -22, "bf16": 2.0 ** -16}
HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}     # of one rounding to the type, relative


def rows_of(tables, b, tokens, bs):
    """(block, slot) of the listed tokens of sequence b."""
    t = torch.as_tensor(tokens, dtype=torch.long)
    return tables[b].long()[t // bs], t % bs


def attention(k, v, q, scale, dtype):
    """One row: k, v [n][D], q [G][D] (any type): (out [G][D], tol [G][D])."""
    G, D = q.shape
    n = k.shape[0]
    if n == 0:
        return torch.zeros(G, D, dtype=torch.float64), torch.zeros(G, D, dtype=torch.float64)
    k, v, q = k.double(), v.double(), q.double()
    s = (q @ k.t()) * scale
    out = torch.zeros(G, D, dtype=torch.float64)
    tol = torch.full((G, D), U32, dtype=torch.float64)
    for g in range(G):
        if bool(torch.isnan(s[g]).any()) or bool((s[g] == math.inf).any()) or not bool(torch.isfinite(s[g]).any()):
            tol[g] = 0.0            # zeros, exactly
            continue
        live = s[g] > -math.inf
        w = torch.exp(s[g][live] - s[g].max())
        W = w.sum()
        out[g] = (w @ v[live]) / W
        A = (w @ v[live].abs()) / W
        S = abs(scale) * float((q[g].abs() * k[live].abs()).sum(1).max())
        rel = EPS_P[dtype] + LAMBDA * U32 * (2 * math.sqrt(64 + -(-n // 16)) + 4 * (math.sqrt(D) + 2) * S + 2)
        lo = LAMBDA * math.sqrt(n) * U32 / 2 / float(W) * float(v[live].abs().max()) if dtype == "fp16" else 0.0
        tol[g] = A * rel + lo + U32
    return out, tol


def small_weights(kv, q, tables, b, n):
    """Gives sequence b's first token a score of 0 and values of 0, its other n -
    1 ones weights of 2^-15.3 and values of 1: fp16 holds such a weight in steps
    of 2^-24 of the largest, times 2^7 in steps of 2^-31, half of one off at most.
    The bound of (1 - weight of the first): every weight off by 2^-32, and the
    relative part of attention()."""
    bs = kv.shape[3]
    q[:, b] = 0
    q[:, b, :, 0] = 1
    blk, slot = rows_of(tables, b, range(n), bs)
    kv[0][:, blk, slot], kv[1][:, blk, slot] = 0, 1
    kv[0][:, blk[1:], slot[1:], :, 0] = -10.6
    kv[1][:, blk[0], slot[0]] = 0
    w = (n - 1) * math.exp(float(torch.tensor(-10.6, dtype=kv.dtype)))
    rel = EPS_P["fp16"] + LAMBDA * U32 * (2 * math.sqrt(64 + -(-n // 16)) + 4 * (math.sqrt(kv.shape[5]) + 2) * 10.7 + 2)
    return w / (1 + w), n * 2.0 ** -32 + w / (1 + w) * rel + U32


def decode(kv, q, tables, scale, dtype, tokens_of):
    """kv [2][L][blocks][bs][H][D], q [L][B][Hq][D] on the CPU; tokens_of(l, b, g)
    lists the tokens a row attends to."""
    L, B, HQ, D = q.shape
    bs, H = kv.shape[3], kv.shape[4]
    G = HQ // H
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for l in range(L):
        for b in range(B):
            for g in range(H):
                blk, slot = rows_of(tables, b, tokens_of(l, b, g), bs)
                at = slice(g * G, (g + 1) * G)
                out[l, b, at], tol[l, b, at] = attention(kv[0, l, blk, slot, g], kv[1, l, blk, slot, g], q[l, b, at],
                                                         scale, dtype)
    return out, tol


def rotate(x, cos, sin, interleaved):
    """x [..., D] float64, cos and sin [..., h]."""
    h = cos.shape[-1]
    y = x.clone()
    a, b = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def select(lo, hi, q, n, keep_first, keep_last, count):
    """lo, hi [n][H][D], q [Hq][D]: lists [H][count]."""
    H = lo.shape[1]
    G = q.shape[0] // H
    out = torch.full((H, count), -1, dtype=torch.int32)
    for g in range(H):
        x = q[g * G:(g + 1) * G].double()
        score = (x.clamp(min=0).sum(0) * hi[:, g].double() + x.clamp(max=0).sum(0) * lo[:, g].double()).sum(-1)
        score = [math.inf if math.isnan(s) else s for s in score.tolist()]
        must = [j for j in range(n) if j < keep_first or j >= n - keep_last]
        rest = sorted((j for j in range(n) if j not in set(must)), key=lambda j: (-score[j], j))
        chosen = sorted((must + rest)[:min(count, n)])
        out[g, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
    return out


def worst(got, want, tol):
    """Largest |got - want| / tol; infinite where one is not finite, or an
    exact value is missed."""
    got = got.double().cpu()
    err = (got - want).abs()
    ratio = torch.where(tol > 0, err / tol.clamp(min=1e-300), torch.where(err > 0, math.inf, 0.0))
    ratio = torch.where(torch.isfinite(got), ratio, torch.tensor(math.inf, dtype=torch.float64))
    return float(ratio.max()) if ratio.numel() else 0.0


# ---- inputs whose scores are exact --------------------------------------------------
# All keys and values are 0 but those of a few live tokens, whose keys are -1 in
# the first dim and whose values are of one sign; queries are x in the first dim
# alone, the scale is 1.  So scores are 0 and -x, exactly, every group of 16 tokens
# has the largest among them, sums of the others' weights are whole numbers, and
# what is left of a row's error is that of the live tokens' weights w = exp(-x):
#   the scaled score and what is taken from it, |x| <= 2: (5.8 + 4) u ln 2, and the
#   exponential's ulp, 2 u: 9 u; of two live tokens at most 2 * 3 parts added to others,
#   2 u each: 12 u; 2 live weights, and 14 binades that the weight sum can pass: 16
#   u; division, factors between wavefronts and partitions (all 1): 4 u; 41 u in all,
# and the parts that a weight is split into (a part is off by half a step of what it
# rounds): 2^-22 of fp16's two and of bf16's three, 2^-17 of bf16's two.
CHAIN = 41 * U32
PARTS = {("fp16", 2): 2.0 ** -22, ("bf16", 2): 2.0 ** -17, ("bf16", 3): 2.0 ** -22}


def split(w, dtype, parts):
    """w (float64) as the sum of `parts` roundings to the type, each of what the
    ones before leave; fp16 takes it times 2^7."""
    t, up = TYPES[dtype], 128.0 if dtype == "fp16" else 1.0
    left, total = (w * up).float(), torch.zeros_like(w)
    for _ in range(parts):
        part = left.to(t).float()
        left, total = left - part, total + part.double()
    return total / up


def telling(dtype, parts):
    """16 queries x whose weights lose most with one part less than `parts`."""
    x = torch.arange(0.25, 2.0, 2.0 ** -7, dtype=torch.float64).to(TYPES[dtype]).double().unique()
    w = torch.exp(-x)
    loss = (split(w, dtype, parts - 1) / w - 1).abs()
    return x[loss.argsort(descending=True)[:16]]


def exact_scores(kv, q, tables, live, dtype, parts):
    """Fills kv and q; live: (sequence, token) pairs, at most two of a sequence's."""
    bs, D = kv.shape[3], kv.shape[5]
    x = telling(dtype, parts)
    kv.zero_()
    q.zero_()
    rows = torch.arange(q[..., 0].numel()).view(q.shape[:3])
    q[..., 0] = x[rows * 5 % 16].to(q.dtype)
    v = (1.0 + torch.arange(D) % 8 / 8).to(kv.dtype)
    for b, t in live:
        blk, slot = int(tables[b, t // bs]), t % bs
        kv[0, :, blk, slot, :, 0] = -1
        kv[1, :, blk, slot] = v


def tiny_weights(n):
    """What a row of small_weights() comes to, and its bound: the score -10.6 is one
    product and exact, so a weight is off by what scaling it and taking the largest
    from it round, 15.3 (1 + 1 + 1) u ln 2, and the exponential's 2 u, 34 u, or, of a
    partition without the first token, by what the factor does to which its maximum
    goes through a record, 15.3 (2 + 1 + 1) u ln 2 + 2 u = 44 u; its two parts by 2^-32 of
    the largest; the sums as in attention()."""
    w = (n - 1) * math.exp(float(torch.tensor(-10.6, dtype=torch.float16)))
    return w / (1 + w), n * 2.0 ** -32 + w / (1 + w) * U32 * (44 + 4 + LAMBDA * 2 * math.sqrt(64 + -(-n // 16)))


def exact_rows(q, D, ctx, live):
    """The 64-bit outputs for inputs of exact_scores(); live: how many live tokens each sequence attends to."""
    w = torch.exp(-q[..., :1].double())
    k, n = (torch.tensor(x, dtype=torch.float64)[None, :, None, None] for x in (live, ctx))
    v = 1.0 + torch.arange(D, dtype=torch.float64) % 8 / 8
    return k * w * v / torch.clamp(n - k + k * w, min=1e-9)


def check_exact(out, q, ctx, live, dtype, parts):
    """The largest error of outputs of such inputs, in bounds."""
    want = exact_rows(q, q.shape[3], ctx, live)
    return worst(out, want, want * (PARTS[dtype, parts] + CHAIN))


def guarded(shape, dtype, value, device="cuda"):
    """(a tensor of `shape` inside a buffer filled with `value`, a check that nothing around it changed)."""
    n = math.prod(shape)
    flat = torch.full((n + 8192,), value, dtype=dtype, device=device)

    def untouched():
        return bool((flat[:4096] == value).all()) and bool((flat[4096 + n:] == value).all())
    return flat[4096:4096 + n].view(shape), untouched
