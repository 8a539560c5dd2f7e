"""Runs calls of the operators for long contexts over a stand-in HIP runtime
(fake_hip.c) and prints, as JSON, what each returns and which kernels it
launches.  A process of its own, without torch:

    python operator_calls.py FAKE_HIP.so LIBLLMIG.so < calls.json

A call is {"op": name, ...}: the arguments that differ from those of a small
valid call.  Device addresses are numbers that nothing reads."""
import ctypes
import json
import re
import sys

import numpy as np

U32, I32, I64, U64, P = ctypes.c_uint32, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_void_p


class Desc(ctypes.Structure):
    _fields_ = [(n, I32) for n in ("num_layers", "num_blocks", "block_size", "num_kv_heads", "head_dim", "elem_bytes")] \
        + [("k_ptrs", ctypes.POINTER(U64)), ("v_ptrs", ctypes.POINTER(U64)), ("k_layout", I32), ("v_layout", I32)]


class Append(ctypes.Structure):
    _fields_ = [("dtype", I32), ("batch", I32), ("q_heads", I32), ("table_stride", I32), ("q", P), ("k", P), ("v", P),
                ("q_out", P), ("q_layer", I64), ("q_token", I64), ("k_layer", I64), ("k_token", I64), ("v_layer", I64),
                ("v_token", I64), ("tables", P), ("from_toks", P), ("n_toks", P), ("first_pos", P), ("cos_sin", P),
                ("positions", I32), ("rotary_dim", I32), ("interleaved", I32)]


class Divisor(ctypes.Structure):
    _fields_ = [("d", U32), ("m", U32), ("shift", U32)]


# The kernels' argument structures, as the sources declare them (to the last field that a test reads).
class AppendArgs(ctypes.Structure):
    _fields_ = [("pointers", U64 * 13), ("first_unit", U32), ("num_layers", U32), ("num_blocks", U32), ("block_size", U32),
                ("table_stride", U32), ("tile_bytes", U32), ("q_heads", U32), ("kv_heads", U32), ("tokens", U32),
                ("batch", U32), ("rows_heads", U32 * 3), ("row_chunks", U32), ("lanes", U32), ("half", U32),
                ("interleaved", U32), ("wide", U32), ("layouts", I32 * 2), ("one_each", U32), ("tensor", U32),
                ("by_slice", Divisor), ("by_layer", Divisor)]


class BoundsArgs(ctypes.Structure):
    _fields_ = [("pointers", U64 * 3), ("num_layers", U32), ("num_blocks", U32), ("block_size", U32), ("table_stride", U32),
                ("tile_bytes", U32), ("batch", U32), ("slot_chunks", U32), ("rows", U32), ("side", U32), ("one_each", U32),
                ("first_item", U32), ("by_slice", Divisor), ("by_group", Divisor)]


class SelectArgs(ctypes.Structure):
    _fields_ = [("pointers", U64 * 5), ("num_layers", U32), ("num_blocks", U32), ("batch", U32), ("q_heads", U32),
                ("kv_heads", U32), ("table_stride", U32), ("keep_first", U32), ("keep_last", U32), ("count", U32),
                ("blocks", U32), ("first_item", U32), ("per_row", U32), ("parts", U32), ("slices", U32)]


class AttnArgs(ctypes.Structure):
    _fields_ = [("pointers", U64 * 5), ("scale", ctypes.c_float), ("num_layers", U32), ("batch", U32), ("q_heads", U32),
                ("kv_heads", U32), ("block_size", U32), ("table_stride", U32), ("item_base", U32), ("layer_items", U32)]


STRUCTS = {"append_rotary_rows": AppendArgs, "append_rotary_slots": AppendArgs, "append_rotary_dims": AppendArgs,
           "key_bounds_rows": BoundsArgs, "score_blocks": SelectArgs, "list_blocks": SelectArgs, "attn_partial_mfma": AttnArgs}


def fields(args):
    out = {}
    for name, kind in args._fields_:
        v = getattr(args, name)
        if name != "pointers":
            out[name] = v.d if kind is Divisor else list(v) if isinstance(v, ctypes.Array) else v
    return out


launches = []


@ctypes.CFUNCTYPE(None, ctypes.c_char_p, ctypes.POINTER(U32), U64, ctypes.c_void_p)
def on_launch(name, gb, lds, args):
    m = re.search(r"\d+([a-z]+_[a-z_]+?)(?:I|E|N)", name.decode().split("GLOBAL__N_1")[-1])
    launches.append({"kernel": m.group(1), "grid": gb[0], "block": gb[3],
                     "template": [int(x) for x in re.findall(r"Li(\d+)E", name.decode())]})
    if m.group(1) in STRUCTS:
        launches[-1]["args"] = fields(STRUCTS[m.group(1)].from_address(args))


fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
fake.fake_hip_on_launch(on_launch)
lib = ctypes.CDLL(sys.argv[2])
pools = {}


def pool(layers=1, blocks=64, bs=16, heads=2, dim=64, elem=2, layouts=(0, 0), at=1):
    key = (layers, blocks, bs, heads, dim, elem, tuple(layouts), at)
    if key not in pools:
        size = (blocks * bs * heads * dim * elem + 255) // 256 * 256
        ptr = [(at << 43) + i * size for i in range(2 * layers)]
        desc = Desc(layers, blocks, bs, heads, dim, elem, (U64 * layers)(*ptr[:layers]), (U64 * layers)(*ptr[layers:]),
                    *layouts)
        h = P()
        assert lib.llmig_pool_create(ctypes.byref(desc), ctypes.byref(h)) == 0
        pools[key] = h
    return pools[key]


def lens(x):
    return None if x is None else np.asarray(x, np.int32)


def at(a):
    return None if a is None else P(a.ctypes.data)


def dev(n):
    return P(n) if n else None


A = [0] + [k << 44 for k in range(1, 8)]      # device addresses


def append(pool_args=None, no_pool=False, from_toks=(5, 0), n_toks=(1, 20), first_pos=None, **kw):
    f, n, p = lens(from_toks), lens(n_toks), lens(first_pos)
    pool_args = pool_args or {}
    row = pool_args.get("heads", 2) * pool_args.get("dim", 64)
    d = dict(dtype=1, batch=0 if n is None else len(n), q_heads=4, table_stride=4, q=A[1], k=A[2], v=A[3], q_out=A[4],
             q_layer=2 * row * 21, q_token=2 * row, k_layer=row * 21, k_token=row, v_layer=row * 21, v_token=row,
             tables=A[5], cos_sin=A[6], positions=100, rotary_dim=64, interleaved=0)
    d.update(kw)
    desc = Append(from_toks=f.ctypes.data if f is not None else None, n_toks=n.ctypes.data if n is not None else None,
                  first_pos=p.ctypes.data if p is not None else None, **d)
    return lib.llmig_append_rotary(None if no_pool else pool(**pool_args), ctypes.byref(desc), None), None


def bounds(pool_args=None, bounds_args=None, no_pool=False, no_bounds=False, dtype=1, batch=2, tables=A[1], table_stride=4,
           from_toks=(5, 0), ctx_lens=(6, 40)):
    f, c = lens(from_toks), lens(ctx_lens)
    b = dict(bs=1, at=2)
    b.update(bounds_args or {})
    return lib.llmig_key_bounds(None if no_pool else pool(**(pool_args or {})), None if no_bounds else pool(**b), dtype,
                                batch, dev(tables), table_stride, at(f), at(c), None), None


def select(bounds_args=None, no_bounds=False, dtype=1, block_size=16, q=A[1], batch=2, q_heads=4, tables=A[2],
           table_stride=8, ctx_lens=(100, 40), keep_first=1, keep_last=1, count=4, workspace=A[3], less=0, blocks=A[4]):
    c = lens(ctx_lens)
    b = dict(bs=1, at=2)
    b.update(bounds_args or {})
    p = None if no_bounds else pool(**b)
    n = I64(-1)
    rc = lib.llmig_select_blocks_workspace(p, block_size, at(c), batch, ctypes.byref(n))
    return lib.llmig_select_blocks(p, dtype, block_size, dev(q), batch, q_heads, dev(tables), table_stride, at(c), keep_first,
                                   keep_last, count, dev(workspace), I64(max(0, n.value) - less), dev(blocks), None), n.value


def attend(pool_args=None, no_pool=False, dtype=1, q=A[1], batch=2, q_heads=4, tables=A[2], table_stride=8,
           ctx_lens=(100, 40), blocks=A[4], count=4, workspace=A[3], less=0, out=A[5]):
    c = lens(ctx_lens)
    p = None if no_pool else pool(**(pool_args or {}))
    n = I64(-1)
    lib.llmig_decode_attention_blocks_workspace(p, at(c), batch, q_heads, count, ctypes.byref(n))
    return lib.llmig_decode_attention_blocks(p, dtype, dev(q), batch, q_heads, dev(tables), table_stride, at(c), dev(blocks),
                                             count, ctypes.c_float(0.1), dev(workspace), I64(max(0, n.value) - less),
                                             dev(out), None), n.value


def prefix(pool_args=None, no_pool=False, dtype=1, q=A[1], batch=None, q_heads=4, tables=A[2], table_stride=8,
           ctx_lens=(100, 70), prefix_blocks=4, workspace=A[3], less=0, out=A[5]):
    c = lens(ctx_lens)
    batch = (0 if c is None else len(c)) if batch is None else batch
    p = None if no_pool else pool(**(pool_args or {}))
    n = I64(-1)
    lib.llmig_decode_attention_prefix_workspace(p, at(c), batch, q_heads, prefix_blocks, ctypes.byref(n))
    return lib.llmig_decode_attention_prefix(p, dtype, dev(q), batch, q_heads, dev(tables), table_stride, at(c),
                                             prefix_blocks, ctypes.c_float(0.1), dev(workspace),
                                             I64(max(0, n.value) - less), dev(out), None), n.value


def decode(pool_args=None, q_heads=4, table_stride=8, ctx_lens=(100, 70), form="workspace"):
    """llmig_decode_attention, its form without a workspace, or carrying a stage."""
    c = lens(ctx_lens)
    p = pool(**(pool_args or {}))
    head = (p, 1, dev(A[1]), len(c), q_heads, dev(A[2]), table_stride, at(c), ctypes.c_float(0.1))
    room = (dev(A[3]), I64(1 << 50), dev(A[5]))
    if form == "noalloc":
        return lib.llmig_decode_attention_noalloc(*head, dev(A[5]), None), None
    if form == "migrate":
        return lib.llmig_decode_attention_migrate(*head, *room, pool(**dict(pool_args or {}, at=2)), 1, dev(A[6]), I64(0),
                                                  I64(1), None), None
    return lib.llmig_decode_attention(*head, *room, None), None


OPS = {f.__name__: f for f in (append, bounds, select, attend, prefix, decode)}


def main():
    results = []
    for c in json.load(sys.stdin):
        launches.clear()
        rc, workspace = OPS[c.pop("op")](**c)
        results.append({"rc": rc, "workspace": workspace, "launches": list(launches)})
    json.dump(results, sys.stdout)


main()
