// Append of new tokens to a paged cache with the position rotation applied on
// the way (llmig_append_rotary).  Part of the single translation unit built
// from llmig.hip.
//
// A head's row x of a token at position p, with h = rotary_dim / 2 angles
// a_i = p * frequency_i (their cosines and sines come in a table):
//     half-split   y[i] = x[i] cos a_i - x[i + h] sin a_i
//                  y[i + h] = x[i + h] cos a_i + x[i] sin a_i,    i < h
//     interleaved  the same for the pairs (2i, 2i + 1);
// elements from rotary_dim on pass through.  Computed in fp32 and rounded once
// to the pool's type.  Keys go rotated, values as they are into the slots that
// the block tables give, queries rotated into an array of their own.
#pragma once

#include "common.h"

namespace {

constexpr int kAppendMaxBatch = 256;    // sequences per call (their ranges ride in the kernel arguments)

struct AppendArgs {
    const uint64_t *tab;         // pool table: K bases then V bases
    const uint8_t *x[3];         // queries, keys, values
    uint64_t layer_bytes[3], token_bytes[3];
    uint8_t *q_out;              // [L][tokens][q_heads][D]
    const int32_t *tables;       // [B][table_stride]
    const float *cos_sin;        // [positions][rotary]: cosines, then sines
    uint32_t first_unit;         // this launch's first unit
    uint32_t num_layers, num_blocks, block_size, table_stride, tile_bytes;
    uint32_t q_heads, kv_heads, tokens, batch;
    uint32_t rows_heads[3];      // append_rotary_rows: query, key and value heads that it moves
    uint32_t row_chunks;         // head_dim / 8
    uint32_t lanes;              // of a unit
    uint32_t half;               // rotary_dim / 2
    uint32_t interleaved;
    uint32_t wide;               // the table's rows can be read 16 bytes at a time
    int32_t layouts[2];
    uint32_t one_each;           // every sequence has one new token
    uint32_t tensor;             // block by block: 0 keys, 1 values
    Divisor by_slice, by_layer, by_row, by_block;
    Divisor by_group, by_groups; // append_rotary_slots: slots that adjoin in a wavefront, such groups of a block
    // tokens (block by block: blocks) of the first s + 1 sequences
    uint32_t unit_end[kAppendMaxBatch];
    int32_t from[kAppendMaxBatch];        // slot of the first new token of sequence s
    int32_t pos[kAppendMaxBatch];         // its position
    // tokens of the first s sequences (block by block)
    uint32_t token_first[kAppendMaxBatch];
};

template <int BF16>
__device__ __forceinline__ float from16(uint32_t bits)
{
    if constexpr (BF16)
        return __builtin_bit_cast(float, bits << 16);
    else
        return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
}

// Nearest even; a NaN stays one.
template <int BF16>
__device__ __forceinline__ uint32_t round16(float x)
{
    if constexpr (BF16)
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
    else
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
}

template <int BF16>
__device__ __forceinline__ void unpack8(u32x4 v, float *x)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = from16<BF16>(v[e] & 0xffffu);
        x[2 * e + 1] = from16<BF16>(v[e] >> 16);
    }
}

template <int BF16>
__device__ __forceinline__ u32x4 pack8(const float *x)
{
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = round16<BF16>(x[2 * e]) | round16<BF16>(x[2 * e + 1]) << 16;
    return v;
}

// Four, or eight, consecutive floats of the table, 16-byte aligned.
__device__ __forceinline__ void table4(const float *p, float *x)
{
    const u32x4 v = *(const LLMIG_GLOBAL u32x4 *)p;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        x[e] = __uint_as_float(v[e]);
}

__device__ __forceinline__ void table8(const float *p, float *x)
{
    table4(p, x);
    table4(p + 4, x + 4);
}

// Dims 8c .. 8c + 7 of the rotated row whose chunks start at `row`.
template <int BF16>
__device__ __forceinline__ u32x4 rotated_chunk(const AppendArgs &a, const uint8_t *row, uint32_t c, const float *cs)
{
    const uint32_t h = a.half, d0 = 8u * c;
    const u32x4 own = load16(row + 16u * c);
    if (d0 >= 2u * h)
        return own;
    float x[8], y[8], co[8], si[8];
    unpack8<BF16>(own, x);
    if (a.interleaved) {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
            const uint32_t i = d0 / 2u + e;
            const bool turns = i < h;
            const float c1 = turns ? cs[i] : 1.f, s1 = turns ? cs[h + i] : 0.f;
            y[2 * e] = turns ? x[2 * e] * c1 - x[2 * e + 1] * s1 : x[2 * e];
            y[2 * e + 1] = turns ? x[2 * e + 1] * c1 + x[2 * e] * s1 : x[2 * e + 1];
        }
    } else if (h % 8u == 0) {       // the partners are a chunk, too
        const bool low = d0 < h;
        float z[8];
        unpack8<BF16>(load16(row + 2u * (low ? d0 + h : d0 - h)), z);
        const float *at = cs + (low ? d0 : d0 - h);
        if (a.wide) {
            table8(at, co);
            table8(at + h, si);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 8; ++e) {
                co[e] = at[e];
                si[e] = at[h + e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            y[e] = low ? x[e] * co[e] - z[e] * si[e] : x[e] * co[e] + z[e] * si[e];
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
            const uint32_t d = d0 + e, i = d < h ? d : d - h;
            y[e] = x[e];
            if (d < 2u * h) {
                const float z = from16<BF16>(((const LLMIG_GLOBAL uint16_t *)row)[d < h ? d + h : d - h]);
                y[e] = d < h ? x[e] * cs[i] - z * cs[h + i] : x[e] * cs[i] + z * cs[h + i];
            }
        }
    }
    return pack8<BF16>(y);
}

// Stores chunk c of head `head`, slot `slot`, where the layout puts it.
__device__ __forceinline__ void store_chunk(uint8_t *tile, int32_t layout, uint32_t slot, uint32_t head, uint32_t c,
                                            const AppendArgs &a, u32x4 v)
{
    const uint32_t rc = a.row_chunks, bs = a.block_size;
    if (layout == LLMIG_LAYOUT_HDN) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            *(LLMIG_GLOBAL uint16_t *)(tile + ((head * rc + c) * 8u + e) * bs * 2u + slot * 2u) =
                static_cast<uint16_t>(v[e / 2] >> (16u * (e & 1u)));
        return;
    }
    const uint32_t at = layout == LLMIG_LAYOUT_NHD   ? (slot * a.kv_heads + head) * rc + c
                        : layout == LLMIG_LAYOUT_HND ? (head * bs + slot) * rc + c
                                                     : (head * rc + c) * bs + slot;
    store16(tile + at * 16u, v);
}

// The sequence that unit i of a call belongs to: the first whose units end past it.
__device__ __forceinline__ uint32_t sequence_of(const uint32_t *unit_end, uint32_t batch, uint32_t i)
{
    uint32_t s = 0, hi = batch - 1;
    while (s < hi) {
        const uint32_t mid = (s + hi) / 2u;
        if (unit_end[mid] <= i)
            s = mid + 1u;
        else
            hi = mid;
    }
    return s;
}

// The rows of one token that a lane moves: two chunks of a head, of LG layers
// from layer0 on, all loads in flight.  Half-split, two that turn are the halves
// of the same eight pairs; the table's entries are read once for all.  FAST: rotary_dim
// is a multiple of 16 and the table 16-byte aligned; else each chunk looks for
// its own partners.
template <int BF16, int LG, int FAST>
__device__ __forceinline__ void move_pair(const AppendArgs &a, uint32_t kind, uint32_t head, uint32_t p, uint32_t layer0,
                                          uint64_t token, const float *cs, uint32_t slot, uint32_t id)
{
    const uint32_t h = a.half;
    const uint64_t layer_bytes = kind == 0 ? a.layer_bytes[0] : kind == 1 ? a.layer_bytes[1] : a.layer_bytes[2];
    const uint8_t *row = (kind == 0 ? a.x[0] : kind == 1 ? a.x[1] : a.x[2]) +
                         token * (kind == 0 ? a.token_bytes[0] : kind == 1 ? a.token_bytes[1] : a.token_bytes[2]) +
                         head * a.row_chunks * 16u;
    const bool splits = FAST && kind != 2 && !a.interleaved;
    const bool halves = splits && 8u * p < h;
    // the head's other chunks in two runs, so that neighbouring lanes' chunks adjoin
    const uint32_t skip = splits ? h / 4u : 0u, run = (a.row_chunks - skip + 1u) / 2u;
    const uint32_t c0 = halves ? p : splits ? skip + p - h / 8u : p, c1 = halves ? p + h / 8u : c0 + run;
    const bool two = c1 < a.row_chunks;
    bool turn0 = kind != 2 && h > 0, turn1 = turn0;
    float co[8], si[8];
    if constexpr (FAST) {
        turn0 = halves || (kind != 2 && a.interleaved && 4u * c0 < h);
        turn1 = halves || (kind != 2 && a.interleaved && 4u * c1 < h);
        if (halves) {
            table8(cs + 8u * p, co);
            table8(cs + h + 8u * p, si);
        } else if (turn0) {
            table4(cs + 4u * c0, co);
            table4(cs + h + 4u * c0, si);
            if (turn1) {
                table4(cs + 4u * c1, co + 4);
                table4(cs + h + 4u * c1, si + 4);
            }
        }
    }
    u32x4 x0[LG], x1[LG];
#pragma unroll
    for (uint32_t l = 0; l < LG; ++l) {
        const uint8_t *at = row + min(layer0 + l, a.num_layers - 1u) * layer_bytes;
        if (FAST || !turn0) {
            x0[l] = load16(at + 16u * c0);
            x1[l] = load16(at + 16u * (two ? c1 : c0));
        } else {
            x0[l] = rotated_chunk<BF16>(a, at, c0, cs);
            x1[l] = rotated_chunk<BF16>(a, at, two ? c1 : c0, cs);
        }
    }
    if (FAST && turn0) {
#pragma unroll
        for (uint32_t l = 0; l < LG; ++l) {
            float u[8], v[8], y[8], z[8];
            unpack8<BF16>(x0[l], u);
            unpack8<BF16>(x1[l], v);
            if (a.interleaved) {
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) {
                    y[2 * e] = u[2 * e] * co[e] - u[2 * e + 1] * si[e];
                    y[2 * e + 1] = u[2 * e + 1] * co[e] + u[2 * e] * si[e];
                    z[2 * e] = v[2 * e] * co[4 + e] - v[2 * e + 1] * si[4 + e];
                    z[2 * e + 1] = v[2 * e + 1] * co[4 + e] + v[2 * e] * si[4 + e];
                }
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) {
                    y[e] = u[e] * co[e] - v[e] * si[e];
                    z[e] = v[e] * co[e] + u[e] * si[e];
                }
            }
            x0[l] = pack8<BF16>(y);
            x1[l] = turn1 ? pack8<BF16>(z) : x1[l];
        }
    }
#pragma unroll
    for (uint32_t l = 0; l < LG; ++l) {
        const uint32_t layer = layer0 + l;
        if (layer >= a.num_layers)
            break;
        if (kind == 0) {
            uint8_t *at = a.q_out + ((static_cast<uint64_t>(layer) * a.tokens + token) * a.q_heads + head) * a.row_chunks * 16u;
            store16(at + c0 * 16u, x0[l]);
            if (two)
                store16(at + c1 * 16u, x1[l]);
        } else if (id < a.num_blocks) {       // an id outside the pool is not written
            uint8_t *tile = reinterpret_cast<uint8_t *>(table_entry(a.tab, layer + (kind - 1u) * a.num_layers)) +
                            static_cast<uint64_t>(id) * a.tile_bytes;
            store_chunk(tile, kind == 1 ? a.layouts[0] : a.layouts[1], slot, head, c0, a, x0[l]);
            if (two)
                store_chunk(tile, kind == 1 ? a.layouts[0] : a.layouts[1], slot, head, c1, a, x1[l]);
        }
    }
}

// Unit: (token, LG layers).  A token's rows, one after the other: each row is read
// and written once as whole lines, and nothing is shared but the table's entries.
// Bound by HBM where there is enough of it: queries of 32 heads of 128, 8 layers of
// 5777 tokens, 757 MB in 130 us, 5.8 TB/s; a decode step's tokens (32 layers of 61
// tokens, 32 query and 8 KV heads) are one round of workgroups, 48 MB in 13.2 us,
// where a plain copy of 48 MB takes 10.5; one token of one layer is a launch, 3.5 us.
template <int BF16, int LG, int FAST>
__global__ void __launch_bounds__(kThreads) append_rotary_rows(const AppendArgs a)
{
    const uint32_t unit_here = divide(blockIdx.x, a.by_slice), unit = a.first_unit + unit_here;
    const uint32_t slice = blockIdx.x - unit_here * a.by_slice.d;
    const uint32_t token = divide(unit, a.by_layer), layer0 = (unit - token * a.by_layer.d) * LG;
    const uint32_t s = a.one_each ? token : sequence_of(a.unit_end, a.batch, token);
    const uint32_t j = token - (s > 0 ? a.unit_end[s - 1] : 0u);
    const uint32_t slot_no = static_cast<uint32_t>(a.from[s]) + j;
    const uint32_t blk = divide(slot_no, a.by_block);
    const uint32_t id = table_id(a.tables, s, a.table_stride, blk);
    const float *cs = a.cos_sin + static_cast<uint64_t>(static_cast<uint32_t>(a.pos[s]) + j) * 2u * a.half;
    const uint32_t lane = slice * kThreads + threadIdx.x;
    if (lane >= a.lanes)
        return;
    uint32_t head = divide(lane, a.by_row);          // by_row: lanes of a head
    const uint32_t p = lane - head * a.by_row.d;
    const uint32_t kind = head < a.rows_heads[0] ? 0u : head < a.rows_heads[0] + a.rows_heads[1] ? 1u : 2u;
    head -= kind == 0 ? 0u : kind == 1 ? a.rows_heads[0] : a.rows_heads[0] + a.rows_heads[1];
    move_pair<BF16, LG, FAST>(a, kind, head, p, layer0, token, cs, slot_no - blk * a.block_size, id);
}

// The slots of a block that a call writes.
struct BlockSlots {
    uint32_t id, lo, hi;        // slots [lo, hi) of block id
    int64_t token, pos;         // slot x is row token + x of the call, at position pos + x
};

__device__ __forceinline__ BlockSlots block_slots(const AppendArgs &a, uint32_t i)
{
    const uint32_t s = sequence_of(a.unit_end, a.batch, i);
    const uint32_t from = static_cast<uint32_t>(a.from[s]);
    const uint32_t blk = divide(from, a.by_block) + i - (s > 0 ? a.unit_end[s - 1] : 0u);
    const uint32_t tokens = (s + 1u < a.batch ? a.token_first[s + 1u] : a.tokens) - a.token_first[s];
    const uint32_t slot0 = blk * a.block_size;
    BlockSlots b;
    b.id = table_id(a.tables, s, a.table_stride, blk);
    b.lo = from > slot0 ? from - slot0 : 0u;
    b.hi = min(a.block_size, from + tokens - slot0);
    const int64_t past = static_cast<int64_t>(slot0) - from;
    b.token = a.token_first[s] + past;
    b.pos = a.pos[s] + past;
    return b;
}

// Several tokens of a sequence into tiles whose tokens do not lie in one piece:
// a token by itself writes 16 (HCNX) or 2 bytes (HDN) in a place, which DRAM
// answers with a third of its rate, so a workgroup takes the tokens of a block.
//
// HCNX.  Unit: (block, LG layers); a lane takes a pair of chunks of one slot, a
// wavefront 8 slots of 8 pairs: it reads and writes whole 128-byte lines.  Keys of
// 32 heads of 128, 8 layers of 5777 tokens, 757 MB in 146 us, 5.2 TB/s (the writes
// go to one of eight places of a tile each).
template <int BF16, int LG, int FAST>
__global__ void __launch_bounds__(kThreads) append_rotary_slots(const AppendArgs a)
{
    const uint32_t unit_here = divide(blockIdx.x, a.by_slice), unit = a.first_unit + unit_here;
    const uint32_t slice = blockIdx.x - unit_here * a.by_slice.d;
    const uint32_t i = divide(unit, a.by_layer), layer0 = (unit - i * a.by_layer.d) * LG;
    const BlockSlots b = block_slots(a, i);
    const uint32_t lane = slice * kThreads + threadIdx.x;
    const uint32_t q = divide(lane, a.by_group), r = divide(q, a.by_row), p = q - r * a.by_row.d;
    const uint32_t head = divide(r, a.by_groups);
    const uint32_t slot = (r - head * a.by_groups.d) * a.by_group.d + lane - q * a.by_group.d;
    if (lane >= a.lanes || slot < b.lo || slot >= b.hi)
        return;
    move_pair<BF16, LG, FAST>(a, 1u + a.tensor, head, p, layer0, static_cast<uint64_t>(b.token + slot),
                              a.cos_sin + static_cast<uint64_t>(b.pos + slot) * 2u * a.half, slot, b.id);
}

// HDN.  Unit: (block, layer); a lane turns 8 dims of 8 slots round in
// registers, and LDS puts the lanes' pieces in the tile's order, so that a
// wavefront stores whole KiB.  Slots that the call does not write keep theirs.
// Values of the call above, 757 MB in 152 us, 5.0 TB/s; a CU holds three workgroups
// (140 registers, most of them for the rotation of eight rows of keys, which values
// do without; its LDS would hold four), and bank conflicts take 5% of the cycles.
template <int BF16>
__global__ void __launch_bounds__(kThreads) append_rotary_dims(const AppendArgs a)
{
    // a lane's 8 pieces of 16 bytes; after the lanes of a chunk one of padding,
    // so that lanes of one dim and different chunks write to different banks
    __shared__ u32x4 turned[kThreads * 9];
    const uint32_t unit_here = divide(blockIdx.x, a.by_slice), unit = a.first_unit + unit_here;
    const uint32_t slice = blockIdx.x - unit_here * a.by_slice.d;
    const uint32_t i = divide(unit, a.by_layer), layer = unit - i * a.num_layers;
    const BlockSlots b = block_slots(a, i);
    const uint32_t kind = 1u + a.tensor, along = a.by_row.d;       // groups of 8 slots
    if (b.id >= a.num_blocks)
        return;
    uint8_t *tile = reinterpret_cast<uint8_t *>(table_entry(a.tab, layer + a.tensor * a.num_layers)) +
                    static_cast<uint64_t>(b.id) * a.tile_bytes;
    const uint32_t chunks = a.by_slice.d > 1u ? kThreads / along : a.lanes / along;    // of a workgroup
    const uint32_t first = slice * chunks;                                             // its first (head, chunk)
    const uint32_t here = min(chunks, a.kv_heads * a.row_chunks - first);
    const uint32_t mine = divide(threadIdx.x, a.by_row), g = threadIdx.x - mine * along;
    auto whole = [&](uint32_t group) { return 8u * group >= b.lo && 8u * group + 8u <= b.hi; };
    if (mine < here) {
        const uint32_t head = (first + mine) / a.row_chunks, c = first + mine - head * a.row_chunks;
        const uint8_t *rows = a.x[kind] + layer * a.layer_bytes[kind] + head * a.row_chunks * 16u;
        u32x4 x[8];
#pragma unroll
        for (uint32_t t = 0; t < 8; ++t) {
            const uint32_t slot = min(max(8u * g + t, b.lo), b.hi - 1u);
            const uint8_t *row = rows + static_cast<uint64_t>(b.token + slot) * a.token_bytes[kind];
            x[t] = a.tensor == 0 ? rotated_chunk<BF16>(a, row, c, a.cos_sin + static_cast<uint64_t>(b.pos + slot) * 2u * a.half)
                                 : load16(row + 16u * c);
        }
        if (whole(g)) {
#pragma unroll
            for (uint32_t d = 0; d < 8; ++d) {       // dim d of the eight slots
                u32x4 y;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    y[k] = __builtin_amdgcn_perm(x[2 * k + 1][d / 2], x[2 * k][d / 2], d % 2 ? 0x07060302u : 0x05040100u);
                turned[mine * (8u * along + 1u) + d * along + g] = y;
            }
        } else {
#pragma unroll
            for (uint32_t t = 0; t < 8; ++t)
                if (8u * g + t >= b.lo && 8u * g + t < b.hi)
                    store_chunk(tile, LLMIG_LAYOUT_HDN, 8u * g + t, head, c, a, x[t]);
        }
    }
    __syncthreads();
    uint8_t *out = tile + static_cast<uint64_t>(first) * 8u * a.block_size * 2u;
    for (uint32_t k = threadIdx.x; k < here * 8u * along; k += kThreads) {
        const uint32_t row = divide(k, a.by_row);                 // (chunk, dim)
        if (whole(k - row * along))
            store16(out + k * 16u, turned[k + row / 8u]);
    }
}

// Whether tiles whose tokens do not lie in one piece are written block by block: one
// or two launches more, and a workgroup for a block that may get a single token, so
// it takes enough tokens a block, and bytes (of keys and values).  Token by token /
// block by block, HCNX keys and HDN values of 16 tokens a block, us: 0.3 MB 8.8 /
// 14.9, 5.0 MB (10 tokens a block) 20.8 / 23.3, 5.3 MB (full ones) 21.2 / 22.2, 9.7 MB
// 35.2 / 26.7, 21 MB 74.7 / 42.0, 30 MB (5 tokens a block) 110 / 92, 8.5 MB of one or two
// 37.7 / 57.4; both HCNX 12.7 / 19.0 at 5.3 MB, 28.1 / 23.5 at 9.7; both HDN 32.0 / 29.3
// and 54.9 / 33.8.
inline bool append_by_blocks(int64_t tokens, int64_t blocks, int64_t bytes)
{
    return tokens >= 4 * blocks && bytes >= 6 << 20;
}

// Layers of a token that a workgroup moves, for `work` workgroups of one layer.
// With two the setup (the sequence, the block, the table's entries) is paid half
// as often; with one there are more of them to start on an empty chip.  One / two
// layers, 32 query and 8 KV heads of 128: 8 layers of 4872 tokens 194 / 183 us, 32
// of 256 43.6 / 40.8, 32 of 61 (3904 workgroups) level, 32 of 8 4.7 / 5.2.
inline uint32_t append_layers(uint64_t work)
{
    return work >= 3000 ? 2 : 1;
}

template <int BF16, int LG, int FAST>
const void *append_kernel(bool slots)
{
    return slots ? reinterpret_cast<const void *>(&append_rotary_slots<BF16, LG, FAST>)
                 : reinterpret_cast<const void *>(&append_rotary_rows<BF16, LG, FAST>);
}

template <int BF16>
const void *append_kernel(bool slots, uint32_t layers, bool fast)
{
    return !fast         ? append_kernel<BF16, 1, 0>(slots)
           : layers == 2 ? append_kernel<BF16, 2, 1>(slots)
                         : append_kernel<BF16, 1, 1>(slots);
}

} // namespace
