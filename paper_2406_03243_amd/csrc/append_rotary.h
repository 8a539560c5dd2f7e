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
    uint32_t first_unit;         // this launch's first (token, layer)
    uint32_t num_layers, num_blocks, block_size, table_stride, tile_bytes;
    uint32_t q_heads, kv_heads, tokens, batch;
    uint32_t row_chunks;         // head_dim / 8
    uint32_t token_chunks;       // 16-byte chunks of one token and layer: (q_heads + 2 kv_heads) * row_chunks
    uint32_t half;               // rotary_dim / 2
    uint32_t interleaved;
    uint32_t wide;               // the table's rows can be read 16 bytes at a time
    int32_t layouts[2];
    Divisor by_slice, by_layer, by_row, by_block;
    uint32_t token_end[kAppendMaxBatch];  // tokens of the first s + 1 sequences
    int32_t from[kAppendMaxBatch];        // slot of the first new token of sequence s
    int32_t pos[kAppendMaxBatch];         // its position
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

// Eight consecutive floats of the table.
__device__ __forceinline__ void table8(const float *p, bool wide, float *x)
{
    if (wide) {
        const u32x4 a = *(const LLMIG_GLOBAL u32x4 *)p, b = *(const LLMIG_GLOBAL u32x4 *)(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = __uint_as_float(a[e]);
            x[4 + e] = __uint_as_float(b[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = ((const LLMIG_GLOBAL float *)p)[e];
    }
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
        table8(at, a.wide, co);
        table8(at + h, a.wide, si);
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
    *(LLMIG_GLOBAL u32x4 *)(tile + at * 16u) = v;
}

// A workgroup takes 256 chunks of one (token, layer): items in the order
// token, layer, slice, so that a token's table row stays in the caches.
template <int BF16>
__global__ void __launch_bounds__(kThreads) append_rotary_rows(const AppendArgs a)
{
    const uint32_t unit_here = divide(blockIdx.x, a.by_slice), unit = a.first_unit + unit_here;
    const uint32_t slice = blockIdx.x - unit_here * a.by_slice.d;
    const uint32_t token = divide(unit, a.by_layer), layer = unit - token * a.num_layers;
    uint32_t s = 0, hi = a.batch - 1;     // the first sequence whose tokens end past it
    while (s < hi) {
        const uint32_t mid = (s + hi) / 2u;
        if (a.token_end[mid] <= token)
            s = mid + 1u;
        else
            hi = mid;
    }
    const uint32_t j = token - (s > 0 ? a.token_end[s - 1] : 0u);
    const uint32_t slot_no = static_cast<uint32_t>(a.from[s]) + j;
    const uint32_t blk = divide(slot_no, a.by_block), slot = slot_no - blk * a.block_size;
    const uint32_t id = table_id(a.tables, s, a.table_stride, blk);
    const float *cs = a.cos_sin + static_cast<uint64_t>(static_cast<uint32_t>(a.pos[s]) + j) * 2u * a.half;

    const uint32_t chunk = slice * kThreads + threadIdx.x;
    if (chunk >= a.token_chunks)
        return;
    uint32_t head = divide(chunk, a.by_row);
    const uint32_t c = chunk - head * a.row_chunks;
    const uint32_t kind = head < a.q_heads ? 0u : head < a.q_heads + a.kv_heads ? 1u : 2u;
    head -= kind == 0 ? 0u : kind == 1 ? a.q_heads : a.q_heads + a.kv_heads;
    const uint8_t *row = (kind == 0 ? a.x[0] : kind == 1 ? a.x[1] : a.x[2]) +
                         layer * (kind == 0 ? a.layer_bytes[0] : kind == 1 ? a.layer_bytes[1] : a.layer_bytes[2]) +
                         token * (kind == 0 ? a.token_bytes[0] : kind == 1 ? a.token_bytes[1] : a.token_bytes[2]) +
                         head * a.row_chunks * 16u;
    const u32x4 v = kind == 2 ? load16(row + 16u * c) : rotated_chunk<BF16>(a, row, c, cs);
    if (kind == 0) {
        const uint64_t at = (static_cast<uint64_t>(layer) * a.tokens + token) * a.q_heads + head;
        *(LLMIG_GLOBAL u32x4 *)(a.q_out + (at * a.row_chunks + c) * 16u) = v;
    } else if (id < a.num_blocks) {       // an id outside the pool is not written
        uint8_t *tile = reinterpret_cast<uint8_t *>(table_entry(a.tab, (kind - 1u) * a.num_layers + layer)) +
                        static_cast<uint64_t>(id) * a.tile_bytes;
        store_chunk(tile, a.layouts[kind - 1u], slot, head, c, a, v);
    }
}

} // namespace
