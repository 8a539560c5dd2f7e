// Bounds of each block's keys, and the choice of blocks by them: the two steps
// before decode attention over listed blocks.  Part of the single translation
// unit built from llmig.hip.
//
// Bounds: per (layer, block, KV head, dim) the least and the largest key of the
// block's tokens, lo and hi.  Any key k of the block then has, for a query q,
//     q . k <= sum_d max(q_d lo_d, q_d hi_d) = sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d.
// Score of a block for a KV head's group of query heads: the sum of that bound
// over the group, one product with P = sum_h max(q_h, 0), N = sum_h min(q_h, 0):
//     score_j = sum_d P_d hi_jd + N_d lo_jd.
// Scores are compared with each other, so they are summed in 64 bits: products
// of 16-bit values are exact there, and which block is listed does not hang on
// the order of a sum.
#pragma once

#include "append_rotary.h"

namespace {

struct BoundsArgs {
    const uint64_t *tab;         // the pool's table (K bases first)
    const uint64_t *bounds_tab;  // the bounds' table: least (K) then largest (V) bases
    const int32_t *tables;
    uint32_t num_layers, num_blocks, block_size, table_stride, tile_bytes, batch;
    uint32_t slot_chunks;        // 16-byte chunks of a token's keys, and of a block's bounds
    uint32_t first_item;
    Divisor by_slice, by_block;  // by_block: division by the blocks of the call
    uint32_t blocks;             // blocks of the call
    uint32_t block_end[kAppendMaxBatch];  // blocks of the first s + 1 sequences
    int32_t first_block[kAppendMaxBatch]; // first block of sequence s to bring up to date
    int32_t tokens[kAppendMaxBatch];      // tokens of sequence s
};

// A lane takes 8 dims of one block's keys over its tokens.  A NaN key makes
// both of its bounds NaN.
template <int BF16>
__global__ void __launch_bounds__(kThreads) key_bounds_rows(const BoundsArgs a)
{
    const uint32_t item = a.first_item + blockIdx.x;
    const uint32_t unit = divide(item, a.by_slice), slice = item - unit * a.by_slice.d;
    const uint32_t layer = divide(unit, a.by_block), i = unit - layer * a.blocks;
    uint32_t s = 0, hi = a.batch - 1;
    while (s < hi) {
        const uint32_t mid = (s + hi) / 2u;
        if (a.block_end[mid] <= i)
            s = mid + 1u;
        else
            hi = mid;
    }
    const uint32_t blk = static_cast<uint32_t>(a.first_block[s]) + i - (s > 0 ? a.block_end[s - 1] : 0u);
    const uint32_t id = table_id(a.tables, s, a.table_stride, blk);
    const uint32_t held = min(static_cast<uint32_t>(a.tokens[s]) - blk * a.block_size, a.block_size);
    const uint32_t chunk = slice * kThreads + threadIdx.x;
    if (chunk >= a.slot_chunks || id >= a.num_blocks)
        return;
    const uint8_t *row = reinterpret_cast<const uint8_t *>(table_entry(a.tab, layer)) +
                         static_cast<uint64_t>(id) * a.tile_bytes + chunk * 16u;
    float lo[8], up[8];
    unpack8<BF16>(load16(row), lo);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        up[e] = lo[e];
#pragma unroll 8
    for (uint32_t t = 1; t < held; ++t) {
        float x[8];
        unpack8<BF16>(load16(row + static_cast<uint64_t>(t) * a.slot_chunks * 16u), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            lo[e] = x[e] < lo[e] || x[e] != x[e] ? x[e] : lo[e];
            up[e] = x[e] > up[e] || x[e] != x[e] ? x[e] : up[e];
        }
    }
    const uint64_t at = (static_cast<uint64_t>(id) * a.slot_chunks + chunk) * 16u;
    *(LLMIG_GLOBAL u32x4 *)(table_entry(a.bounds_tab, layer) + at) = pack8<BF16>(lo);
    *(LLMIG_GLOBAL u32x4 *)(table_entry(a.bounds_tab, a.num_layers + layer) + at) = pack8<BF16>(up);
}

// ---------------------------------------------------------------------------
// Scores and the choice.

struct SelectArgs {
    const uint64_t *tab;         // the bounds' table: least (K) then largest (V) bases
    const uint8_t *q;            // [L][B][Hq][D]
    const int32_t *tables;
    uint64_t *keys;              // [L][sum of n_s][H]: the scores, as words of the same order
    int32_t *out;                // [L][B][H][count]
    uint32_t num_layers, num_blocks, batch, q_heads, kv_heads, table_stride;
    uint32_t keep_first, keep_last, count;
    uint32_t blocks;             // sum of the sequences' blocks
    uint32_t first_item;         // this launch's first item
    uint32_t parts;              // score_blocks: workgroups of the longest sequence, one layer and slice
    uint32_t slices;             // score_blocks: 256-lane slices of a row of bounds
    uint32_t block_end[kAppendMaxBatch];  // blocks of the first s + 1 sequences
};

constexpr uint32_t kScoreBlocks = 32;     // blocks that a row of lanes of score_blocks takes one after the other

// A score as a word: unsigned order is the scores' order, NaN is the highest
// (a block whose bounds say nothing is not left out), and -0 equals 0.
__device__ __forceinline__ uint64_t score_key(double x)
{
    x += 0.0;
    if (x != x)
        x = INFINITY;
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// A lane takes 8 dims of one KV head, its sums P and N in registers, over the
// blocks of its part; the D / 8 lanes of a head add up.
template <int BF16, int D>
__global__ void __launch_bounds__(kThreads) score_blocks(const SelectArgs a)
{
    constexpr uint32_t C = D / 8;
    uint32_t w = a.first_item + blockIdx.x;
    const uint32_t part = w % a.parts;
    w /= a.parts;
    const uint32_t slice = w % a.slices;
    w /= a.slices;
    const uint32_t s = w % a.batch, layer = w / a.batch;
    const uint32_t first = s > 0 ? a.block_end[s - 1] : 0u;
    const uint32_t n = a.block_end[s] - first;
    const uint32_t row = a.kv_heads * C;                     // chunks of a block's bounds
    const uint32_t rows = row < kThreads ? kThreads / row : 1u;    // rows of lanes in the workgroup
    const uint32_t r = row < kThreads ? threadIdx.x / row : 0u;
    const uint32_t chunk = row < kThreads ? threadIdx.x % row : slice * kThreads + threadIdx.x;
    const uint32_t j0 = part * rows * kScoreBlocks;
    if (n <= a.count || j0 >= n)       // every block of a short sequence is listed
        return;
    const bool in = r < rows && chunk < row;
    const uint32_t head = in ? chunk / C : 0u, c = in ? chunk % C : 0u;
    const uint32_t G = a.q_heads / a.kv_heads;
    double p[8], m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        p[e] = m[e] = 0.0;
    for (uint32_t h = 0; h < G; ++h) {
        float x[8];
        unpack8<BF16>(load16(a.q + (((static_cast<uint64_t>(layer) * a.batch + s) * a.q_heads + head * G + h) * C + c) * 16u), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] += x[e] < 0.f ? 0.0 : static_cast<double>(x[e]);
            m[e] += x[e] > 0.f ? 0.0 : static_cast<double>(x[e]);
        }
    }
    const uint8_t *lo = reinterpret_cast<const uint8_t *>(table_entry(a.tab, layer));
    const uint8_t *hi = reinterpret_cast<const uint8_t *>(table_entry(a.tab, a.num_layers + layer));
    for (uint32_t k = 0; k < kScoreBlocks; ++k) {
        const uint32_t j = j0 + k * rows + r;
        if (j0 + k * rows >= n)
            break;
        const bool here = in && j < n;
        double sum = 0.0;
        if (here) {
            const uint32_t id = min(table_id(a.tables, s, a.table_stride, j), a.num_blocks - 1u);
            const uint64_t at = (static_cast<uint64_t>(id) * row + chunk) * 16u;
            float x[8], y[8];
            unpack8<BF16>(load16(hi + at), x);
            unpack8<BF16>(load16(lo + at), y);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum += p[e] * static_cast<double>(x[e]) + m[e] * static_cast<double>(y[e]);
        }
#pragma unroll
        for (uint32_t d = 1; d < C; d *= 2)
            sum += __shfl_xor(sum, d);
        if (here && c == 0)
            a.keys[(static_cast<uint64_t>(layer) * a.blocks + first + j) * a.kv_heads + head] = score_key(sum);
    }
}

// Lists the `count` highest keys of a row (layer, sequence, KV head), one
// workgroup a row: a radix search for the key of the last one listed, a byte a
// pass, then one walk through the blocks in order.
__global__ void __launch_bounds__(kThreads) list_blocks(const SelectArgs a)
{
    uint32_t w = a.first_item + blockIdx.x;
    const uint32_t g = w % a.kv_heads;
    w /= a.kv_heads;
    const uint32_t s = w % a.batch, layer = w / a.batch;
    const uint32_t first = s > 0 ? a.block_end[s - 1] : 0u;
    const uint32_t n = a.block_end[s] - first;
    int32_t *out = a.out + ((static_cast<uint64_t>(layer) * a.batch + s) * a.kv_heads + g) * a.count;
    if (n <= a.count) {
        for (uint32_t k = threadIdx.x; k < a.count; k += kThreads)
            out[k] = k < n ? static_cast<int32_t>(k) : -1;
        return;
    }
    const uint64_t *keys = a.keys + (static_cast<uint64_t>(layer) * a.blocks + first) * a.kv_heads + g;
    // blocks that are always listed stand above every score (count holds them)
    auto key = [&](uint32_t j) {
        return j < a.keep_first || j >= n - a.keep_last ? ~0ull : keys[static_cast<uint64_t>(j) * a.kv_heads];
    };
    __shared__ uint32_t bins[256];
    __shared__ uint32_t sh_bin, sh_need;
    __shared__ uint32_t wave_sum[2][kThreads / 64];
    uint64_t prefix = 0;
    uint32_t need = a.count;           // of the keys that begin with prefix, these many are listed
    for (int shift = 56; shift >= 0; shift -= 8) {
        bins[threadIdx.x] = 0;
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < n; j += kThreads) {
            const uint64_t k = key(j);
            if (shift == 56 || k >> (shift + 8) == prefix)
                atomicAdd(&bins[static_cast<uint32_t>(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t b = 255, left = need;
            while (b > 0 && bins[b] < left) {
                left -= bins[b];
                --b;
            }
            sh_bin = b;
            sh_need = left;
        }
        __syncthreads();
        prefix = prefix << 8 | sh_bin;
        need = sh_need;
        __syncthreads();
    }
    // in order: every key above the last one listed, and the first `need` equal to it
    uint32_t listed = 0, equal = 0;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    for (uint32_t j0 = 0; j0 < n; j0 += kThreads) {
        const uint32_t j = j0 + threadIdx.x;
        const uint64_t k = j < n ? key(j) : 0ull;
        const bool above = j < n && k > prefix, same = j < n && k == prefix;
        const uint64_t below = (1ull << lane) - 1ull;
        const uint64_t same_mask = __ballot(same);
        if (lane == 0)
            wave_sum[0][wave] = __popcll(same_mask);
        __syncthreads();
        uint32_t rank = equal + __popcll(same_mask & below), all_same = 0;
        for (uint32_t x = 0; x < kThreads / 64; ++x) {
            rank += x < wave ? wave_sum[0][x] : 0u;
            all_same += wave_sum[0][x];
        }
        const bool take = above || (same && rank < need);
        const uint64_t take_mask = __ballot(take);
        if (lane == 0)
            wave_sum[1][wave] = __popcll(take_mask);
        __syncthreads();
        uint32_t at = listed + __popcll(take_mask & below), all_take = 0;
        for (uint32_t x = 0; x < kThreads / 64; ++x) {
            at += x < wave ? wave_sum[1][x] : 0u;
            all_take += wave_sum[1][x];
        }
        if (take)
            out[at] = static_cast<int32_t>(j);
        listed += all_take;
        equal += all_same;
    }
}

} // namespace
