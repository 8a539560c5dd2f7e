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
// Scores are compared with each other, so they are summed in 64 bits, in one order
// for every block: equal bounds give equal scores, and a call's choice repeats.
// (The sum is exact where its terms span few enough exponents for 53 bits; else
// blocks whose scores differ by its rounding may change places.)
#pragma once

#include "append_rotary.h"

namespace {

struct BoundsArgs {
    const uint64_t *tab;         // the pool's table (K bases first)
    const uint64_t *bounds_tab;  // the bounds' table: least (K) then largest (V) bases
    const int32_t *tables;
    uint32_t num_layers, num_blocks, block_size, table_stride, tile_bytes, batch;
    uint32_t slot_chunks;        // 16-byte chunks of a token's keys, and of a block's bounds
    uint32_t rows;               // rows of lanes that share a block's tokens
    uint32_t side;               // blocks side by side in a workgroup
    uint32_t one_each;           // every sequence has one block
    uint32_t first_item;
    Divisor by_slice, by_group;  // by_group: division by the groups of `side` blocks of the call
    Divisor by_chunk, by_row;    // by the chunks of a slice, by rows
    uint32_t blocks;             // blocks of the call
    uint32_t block_end[kAppendMaxBatch];  // blocks of the first s + 1 sequences
    int32_t first_block[kAppendMaxBatch]; // first block of sequence s to bring up to date
    int32_t tokens[kAppendMaxBatch];      // tokens of sequence s
};

// The less, and the larger; a NaN on either side stays one.
__device__ __forceinline__ float less_of(float a, float b)
{
    return b < a || b != b ? b : a;
}

__device__ __forceinline__ float larger_of(float a, float b)
{
    return b > a || b != b ? b : a;
}

// A lane takes 8 dims of one block's keys over its row's share of the tokens,
// eight loads in flight; the rows meet in LDS.  Blocks of few heads stand side by
// side (SIDE), so that every lane has 8 tokens where the block has them (23 layers of
// 2 heads of 64, 7 requests of up to 3431 tokens, 32 a block: a block a workgroup 58
// us, 4 of them 20).  A NaN key makes both of its bounds NaN.
//
// A block that several sequences bring up to date is stored by each of them: equal
// bytes, as the caller guarantees that they hold the same number of its tokens.  (To
// find a sequence that holds more, comparing every other one's id at that place, took
// 0.3 us of 8.3 for 32 requests, and 7.5 instead of 4.7 for 256 of one KV head.)
//
// Every key is read once, so HBM bounds it: prompts of up to 32768 tokens, 4 layers of
// 8 heads of 128, 515 MB in 90 us, 5.7 TB/s; one block each of 32 requests, 32 layers,
// 22 MB in 7.9 us, of which some 4 start and end a launch.
template <int BF16, int SIDE>
__global__ void __launch_bounds__(kThreads) key_bounds_rows(const BoundsArgs a)
{
    __shared__ u32x4 part[2][kThreads];
    const uint32_t item = a.first_item + blockIdx.x;
    const uint32_t unit = divide(item, a.by_slice), slice = item - unit * a.by_slice.d;
    const uint32_t layer = divide(unit, a.by_group), group = unit - layer * a.by_group.d;
    const uint32_t set = divide(threadIdx.x, a.by_chunk), mine = threadIdx.x - set * a.by_chunk.d;
    const uint32_t beside = SIDE ? divide(set, a.by_row) : 0u, r = set - beside * a.rows;
    const uint32_t i = SIDE ? min(group * a.side + beside, a.blocks - 1u) : group;
    const uint32_t s = a.one_each ? i : sequence_of(a.block_end, a.batch, i);
    const uint32_t blk = static_cast<uint32_t>(a.first_block[s]) + i - (s > 0 ? a.block_end[s - 1] : 0u);
    const uint32_t id = table_id(a.tables, s, a.table_stride, blk);
    const uint32_t held = min(static_cast<uint32_t>(a.tokens[s]) - blk * a.block_size, a.block_size);
    const uint32_t chunk = slice * kThreads + mine;
    const bool in = r < a.rows && chunk < a.slot_chunks && id < a.num_blocks &&
                    (!SIDE || (beside < a.side && group * a.side + beside < a.blocks));
    const uint8_t *row = reinterpret_cast<const uint8_t *>(table_entry(a.tab, layer)) +
                         (in ? static_cast<uint64_t>(id) * a.tile_bytes + chunk * 16u : 0u);
    float lo[8], up[8];
    for (uint32_t t = in ? r : 0u, first = 1; t < held || first; t += 8u * a.rows) {
        u32x4 x[8];
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u)       // (a token twice changes nothing)
            x[u] = load16(row + static_cast<uint64_t>(min(t + u * a.rows, held - 1u)) * a.slot_chunks * 16u);
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) {
            float f[8];
            unpack8<BF16>(x[u], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                lo[e] = u == 0 && first ? f[e] : less_of(lo[e], f[e]);
                up[e] = u == 0 && first ? f[e] : larger_of(up[e], f[e]);
            }
        }
        first = 0;
    }
    if (a.rows > 1) {
        part[0][threadIdx.x] = pack8<BF16>(lo);
        part[1][threadIdx.x] = pack8<BF16>(up);
        __syncthreads();
        if (r > 0 || !in)
            return;
        for (uint32_t k = 1; k < a.rows; ++k) {
            float f[8], h[8];
            unpack8<BF16>(part[0][threadIdx.x + k * a.by_chunk.d], f);
            unpack8<BF16>(part[1][threadIdx.x + k * a.by_chunk.d], h);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                lo[e] = less_of(lo[e], f[e]);
                up[e] = larger_of(up[e], h[e]);
            }
        }
    }
    if (!in)
        return;
    const uint64_t at = (static_cast<uint64_t>(id) * a.slot_chunks + chunk) * 16u;
    *(LLMIG_GLOBAL u32x4 *)(table_entry(a.bounds_tab, layer) + at) = pack8<BF16>(lo);
    *(LLMIG_GLOBAL u32x4 *)(table_entry(a.bounds_tab, a.num_layers + layer) + at) = pack8<BF16>(up);
}

inline const void *key_bounds_kernel(int bf16, bool side)
{
    return bf16 ? side ? reinterpret_cast<const void *>(&key_bounds_rows<1, 1>)
                       : reinterpret_cast<const void *>(&key_bounds_rows<1, 0>)
           : side ? reinterpret_cast<const void *>(&key_bounds_rows<0, 1>)
                  : reinterpret_cast<const void *>(&key_bounds_rows<0, 0>);
}

// ---------------------------------------------------------------------------
// Scores and the choice.

struct SelectArgs {
    const uint64_t *tab;         // the bounds' table: least (K) then largest (V) bases
    const uint8_t *q;            // [L][B][Hq][D]
    const int32_t *tables;
    uint64_t *keys;              // the scores, as words of the same order: [L][sequence][H][its blocks]
    int32_t *out;                // [L][B][H][count]
    uint32_t num_layers, num_blocks, batch, q_heads, kv_heads, table_stride;
    uint32_t keep_first, keep_last, count;
    uint32_t blocks;             // sum of the sequences' blocks
    uint32_t first_item;         // this launch's first item
    uint32_t per_row;            // score_blocks: blocks that a row of lanes takes, one after the other
    uint32_t parts;              // score_blocks: workgroups of the longest sequence, one layer and slice
    uint32_t slices;             // score_blocks: 256-lane slices of a row of bounds
    uint32_t block_end[kAppendMaxBatch];  // blocks of the first s + 1 sequences
};

// Where the keys of (layer, sequence, KV head) start; `first` blocks of other
// sequences come before the sequence's n.
__device__ __forceinline__ uint64_t key_row(const SelectArgs &a, uint32_t layer, uint32_t first, uint32_t n, uint32_t g)
{
    return (static_cast<uint64_t>(layer) * a.blocks + first) * a.kv_heads + static_cast<uint64_t>(g) * n;
}

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

// x of another lane of the row of 16 (DPP control CTRL).
template <int CTRL>
__device__ __forceinline__ double of_lane(double x)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 v = __builtin_bit_cast(i32x2, x);
    return __builtin_bit_cast(double, i32x2{__builtin_amdgcn_update_dpp(0, v.x, CTRL, 0xf, 0xf, false),
                                            __builtin_amdgcn_update_dpp(0, v.y, CTRL, 0xf, 0xf, false)});
}

constexpr int kLaneXor1 = 0xB1, kLaneXor2 = 0x4E, kLaneXor7 = 0x141, kLaneXor8 = 0x128;

// The sums over C lanes (8 or 16, a head's) of four values: lane c gets that of
// value c / (C / 4).  Lanes l and l ^ mask exchange what the other keeps, then the
// few lanes of each value add up.  Each value's sum is the same tree, so equal
// values give equal sums.
template <uint32_t C>
__device__ __forceinline__ double sums_of_four(const double *s, uint32_t c)
{
    constexpr int kFirst = C == 16 ? kLaneXor8 : kLaneXor7, kSecond = C == 16 ? kLaneXor7 : kLaneXor2;
    const bool upper = c & (C / 2), odd = c & (C / 4);
    const double a = (upper ? s[2] : s[0]) + of_lane<kFirst>(upper ? s[0] : s[2]);
    const double b = (upper ? s[3] : s[1]) + of_lane<kFirst>(upper ? s[1] : s[3]);
    double x = (odd ? b : a) + of_lane<kSecond>(odd ? a : b);
    if constexpr (C == 16)
        x += of_lane<kLaneXor2>(x);
    return x + of_lane<kLaneXor1>(x);
}

// A lane takes 8 dims of one KV head, its sums P and N in registers, over the
// consecutive blocks of its row of lanes, four blocks' bounds in flight; the D / 8
// lanes of a head add up, and each keeps the score of one block in D / 8, so that
// scores leave as whole lines.  The bounds are read once: 12 requests of up to 65536
// tokens, 4 layers of 8 heads of 128, 352 MB in 66 us, 5.3 TB/s; 32 of up to 4000, 32
// layers, 460 MB in 101, 4.5.  HBM bounds it, at what it gives for rows of 2 KiB here and
// there: sums in 32 bits would take 3% less, more blocks a row of lanes the same (sums
// across lanes through LDS, and without the bounds' loads a step ahead, 79 us).
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
    if (n <= a.count || part * rows * a.per_row >= n)      // every block of a short sequence is listed
        return;
    const bool in = r < rows && chunk < row;
    const uint32_t head = in ? chunk / C : 0u, c = threadIdx.x % C;
    const uint32_t G = a.q_heads / a.kv_heads;
    double p[8], m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        p[e] = m[e] = 0.0;
    const uint8_t *q = a.q + (((static_cast<uint64_t>(layer) * a.batch + s) * a.q_heads + head * G) * C + c) * 16u;
    for (uint32_t h0 = 0; h0 < G; h0 += 4u) {
        u32x4 x[4];
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u)
            x[u] = load16(q + min(h0 + u, G - 1u) * C * 16u);
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u) {
            float f[8];
            unpack8<BF16>(x[u], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = h0 + u < G ? f[e] : 0.f;
                p[e] += static_cast<double>(v < 0.f ? 0.f : v);
                m[e] += static_cast<double>(v > 0.f ? 0.f : v);
            }
        }
    }
    const uint8_t *lo = reinterpret_cast<const uint8_t *>(table_entry(a.tab, layer));
    const uint8_t *hi = reinterpret_cast<const uint8_t *>(table_entry(a.tab, a.num_layers + layer));
    const uint32_t j0 = (part * rows + (in ? r : 0u)) * a.per_row;
    uint64_t *out = a.keys + key_row(a, layer, first, n, head);
    // bounds of four blocks, and the ids of the four after them
    u32x4 x[4], y[4];
    uint32_t ids[4];
    auto look_up = [&](uint32_t k0) {
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u)
            ids[u] = table_id(a.tables, s, a.table_stride, min(j0 + k0 + u, n - 1u));
    };
    auto fetch = [&]() {
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u) {
            const uint64_t at = (static_cast<uint64_t>(min(ids[u], a.num_blocks - 1u)) * row + (in ? chunk : 0u)) * 16u;
            x[u] = load16(hi + at);
            y[u] = load16(lo + at);
        }
    };
    look_up(0);
    fetch();
    look_up(4);
    uint64_t kept = 0;
    for (uint32_t k0 = 0; k0 < a.per_row; k0 += 4u) {
        u32x4 up4[4], low4[4];
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u) {
            up4[u] = x[u];
            low4[u] = y[u];
        }
        if (k0 + 4u < a.per_row) {
            fetch();
            look_up(k0 + 8u);
        }
        double sum[4];
#pragma unroll
        for (uint32_t u = 0; u < 4u; ++u) {
            float up[8], low[8];
            unpack8<BF16>(up4[u], up);
            unpack8<BF16>(low4[u], low);
            sum[u] = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum[u] = __fma_rn(p[e], static_cast<double>(up[e]), sum[u]);
                sum[u] = __fma_rn(m[e], static_cast<double>(low[e]), sum[u]);
            }
        }
        // lane c has the score of block k0 + c / (C / 4); every C blocks, or at the
        // end, the lanes that share one take it for different k0
        const double score = sums_of_four<C>(sum, c);
        const uint32_t mine = c % (C / 4) * 4u + c / (C / 4);
        if (c % (C / 4) == k0 / 4u % (C / 4))
            kept = score_key(score);
        const uint32_t done = k0 + 4u;             // per_row is a multiple of C, or less than C
        if (done % C == 0 || done >= a.per_row) {
            const uint32_t k = (done - 1u) / C * C + mine, j = j0 + k;
            if (in && k < done && j < n)
                out[j] = kept;
        }
    }
}

// Blocks of a row of lanes, for `work` rows of lanes times blocks in all: more of
// them share the setup (the sums of the queries), if enough workgroups are left to
// fill the chip.  12 requests of up to 65536 tokens, 4 layers of 8 heads, 8 / 16 / 32
// blocks 81 / 68 / 69 us; 16 of up to 32000, one layer, 19.5 / 19.5 / 19.2.
inline uint32_t score_blocks_per_row(uint64_t work)
{
    return work >= 16 * 1024 ? 16 : work >= 8 * 512 ? 8 : 4;
}

// The parallel part of a pass of the search below: of the counts of 256 bins,
// which one holds the need-th key from the top, and how many of it are needed.
// The T threads' first 256, or the 64 lanes of the only wavefront, hold the bins,
// BINS each, in order from the top.
template <int T>
__device__ __forceinline__ void find_bin(uint32_t *bins, uint32_t *wave_sum, uint32_t *found, uint32_t need)
{
    constexpr uint32_t BINS = T == 64 ? 4 : 1;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, top = 255u - BINS * threadIdx.x;
    uint32_t bin[BINS], mine = 0, sum = 0;
    if (threadIdx.x < 256) {
#pragma unroll
        for (uint32_t k = 0; k < BINS; ++k) {
            bin[k] = bins[top - k];
            mine += bin[k];
        }
        sum = mine;
#pragma unroll
        for (uint32_t d = 1; d < 64; d *= 2) {
            const uint32_t v = __shfl_up(sum, d);
            sum += lane >= d ? v : 0u;
        }
        if (T > 64 && lane == 63)
            wave_sum[wave] = sum;
    }
    if (T > 64)
        __syncthreads();
    if (threadIdx.x < 256) {
        for (uint32_t x = 0; T > 64 && x < wave; ++x)
            sum += wave_sum[x];
        uint32_t before = sum - mine;
#pragma unroll
        for (uint32_t k = 0; k < BINS; ++k) {
            if (before < need && before + bin[k] >= need) {
                found[0] = top - k;
                found[1] = need - before;            // needed of the bin
                found[2] = bin[k];                   // keys in it
            }
            before += bin[k];
            bins[top - k] = 0;
        }
    }
    __syncthreads();
}

// Makes x[0 .. N) the sums of what comes before each entry.
template <uint32_t N>
__device__ __forceinline__ void exclusive_sums(uint32_t *x)
{
    if (threadIdx.x < 64) {
        uint32_t before = 0;
#pragma unroll
        for (uint32_t k = 0; k < N; k += 64) {
            const uint32_t at = k + threadIdx.x, v = at < N ? x[at] : 0u;
            uint32_t sum = v;
#pragma unroll
            for (uint32_t d = 1; d < 64; d *= 2) {
                const uint32_t y = __shfl_up(sum, d);
                sum += threadIdx.x >= d ? y : 0u;
            }
            if (at < N)
                x[at] = before + sum - v;
            before += __shfl(sum, 63);
        }
    }
    __syncthreads();
}

// Lists the `count` highest keys of a row (layer, sequence, KV head), one
// workgroup a row: a radix search for the key of the last one listed, a byte a
// pass, which ends as soon as all keys that begin alike are listed; then the
// listed ones leave in order.  KPT: a thread holds that many keys, which are
// read once; 0: rows too long for that read them from memory in each pass.  A pass
// is a chain of LDS adds and three barriers, some 0.5 us, and that chain is what a
// call takes: 24 rows of up to 563 blocks 5.6 us, 384 of up to 4096 12.
template <int T, int KPT>
__global__ void __launch_bounds__(T) list_blocks(const SelectArgs a)
{
    constexpr uint32_t kWaves = T / 64, kHeld = KPT ? KPT : 1;
    uint32_t w = a.first_item + blockIdx.x;
    const uint32_t g = w % a.kv_heads;
    w /= a.kv_heads;
    const uint32_t s = w % a.batch, layer = w / a.batch;
    const uint32_t first = s > 0 ? a.block_end[s - 1] : 0u;
    const uint32_t n = a.block_end[s] - first;
    int32_t *out = a.out + ((static_cast<uint64_t>(layer) * a.batch + s) * a.kv_heads + g) * a.count;
    if (n <= a.count) {
        for (uint32_t k = threadIdx.x; k < a.count; k += T)
            out[k] = k < n ? static_cast<int32_t>(k) : -1;
        return;
    }
    const uint64_t *keys = a.keys + key_row(a, layer, first, n, g);
    // blocks that are always listed stand above every score (count holds them)
    auto key_of = [&](uint32_t j) {
        return j < a.keep_first || j >= n - a.keep_last ? ~0ull : keys[j];
    };
    __shared__ uint32_t bins[256], wave_sum[kWaves], found[3];
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    uint64_t held[kHeld];
    if constexpr (KPT > 0)
#pragma unroll
        for (uint32_t i = 0; i < KPT; ++i) {
            const uint32_t j = i * T + threadIdx.x;
            held[i] = j < n ? key_of(j) : 0ull;      // (no score's key: those of -inf are above it)
        }
    auto each = [&](auto &&f) {
        if constexpr (KPT > 0) {
#pragma unroll
            for (uint32_t i = 0; i < KPT; ++i)
                f(i * T + threadIdx.x, held[i]);
        } else {
            for (uint32_t j = threadIdx.x; j < n; j += T)
                f(j, key_of(j));
        }
    };
    for (uint32_t k = threadIdx.x; k < 256u; k += T)
        bins[k] = 0;
    __syncthreads();
    uint64_t prefix = 0;
    uint32_t need = a.count;           // of the keys that begin with prefix, these many are listed
    int shift = 56;
    bool ties = true;                  // whether not all of them are
    for (; shift >= 0 && ties; shift -= 8) {
        each([&](uint32_t j, uint64_t k) {
            const bool counts = j < n && (shift == 56 || k >> (shift + 8) == prefix);
            const uint32_t bin = static_cast<uint32_t>(k >> shift) & 255u;
            if (shift == 56) {       // sign and exponent: the keys of a wavefront mostly share a bin
                const uint64_t left = __ballot(counts);
                if (!left)
                    return;
                const uint32_t first_lane = __ffsll(static_cast<unsigned long long>(left)) - 1;
                const uint32_t common = __builtin_amdgcn_readlane(bin, first_lane);
                const uint64_t alike = __ballot(counts && bin == common);
                if (lane == first_lane)
                    atomicAdd(&bins[common], static_cast<uint32_t>(__popcll(alike)));
                else if (counts && bin != common)
                    atomicAdd(&bins[bin], 1u);
                return;
            }
            if (counts)
                atomicAdd(&bins[bin], 1u);
        });
        __syncthreads();
        find_bin<T>(bins, wave_sum, found, need);
        prefix = prefix << 8 | found[0];
        need = found[1];
        ties = found[1] != found[2];
    }
    shift += 8;
    // every key that begins above prefix, and the first `need` that begin with it
    const uint64_t below = (1ull << lane) - 1ull;
    if constexpr (KPT > 0) {
        __shared__ uint32_t chunk[KPT * kWaves];     // of 64 blocks each, in order
        uint32_t take = 0, same = 0;                 // a bit per key held
#pragma unroll
        for (uint32_t i = 0; i < KPT; ++i) {
            const uint64_t top = held[i] >> shift;
            if (i * T + threadIdx.x < n && top >= prefix) {
                take |= 1u << i;
                same |= top == prefix ? 1u << i : 0u;
            }
        }
        auto rank = [&](uint32_t flags, auto &&f) {
#pragma unroll
            for (uint32_t i = 0; i < KPT; ++i) {
                const uint64_t mask = __ballot(flags >> i & 1u);
                if (lane == 0)
                    chunk[i * kWaves + wave] = __popcll(mask);
            }
            __syncthreads();
            exclusive_sums<KPT * kWaves>(chunk);
#pragma unroll
            for (uint32_t i = 0; i < KPT; ++i) {
                const uint64_t mask = __ballot(flags >> i & 1u);
                f(i, chunk[i * kWaves + wave] + static_cast<uint32_t>(__popcll(mask & below)));
            }
        };
        if (ties) {
            uint32_t kept = take & ~same;
            rank(same, [&](uint32_t i, uint32_t at) { kept |= at < need ? same & 1u << i : 0u; });
            take = kept;
            __syncthreads();
        }
        rank(take, [&](uint32_t i, uint32_t at) {
            if (take >> i & 1u)
                out[at] = static_cast<int32_t>(i * T + threadIdx.x);
        });
        return;
    }
    __shared__ uint32_t sums[2][kWaves];
    uint32_t listed = 0, equal = 0;
    for (uint32_t i = 0; i * T < n; ++i) {
        const uint32_t j = i * T + threadIdx.x;
        const uint64_t top = (j < n ? key_of(j) : 0ull) >> shift;
        const bool same = j < n && top == prefix;
        bool take = j < n && top >= prefix;
        if (ties) {
            const uint64_t same_mask = __ballot(same);
            if (lane == 0)
                sums[0][wave] = __popcll(same_mask);
            __syncthreads();
            uint32_t rank = equal + __popcll(same_mask & below);
            for (uint32_t x = 0; x < kWaves; ++x) {
                rank += x < wave ? sums[0][x] : 0u;
                equal += sums[0][x];
            }
            take = take && (!same || rank < need);
        }
        const uint64_t take_mask = __ballot(take);
        if (lane == 0)
            sums[1][wave] = __popcll(take_mask);
        __syncthreads();
        uint32_t at = listed + __popcll(take_mask & below);
        for (uint32_t x = 0; x < kWaves; ++x) {
            at += x < wave ? sums[1][x] : 0u;
            listed += sums[1][x];
        }
        if (take)
            out[at] = static_cast<int32_t>(j);
        __syncthreads();
    }
}

// The kernel for rows of at most `longest` blocks, and its threads.  384 rows of up
// to 4096 blocks, 256 / 512 / 1024 threads 16.4 / 12.4 / 11.9 us; 24 of up to 563 take
// 5.6 with 256; 8192 of up to 250, 256 / 64 threads 25.1 / 13.1, 64 of them 5.6 / 5.1.
// More keys a thread than a row needs cost time: 5 rows of 5829 blocks, 8 / 16 of them
// 8.9 / 12.6 us.
inline const void *list_kernel(uint32_t longest, uint32_t *threads)
{
    *threads = longest <= 256 ? 64 : longest <= 1024 ? 256 : 1024;
    return longest <= 256     ? reinterpret_cast<const void *>(&list_blocks<64, 4>)
           : longest <= 1024  ? reinterpret_cast<const void *>(&list_blocks<256, 4>)
           : longest <= 4096  ? reinterpret_cast<const void *>(&list_blocks<1024, 4>)
           : longest <= 8192  ? reinterpret_cast<const void *>(&list_blocks<1024, 8>)
           : longest <= 16384 ? reinterpret_cast<const void *>(&list_blocks<1024, 16>)
                              : reinterpret_cast<const void *>(&list_blocks<1024, 0>);
}

} // namespace
