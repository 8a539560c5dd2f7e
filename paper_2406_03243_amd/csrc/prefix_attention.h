// Decode attention over a prefix that the sequences of a batch share
// (llmig_decode_attention_prefix).  Part of the single translation unit built
// from llmig.hip.
//
// The query rows of all sequences behind the prefix, M = sequences x group of
// each KV head, attend to the same K and V, which are read once for all of
// them: S = K Q^T and O = V^T P^T are products of M columns.  prefix_rows cuts
// the prefix into partitions and leaves a record (maximum, weight sum,
// weighted V sum) per partition and row; attn_partial_mfma (decode_attention.h,
// kAttnOwn) takes each sequence's own tokens and joins both by the maxima, or, of
// own tokens cut into several partitions and of many partitions of the prefix,
// leaves records for prefix_join.
#pragma once

#include "append_rotary.h"
#include "decode_attention.h"

#include <type_traits>

namespace {

constexpr uint32_t kPrefixTile = 64;      // tokens of K and V in LDS at a time

struct PrefixArgs {
    const uint64_t *tab;         // pool table: K bases then V bases
    const uint8_t *q;            // [L][B][Hq][D]
    const int32_t *table;        // the prefix's blocks
    float *ws;                   // records [L][parts][members][Hq][D + kAttnHeader]
    float scale;
    uint32_t num_layers, batch, q_heads, kv_heads, num_blocks, block_size;
    uint32_t tokens;             // of the prefix
    uint32_t part_tokens, parts; // a partition's tokens (a multiple of kPrefixTile), partitions
    uint32_t members;            // sequences behind the prefix
    uint32_t chunks;             // workgroups that share a partition's rows
    Divisor by_block;
    uint8_t member[kAttnMaxBatch];        // their numbers in the batch
};

struct PrefixJoinArgs {
    const float *prefix, *own;   // records
    float *out;                  // [L][B][Hq][D]
    uint32_t num_layers, batch, q_heads, parts, members, n_records;
    uint32_t seqs;               // sequences that left records
    uint32_t row_base;           // this launch's first row
    uint32_t seq_end[kAttnMaxBatch];      // own records of the first s + 1 of them
    uint16_t member[kAttnMaxBatch];       // sequence s's place among the members (members: none)
    uint8_t seq[kAttnMaxBatch];           // its number in the batch
};

typedef float f32x16_t __attribute__((ext_vector_type(16)));

template <int BF16>
__device__ __forceinline__ f32x16_t mfma_32(u32x4 a, u32x4 b, f32x16_t c)
{
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c,
                                                      0, 0, 0);
}

// The larger, and the sum, of x of lanes l and l + 32, in both.
__device__ __forceinline__ float max_of_halves(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

__device__ __forceinline__ float sum_of_halves(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// A multiple of 8 tokens a block (ALIGNED) puts each 8 tokens in one, so their
// row is found with scalar instructions.
//
// One workgroup: a partition of one (layer, KV head) against 32 * WM query
// rows.  Of its four wavefronts WM split the rows, 32 each (the columns of one
// MFMA), and 4 / WM the tokens of each tile.
//
// The weights go through the matrix cores twice, as their 16-bit rounding and that
// of the rest (16 bits alone are off by 2^-9 of a weight), so a KV head takes 6 M D
// operations a token.  Many rows are bound by those: 4 layers of 8 heads of 128, 512
// rows, 16384 tokens, 206 GFLOP in 205 us, 1.0 PFLOP/s, the matrix cores busy 55% of
// the cycles at the clock that their power leaves (about 1.9 GHz), the rest weights and reads
// of LDS; without the loads from memory 165 us.  Few rows are bound by HBM: 8 layers of
// 32 heads, 40 rows, 4096 tokens, 537 MB in 109 us, 5.0 TB/s with two workgroups a
// CU, a tile of each on its way.  Against it were measured: a wavefront a tile of 32
// tokens and two of them on their way (three workgroups of two wavefronts a CU) 112 to
// 132 us, and up to 1.5 times as long where the chip is not full; tiles of 128 tokens
// level; hand-ordered instructions between the products level or slower.
template <int BF16, int D, int WM, int ALIGNED>
__global__ void __launch_bounds__(kThreads, 2) prefix_rows(const PrefixArgs a)
{
    constexpr int KS = D / 16;                     // k-steps of the QK product
    constexpr int MT = D / 32;                     // 32-dim tiles of the PV product
    constexpr uint32_t LPR = D / 8;                // 16-byte chunks of a row
    constexpr uint32_t RB = D * 2;                 // bytes of a row
    constexpr uint32_t RPB = 128 / D;              // rows per 256 bytes
    constexpr uint32_t T = kPrefixTile;
    constexpr int STEPS = T * WM / 128;            // of 32 tokens a wavefront takes of a tile
    constexpr int CPT = T * LPR / kThreads;    // chunks of K, and of V, a thread brings per tile
    constexpr uint32_t RPI = kThreads / LPR;       // rows that the threads bring at a time
    constexpr float kLog2e = 1.4426950408889634f;
    constexpr uint32_t kTileBytes = T * RB;
    // Two tiles, K and V, the one in work and the one on its way: arrays of their
    // own, so that the compiler sees which loads a read has to wait for.
    __shared__ __align__(16) uint8_t tile_a[2 * kTileBytes], tile_b[2 * kTileBytes];
    static_assert(4 * 16 * D * 4 <= 2 * kTileBytes, "the merge of 16 rows fits");
    __shared__ float sh_m[4][32], sh_l[4][32], sh_c[4][32];

    // The workgroups that read the same tokens (a partition's row chunks, then
    // its KV heads, whose rows adjoin) follow each other on one XCD.
    uint32_t chunk, g, unit;
    {
        const uint32_t per = a.kv_heads * a.chunks, lin = blockIdx.x;
        const uint32_t full = gridDim.x - gridDim.x % (8u * per);
        uint32_t k = lin;
        if (lin < full)
            k = (lin / 8u / per * 8u + lin % 8u) * per + lin / 8u % per;
        chunk = uniform(k % a.chunks);
        g = uniform(k / a.chunks % a.kv_heads);
        unit = uniform(k / per);
    }
    const uint32_t layer = unit / a.parts, part = unit - layer * a.parts;
    const uint32_t t_begin = part * a.part_tokens, t_end = min(t_begin + a.part_tokens, a.tokens);
    const uint32_t wave = uniform(threadIdx.x / 64), lane = threadIdx.x % 64;
    const uint32_t wm = wave % WM, wt = wave / WM;
    const uint32_t l32 = lane % 32, half = lane / 32;
    const uint32_t G = a.q_heads / a.kv_heads, M = a.members * G;
    const uint8_t *kbase = reinterpret_cast<const uint8_t *>(table_entry(a.tab, layer));
    const uint8_t *vbase = reinterpret_cast<const uint8_t *>(table_entry(a.tab, a.num_layers + layer));

    // Q^T fragments (B operand): dims 16 * ks + 8 * half .. + 8 of the lane's row;
    // rows past the last: the last again, stored nowhere.  A negative scale turns
    // the queries' signs, so that scores rise with their products.
    u32x4 qf[KS];
    {
        const uint32_t r = min(chunk * 32u * WM + wm * 32u + l32, M - 1u);
        const uint64_t q_row = (static_cast<uint64_t>(layer) * a.batch + a.member[r / G]) * a.q_heads + g * G + r % G;
        const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            qf[ks] = load16(a.q + (q_row * D + 16 * ks + 8 * half) * 2) ^ sign;
    }

    // A tile's rows go from memory straight into LDS: load i of a thread brings 16
    // bytes of token th + i * RPI while the tile before is worked on, and the ids of
    // the blocks are looked up one tile ahead of that.  Past the partition's end
    // valid rows repeat; they weigh 0.  Slot c of token t in LDS takes the row's
    // 16-byte chunk c ^ swizzle(t), so that what is read at once falls on distinct
    // banks: of K a chunk of each of 16 rows, of V four chunks of each of 4 rows.
    auto k_swizzle = [](uint32_t t) { return (t / RPB) % LPR; };
    auto v_swizzle = [](uint32_t t) { return t / RPB % (4u / RPB) * 4u ^ t / 4u % 4u; };
    static_assert(RPI % 16 == 0, "a thread's rows swizzle alike");
    const uint32_t th = threadIdx.x / LPR, tc = threadIdx.x % LPR;
    uint32_t ids[CPT];
    // ALIGNED: the first of the 8 tokens (t_end is a multiple of 8) to which the
    // wavefront's rows of load i belong; else the thread's token.
    const uint32_t wave_row = wave * (64u / LPR);
    auto token_of = [&](uint32_t t0, uint32_t i) {
        return ALIGNED ? min(t0 + (i * RPI + wave_row) / 8u * 8u, t_end - 8u) : min(t0 + i * RPI + th, t_end - 1u);
    };
    auto block_of = [&](uint32_t t) {       // (ALIGNED: the divisor is not 1)
        return ALIGNED ? __umulhi(t, a.by_block.m) >> a.by_block.shift : divide(t, a.by_block);
    };
    const uint64_t lane_row = ALIGNED ? static_cast<uint64_t>(th % 8u) * a.kv_heads * RB : 0u;
    const uint8_t *k_lane = kbase + lane_row + 16u * (tc ^ k_swizzle(th)), *v_lane = vbase + lane_row + 16u * (tc ^ v_swizzle(th));
    auto look_up = [&](uint32_t t0) {
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const uint32_t blk = block_of(token_of(t0, i));
            ids[i] = ALIGNED ? static_cast<uint32_t>(id_entry(a.table, uniform(blk))) : static_cast<uint32_t>(a.table[blk]);
        }
    };
    auto fetch = [&](uint8_t *tile, uint32_t t0) {
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const uint32_t t = token_of(t0, i), blk = block_of(t);
            const uint64_t slot = static_cast<uint64_t>(min(ids[i], a.num_blocks - 1u)) * a.block_size + (t - blk * a.block_size);
            const uint64_t at = (slot * a.kv_heads + g) * RB;
            uint8_t *to = tile + (i * RPI + wave_row) * RB;
            __builtin_amdgcn_global_load_lds((const void LLMIG_GLOBAL *)(k_lane + at), (void LLMIG_LDS *)to, 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const void LLMIG_GLOBAL *)(v_lane + at), (void LLMIG_LDS *)(to + kTileBytes), 16,
                                             0, 0);
        }
    };

    // Operands out of LDS.  K (A operand): token l32, dims 16 * ks + 8 * half .. + 8.
    // V^T (A operand: dim 32 * mt + l32) by transposing reads: lane r16 of a
    // 16-lane group receives element r16 % 4 of the 8 bytes that lane 4 * q +
    // r16 / 4 of its group addresses, for q = 0..3: tokens 4 * half + q of 8.
    const uint32_t r16 = lane % 16;
    const uint32_t k_at = l32 * RB, k_x = 16u * (half ^ k_swizzle(l32));
    const uint32_t v_row = 4u * half + r16 / 4u;
    const uint32_t v_at = v_row * RB + 8u * (r16 % 2u), v_x = 16u * ((2u * (lane / 16u % 2u) + r16 % 4u / 2u) ^ v_swizzle(v_row));

    const float qk_scale = fabsf(a.scale) * kLog2e;
    float m = -INFINITY, lsum = 0.f;
    f32x16_t acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            acc[mt][i] = 0.f;

    // A tile in LDS; TAIL: the partition ends in it.
    auto work = [&](const uint8_t *tile, uint32_t t0, auto tail_c) {
        constexpr bool TAIL = decltype(tail_c)::value;
        const uint8_t *kt = tile + wt * (32u * STEPS) * RB, *vt = kt + kTileBytes;
        auto k_rows = [&](int step, int ks) {
            return *reinterpret_cast<const u32x4 *>(kt + 32 * step * RB + k_at + (k_x ^ (32u * ks)));
        };
        auto v_rows = [&](int step, int n, int mt) {
            typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
            u64x2 v;
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j)
                v[j] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (LLMIG_LDS i16x4_t *)(vt + (32 * step + 16 * n + 8 * j) * RB + v_at + (v_x ^ (64u * mt) ^ (32u * j)))));
            return __builtin_bit_cast(u32x4, v);
        };
        f32x16_t s;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            s[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            s = mfma_32<BF16>(k_rows(0, ks), qf[ks], s);
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
            // element i of s is token first + 8 * (i / 4) + i % 4, of query row l32
            const uint32_t first = t0 + 32u * (wt * STEPS + step) + 4u * half;
            if constexpr (TAIL) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[i] = first + 8u * (i / 4) + i % 4 < t_end ? s[i] : -INFINITY;
            }
            // The maximum that weights are taken against moves only when a score
            // exceeds it by 2^8: the sums have the room (fp16 weights reach 2^15), and
            // the accumulators are rescaled seldom.
            float mx = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i)
                mx = fmaxf(mx, s[i]);
            mx *= qk_scale;
            if (__ballot(mx > m + 8.f)) {
                const float m_new = fmaxf(m, max_of_halves(mx));
                const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
                lsum *= c;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    acc[mt] = acc[mt] * c;
                m = m_new;
            }
            const float m_sub = m == -INFINITY ? 0.f : m - attn_weights_up(BF16);
            // From here on to the end of the step products and weights alternate:
            // the next 32 tokens' scores beside the first 16 tokens' weights, those
            // tokens' part of O^T += V^T . P^T beside the other 16 tokens' weights.
            uint32_t hi[8], lo[8];
            auto weights = [&](int n) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int k = 8 * n + i;
                    p[i] = __builtin_amdgcn_exp2f(s[k] * qk_scale - m_sub);
                    if constexpr (TAIL)         // (a scale of 0 would make NaN of the mask's -inf)
                        p[i] = first + 8u * (k / 4) + k % 4 < t_end ? p[i] : 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lsum += p[2 * i] + p[2 * i + 1];
                    split_weights<BF16>(p[2 * i], p[2 * i + 1], &hi[4 * n + i], &lo[4 * n + i]);
                }
            };
            // the weights as their 16-bit rounding and the 16-bit rounding of the rest
            auto values = [&](int n, const u32x4 *vf) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    acc[mt] = mfma_32<BF16>(vf[mt], u32x4{hi[4 * n], hi[4 * n + 1], hi[4 * n + 2], hi[4 * n + 3]}, acc[mt]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    acc[mt] = mfma_32<BF16>(vf[mt], u32x4{lo[4 * n], lo[4 * n + 1], lo[4 * n + 2], lo[4 * n + 3]}, acc[mt]);
            };
            u32x4 v0[MT], v1[MT];
            f32x16_t s_next;
            const bool next = step + 1 < STEPS;
            if (next) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s_next[i] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    s_next = mfma_32<BF16>(k_rows(step + 1, ks), qf[ks], s_next);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                v0[mt] = v_rows(step, 0, mt);
            weights(0);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                v1[mt] = v_rows(step, 1, mt);
            // (a wavefront in its products goes first: 2% against the other one of
            // the SIMD being let in between)
            __builtin_amdgcn_s_setprio(1);
            values(0, v0);
            weights(1);
            values(1, v1);
            __builtin_amdgcn_s_setprio(0);
            if (next)
                s = s_next;
        }
    };

    // A whole tile: every thread's part of it has landed, the tile after it is
    // requested, then the work.
    auto landed = [&]() {
        __builtin_amdgcn_s_waitcnt(kWaitVm0);
        __syncthreads();
    };
    auto turn = [&](const uint8_t *tile, uint8_t *next, uint32_t t0) {
        landed();
        if (t0 + T < t_end) {
            fetch(next, t0 + T);
            look_up(t0 + 2 * T);
        }
        work(tile, t0, std::false_type());
    };
    look_up(t_begin);
    fetch(tile_a, t_begin);
    look_up(t_begin + T);
    uint32_t t0 = t_begin;
    for (; t0 + 2 * T <= t_end; t0 += 2 * T) {
        turn(tile_a, tile_b, t0);
        turn(tile_b, tile_a, t0 + T);
    }
    if (t0 + T <= t_end) {
        turn(tile_a, tile_b, t0);
        t0 += T;
    }
    if (t0 < t_end) {
        landed();
        work((t0 - t_begin) / T % 2u ? tile_b : tile_a, t0, std::true_type());
    }

    // The records leave in whole rows, through LDS, 16 rows of each wavefront at a
    // time; wavefronts that split the tokens meet there.  (Chunk c of row r stands at
    // c ^ r, so that what is written at once falls on distinct banks; G is a power of
    // two.  With divisions by G, a row's factors found for each of its chunks and
    // conflicts, this took 6 us of a workgroup's time, now 1.5.)
    lsum = sum_of_halves(lsum);
    if (half == 0) {
        sh_m[wave][l32] = m;
        sh_l[wave][l32] = lsum;
    }
    float *so = reinterpret_cast<float *>(tile_a);                // [wave][16 rows][D]
    const uint32_t g_log = 31u - __builtin_clz(G);
    float *recs = a.ws + ((static_cast<uint64_t>(layer) * a.parts + part) * a.members * a.q_heads + g * G) * (D + kAttnHeader);
    auto record = [&](uint32_t row) {
        return recs + static_cast<uint64_t>((row >> g_log) * a.q_heads + (row & (G - 1u))) * (D + kAttnHeader);
    };
    __syncthreads();
    if (threadIdx.x < 32u * WM) {
        const uint32_t w0 = threadIdx.x / 32u, rr = threadIdx.x % 32u, row = chunk * 32u * WM + threadIdx.x;
        float mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < 4 / WM; ++w)
            mm = fmaxf(mm, sh_m[w * WM + w0][rr]);
#pragma unroll
        for (uint32_t w = 0; w < 4 / WM; ++w) {
            const float mw = sh_m[w * WM + w0][rr];
            // (no weight: a factor of 1 would do as well, but for a NaN sum)
            const float c = mw == -INFINITY ? 1.f : exp2f(mw - mm);
            ll += sh_l[w * WM + w0][rr] * c;
            sh_c[w * WM + w0][rr] = c;
        }
        if (row < M)              // the maximum in the natural base, as attn_partial_mfma leaves it
            *(LLMIG_GLOBAL f32x4_t *)record(row) = f32x4_t{mm == -INFINITY ? -INFINITY : mm / kLog2e, ll, 0.f, 0.f};
    }
#pragma unroll
    for (uint32_t rt = 0; rt < 2; ++rt) {
        if (rt > 0)
            __syncthreads();
        if (l32 / 16u == rt) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4_t *>(so + (wave * 16u + r16) * D + 4u * ((8u * mt + 2u * i + half) ^ r16)) =
                        f32x4_t{acc[mt][4 * i], acc[mt][4 * i + 1], acc[mt][4 * i + 2], acc[mt][4 * i + 3]};
        }
        __syncthreads();
        constexpr uint32_t kRows = kThreads / (D / 4);                // rows stored at a time
        const uint32_t d4 = threadIdx.x % (D / 4), r0 = threadIdx.x / (D / 4);
#pragma unroll
        for (uint32_t k = 0; k < WM * 16u / kRows; ++k) {
            const uint32_t r = k * kRows + r0, w0 = r / 16u, rr = r % 16u, row = chunk * 32u * WM + w0 * 32u + 16u * rt + rr;
            f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t w = 0; w < 4 / WM; ++w) {
                const uint32_t v = w * WM + w0;
                const f32x4_t x = *reinterpret_cast<const f32x4_t *>(so + (v * 16u + rr) * D + 4u * (d4 ^ rr));
                o = WM == 4 ? x : o + x * sh_c[v][16 * rt + rr];
            }
            if (row < M)
                *(LLMIG_GLOBAL f32x4_t *)(record(row) + kAttnHeader + 4 * d4) = o;
        }
    }
}

// Joins the records of the prefix and of own tokens that left some; bound by reading
// them and the launch (8 sequences of 8 heads of 128 and 4 query heads each, 33 records
// a row, 4.9 us).  D / 4 lanes
// a row (layer, sequence, query head) and record, SUB of them side by side, each
// with every SUB-th record, eight records' loads in flight; they meet in LDS.
template <int D, int SUB>
__global__ void __launch_bounds__(kThreads) prefix_join(const PrefixJoinArgs a)
{
    constexpr uint32_t kQuads = D / 4, kRec = D + kAttnHeader, kRows = kThreads / (kQuads * SUB);
    const uint32_t d4 = threadIdx.x % kQuads, sub = threadIdx.x / kQuads % SUB, mine = threadIdx.x / (kQuads * SUB);
    const uint32_t rows = a.num_layers * a.seqs * a.q_heads;
    const uint32_t r0 = a.row_base + blockIdx.x * kRows + mine;
    const uint32_t r = min(r0, rows - 1u);
    const uint32_t h = r % a.q_heads, s = r / a.q_heads % a.seqs, layer = r / a.q_heads / a.seqs;
    const uint32_t first = s > 0 ? a.seq_end[s - 1] : 0u;
    const uint32_t place = a.member[s], shared = place < a.members ? a.parts : 0u;
    const uint32_t all = shared + a.seq_end[s] - first;
    const float *pre = a.prefix + ((static_cast<uint64_t>(layer) * a.parts * a.members + place) * a.q_heads + h) * kRec;
    const float *own = a.own + ((static_cast<uint64_t>(layer) * a.n_records + first) * a.q_heads + h) * kRec;
    const uint64_t pre_step = static_cast<uint64_t>(a.members) * a.q_heads * kRec;
    const uint64_t own_step = static_cast<uint64_t>(a.q_heads) * kRec;
    float m = -INFINITY, l = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m2, float l2, f32x4_t v) {
        const float mm = fmaxf(m, m2);
        if (mm == -INFINITY) {      // no weight on either side; a NaN sum stays one
            l += l2;
            return;
        }
        const float c1 = __expf(m - mm), c2 = __expf(m2 - mm);
        l = l * c1 + l2 * c2;
        acc = acc * c1 + v * c2;
        m = mm;
    };
    for (uint32_t p0 = sub; p0 < all; p0 += 8 * SUB) {
        float2 ml[8];
        f32x4_t v[8];
#pragma unroll
        for (uint32_t u = 0; u < 8; ++u) {
            const uint32_t p = p0 + u * SUB;
            ml[u] = make_float2(-INFINITY, 0.f);
            v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (p < all) {
                const float *src = p < shared ? pre + p * pre_step : own + (p - shared) * own_step;
                ml[u] = *reinterpret_cast<const float2 *>(src);
                v[u] = *reinterpret_cast<const f32x4_t *>(src + kAttnHeader + 4 * d4);
            }
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            add(ml[u].x, ml[u].y, v[u]);
    }
    if constexpr (SUB > 1) {
        __shared__ float2 sh_ml[kRows][SUB];
        __shared__ f32x4_t sh_v[kRows][SUB][kQuads];
        sh_v[mine][sub][d4] = acc;
        if (d4 == 0)
            sh_ml[mine][sub] = make_float2(m, l);
        __syncthreads();
        if (sub > 0)
            return;
#pragma unroll
        for (int u = 1; u < SUB; ++u)
            add(sh_ml[mine][u].x, sh_ml[mine][u].y, sh_v[mine][u][d4]);
    }
    if (r0 < rows)
        reinterpret_cast<f32x4_t *>(a.out)[((static_cast<uint64_t>(layer) * a.batch + a.seq[s]) * a.q_heads + h) * kQuads + d4] =
            l > 0.f ? acc / l : f32x4_t{0.f, 0.f, 0.f, 0.f};
}

// The join of `rows` rows of at most `most` records; its rows per workgroup.
// Side by side where the rows alone leave the chip empty.
inline const void *prefix_join_kernel(int head_dim, uint64_t rows, uint32_t most, uint32_t *per)
{
    *per = kThreads / (head_dim / 4);
    if (most > 8 && rows / *per < 512) {
        *per /= 8;
        return head_dim == 64 ? reinterpret_cast<const void *>(&prefix_join<64, 8>)
                              : reinterpret_cast<const void *>(&prefix_join<128, 8>);
    }
    return head_dim == 64 ? reinterpret_cast<const void *>(&prefix_join<64, 1>)
                          : reinterpret_cast<const void *>(&prefix_join<128, 1>);
}

template <int BF16, int D, int ALIGNED>
const void *prefix_kernel(uint32_t wm)
{
    return wm == 2 ? reinterpret_cast<const void *>(&prefix_rows<BF16, D, 2, ALIGNED>)
                   : reinterpret_cast<const void *>(&prefix_rows<BF16, D, 4, ALIGNED>);
}

template <int BF16, int D>
const void *prefix_kernel(uint32_t wm, bool aligned)
{
    return aligned ? prefix_kernel<BF16, D, 1>(wm) : prefix_kernel<BF16, D, 0>(wm);
}

inline const void *prefix_kernel_for(int bf16, int head_dim, uint32_t wm, bool aligned)
{
    if (head_dim == 64)
        return bf16 ? prefix_kernel<1, 64>(wm, aligned) : prefix_kernel<0, 64>(wm, aligned);
    return bf16 ? prefix_kernel<1, 128>(wm, aligned) : prefix_kernel<0, 128>(wm, aligned);
}

// Whether the workgroups of the own tokens join the records of so many partitions
// themselves.  It saves a launch and a record per row, but one workgroup reads the
// partitions of its rows in turns of eight, which prefix_join reads side by side.
// Joined / left to prefix_join, us: 2 layers of 8 heads, 30 sequences of 4 query heads
// behind 4320 tokens, 4 partitions 41.9 / 43.6, 8 33.2 / 36.7, 16 30.9 / 33.1; one layer, 2
// behind 8192, 12 of them 27.1 / 27.3, 16 25.7 / 24.5, 32 27.5 / 20.7.
constexpr uint32_t kPrefixJoined = 12;

inline bool prefix_joins(uint32_t parts)
{
    return parts <= kPrefixJoined;
}

// How the prefix of a call is cut: wavefronts of a workgroup that split the
// rows, workgroups that share a partition, partitions; and about how long that
// takes.
struct PrefixCut {
    uint32_t wm, chunks, part_tokens, parts;
    int64_t ns;
};

// Partitions fill the chip, two workgroups a CU; each costs a record per row,
// written and read again.  What a cut takes was measured for 31 shapes (1 to 33
// layers, 4 to 32 heads, 6 to 512 rows, prefixes of 128 to 16384 tokens, 1 to 64
// partitions) and is, in rounds of 512 workgroups, beyond what all cuts take,
//     2 us + tiles of a partition x 1.2 us (x 1.5 with two a CU) + 0.2 ns a record
//     + 0.4 us a partition where they are joined at once, 5 us where they are not,
// for head_dim 128: the partitions that this puts first were within 0.8% of the
// best ones on average, 9% at most (8 heads, 512 rows, 8192 tokens: 1 partition
// 204 us, 4 65, 8 47, 12 53, 32 69).
constexpr int64_t kPrefixStartNs = 2000, kPrefixTileNs = 1200, kPrefixJoinNs = 400, kPrefixApartNs = 5000;
constexpr uint32_t kPrefixMostParts = 128;

inline int64_t prefix_cut_ns(int64_t workgroups, int64_t tiles, int64_t parts, int64_t records, int64_t head_dim)
{
    const int64_t rounds = (workgroups + 511) / 512, last = workgroups - (rounds - 1) * 512;
    const int64_t work = tiles * kPrefixTileNs * (128 + head_dim) / 256;
    return rounds * kPrefixStartNs + work * ((rounds - 1) * 15 + (last <= 256 ? 10 : 15)) / 10 +
           records * head_dim * 20 / 12800 +
           (prefix_joins(static_cast<uint32_t>(parts)) ? parts * kPrefixJoinNs : kPrefixApartNs);
}

inline PrefixCut prefix_cut(uint32_t rows, int64_t tokens, int64_t layer_heads, int64_t head_dim)
{
    PrefixCut c;
    c.wm = rows <= 64 ? 2 : 4;
    c.chunks = (rows + 32 * c.wm - 1) / (32 * c.wm);
    c.ns = -1;
    constexpr uint32_t tile = kPrefixTile;
    const int64_t tiles = (tokens + tile - 1) / tile, most = std::min<int64_t>(tiles, kPrefixMostParts);
    for (int64_t want = 1; want <= most; ++want) {
        const int64_t per = (tiles + want - 1) / want, parts = (tiles + per - 1) / per;
        const int64_t ns = prefix_cut_ns(parts * layer_heads * c.chunks, per, parts, parts * rows * layer_heads, head_dim);
        if (parts == want && (c.ns < 0 || ns < c.ns)) {
            c.ns = ns;
            c.parts = static_cast<uint32_t>(parts);
            c.part_tokens = static_cast<uint32_t>(per * tile);
        }
    }
    return c;
}

// Whether reading the prefix once pays.  It costs a launch or two more than plain
// attention, and every row reads its record again, 0.2 ns.  Plain attention reads the
// prefix for each of `members` sequences, after the first mostly out of the caches: 10
// to 14 TB/s where an XCD's share of the layers fits into its L2 (8 of head_dim 64 and
// of one KV head), 7 to 10 else; and a workgroup of its own costs more than the quarter
// of one that a short rest of a sequence takes.  Prefix / plain, us: one layer of 8
// heads of 128 and 4 query heads each, 7 sequences behind 2000 tokens 17.7 / 14.8, 8
// behind 8192 23.2 / 32.0, 64 behind 512 18.9 / 18.3; 8 query heads each, 16 behind 2000
// 22.2 / 23.0 (the rule takes the latter here), 64 behind 2000 28 / 73; 8 layers, 16 behind 512 21.5 / 25.3, 8 behind 2000
// 26 / 68; 9 layers of 32 heads, 8 behind 160 26 / 41; 6 layers of 8 heads and 8 query
// heads each, 47 behind 64 22.8 / 18.4; 23 layers of one head, 7 behind 2400 22 / 38.
inline bool prefix_pays(const PrefixCut &c, int64_t members, int64_t group, int64_t tokens, int64_t layers, int64_t heads,
                        int64_t head_dim)
{
    const double layer_bytes = static_cast<double>(tokens) * heads * head_dim * 4;
    const bool cached = head_dim == 128 && heads > 1 && layer_bytes * std::max<int64_t>(1, layers / 8) <= 4 << 20;
    const double workgroups = static_cast<double>(layers) * heads * members;
    const double plain_ns = layer_bytes * layers * members / (cached ? 12500. : 8500.) +
                            (workgroups >= 1024 ? 3.5 * workgroups : 0.);
    return c.ns + 4000 + members * group * layers * heads * head_dim * 20 / 12800 < plain_ns;
}

} // namespace
