// Decode attention over a prefix that the sequences of a batch share
// (llmig_decode_attention_prefix).  Part of the single translation unit built
// from llmig.hip.
//
// The query rows of all sequences behind the prefix, M = sequences x group of
// each KV head, attend to the same K and V, which are read once for all of
// them: S = K Q^T and O = V^T P^T are products of M columns.  prefix_rows cuts
// the prefix into partitions and leaves a record (maximum, weight sum,
// weighted V sum) per partition and row; attn_partial_mfma leaves the records
// of each sequence's own tokens (decode_attention.h, kAttnOwn), and prefix_join
// joins both by the maxima.
#pragma once

#include "append_rotary.h"
#include "decode_attention.h"

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
    uint32_t row_base;           // this launch's first row
    uint32_t seq_end[kAttnMaxBatch];      // own records of the first s + 1 sequences
    uint16_t member[kAttnMaxBatch];       // sequence s's place among the members (members: none)
    uint8_t seq[kAttnMaxBatch];           // its number in the batch
};

// x of the lane 16, or 32, lanes away (in either direction of its row pair,
// half pair): the larger, and the sum.
__device__ __forceinline__ float max_of_rows(float x)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float sum_of_rows(float x)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Two weights as their 16-bit roundings and the 16-bit roundings of what these
// leave, the first weight in the low halves.
template <int BF16>
__device__ __forceinline__ void split_weights(float p0, float p1, uint32_t *hi, uint32_t *lo)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    if constexpr (BF16) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0, p1}), bf16x2));
        *hi = h;
        *lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0 - __uint_as_float(h << 16),
                                                                          p1 - __uint_as_float(h & 0xffff0000u)}), bf16x2));
    } else {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        const f16x2 h = __builtin_convertvector((f32x2{p0, p1}), f16x2);
        *hi = __builtin_bit_cast(uint32_t, h);
        *lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{p0 - static_cast<float>(h.x),
                                                                          p1 - static_cast<float>(h.y)}), f16x2));
    }
}

// One workgroup: a partition of one (layer, KV head) against 32 * WM query
// rows.  Of its four wavefronts WM split the rows, 32 each (two MFMA columns
// of 16), and 4 / WM the tokens of each tile.
template <int BF16, int D, int WM>
__global__ void __launch_bounds__(kThreads, 2) prefix_rows(const PrefixArgs a)
{
    constexpr int KS = D / 32;                     // k-steps of the QK product
    constexpr int MT = D / 16;                     // 16-dim tiles of the PV product
    constexpr int LPR = D / 8;                     // 16-byte chunks of a row
    constexpr int RB = D * 2;                      // bytes of a row
    constexpr int RPB = 128 / D;                   // rows per 256 bytes
    constexpr int TT = kPrefixTile / 16 * WM / 4;  // 16-token groups of a tile per wavefront
    constexpr int STEP = TT > 1 ? 2 : 1;           // groups taken at a time
    constexpr int CPT = kPrefixTile * LPR / kThreads;   // chunks of K, and of V, a thread brings per tile
    constexpr float kLog2e = 1.4426950408889634f;
    constexpr int kTileBytes = kPrefixTile * RB;
    constexpr int kMergeRow = D + 4;
    __shared__ __align__(16) uint8_t smem[2][2][kTileBytes];      // buffer, K or V
    static_assert(4 * 16 * kMergeRow * 4 <= 4 * kTileBytes, "the merge of 16 rows fits");
    __shared__ float sh_m[4][32], sh_l[4][32];

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
    const uint32_t r16 = lane % 16, g4 = lane / 16;
    const uint32_t G = a.q_heads / a.kv_heads, M = a.members * G;
    const uint8_t *kbase = reinterpret_cast<const uint8_t *>(table_entry(a.tab, layer));
    const uint8_t *vbase = reinterpret_cast<const uint8_t *>(table_entry(a.tab, a.num_layers + layer));

    // Q^T fragments (B operand): dims 32 * ks + 8 * g4 .. + 8 of the lane's row
    // of each column block; rows past the last: the last again, stored nowhere.
    const uint32_t row0 = chunk * 32u * WM + wm * 32u;
    u32x4 qf[2][KS];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
        const uint32_t r = min(row0 + 16u * rt + r16, M - 1u);
        const uint64_t q_row = (static_cast<uint64_t>(layer) * a.batch + a.member[r / G]) * a.q_heads + g * G + r % G;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            // a negative scale: the queries' signs turn, so that scores rise
            // with their products
            qf[rt][ks] = load16(a.q + (q_row * D + 32 * ks + 8 * g4) * 2) ^ (a.scale < 0.f ? 0x80008000u : 0u);
        }
    }

    // A tile's rows: thread's chunk of token th + i * (kThreads / LPR), brought
    // into registers while the tile before it is worked on, and their blocks'
    // ids one tile ahead of them.  Tokens past the partition's end repeat its
    // last one; they weigh 0.
    const uint32_t th = threadIdx.x / LPR, tc = threadIdx.x % LPR;
    u32x4 kr[CPT], vr[CPT];
    uint32_t ids[CPT];
    auto token_of = [&](uint32_t t0, int i) { return min(t0 + th + i * (kThreads / LPR), t_end - 1u); };
    auto look_up = [&](uint32_t t0) {
#pragma unroll
        for (int i = 0; i < CPT; ++i)
            ids[i] = static_cast<uint32_t>(a.table[divide(token_of(t0, i), a.by_block)]);
    };
    auto fetch = [&](uint32_t t0) {
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const uint32_t t = token_of(t0, i), blk = divide(t, a.by_block);
            const uint64_t slot = static_cast<uint64_t>(min(ids[i], a.num_blocks - 1u)) * a.block_size + (t - blk * a.block_size);
            const uint64_t at = (slot * a.kv_heads + g) * RB + 16u * tc;
            kr[i] = *(const LLMIG_GLOBAL u32x4 *)(kbase + at);
            vr[i] = *(const LLMIG_GLOBAL u32x4 *)(vbase + at);
        }
    };
    // 16-byte chunk c of token t sits at chunk c ^ swz(t) of its row, so that
    // reads of 16 rows at once fall on distinct banks.
    auto swz = [](uint32_t t) { return (t / RPB) % LPR; };
    auto put = [&](uint32_t buf) {
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
            const uint32_t t = th + i * (kThreads / LPR), at = t * RB + 16u * (tc ^ swz(t));
            *reinterpret_cast<u32x4 *>(&smem[buf][0][at]) = kr[i];
            *reinterpret_cast<u32x4 *>(&smem[buf][1][at]) = vr[i];
        }
    };

    const float qk_scale = fabsf(a.scale) * kLog2e;
    float m[2] = {-INFINITY, -INFINITY}, lsum[2] = {0.f, 0.f};
    f32x4_t acc[2][MT];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            acc[rt][mt] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    look_up(t_begin);
    fetch(t_begin);
    look_up(t_begin + kPrefixTile);
    put(0);
    uint32_t buf = 0;
    for (uint32_t t0 = t_begin; t0 < t_end; t0 += kPrefixTile, buf ^= 1u) {
        __syncthreads();                      // the tile is in LDS, and the one before it is done with
        const bool more = t0 + kPrefixTile < t_end;
        if (more) {
            fetch(t0 + kPrefixTile);
            look_up(t0 + 2 * kPrefixTile);
        }
        const bool tail = t0 + kPrefixTile > t_end;
        const uint8_t *kt = smem[buf][0], *vt = smem[buf][1];
#pragma unroll
        for (int step = 0; step < TT; step += STEP) {
            const uint32_t tb = 16u * (wt * TT + step);
            // S^T = K . Q^T
            f32x4_t s[2][STEP];
#pragma unroll
            for (int u = 0; u < STEP; ++u) {
                const uint32_t t = tb + 16u * u + r16;
                s[0][u] = s[1][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const u32x4 kf = *reinterpret_cast<const u32x4 *>(kt + t * RB + 16u * ((4u * ks + g4) ^ swz(t)));
                    s[0][u] = mfma_qk<BF16>(kf, qf[0][ks], s[0][u]);
                    s[1][u] = mfma_qk<BF16>(kf, qf[1][ks], s[1][u]);
                }
            }
            // softmax of query row r16 of each column block over the lane's
            // tokens tb + 16 * u + 4 * g4 + i.  The maximum that weights are
            // taken against moves only when a score exceeds it by 2^8: the
            // sums have the room, and the accumulators are rescaled seldom.
            uint32_t ph[2][STEP][2], pl[2][STEP][2];
            if (tail)
#pragma unroll
                for (int u = 0; u < STEP; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (t0 + tb + 16u * u + 4u * g4 + i >= t_end)
                            s[0][u][i] = s[1][u][i] = -INFINITY;
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) {
                float mx = -INFINITY;
#pragma unroll
                for (int u = 0; u < STEP; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mx = fmaxf(mx, s[rt][u][i]);
                mx *= qk_scale;
                if (__ballot(mx > m[rt] + 8.f)) {
                    const float m_new = fmaxf(m[rt], max_of_rows(mx));
                    const float c = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[rt] - m_new);
                    lsum[rt] *= c;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        acc[rt][mt] = acc[rt][mt] * c;
                    m[rt] = m_new;
                }
                const float m_sub = m[rt] == -INFINITY ? 0.f : m[rt];
#pragma unroll
                for (int u = 0; u < STEP; ++u) {
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        p[i] = __builtin_amdgcn_exp2f(s[rt][u][i] * qk_scale - m_sub);
                    if (tail)       // (a scale of 0 would make NaN of the mask's -inf)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            p[i] = t0 + tb + 16u * u + 4u * g4 + i < t_end ? p[i] : 0.f;
                    lsum[rt] += (p[0] + p[1]) + (p[2] + p[3]);
                    split_weights<BF16>(p[0], p[1], &ph[rt][u][0], &pl[rt][u][0]);
                    split_weights<BF16>(p[2], p[3], &ph[rt][u][1], &pl[rt][u][1]);
                }
            }
            // O^T += V^T . P^T, the weights as their 16-bit rounding and the
            // 16-bit rounding of the rest
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                uint64_t vf[STEP];
#pragma unroll
                for (int u = 0; u < STEP; ++u) {
                    const uint32_t t = tb + 16u * u + 4u * g4 + r16 / 4u;
                    const uint32_t c = 2u * mt + r16 % 4u / 2u;
                    vf[u] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (LLMIG_LDS i16x4_t *)(vt + t * RB + 16u * (c ^ swz(t)) + 8u * (r16 % 2u))));
                }
                typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
                const u32x4 v = __builtin_bit_cast(u32x4, u64x2{vf[0], vf[STEP - 1]});
#pragma unroll
                for (int rt = 0; rt < 2; ++rt) {
                    const uint32_t(&h)[STEP][2] = ph[rt], (&l)[STEP][2] = pl[rt];
                    if constexpr (STEP == 2) {
                        acc[rt][mt] = mfma_qk<BF16>(v, u32x4{h[0][0], h[0][1], h[1][0], h[1][1]}, acc[rt][mt]);
                        acc[rt][mt] = mfma_qk<BF16>(v, u32x4{l[0][0], l[0][1], l[1][0], l[1][1]}, acc[rt][mt]);
                    } else {        // 16 tokens: both parts in one product, against the same V rows twice
                        acc[rt][mt] = mfma_qk<BF16>(v, u32x4{h[0][0], h[0][1], l[0][0], l[0][1]}, acc[rt][mt]);
                    }
                }
            }
        }
        if (more)
            put(buf ^ 1u);
    }

    // The wavefronts that split the tokens meet in LDS, 16 rows of each at a
    // time, and the records leave in whole rows.
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
        lsum[rt] = sum_of_rows(lsum[rt]);
    float *so = reinterpret_cast<float *>(&smem[0][0][0]);        // [wave][16 rows][kMergeRow]
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
        __syncthreads();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            *reinterpret_cast<f32x4_t *>(so + (wave * 16u + r16) * kMergeRow + 16 * mt + 4 * g4) = acc[rt][mt];
        if (g4 == 0) {
            sh_m[wave][16 * rt + r16] = m[rt];
            sh_l[wave][16 * rt + r16] = lsum[rt];
        }
        __syncthreads();
        for (uint32_t x = threadIdx.x; x < WM * 16u * (D / 4); x += kThreads) {
            const uint32_t r = x / (D / 4), d4 = x % (D / 4), w0 = r / 16u, rr = r % 16u;
            const uint32_t row = chunk * 32u * WM + w0 * 32u + 16u * rt + rr;
            if (row >= M)
                continue;
            float mm = -INFINITY, ll = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < 4 / WM; ++w)
                mm = fmaxf(mm, sh_m[w * WM + w0][16 * rt + rr]);
            f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t w = 0; w < 4 / WM; ++w) {
                const uint32_t v = w * WM + w0;
                const float mw = sh_m[v][16 * rt + rr];
                // (no weight: a factor of 1 would do as well, but for a NaN sum)
                const float c = mw == -INFINITY ? 1.f : exp2f(mw - mm);
                ll += sh_l[v][16 * rt + rr] * c;
                o += *reinterpret_cast<const f32x4_t *>(so + (v * 16u + rr) * kMergeRow + 4 * d4) * c;
            }
            float *rec = a.ws + (((static_cast<uint64_t>(layer) * a.parts + part) * a.members + row / G) * a.q_heads + g * G +
                                 row % G) * (D + kAttnHeader);
            *(LLMIG_GLOBAL f32x4_t *)(rec + kAttnHeader + 4 * d4) = o;
            if (d4 == 0)          // the maximum in the natural base, as attn_partial_mfma leaves it
                *(LLMIG_GLOBAL f32x4_t *)rec = f32x4_t{mm == -INFINITY ? -INFINITY : mm / kLog2e, ll, 0.f, 0.f};
        }
    }
}

// Joins the records of the prefix and of a sequence's own tokens.  D / 4 lanes
// a row (layer, sequence, query head) and record, SUB of them side by side, each
// with every SUB-th record, eight records' loads in flight; they meet in LDS.
template <int D, int SUB>
__global__ void __launch_bounds__(kThreads) prefix_join(const PrefixJoinArgs a)
{
    constexpr uint32_t kQuads = D / 4, kRec = D + kAttnHeader, kRows = kThreads / (kQuads * SUB);
    const uint32_t d4 = threadIdx.x % kQuads, sub = threadIdx.x / kQuads % SUB, mine = threadIdx.x / (kQuads * SUB);
    const uint32_t rows = a.num_layers * a.batch * a.q_heads;
    const uint32_t r0 = a.row_base + blockIdx.x * kRows + mine;
    const uint32_t r = min(r0, rows - 1u);
    const uint32_t h = r % a.q_heads, s = r / a.q_heads % a.batch, layer = r / a.q_heads / a.batch;
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

// The join for at most `most` records a row; its rows per workgroup.
inline const void *prefix_join_kernel(int head_dim, uint32_t most, uint32_t *rows)
{
    *rows = kThreads / (head_dim / 4) / (most <= 8 ? 1u : 8u);
    if (head_dim == 64)
        return most <= 8 ? reinterpret_cast<const void *>(&prefix_join<64, 1>) : reinterpret_cast<const void *>(&prefix_join<64, 8>);
    return most <= 8 ? reinterpret_cast<const void *>(&prefix_join<128, 1>) : reinterpret_cast<const void *>(&prefix_join<128, 8>);
}

template <int BF16, int D>
const void *prefix_kernel(uint32_t wm)
{
    return wm == 1   ? reinterpret_cast<const void *>(&prefix_rows<BF16, D, 1>)
           : wm == 2 ? reinterpret_cast<const void *>(&prefix_rows<BF16, D, 2>)
                     : reinterpret_cast<const void *>(&prefix_rows<BF16, D, 4>);
}

inline const void *prefix_kernel_for(int bf16, int head_dim, uint32_t wm)
{
    if (head_dim == 64)
        return bf16 ? prefix_kernel<1, 64>(wm) : prefix_kernel<0, 64>(wm);
    return bf16 ? prefix_kernel<1, 128>(wm) : prefix_kernel<0, 128>(wm);
}

// How the prefix of a call is cut: wavefronts of a workgroup that split the
// rows, workgroups that share a partition, partitions.
struct PrefixCut {
    uint32_t wm, chunks, part_tokens, parts;
};

inline PrefixCut prefix_cut(uint32_t rows, int64_t tokens, int64_t layer_heads)
{
    PrefixCut c;
    c.wm = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    c.chunks = (rows + 32 * c.wm - 1) / (32 * c.wm);
    const int64_t tiles = (tokens + kPrefixTile - 1) / kPrefixTile;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(tiles, 512 / std::max<int64_t>(1, layer_heads * c.chunks)));
    const int64_t per = (tiles + want - 1) / want;
    c.part_tokens = static_cast<uint32_t>(per * kPrefixTile);
    c.parts = static_cast<uint32_t>((tiles + per - 1) / per);
    return c;
}

} // namespace
