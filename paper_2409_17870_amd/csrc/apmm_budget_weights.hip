// What attention of the new tokens gives each token of the four-bit cache (apmm_kv_attention.h has the scores):
//
//   w_j = decay w_j + sum over rows i of p_ij,   p_ij = 2^(x_ij - m_i) / l_i,  m_i = max_j x_ij,  l_i = sum_j 2^(x_ij - m_i)
//
// Rows are the queries of a sequence's new tokens and of the query heads that share a key/value head.  Two passes over the keys: one for m and l of each row, whose lanes hold those of some keys each and
// meet at the end, one that owns some keys and goes through the rows.  No sum's order depends on timing.  (m and 1 / l are kept apart: one number m + log2(l) would be rounded to 2^-24 of itself, which
// is more than the sums' own error.)
#include <algorithm>

#include "apmm_budget.h"

namespace apmm {

namespace {

constexpr int kStep = 32;     // keys of a step of the first pass
constexpr int kWaves = 4;
constexpr int kKeys = 64;     // keys of a wave of the second pass
constexpr int kChunk = 4;     // tiles of 16 rows that are in LDS at a time there

struct RowFactor { float base, by; };  // -m and 1 / l; zeros for a row that sees nothing

// The odd integers 2 u - 15 of a word of codes as operand words (nibbles 0 and 4, 1 and 5, 2 and 6, 3 and 7): a code in bits 1 to 4 under the upper bits of 1024 is 1024 + 2 u, in bits 4 to 7 under those of
// 128 it is 128 + 2 u.  The attention's operands, u 2^-24, take five operations in place of eleven, and leave a score off by 2^-17 of itself where these leave 2^-24 (the matrix unit keeps fewer bits of
// products of subnormal numbers): too much for weights that are a result of 32 bits.
__device__ __forceinline__ half8 odd_operand(uint32_t w)
{
    const half2v less2 = {(_Float16)-1039.0f, (_Float16)-1039.0f}, less4 = {(_Float16)-143.0f, (_Float16)-143.0f};
    const uint32_t h = w >> 8;
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, ((w << 1) & 0x001e001eu) | 0x64006400u) + less2);
    r.y = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, (w & 0x00f000f0u) | 0x58005800u) + less4);
    r.z = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, ((w >> 7) & 0x001e001eu) | 0x64006400u) + less2);
    r.w = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, (h & 0x00f000f0u) | 0x58005800u) + less4);
    return __builtin_bit_cast(half8, r);
}

// The places of a lane's codes (its part of key lane % 16 of 16) and of the scales of its four scores
template <int D>
struct Keys {
    half8 k[D / 32];
    float s[4];
};
template <int D>
struct KeyCodes {
    uint32_t k[D / 32];
    uint2 s;
};
template <int D>
__device__ __forceinline__ void load_keys(const KvAttentionArgs &a, int head, int key, int page, KeyCodes<D> &s)
{
    const int shift = a.c.page_shift, n = kv_lane() & 15, g = kv_lane() >> 4;
    const int64_t place = ((((int64_t)max(page, 0) * a.c.heads + head) * 2) << shift) + (key & ((1 << shift) - 1));
    const uint8_t *keys = a.c.codes + place * (D / 2) + n * (D / 2) + g * (D / 8);
    if constexpr (D == 128) {
        const uint4 w = *reinterpret_cast<const uint4 *>(keys);
        s.k[0] = w.x; s.k[1] = w.y; s.k[2] = w.z; s.k[3] = w.w;
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(keys);
        s.k[0] = w.x; s.k[1] = w.y;
    }
    s.s = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(a.c.scales + place) + g * 8);
}
template <int D, bool BF16>
__device__ __forceinline__ void make_keys(const KeyCodes<D> &from, Keys<D> &to)
{
#pragma unroll
    for (int i = 0; i < D / 32; ++i) to.k[i] = odd_operand(from.k[i]);
    to.s[0] = kv_low<BF16>(from.s.x); to.s[1] = kv_high<BF16>(from.s.x);
    to.s[2] = kv_low<BF16>(from.s.y); to.s[3] = kv_high<BF16>(from.s.y);
}

// Rows of a wave as operands: row `row` (lane % 16 of a tile) of a sequence, channels j and j + 4 of eight to a word as the keys' codes lie.  binary16 numbers as they are; bfloat16 ones times a power of two
// that puts the row's largest just below 2^15: numbers below 2^-24 of that lose bits, 2^-39 of it at most.  `factor` is what makes a score, in powers of two, of a product and the key's scale.
template <int D, bool BF16>
__device__ __forceinline__ void load_rows(const KvAttentionArgs &a, int start, int head, int row, half8 (&q)[D / 32], float &factor)
{
    const int g = kv_lane() >> 4, at = kv_divide(row, a.by_groups);
    uint32_t x[D / 8];
    kv_load(a.q.data + (int64_t)(start + at) * a.q.token_stride + (int64_t)(head * a.groups + row - at * a.groups) * a.q.head_stride + g * (D / 4), a.q.aligned, x);
    float by = 1.0f;
    if (BF16) {
        uint32_t bits2 = 0, bits = 0;  // of the largest finite magnitude
#pragma unroll
        for (int i = 0; i < D / 8; ++i) bits2 = kv_fold_max(bits2, x[i] & 0x7fff7fffu);
        bits = max(bits2 & 0xffffu, bits2 >> 16);
        if (bits >= 0x7f80u) {
            bits = 0;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) bits = kv_finite_max<true>(kv_finite_max<true>(bits, x[i] & 0x7fffu), (x[i] >> 16) & 0x7fffu);
        }
        bits = max(bits, (uint32_t)__shfl_xor((int)bits, 16));
        bits = max(bits, (uint32_t)__shfl_xor((int)bits, 32));
        const int e = min(15 - ((int)(bits >> 7) - 126), 100);  // (rows of the smallest numbers, and of zeros)
        by = ldexpf(1.0f, e);
        factor = fminf(fmaxf(ldexpf(a.scale * 1.44269504088896341f, -e), 0x1p-149f), -kLowest);
    } else {
        factor = fminf(a.scale * 1.44269504088896341f, -kLowest);
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t u = x[4 * i + j / 2], v = x[4 * i + j / 2 + 2];
            if (BF16) w[j] = kv_half_pair((j & 1 ? kv_high<true>(u) : kv_low<true>(u)) * by, (j & 1 ? kv_high<true>(v) : kv_low<true>(v)) * by);
            else w[j] = __builtin_amdgcn_perm(v, u, j & 1 ? 0x07060302u : 0x05040100u);
        }
        q[i] = __builtin_bit_cast(half8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

// First pass.  A workgroup has R tiles of 16 rows and a piece of the keys that they see, its waves take steps in turn.
template <int D, bool BF16, int R>
__global__ __launch_bounds__(64 * kWaves) void kv_statistics_kernel(KvAttentionArgs a, KvPart part, RowFactor *factors)
{
    constexpr int W = D / 32, T = 16 * R;
    __shared__ float bases[kWaves][T], totals[kWaves][T];
    const int slot = kv_divide(blockIdx.x, a.c.by_heads), head = blockIdx.x - slot * a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4;
    KvItem<kStep> it;
    const bool there = kv_item<kStep, T>(a, part, slot, it);
    if (part.target && threadIdx.x == 0) {
        KvPieceNote note = {};
        if (there && it.part == 0 && it.pieces > 1) note = {it.s.start, it.row0, min(it.rows, T), min(it.pieces, part.slots - slot)};  // (no more than there are slots: as in kv_note)
        kv_partial(a.partial, part, a.c.heads, 0).note[(int64_t)slot * a.c.heads + head] = note;
    }
    if (!there) return;
    const int rows = min(it.rows, T);
    half8 q[R][W];
    float factor[R], top[R], total[R];
    int pos[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = it.row0 + min(16 * r + n, rows - 1);
        load_rows<D, BF16>(a, it.s.start, head, row, q[r], factor[r]);
        pos[r] = it.s.first + kv_divide(row, a.by_groups);
        top[r] = kLowest;
        total[r] = 0.0f;
    }
    const int first_pos = it.s.first + kv_divide(it.row0, a.by_groups), last_pos = it.s.first + kv_divide(it.row0 + rows - 1, a.by_groups);
    int v = it.from + wave, ids = kv_page_ids(a, it, v, kWaves), id = 0;
    for (; v < it.to; v += kWaves) {
        const int key0 = it.key_of(v), page0 = __builtin_amdgcn_readlane(ids, id), page1 = __builtin_amdgcn_readlane(ids, id + 1);
        id += 2;
        if (id == 64) {
            ids = kv_page_ids(a, it, v + kWaves, kWaves);
            id = 0;
        }
        KeyCodes<D> codes[2];
        load_keys<D>(a, head, key0, page0, codes[0]);
        load_keys<D>(a, head, key0 + 16, page1, codes[1]);
        Keys<D> keys[2];
        make_keys<D, BF16>(codes[0], keys[0]);
        make_keys<D, BF16>(codes[1], keys[1]);
        const bool all = key0 + kStep <= it.s.keys && key0 + kStep - 1 <= first_pos && page0 >= 0 && page1 >= 0 && (!a.window || key0 > last_pos - a.window || key0 + kStep <= a.sinks);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (16 * r >= rows) break;
            float x[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float4v s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < W; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys[t].k[i], q[r][i], s, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[4 * t + i] = s[i] * keys[t].s[i] * factor[r];
            }
            if (!all) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = key0 + 16 * (i / 4) + 4 * g + i % 4, end = (i < 4 ? page0 : page1) >= 0 ? min(it.s.keys, pos[r] + 1) : 0;
                    const bool hidden = (key >= end) | ((a.window != 0) & (key <= pos[r] - a.window) & (key >= a.sinks));
                    x[i] = hidden ? -__builtin_inff() : x[i];
                }
            }
            const float high = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))), to = fmaxf(top[r], high);
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += __builtin_amdgcn_exp2f(x[i] - to);
            total[r] = fmaf(total[r], __builtin_amdgcn_exp2f(top[r] - to), sum);
            top[r] = to;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float to = fmaxf(fmaxf(top[r], __shfl_xor(top[r], 16)), fmaxf(__shfl_xor(top[r], 32), __shfl_xor(top[r], 48)));
        float t = total[r] * __builtin_amdgcn_exp2f(top[r] - to);
        t += __shfl_xor(t, 16);
        t += __shfl_xor(t, 32);
        if (g == 0) {
            bases[wave][16 * r + n] = to;
            totals[wave][16 * r + n] = t;
        }
    }
    __syncthreads();
    for (int r = threadIdx.x; r < rows; r += 64 * kWaves) {
        float to = bases[0][r], t = 0.0f;
#pragma unroll
        for (int i = 1; i < kWaves; ++i) to = fmaxf(to, bases[i][r]);
#pragma unroll
        for (int i = 0; i < kWaves; ++i) t = fmaf(totals[i][r], __builtin_amdgcn_exp2f(bases[i][r] - to), t);
        if (it.pieces == 1) {
            const int row = it.row0 + r, at = kv_divide(row, a.by_groups);
            factors[(int64_t)(it.s.start + at) * a.c.heads * a.groups + head * a.groups + row - at * a.groups] = t == 0.0f ? RowFactor{0.0f, 0.0f} : RowFactor{-to, 1.0f / t};
        } else {
            kv_partial(a.partial, part, a.c.heads, 0).row[((int64_t)slot * a.c.heads + head) * T + r] = make_float2(to, t);
        }
    }
}

// Joins the pieces of tiles whose keys were cut: a lane to a row
__global__ __launch_bounds__(64) void kv_statistics_join_kernel(KvAttentionArgs a, KvPart part, RowFactor *factors)
{
    const int item = blockIdx.x, head = item - kv_divide(item, a.c.by_heads) * a.c.heads, r = threadIdx.x;
    const KvPartial partial = kv_partial(a.partial, part, a.c.heads, 0);
    const KvPieceNote note = partial.note[item];
    if (note.pieces == 0 || r >= note.rows) return;
    float to = kLowest, total = 0.0f;
    for (int i = 0; i < note.pieces; ++i) {
        const float2 p = partial.row[((int64_t)item + (int64_t)i * a.c.heads) * part.tile + r];
        const float top = fmaxf(to, p.x);
        total = fmaf(total, __builtin_amdgcn_exp2f(to - top), p.y * __builtin_amdgcn_exp2f(p.x - top));
        to = top;
    }
    const int row = note.row0 + r, at = kv_divide(row, a.by_groups);
    factors[(int64_t)(note.start + at) * a.c.heads * a.groups + head * a.groups + row - at * a.groups] = total == 0.0f ? RowFactor{0.0f, 0.0f} : RowFactor{-to, 1.0f / total};
}

// Second pass.  A workgroup takes 256 keys of a head at a time, 64 to a wave, and goes through the rows that may see them: each of its waves makes operands of 16 rows, which all read from LDS.
template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves) void kv_weights_kernel(KvAttentionArgs a, KvWeights out, float decay, const RowFactor *factors)
{
    constexpr int W = D / 32, KT = kKeys / 16;
    __shared__ __align__(16) half8 rows_q[kChunk][W][64];
    __shared__ float4v rows_f[kChunk][16];  // factor, base, by
    __shared__ int rows_pos[kChunk][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4, head = blockIdx.y;
    for (int unit = blockIdx.x;; unit += gridDim.x) {
        int b, rest;
        auto count = [&](int at) {
            const KvSequence s = kv_sequence(a.c, at);
            return s.n ? (s.keys + kWaves * kKeys - 1) / (kWaves * kKeys) : 0;  // (fewer than 2^31 in all: kv_weights_blocks)
        };
        if (!kv_find(a.c.sequences, unit, b, rest, count)) return;
        const KvSequence s = kv_sequence(a.c, b);
        const int block0 = rest * kWaves * kKeys, key0 = block0 + wave * kKeys;
        KeyCodes<D> codes[KT];
        int pages[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const int key = key0 + 16 * t;
            pages[t] = key < s.keys ? a.c.table[b * a.c.table_stride + (key >> a.c.page_shift)] : -1;
            if (pages[t] >= a.c.pages) pages[t] = -1;
            load_keys<D>(a, head, key, pages[t], codes[t]);
        }
        // rows whose position is that of the block's first key or later, and under a window those that see its last key or have it among the first ones
        const int rows = s.n * a.groups;
        const int first_token = max(block0 - s.first, 0);
        int last_token = s.n;  // (behind the last)
        if (a.window && block0 >= a.sinks) last_token = (int)min((int64_t)s.n, max((int64_t)block0 + kWaves * kKeys - 1 + a.window - s.first, (int64_t)0));
        const int row_end = min(last_token * a.groups, rows);
        float sums[KT][4];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[t][i] = 0.0f;
        Keys<D> keys[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) make_keys<D, BF16>(codes[t], keys[t]);
        for (int row0 = first_token * a.groups / 16 * 16; row0 < row_end; row0 += 16 * kChunk) {
            __syncthreads();
            if (row0 + 16 * wave < row_end) {
                const int row = min(row0 + 16 * wave + n, rows - 1), at = kv_divide(row, a.by_groups);
                half8 q[W];
                float factor;
                load_rows<D, BF16>(a, s.start, head, row, q, factor);
#pragma unroll
                for (int i = 0; i < W; ++i) rows_q[wave][i][lane] = q[i];
                if (g == 0) {
                    RowFactor f = factors[(int64_t)(s.start + at) * a.c.heads * a.groups + head * a.groups + row - at * a.groups];
                    if (row0 + 16 * wave + n >= rows) f.by = 0.0f;  // (the last row again)
                    rows_f[wave][n] = float4v{factor, f.base, f.by, 0.0f};
                    rows_pos[wave][n] = row0 + 16 * wave + n < rows ? s.first + at : -1;
                }
            }
            __syncthreads();
            const int tiles = min((row_end - row0 + 15) / 16, kChunk);
            for (int tile = 0; tile < tiles; ++tile) {
                half8 q[W];
#pragma unroll
                for (int i = 0; i < W; ++i) q[i] = rows_q[tile][i][lane];
                const float4v f = rows_f[tile][n];
                const int pos = rows_pos[tile][n], from = __builtin_amdgcn_readfirstlane(rows_pos[tile][0]), last = min(row0 + 16 * tile + 15, rows - 1), to = s.first + kv_divide(last, a.by_groups);
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    const int key = key0 + 16 * t;
                    float4v x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < W; ++i) x = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys[t].k[i], q[i], x, 0, 0, 0);
                    const bool all = row0 + 16 * tile + 16 <= rows && key + 16 <= s.keys && key + 15 <= from && pages[t] >= 0 && (!a.window || key > to - a.window || key + 16 <= a.sinks);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float y = x[i] * keys[t].s[i];
                        if (all) {
                            sums[t][i] = fmaf(__builtin_amdgcn_exp2f(fmaf(y, f[0], f[1])), f[2], sums[t][i]);
                        } else {
                            const int k = key + 4 * g + i;
                            const bool hidden = (k > pos) | (k >= s.keys) | (pages[t] < 0) | ((a.window != 0) & (k <= pos - a.window) & (k >= a.sinks));
                            const float p = hidden ? 0.0f : __builtin_amdgcn_exp2f(fmaf(y, f[0], f[1])) * f[2];
                            sums[t][i] += p;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = sums[t][i];
#pragma unroll
                for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
                const int key = key0 + 16 * t + 4 * g + i;
                if (n == 4 * t + i && key < s.keys && key < out.capacity) {
                    float *w = out.data + b * out.sequence_stride + head * out.head_stride + key;
                    *w = decay == 0.0f ? v : fmaf(decay, *w, v);
                }
            }
    }
}

template <int D, bool BF16>
void launch(const KvAttentionArgs &a, const KvWeights &w, float decay, const KvWeightsPlan &p, hipStream_t stream)
{
    RowFactor *factors = reinterpret_cast<RowFactor *>(reinterpret_cast<uint8_t *>(a.partial) + p.pieces_bytes);
    const dim3 first((uint32_t)((int64_t)p.part.slots * a.c.heads));
    if (p.row_tiles == 1) kv_statistics_kernel<D, BF16, 1><<<first, dim3(64 * kWaves), 0, stream>>>(a, p.part, factors);
    else kv_statistics_kernel<D, BF16, 4><<<first, dim3(64 * kWaves), 0, stream>>>(a, p.part, factors);
    if (p.part.target) kv_statistics_join_kernel<<<first, dim3(64), 0, stream>>>(a, p.part, factors);
    kv_weights_kernel<D, BF16><<<dim3((uint32_t)p.groups, (uint32_t)a.c.heads), dim3(64 * kWaves), 0, stream>>>(a, w, decay, factors);
}

}  // namespace

// Blocks of keys that the second pass may have
int64_t kv_weights_blocks(const KvArgs &c)
{
    return (std::min<int64_t>((int64_t)c.width << c.page_shift, kKvMost) + kWaves * kKeys - 1) / (kWaves * kKeys) * c.sequences;
}

KvWeightsPlan kv_weights_plan(const KvArgs &c, int groups, int window, int sinks)
{
    KvWeightsPlan p = {};
    const int64_t rows = (int64_t)c.tokens * groups, sequences = std::min(c.sequences, c.tokens);
    p.row_tiles = rows <= 16 || c.tokens <= c.sequences ? 1 : 4;
    p.rows = rows * c.heads;
    KvPart &t = p.part;
    t.tile = 16 * p.row_tiles;
    t.to_rows = INT32_MAX;
    t.least = 32;
    const int64_t tiles = std::min(c.tokens * (int64_t)((groups + t.tile - 1) / t.tile), rows / t.tile + sequences);
    int64_t most_steps = (((int64_t)c.width << c.page_shift) + kStep - 1) / kStep;
    if (window) most_steps = std::min<int64_t>(most_steps, kv_window_steps(window, sinks, (t.tile + groups - 2) / groups, kStep));
    t.target = tiles * c.heads >= 4096 || most_steps <= t.least ? 0 : std::max(1024 / c.heads, 1);
    t.slots = (int)(tiles + (t.target ? t.target + 1 : 0));
    if (t.target) {
        const KvPartial at = kv_partial(nullptr, t, c.heads, 0);
        p.pieces_bytes = reinterpret_cast<size_t>(at.note + (int64_t)t.slots * c.heads);
    }
    p.groups = std::max<int64_t>(1, std::min<int64_t>(kv_weights_blocks(c), std::max(1, 4096 / c.heads)));
    return p;
}

size_t kv_weights_bytes(const KvWeightsPlan &p) { return p.pieces_bytes + p.rows * sizeof(RowFactor); }
int64_t kv_weights_items(const KvWeightsPlan &p, int heads) { return std::max((int64_t)p.part.slots, p.groups) * heads * 64 * kWaves; }

hipError_t launch_kv_weights(const KvAttentionArgs &a, const KvWeights &w, float decay, const KvWeightsPlan &p, hipStream_t stream)
{
    if (a.c.head_dim == 128) a.c.bf16 ? launch<128, true>(a, w, decay, p, stream) : launch<128, false>(a, w, decay, p, stream);
    else a.c.bf16 ? launch<64, true>(a, w, decay, p, stream) : launch<64, false>(a, w, decay, p, stream);
    return hipGetLastError();
}

}  // namespace apmm
