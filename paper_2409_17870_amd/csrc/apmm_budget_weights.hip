// What attention of the new tokens gives each token of the four-bit cache (apmm_kv_attention.h has the scores):
//
//   w_j = decay w_j + sum over rows i of p_ij,   p_ij = 2^(x_ij - m_i) / l_i,  m_i = max_j x_ij,  l_i = sum_j 2^(x_ij - m_i)
//
// Rows are the queries of a sequence's new tokens and of the query heads that share a key/value head.  Two passes over the keys: one for m and l of each row, whose lanes hold those of some keys each and
// meet at the end, one that owns some keys and goes through the rows.  No sum's order depends on timing.  (m and 1 / l are kept apart: one number m + log2(l) would be rounded to 2^-24 of itself, which
// is more than the sums' own error.)
//
// Few rows of a sequence (up to 16: token generation): both passes have the same workgroups, a piece of the keys each; the second joins the pieces' m and l as it begins.  The first keeps its scores for the second, a
// number for each row and key, where they are no more than 2^26; else, and for the sequences of few rows beside others of many, the second makes them again from the keys.  8 sequences of up to 32768 tokens, 8 key/value
// heads of 128: 4 query heads to one 51 us with scores kept (35 and 13; 111 MB of keys, 26 MB of scores written and read) and 78 with scores made twice (34 and 40), 6 60 and 78; 4 sequences of 8 to one 39 and 49, 16 to one
// of 4 heads 32 and 35; one sequence of 3000 tokens 19 and 24.  Bound by HBM and, at the beginnings, by the way from lengths to pages to codes.
// Many: the second pass has blocks of 256 keys (fewer where there are few of them), as operands in registers, and every row that sees some of them comes by through LDS, as the first pass left it in the workspace (RowTiles).  4096 tokens
// of 32 heads of 128: 100 and 110 us where calls follow each other (120 and 128 in the first twenty after a pause).  Bound by the vector unit in the first pass: 11 instructions a score, of which the exponential takes the time of two, busy for
// 92 % of the cycles in which its compute unit has work, which are 88 % of all.  In the second pass (9 instructions) no unit is full: vector 72 %, LDS 58 %, matrix 30 % of the cycles with work, which are 81 % of all, since each workgroup has one
// block here and the first ones have the most rows.  When the passes took 115 and 122 us: the first one with the rows in registers, three waves to a vector unit, 126; half as many workgroups, each with a first and a last block, 10 more in
// all; the next tile's operands read ahead, or its products made ahead, which take registers that a fourth wave to a SIMD has, 2 and 10 more.
#include <algorithm>
#include <type_traits>

#include "apmm_budget.h"

namespace apmm {

namespace {

constexpr int kStep = 32;     // keys of a step of the first pass
constexpr int kWaves = 4;
constexpr int kFew = 16;      // rows of a sequence that are few
constexpr int64_t kMostScores = 64 << 20;  // few rows' that are kept in the workspace
constexpr int kChunk = 4;     // tiles of 16 rows that are in LDS at a time
constexpr int kFold = 8;      // of these whose weights are one sum

struct RowFactor { float base, by; };  // -m and 1 / l; zeros for a row that sees nothing

// Many rows' operands and factors, by tiles of 16 rows of a sequence, as the first pass leaves them for the second, which reads each tile once for every 128 keys or so: rows where they lie are a power of two
// apart as a rule and meet in few channels of L2 (4096 tokens of 32 heads: 155 us of the second pass with rows from there).
struct RowTiles {
    uint8_t *operands;    // [tile][head][operand][lane] of 16 bytes
    RowFactor *factors;   // [tile][head][16]
    float *scales;        // [tile][head][16]: what makes a score of a product and the key's scale
};
// Few rows' scores, in powers of two, by the first pass for the second: of each row of the call and head as many as the page table has tokens, of those keys that the row's tile visits
struct RowScores {
    float *data;
    int64_t stride;
    __device__ __forceinline__ float *of(const KvAttentionArgs &a, int row, int head) const { return data + ((int64_t)row * a.c.heads + head) * stride; }
};
// The first tile of sequence b: the tiles of the sequences before it end below
__device__ __forceinline__ int first_tile(const KvAttentionArgs &a, const KvSequence &s, int b) { return (int)((int64_t)s.start * a.groups / 16) + b; }

// The odd integers 2 u - 15 of a word of codes as operand words (nibbles 0 and 4, 1 and 5, 2 and 6, 3 and 7): a code in bits 1 to 4 under the upper bits of 1024 is 1024 + 2 u, in bits 4 to 7 under those of
// 128 it is 128 + 2 u.  The attention's operands, u 2^-24, take five operations in place of eleven, and leave a score off by 2^-17 of itself where these leave 2^-24 (the matrix unit keeps fewer bits of
// products of subnormal numbers): too much for weights that are a result of 32 bits.
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits)
{
    uint32_t r;  // (in one instruction with one of the two in a scalar register; of two literals the compiler makes two)
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "s"(mask), "v"(bits));
    return r;
}
__device__ __forceinline__ half8 odd_operand(uint32_t w)
{
    const half2v less2 = {(_Float16)-1039.0f, (_Float16)-1039.0f}, less4 = {(_Float16)-143.0f, (_Float16)-143.0f};
    const uint32_t h = w >> 8;
    uint4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, and_or(w << 1, 0x001e001eu, 0x64006400u)) + less2);
    r.y = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, and_or(w, 0x00f000f0u, 0x58005800u)) + less4);
    r.z = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, and_or(w >> 7, 0x001e001eu, 0x64006400u)) + less2);
    r.w = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, and_or(h, 0x00f000f0u, 0x58005800u)) + less4);
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
__device__ __forceinline__ void make_rows(const KvAttentionArgs &a, const uint32_t (&x)[D / 8], half8 (&q)[D / 32], float &factor)
{
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
// Their numbers as they lie
template <int D>
__device__ __forceinline__ void load_rows(const KvAttentionArgs &a, int start, int head, int row, int at, uint32_t (&x)[D / 8])
{
    kv_load(a.q.data + (int64_t)(start + at) * a.q.token_stride + (int64_t)(head * a.groups + row - at * a.groups) * a.q.head_stride + (kv_lane() >> 4) * (D / 4), a.q.aligned, x);
}
template <int D, bool BF16>
__device__ __forceinline__ void take_rows(const KvAttentionArgs &a, int start, int head, int row, half8 (&q)[D / 32], float &factor)
{
    uint32_t x[D / 8];
    load_rows<D>(a, start, head, row, kv_divide(row, a.by_groups), x);
    make_rows<D, BF16>(a, x, q, factor);
}

// Pieces of the first pass: a slot's rows' m and l
__device__ __forceinline__ float2 *piece_rows(const KvAttentionArgs &a, float *at, const KvPart &part, int slot, int head) { return reinterpret_cast<float2 *>(at) + ((int64_t)slot * a.c.heads + head) * part.tile; }
// ... and behind these, where rows are many, the notes for their joining
__device__ __forceinline__ KvPieceNote *piece_note(const KvAttentionArgs &a, float *at, const KvPart &part, int slot, int head)
{
    return reinterpret_cast<KvPieceNote *>(piece_rows(a, at, part, part.slots, 0)) + (int64_t)slot * a.c.heads + head;
}
__device__ __forceinline__ RowFactor factor_of(float top, float total) { return total == 0.0f ? RowFactor{0.0f, 0.0f} : RowFactor{-top, 1.0f / total}; }
__device__ __forceinline__ void join(float &top, float &total, float other_top, float other_total)
{
    const float to = fmaxf(top, other_top);
    total = fmaf(total, __builtin_amdgcn_exp2f(top - to), other_total * __builtin_amdgcn_exp2f(other_top - to));
    top = to;
}

// One instruction (fmaxf first makes a quiet NaN of each operand that might be a signalling one, with an instruction of its own)
__device__ __forceinline__ float max_of_three(float x, float y, float z)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
}

// First pass.  A workgroup has R tiles of 16 rows and a piece of the keys that they see, its waves take steps in turn, the next step's codes on their way while one's scores are made.
template <int D, bool BF16, int R, bool SCORES>
__global__ __launch_bounds__(64 * kWaves, 4) void kv_statistics_kernel(KvAttentionArgs a, KvPart part, float *pieces, RowTiles out, RowScores scores)
{
    constexpr int W = D / 32, T = 16 * R;
    __shared__ float bases[kWaves][T], totals[kWaves][T];
    const int slot = kv_divide(blockIdx.x, a.c.by_heads), head = blockIdx.x - slot * a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4;
    KvItem<kStep> it;
    const bool there = kv_item<kStep, T>(a, part, slot, it);
    if (R > 1 && part.target && threadIdx.x == 0) {
        KvPieceNote note = {};
        if (there && it.part == 0 && it.pieces > 1) note = {0, first_tile(a, it.s, it.b) + it.row0 / 16, min(it.rows, T), min(it.pieces, part.slots - slot)};  // (no more than there are slots: as in kv_note)
        *piece_note(a, pieces, part, slot, head) = note;
    }
    if (!there) return;
    const int rows = min(it.rows, T);
    int v = it.from + wave, ids = kv_page_ids(a, it, v, kWaves), id = 0;
    KeyCodes<D> codes[2], next[2];
    if (v < it.to) {
        load_keys<D>(a, head, it.key_of(v), __builtin_amdgcn_readlane(ids, 0), codes[0]);
        load_keys<D>(a, head, it.key_of(v) + 16, __builtin_amdgcn_readlane(ids, 1), codes[1]);
    }
    // one tile's operands are in each wave's registers, several tiles' in LDS, a wave makes one
    __shared__ __align__(16) half8 rows_q[R > 1 ? R : 1][W][R > 1 ? 64 : 1];
    __shared__ float rows_factor[R][16];
    half8 q[W];
    float factor[R], top[R], total[R];
    int pos[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        pos[r] = it.s.first + kv_divide(it.row0 + min(16 * r + n, rows - 1), a.by_groups);
        top[r] = kLowest;
        total[r] = 0.0f;
    }
    take_rows<D, BF16>(a, it.s.start, head, it.row0 + min(16 * (R > 1 ? wave : 0) + n, rows - 1), q, factor[0]);
    if constexpr (R > 1) {
        static_assert(R == kWaves, "a tile to a wave");
#pragma unroll
        for (int i = 0; i < W; ++i) rows_q[wave][i][lane] = q[i];
        if (g == 0) rows_factor[wave][n] = factor[0];
        if (it.part == 0 && 16 * wave < rows) {
            const int64_t tile = (int64_t)(first_tile(a, it.s, it.b) + it.row0 / 16 + wave) * a.c.heads + head;
#pragma unroll
            for (int i = 0; i < W; ++i) reinterpret_cast<half8 *>(out.operands)[(tile * W + i) * 64 + lane] = q[i];
            if (g == 0) out.scales[tile * 16 + n] = factor[0];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) factor[r] = rows_factor[r][n];
    }
    const int first_pos = it.s.first + kv_divide(it.row0, a.by_groups), last_pos = it.s.first + kv_divide(it.row0 + rows - 1, a.by_groups);
    for (; v < it.to; v += kWaves) {
        const int key0 = it.key_of(v), page0 = __builtin_amdgcn_readlane(ids, id), page1 = __builtin_amdgcn_readlane(ids, id + 1);
        id += 2;
        if (id == 64) {
            ids = kv_page_ids(a, it, v + kWaves, kWaves);
            id = 0;
        }
        {   // (behind the last step the same one again: from the cache, and no branch)
            const bool more = v + kWaves < it.to;
            const int key = more ? it.key_of(v + kWaves) : key0;
            load_keys<D>(a, head, key, more ? __builtin_amdgcn_readlane(ids, id) : page0, next[0]);
            load_keys<D>(a, head, key + 16, more ? __builtin_amdgcn_readlane(ids, id + 1) : page1, next[1]);
        }
        Keys<D> keys[2];
        make_keys<D, BF16>(codes[0], keys[0]);
        make_keys<D, BF16>(codes[1], keys[1]);
        const bool all = key0 + kStep <= it.s.keys && key0 + kStep - 1 <= first_pos && page0 >= 0 && page1 >= 0 && (!a.window || key0 > last_pos - a.window || key0 + kStep <= a.sinks);
        if (R > 1) asm volatile("" ::: "memory");  // (the rows' operands are read in each step: held from one to the next they take the registers that a fourth wave has)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (16 * r >= rows) break;
            float x[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float4v s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < W; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys[t].k[i], R > 1 ? rows_q[r][i][R > 1 ? lane : 0] : q[i], s, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[4 * t + i] = s[i] * keys[t].s[i];
            }
            if (!all) {
                int first = key0 + 4 * g, below = a.window ? pos[r] - a.window : INT32_MIN, end = min(it.s.keys, pos[r] + 1);
                asm volatile("" : "+v"(first));  // (else all that follows is done in every step, and only the choice left out)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = first + 16 * (i / 4) + i % 4;
                    const bool hidden = (key >= end) | ((i < 4 ? page0 : page1) < 0) | ((key <= below) & (key >= a.sinks));
                    x[i] = hidden ? -__builtin_inff() : x[i];
                }
            }
            if (SCORES && n < rows) {
                float *const at = scores.of(a, it.s.start * a.groups + it.row0 + n, head) + key0 + 4 * g;
#pragma unroll
                for (int t = 0; t < 2; ++t) *reinterpret_cast<float4 *>(at + 16 * t) = make_float4(x[4 * t] * factor[r], x[4 * t + 1] * factor[r], x[4 * t + 2] * factor[r], x[4 * t + 3] * factor[r]);
            }
            const float high = max_of_three(max_of_three(x[0], x[1], x[2]), max_of_three(x[3], x[4], x[5]), max_of_three(x[6], x[7], x[7])) * factor[r], to = max_of_three(top[r], high, high);
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += __builtin_amdgcn_exp2f(fmaf(x[i], factor[r], -to));
            total[r] = fmaf(total[r], __builtin_amdgcn_exp2f(top[r] - to), sum);
            top[r] = to;
        }
        codes[0] = next[0];
        codes[1] = next[1];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        join(top[r], total[r], __shfl_xor(top[r], 16), __shfl_xor(total[r], 16));
        join(top[r], total[r], __shfl_xor(top[r], 32), __shfl_xor(total[r], 32));
        if (g == 0) {
            bases[wave][16 * r + n] = top[r];
            totals[wave][16 * r + n] = total[r];
        }
    }
    __syncthreads();
    for (int r = threadIdx.x; r < rows; r += 64 * kWaves) {
        float to = bases[0][r], t = totals[0][r];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) join(to, t, bases[i][r], totals[i][r]);
        if (R > 1 && it.pieces == 1) {
            out.factors[((int64_t)(first_tile(a, it.s, it.b) + (it.row0 + r) / 16) * a.c.heads + head) * 16 + r % 16] = factor_of(to, t);
        } else {
            piece_rows(a, pieces, part, slot, head)[r] = make_float2(to, t);
        }
    }
}

// Joins the pieces of tiles of many rows whose keys were cut: a lane to a row
__global__ __launch_bounds__(64) void kv_statistics_join_kernel(KvAttentionArgs a, KvPart part, float *pieces, RowTiles out)
{
    const int slot = kv_divide(blockIdx.x, a.c.by_heads), head = blockIdx.x - slot * a.c.heads, r = threadIdx.x;
    const KvPieceNote note = *piece_note(a, pieces, part, slot, head);
    if (note.pieces == 0 || r >= note.rows) return;
    float to = kLowest, total = 0.0f;
#pragma unroll 4
    for (int i = 0; i < note.pieces; ++i) {
        const float2 p = piece_rows(a, pieces, part, slot + i, head)[r];
        join(to, total, p.x, p.y);
    }
    out.factors[((int64_t)(note.row0 + r / 16) * a.c.heads + head) * 16 + r % 16] = factor_of(to, total);  // (row0: a tile of all sequences' here)
}

// Sums of eight numbers over sixteen lanes: lane n has that of number n / 2
__device__ __forceinline__ float sums_of_eight(const float (&x)[8], int n)
{
    auto other = [](float v, auto ctrl) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    float y[4], z[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (n & 8 ? x[i + 4] : x[i]) + other(n & 8 ? x[i] : x[i + 4], std::integral_constant<int, 0x140>());  // sixteen mirrored
#pragma unroll
    for (int i = 0; i < 2; ++i) z[i] = (n & 4 ? y[i + 2] : y[i]) + other(n & 4 ? y[i] : y[i + 2], std::integral_constant<int, 0x141>());  // eight mirrored
    const float s = (n & 2 ? z[1] : z[0]) + other(n & 2 ? z[0] : z[1], std::integral_constant<int, 0x4e>());
    return s + other(s, std::integral_constant<int, 0xb1>());
}

// A second pass' piece of few rows' first one.  A sequence that has more than one tile of rows all the same has its keys shared out anew among the first tile's workgroups, which go through the tiles.
__device__ __forceinline__ bool few_item(const KvAttentionArgs &a, const KvPart &part, int slot, int head, const KvWeights &out, float decay, KvItem<kStep> &it, int &all_rows, int &tiles, int &first_slot, int &end,
                                         float *&weights)
{
    if (!kv_item<kStep, kFew>(a, part, slot, it)) return false;
    all_rows = it.s.n * a.groups;
    tiles = (all_rows + kFew - 1) / kFew;
    const int tile = it.row0 / kFew;
    first_slot = slot - it.part - (tiles - 1 - tile) * it.pieces;  // (the last tile comes first)
    if (tile) return false;
    if (tiles > 1) {
        const int steps = (it.s.keys + kStep - 1) / kStep;
        it.from = (int)((int64_t)steps * it.part / it.pieces);
        it.to = (int)((int64_t)steps * (it.part + 1) / it.pieces);
        it.sink_steps = it.gap = 0;
    }
    weights = out.data + it.b * out.sequence_stride + head * out.head_stride;
    end = (int)min((int64_t)it.s.keys, out.capacity);
    if (it.gap && decay != 1.0f) {  // keys that a window hides from every row
        const int from = (it.sink_steps + (int)((int64_t)it.gap * it.part / it.pieces)) * kStep, to = min((it.sink_steps + (int)((int64_t)it.gap * (it.part + 1) / it.pieces)) * kStep, end);
        for (int key = from + (int)threadIdx.x; key < to; key += 64 * kWaves) weights[key] = decay == 0.0f ? 0.0f : decay * weights[key];
    }
    return true;
}
// Row min(n, rows - 1) of a tile: its pieces' m and l, quarter g of them to a lane, joined
__device__ __forceinline__ RowFactor tile_row(const KvAttentionArgs &a, const KvPart &part, float *pieces, const KvItem<kStep> &it, int head, int tile, int tiles, int first_slot, int rows, int n, int g)
{
    float top = kLowest, total = 0.0f;
    // (there are slots for all pieces but where starts do not ascend: as in kv_note)
    const int from = first_slot + (tiles - 1 - tile) * it.pieces, there = min(it.pieces, part.slots - from);
#pragma unroll 4
    for (int i = g; i < there; i += 4) {
        const float2 p = piece_rows(a, pieces, part, from + i, head)[min(n, rows - 1)];
        join(top, total, p.x, p.y);
    }
    join(top, total, __shfl_xor(top, 16), __shfl_xor(total, 16));
    join(top, total, __shfl_xor(top, 32), __shfl_xor(total, 32));
    RowFactor f = factor_of(top, total);
    if (n >= rows) f.by = 0.0f;  // (the last row again)
    return f;
}

// Second pass of few rows whose scores the first one has kept: a lane has four keys, a wave eight steps at a time.
__global__ __launch_bounds__(64 * kWaves) void kv_weights_scored_kernel(KvAttentionArgs a, KvPart part, float *pieces, RowScores scores, KvWeights out, float decay)
{
    __shared__ RowFactor factors[kFew];
    __shared__ int positions[kFew];
    const int slot = kv_divide(blockIdx.x, a.c.by_heads), head = blockIdx.x - slot * a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4;
    KvItem<kStep> it;
    int all_rows, tiles, first_slot, end;
    float *weights;
    if (!few_item(a, part, slot, head, out, decay, it, all_rows, tiles, first_slot, end, weights)) return;
    for (int tile = 0; tile < tiles; ++tile) {
        const int rows = min(all_rows - tile * kFew, kFew);
        __syncthreads();
        if (wave == 0) {
            const RowFactor f = tile_row(a, part, pieces, it, head, tile, tiles, first_slot, rows, n, g);
            if (g == 0) {
                factors[n] = f;
                positions[n] = it.s.first + kv_divide(tile * kFew + min(n, rows - 1), a.by_groups);
            }
        }
        __syncthreads();
        for (int v = it.from + 8 * wave + (lane >> 3); v < it.to; v += 8 * kWaves) {
            const int key = it.key_of(v) + 4 * (lane & 7);
            float p[4] = {}, before[4] = {};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((tile || decay != 0.0f) && key + i < end) before[i] = weights[key + i];
#pragma unroll 4
            for (int r = 0; r < rows; ++r) {
                const float4 x = *reinterpret_cast<const float4 *>(scores.of(a, it.s.start * a.groups + tile * kFew + r, head) + key);
                const RowFactor f = factors[r];
                const int pos = positions[r], below = a.window ? pos - a.window : INT32_MIN;
                const float s[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(s[i] + f.base) * f.by;
                    p[i] += (key + i > pos) | ((key + i <= below) & (key + i >= a.sinks)) ? 0.0f : w;  // (what the row's tile did not visit was not written)
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (key + i < end) weights[key + i] = tile ? before[i] + p[i] : decay == 0.0f ? p[i] : fmaf(decay, before[i], p[i]);
        }
    }
}

// Second pass of few rows, on the first one's pieces, which makes the scores again.
template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves, 3) void kv_weights_few_kernel(KvAttentionArgs a, KvPart part, float *pieces, KvWeights out, float decay)
{
    constexpr int W = D / 32;
    const int slot = kv_divide(blockIdx.x, a.c.by_heads), head = blockIdx.x - slot * a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4;
    KvItem<kStep> it;
    int all_rows, tiles, first_slot, end;
    float *weights;
    if (!few_item(a, part, slot, head, out, decay, it, all_rows, tiles, first_slot, end, weights)) return;
    int v = it.from + wave, ids = kv_page_ids(a, it, v, kWaves), id = 0;
    if (v >= it.to) return;
    KeyCodes<D> codes[2], next[2];
    const int column = 16 * (n >> 3) + 4 * g + (n >> 1 & 3);  // of a step's keys, whose sum this lane gets
    float before = 0.0f, next_before = 0.0f;
    auto load = [&](int key, int page0, int page1, KeyCodes<D> (&to)[2], float &w) {
        load_keys<D>(a, head, key, page0, to[0]);
        load_keys<D>(a, head, key + 16, page1, to[1]);
        w = decay != 0.0f ? weights[min(key + column, end - 1)] : 0.0f;
    };
    if (end <= 0) return;
    load(it.key_of(v), __builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1), codes, before);
    half8 q[W];
    RowFactor f;
    float factor;
    int pos, rows, first_pos, last_pos;
    auto take = [&](int tile) {
        rows = min(all_rows - tile * kFew, kFew);
        const int row = tile * kFew + min(n, rows - 1);
        take_rows<D, BF16>(a, it.s.start, head, row, q, factor);
        f = tile_row(a, part, pieces, it, head, tile, tiles, first_slot, rows, n, g);
        pos = n < rows ? it.s.first + kv_divide(row, a.by_groups) : INT32_MIN;
        first_pos = it.s.first + kv_divide(tile * kFew, a.by_groups);
        last_pos = it.s.first + kv_divide(tile * kFew + rows - 1, a.by_groups);
    };
    take(0);
    for (; v < it.to; v += kWaves) {
        const int key0 = it.key_of(v), page0 = __builtin_amdgcn_readlane(ids, id), page1 = __builtin_amdgcn_readlane(ids, id + 1);
        id += 2;
        if (id == 64) {
            ids = kv_page_ids(a, it, v + kWaves, kWaves);
            id = 0;
        }
        {
            const bool more = v + kWaves < it.to;
            load(more ? it.key_of(v + kWaves) : key0, more ? __builtin_amdgcn_readlane(ids, id) : page0, more ? __builtin_amdgcn_readlane(ids, id + 1) : page1, next, next_before);
        }
        Keys<D> keys[2];
        make_keys<D, BF16>(codes[0], keys[0]);
        make_keys<D, BF16>(codes[1], keys[1]);
        float p[8] = {};
        for (int tile = 0; tile < tiles; ++tile) {
            if (tiles > 1) take(tile);
            const bool all = key0 + kStep <= it.s.keys && key0 + kStep - 1 <= first_pos && page0 >= 0 && page1 >= 0 && (!a.window || key0 > last_pos - a.window || key0 + kStep <= a.sinks);
            float x[8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float4v s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < W; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys[t].k[i], q[i], s, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[4 * t + i] = __builtin_amdgcn_exp2f(fmaf(s[i] * keys[t].s[i], factor, f.base)) * f.by;
            }
            if (!all) {
                int first = key0 + 4 * g, below = a.window ? pos - a.window : INT32_MIN, to_key = min(pos + 1, it.s.keys);
                asm volatile("" : "+v"(first));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int key = first + 16 * (i / 4) + i % 4;
                    const bool hidden = (key >= to_key) | ((i < 4 ? page0 : page1) < 0) | ((key <= below) & (key >= a.sinks));
                    x[i] = hidden ? 0.0f : x[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] += x[i];
        }
        const float sum = sums_of_eight(p, n);
        if (!(n & 1) && key0 + column < end) weights[key0 + column] = decay == 0.0f ? sum : fmaf(decay, before, sum);
        codes[0] = next[0];
        codes[1] = next[1];
        before = next_before;
    }
}

// Second pass of many rows.  A workgroup takes 64 KT keys of a head at a time, 16 KT to a wave, and goes through the rows that may see them: each of its waves makes operands of 16 rows, which all read from
// LDS, the next ones on their way from memory meanwhile.
template <int D, bool BF16, int KT>
__global__ __launch_bounds__(64 * kWaves, 2) void kv_weights_many_kernel(KvAttentionArgs a, KvWeights out, float decay, RowTiles in, int from_rows)
{
    constexpr int W = D / 32, kBlock = 16 * KT * kWaves;
    __shared__ __align__(16) half8 rows_q[2][kChunk][W][64];
    __shared__ float4v rows_f[2][kChunk][16];  // factor, base, by, position
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4, units = gridDim.x / a.c.heads;
    const int own = kv_divide(blockIdx.x, a.c.by_heads), head = blockIdx.x - own * a.c.heads;
    for (int round = 0;; ++round) {
        // one round in order, the next in reverse: the blocks of a sequence have fewer rows one by one, so that a first and a last one take as long as two from the middle
        const int unit = round & 1 ? (round + 1) * units - 1 - own : round * units + own;
        int b, rest;
        auto count = [&](int at) {
            const KvSequence s = kv_sequence(a.c, at);
            return s.n * a.groups >= from_rows ? (s.keys + kBlock - 1) / kBlock : 0;  // (fewer than 2^31 in all: kv_weights_blocks)
        };
        if (!kv_find(a.c.sequences, unit, b, rest, count)) return;
        const KvSequence s = kv_sequence(a.c, b);
        const int block0 = rest * kBlock, key0 = block0 + wave * 16 * KT;
        KeyCodes<D> codes[KT];
        uint32_t missing = 0;  // tiles of keys without a page
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const int key = key0 + 16 * t;
            int page = key < s.keys ? a.c.table[b * a.c.table_stride + (key >> a.c.page_shift)] : -1;
            if (page >= a.c.pages) page = -1;
            missing |= page < 0 ? 1u << t : 0u;
            load_keys<D>(a, head, key, page, codes[t]);
        }
        // rows whose position is that of the block's first key or later, and under a window those that see its last key or have it among the first ones
        const int rows = s.n * a.groups, first_token = max(block0 - s.first, 0);
        int last_token = s.n;  // (behind the last)
        if (a.window && block0 >= a.sinks) last_token = (int)min((int64_t)s.n, max((int64_t)block0 + kBlock - 1 + a.window - s.first, (int64_t)0));
        const int row_end = min(last_token * a.groups, rows);
        // sums of kFold chunks' rows, and of these: of 8192 tiles one after the other the sum would be off by 2^-25 of itself 52 times, as a rule (8192 / 3 roundings' root), in two steps by 10
        float sums[KT][4], whole[KT][4];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[t][i] = whole[t][i] = 0.0f;
        auto fold = [&] {
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    whole[t][i] += sums[t][i];
                    sums[t][i] = 0.0f;
                }
        };
        Keys<D> keys[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) make_keys<D, BF16>(codes[t], keys[t]);
        const int tile0 = first_tile(a, s, b);
        half8 q[W] = {};
        RowFactor factor = {};
        float scale = 0.0f;
        auto bring = [&](int row0) {  // this wave's sixteen of the rows from row0 on (or the last ones again)
            const int64_t tile = (int64_t)(tile0 + min(row0 / 16 + wave, (rows - 1) / 16)) * a.c.heads + head;
#pragma unroll
            for (int i = 0; i < W; ++i) q[i] = reinterpret_cast<const half8 *>(in.operands)[(tile * W + i) * 64 + lane];
            factor = in.factors[tile * 16 + n];
            scale = in.scales[tile * 16 + n];
        };
        int row0 = first_token * a.groups / 16 * 16, place = 0, chunks = 0;
        if (row0 < row_end) bring(row0);
        __syncthreads();  // (of the unit before nothing is read from LDS any more)
        for (; row0 < row_end; row0 += 16 * kChunk, place ^= 1) {
#pragma unroll
            for (int i = 0; i < W; ++i) rows_q[place][wave][i][lane] = q[i];
            const int row = row0 + 16 * wave + n;  // (from `rows` on the last row again, without weight: its factors were not written)
            if (g == 0)
                rows_f[place][wave][n] = row < rows ? float4v{scale, factor.base, factor.by, __uint_as_float((uint32_t)(s.first + kv_divide(row, a.by_groups)))} :
                                                      float4v{0.0f, 0.0f, 0.0f, __uint_as_float((uint32_t)INT32_MIN)};
            __syncthreads();
            if (++chunks % kFold == 0) fold();
            if (row0 + 16 * kChunk < row_end) bring(row0 + 16 * kChunk);
            const int tiles = min((row_end - row0 + 15) / 16, kChunk);
            for (int tile = 0; tile < tiles; ++tile) {
                half8 x[W];
#pragma unroll
                for (int i = 0; i < W; ++i) x[i] = rows_q[place][tile][i][lane];
                const float4v r = rows_f[place][tile][n];
                const int pos = (int)__float_as_uint(r[3]), first_row = row0 + 16 * tile, from = s.first + kv_divide(first_row, a.by_groups), to = s.first + kv_divide(min(first_row + 15, rows - 1), a.by_groups);
                const bool all = key0 + 16 * KT <= s.keys && key0 + 16 * KT - 1 <= from && !missing && (!a.window || key0 > to - a.window || key0 + 16 * KT <= a.sinks);
                float4v y[KT];
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    y[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < W; ++i) y[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys[t].k[i], x[i], y[t], 0, 0, 0);
                }
                if (all) {
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sums[t][i] = fmaf(__builtin_amdgcn_exp2f(fmaf(y[t][i] * keys[t].s[i], r[0], r[1])), r[2], sums[t][i]);
                } else {
                    int first = key0 + 4 * g, below = a.window ? pos - a.window : INT32_MIN, to_key = min(pos + 1, s.keys);  // (a row that there is not: pos + 1 is less than any key)
                    asm volatile("" : "+v"(first));
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int k = first + 16 * t + i;
                            const bool hidden = (k >= to_key) | ((missing >> t & 1) != 0) | ((k <= below) & (k >= a.sinks));
                            const float p = __builtin_amdgcn_exp2f(fmaf(y[t][i] * keys[t].s[i], r[0], r[1])) * r[2];
                            sums[t][i] += hidden ? 0.0f : p;
                        }
                }
            }
        }
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = whole[t][i] + sums[t][i];
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
    float *few = a.partial, *many = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(a.partial) + p.few_bytes + p.score_bytes);
    RowTiles tiles;
    tiles.operands = reinterpret_cast<uint8_t *>(many) + p.many_bytes;
    tiles.factors = reinterpret_cast<RowFactor *>(tiles.operands + p.row_tiles * a.c.heads * (D / 32) * 1024);
    tiles.scales = reinterpret_cast<float *>(tiles.factors + p.row_tiles * a.c.heads * 16);
    const dim3 block(64 * kWaves);
    if (p.few.tile) {
        const dim3 groups((uint32_t)((int64_t)p.few.slots * a.c.heads));
        if (p.score_bytes) {
            const RowScores scores = {reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(few) + p.few_bytes), p.score_stride};
            kv_statistics_kernel<D, BF16, 1, true><<<groups, block, 0, stream>>>(a, p.few, few, RowTiles{}, scores);
            kv_weights_scored_kernel<<<groups, block, 0, stream>>>(a, p.few, few, scores, w, decay);
        } else {
            kv_statistics_kernel<D, BF16, 1, false><<<groups, block, 0, stream>>>(a, p.few, few, RowTiles{}, RowScores{});
            kv_weights_few_kernel<D, BF16><<<groups, block, 0, stream>>>(a, p.few, few, w, decay);
        }
    }
    if (p.many.tile) {
        const dim3 groups((uint32_t)((int64_t)p.many.slots * a.c.heads)), units((uint32_t)(p.units * a.c.heads));
        kv_statistics_kernel<D, BF16, 4, false><<<groups, block, 0, stream>>>(a, p.many, many, tiles, RowScores{});
        if (p.many.target) kv_statistics_join_kernel<<<groups, dim3(64), 0, stream>>>(a, p.many, many, tiles);
        if (p.key_tiles == 2) kv_weights_many_kernel<D, BF16, 2><<<units, block, 0, stream>>>(a, w, decay, tiles, p.many.from_rows);
        else if (p.key_tiles == 4) kv_weights_many_kernel<D, BF16, 4><<<units, block, 0, stream>>>(a, w, decay, tiles, p.many.from_rows);
        else kv_weights_many_kernel<D, BF16, 1><<<units, block, 0, stream>>>(a, w, decay, tiles, p.many.from_rows);
    }
}

int64_t blocks_of(const KvArgs &c, int keys) { return (std::min<int64_t>((int64_t)c.width << c.page_shift, kKvMost) + keys - 1) / keys * c.sequences; }

void cut(KvPart &p, const KvArgs &c, int groups, int window, int sinks, int64_t tiles, int wanted, int plenty)
{
    int64_t most_steps = (((int64_t)c.width << c.page_shift) + kStep - 1) / kStep;  // of a sequence, as far as the page table goes
    if (window) most_steps = std::min<int64_t>(most_steps, kv_window_steps(window, sinks, (p.tile + groups - 2) / groups, kStep));
    p.target = tiles * c.heads >= plenty || most_steps <= p.least ? 0 : std::max(wanted / c.heads, 1);
    p.slots = (int)(tiles + (p.target ? p.target + 1 : 0));
}

}  // namespace

// Blocks of keys that the second pass of many rows may have, the smaller ones
int64_t kv_weights_blocks(const KvArgs &c) { return blocks_of(c, 16 * kWaves); }

KvWeightsPlan kv_weights_plan(const KvArgs &c, int groups, int window, int sinks)
{
    KvWeightsPlan p = {};
    const int64_t rows = (int64_t)c.tokens * groups, sequences = std::min(c.sequences, c.tokens);
    // A sequence's rows are as many as the call's where it is the only one, and `groups` where it is said that each has one token.  No more tokens than sequences: one of each as a rule.
    const bool few = rows <= kFew || (c.tokens <= c.sequences && groups <= kFew), many = !few && (c.sequences == 1 || !c.starts);
    if (!many) {
        p.few.tile = kFew;
        p.few.to_rows = few ? INT32_MAX : kFew;
        p.few.least = 32;
        cut(p.few, c, groups, window, sinks, few ? std::min(c.tokens * (int64_t)((groups + kFew - 1) / kFew), rows / kFew + sequences) : sequences, 1024, 4096);  // (8 sequences of up to 32768 tokens: 78 us; 512 pieces 87, 1536 and 2048 85)
        p.few_bytes = (size_t)p.few.slots * c.heads * kFew * sizeof(float2);
        p.score_stride = blocks_of(c, kStep) / c.sequences * kStep;
        if (few && rows * c.heads * p.score_stride <= kMostScores) p.score_bytes = (size_t)(rows * c.heads * p.score_stride) * sizeof(float);
    }
    if (!few) {
        p.many.tile = 64;
        p.many.from_rows = many ? 1 : kFew + 1;
        p.many.to_rows = INT32_MAX;
        p.many.least = 32;
        cut(p.many, c, groups, window, sinks, std::min(c.tokens * (int64_t)((groups + 63) / 64), rows / 64 + sequences), 1024, 1024);
        if (p.many.target) p.many_bytes = (size_t)p.many.slots * c.heads * (64 * sizeof(float2) + sizeof(KvPieceNote));
        p.row_tiles = rows / 16 + c.sequences + 1;
        p.rows_bytes = (size_t)p.row_tiles * c.heads * (c.head_dim / 32 * 1024 + 16 * (sizeof(RowFactor) + sizeof(float)));
        p.key_tiles = blocks_of(c, 64 * kWaves) * c.heads >= 1024 ? 4 : blocks_of(c, 32 * kWaves) * c.heads >= 512 ? 2 : 1;
        p.units = std::max<int64_t>(1, std::min<int64_t>(blocks_of(c, 16 * p.key_tiles * kWaves), std::max(1, (p.key_tiles == 4 ? 512 : 1024) / c.heads)));
    }
    return p;
}

size_t kv_weights_bytes(const KvWeightsPlan &p) { return p.few_bytes + p.score_bytes + p.many_bytes + p.rows_bytes; }
int64_t kv_weights_items(const KvWeightsPlan &p, int heads) { return std::max(std::max((int64_t)p.few.slots, (int64_t)p.many.slots), p.units) * heads * 64 * kWaves; }

hipError_t launch_kv_weights(const KvAttentionArgs &a, const KvWeights &w, float decay, const KvWeightsPlan &p, hipStream_t stream)
{
    if (a.c.head_dim == 128) a.c.bf16 ? launch<128, true>(a, w, decay, p, stream) : launch<128, false>(a, w, decay, p, stream);
    else a.c.bf16 ? launch<64, true>(a, w, decay, p, stream) : launch<64, false>(a, w, decay, p, stream);
    return hipGetLastError();
}

}  // namespace apmm
