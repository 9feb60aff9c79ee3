// Attention over the four-bit key/value cache (layout: apmm_kv.h): what its kernels share.
//
// For a query q of a row and keys j that it sees, with key codes u, value codes w, scales a, b of a token and c = scale log2(e):
//   x_j = c a_j sum_d q_d (2 u_jd - 15)        p_j = 2^(x_j - m)        o_d = sum_j p_j b_j (2 w_jd - 15) / sum_j p_j
// Both sums over products are matrix instructions on binary16 operands with 32-bit accumulators.
//
//   Codes as operands   A code in the low mantissa bits of a binary16 number is the subnormal u 2^-24 (bits 0 to 3) or u 2^-20 (bits 4 to 7), which the matrix unit takes exactly:
//                       five operations make four operand words of one word of eight codes.  The -15 is added outside: -15 sum_d q_d is where the accumulators of the first product start
//                       from, and 15 times the sum of the weights is taken off the second one's result.
//   Queries             times a power of two for each row, so that its largest number is just below 2^11 (2^15 for the channels that meet u 2^-24).  Numbers below 2^-27 of the row's largest may
//                       lose bits, 2^-35 of it at most (bfloat16, and binary16 rows beyond 2^11; other binary16 rows lose none); where the 32 rows of a wave share the power of the largest
//                       one, rows down to 2^-10 of that, below 2^-17 of the row's largest and 2^-25 of it at most.
//   Weights             p_j b_j, rounded once to binary16 (bfloat16 would cost an output of binary16 numbers eight times its own rounding; kv_attention_rows, which waits for memory, adds what
//                       the rounding left as a second number for them).  The value scales may lie anywhere, so each row holds a power of two 2^E above all that it has met, and weights carry the
//                       factor 2^(2 - E) until the end (in p as far as it has the range, kv_rest): at most 2^15, full precision down to 2^-16 of that for p = 1 and b = 2^E, and 2^-27 of it is the least that counts.
//                       The sum of the rounded weights goes with them (dot products with ones).
//   Running maximum     m (and E) are only moved where a score passes m + 13: until then weights are at most 2^13 times larger, for which there is room.  Then the accumulators are scaled;
//                       -m + 2 - E is one number, `base`.  So large a slack is what lets kv_attention_tiles go without a maximum in most steps.
//   Products transposed S^T = K Q^T and O^T = V^T P^T: the rows of S^T in a lane's accumulators are eight (or sixteen) keys that follow each other, if key rows are dealt to the operand's
//                       rows in that order, and those are the lane's part of the operand P^T of the second product.  No weight passes through LDS.
// A row that sees no key has the weight sum 0 and gets zeros.
#pragma once

#include "apmm_kv.h"

namespace apmm {

constexpr int kRowsTile = 16;    // rows of a workgroup of kv_attention_rows_kernel
constexpr int kTilesTile = 64;   // and of half a workgroup of kv_attention_tiles_kernel

constexpr int kRowsStep = 32;    // keys of one step
constexpr int kTilesStep = 32;

// Workgroups of kv_attention_tiles_kernel for tiles
inline int64_t kv_tiles_groups(const KvPart &part, int heads) { return (int64_t)((part.slots + 1) / 2) * heads; }

hipError_t launch_kv_attention_rows(const KvAttentionArgs &a, const KvPart &part, hipStream_t stream);
hipError_t launch_kv_attention_tiles(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream);

// Most steps of a tile under a window, whose queries are at most `later` positions behind the first one's
__host__ __device__ inline int kv_window_steps(int window, int sinks, int later, int step) { return (int)(((int64_t)window + later + step - 1) / step) + 1 + (sinks + step - 1) / step; }

#ifdef __HIPCC__
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float kLowest = -3.402823466e38f;
constexpr float kSlack = 13.0f, kRoom = 2.0f;  // 2^(kSlack + kRoom) is what binary16 has room for, but for the last octave

// A workgroup's part of the call: keys of steps `from` to `to` - 1 (of STEP keys, the hidden ones between the first tokens and the window left out) for rows of one sequence
template <int STEP>
struct KvItem {
    KvSequence s;
    int b, row0, rows;   // first row, rows that there are from there on (may be more than a tile)
    int from, to;
    int sink_steps, gap; // step v lies at v < sink_steps ? v : v + gap
    int pieces, part;    // of the tile; which this is
    __device__ __forceinline__ int key_of(int v) const { return (v < sink_steps ? v : v + gap) * STEP; }
};

// Tiles of a sequence, and steps of the one with most (or a few more)
template <int STEP, int TILE>
__device__ __forceinline__ void kv_extent(const KvAttentionArgs &a, const KvSequence &s, const KvPart &p, int &tiles, int &steps)
{
    const int rows = s.n * a.groups;
    tiles = rows >= p.from_rows && rows <= p.to_rows ? (rows + TILE - 1) / TILE : 0;
    steps = (s.keys + STEP - 1) / STEP;
    if (a.window) steps = min(steps, kv_window_steps(a.window, a.sinks, kv_divide(TILE + a.groups - 2, a.by_groups), STEP));
    if (!tiles) steps = 0;
}

__device__ __forceinline__ int kv_pieces(int steps, int piece)
{
    if (steps <= piece) return 1;
    const int n = (int)((float)steps / (float)piece);  // steps < 2^25; within one of the quotient
    return n * (int64_t)piece >= steps ? ((n - 1) * (int64_t)piece >= steps ? n - 1 : n) : ((n + 1) * (int64_t)piece >= steps ? n + 1 : n + 2);
}

// Piece `slot` of the call; false: there is none
template <int STEP, int TILE>
__device__ __forceinline__ bool kv_item(const KvAttentionArgs &a, const KvPart &p, int slot, KvItem<STEP> &it)
{
    const int lane = kv_lane();
    int piece = 0x7fffffff, tiles, steps;
    KvSequence s = {};
    if (lane < a.c.sequences) s = kv_sequence(a.c, lane);  // the first 64 stay in registers
    kv_extent<STEP, TILE>(a, s, p, tiles, steps);
    if (p.target) {
        float work = (float)tiles * (float)steps, all = (float)tiles;
        for (int at = lane + 64; at < a.c.sequences; at += 64) {
            int t, n;
            kv_extent<STEP, TILE>(a, kv_sequence(a.c, at), p, t, n);
            work += (float)t * (float)n;
            all += (float)t;
        }
        auto sum = [](float v) {
#pragma unroll
            for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
            return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));  // (and what follows from it is the same for the wave)
        };
        work = sum(work);
        all = sum(all);
        // A tile's last piece is half a piece too many on average: so much less than `target` is asked for, and, where the pieces are more than that nevertheless, a whole one
        // (rounding: a piece may be 2^-20 shorter than the work asks for, for which there is one slot more)
        auto length = [&](float pieces) { return __builtin_amdgcn_readfirstlane(max((int)ceilf(fminf(work / pieces * (1.0f - 0x1p-20f), 0x1p30f)), p.least)); };
        const float target = (float)p.target;
        piece = length(fmaxf(target - 0.5f * all, 0.5f * target));
        if (a.c.sequences <= 64 && all < target && sum((float)(tiles * kv_pieces(steps, piece))) > target) piece = length(target - all);
    }
    int rest, l;
    const int pieces = kv_pieces(steps, piece), own = tiles * pieces, to = kv_scan(own);
    const uint64_t past = __ballot(to > slot);
    if (past) {
        l = __ffsll((long long)past) - 1;
        it.b = l;
        rest = slot - (__builtin_amdgcn_readlane(to, l) - __builtin_amdgcn_readlane(own, l));
        it.s.start = __builtin_amdgcn_readlane(s.start, l);
        it.s.n = __builtin_amdgcn_readlane(s.n, l);
        it.s.first = __builtin_amdgcn_readlane(s.first, l);
        it.s.keys = __builtin_amdgcn_readlane(s.keys, l);
        it.pieces = __builtin_amdgcn_readlane(pieces, l);
        tiles = __builtin_amdgcn_readlane(tiles, l);
    } else {
        const int before = __builtin_amdgcn_readlane(to, 63);
        auto count = [&](int at) {
            int t, n;
            if (at + 64 >= a.c.sequences) return 0;
            kv_extent<STEP, TILE>(a, kv_sequence(a.c, at + 64), p, t, n);
            return t * kv_pieces(n, piece);
        };
        if (a.c.sequences <= 64 || !kv_find(a.c.sequences - 64, slot - before, it.b, rest, count)) return false;
        it.b += 64;
        it.s = kv_sequence(a.c, it.b);
        kv_extent<STEP, TILE>(a, it.s, p, tiles, steps);
        it.pieces = kv_pieces(steps, piece);
    }
    int tile = rest;
    it.part = 0;
    if (it.pieces > 1) {
        tile = rest / it.pieces;
        it.part = rest % it.pieces;
    }
    if (tile >= p.turn && tile < 2 * p.turn) tile = p.turn + min(2 * p.turn, tiles) - 1 - tile;
    tile = tiles - 1 - tile;  // (the last queries see the most keys: those first)
    it.row0 = tile * TILE;
    it.rows = it.s.n * a.groups - it.row0;
    const int last = min(it.rows, TILE) - 1, first_pos = it.s.first + kv_divide(it.row0, a.by_groups), last_pos = it.s.first + kv_divide(it.row0 + last, a.by_groups);
    const int end = min(last_pos + 1, it.s.keys), all = end > 0 ? (end + STEP - 1) / STEP : 0;
    const int low = min(a.window ? max(first_pos - a.window + 1, 0) / STEP : 0, all);
    it.sink_steps = min((a.sinks + STEP - 1) / STEP, low);
    it.gap = low - it.sink_steps;
    it.from = 0;
    it.to = all - it.gap;
    if (it.pieces > 1) {
        const int even = max(kv_pieces(it.to, it.pieces), min(piece, p.least));
        it.from = min(it.part * (int64_t)even, (int64_t)it.to);
        it.to = min((it.part + 1) * (int64_t)even, (int64_t)it.to);
    }
    return true;
}

// For the joining of pieces: what lies at a slot and head
struct KvPieceNote {
    int start, row0, rows, pieces;  // pieces: of the tile, no more than there are slots from this one on; 0 where this is not the first of several
};
struct KvPartial {
    float *sums;        // [slot][head][tile row][channel]
    float2 *row;        // [slot][head][tile row]: base and total; the row is sum_i 2^base_i sums_i / sum_i 2^base_i total_i over its pieces
    KvPieceNote *note;  // [slot][head]
};
__host__ __device__ inline KvPartial kv_partial(float *at, const KvPart &part, int heads, int head_dim)
{
    const int64_t rows = (int64_t)part.slots * heads * part.tile;
    KvPartial p;
    p.sums = at;
    p.row = reinterpret_cast<float2 *>(at + rows * head_dim);
    p.note = reinterpret_cast<KvPieceNote *>(p.row + rows);
    return p;
}
template <int STEP>
__device__ __forceinline__ void kv_note(const KvAttentionArgs &a, const KvPart &p, float *partials, int slot, int head, bool there, const KvItem<STEP> &it, bool first)
{
    if (!p.target || !first) return;
    KvPieceNote n = {};
    // (there are slots for all pieces but where starts do not ascend: sequences that share rows may then have more tiles than the host counted)
    if (there && it.part == 0 && it.pieces > 1) n = {it.s.start, it.row0, min(it.rows, p.tile), min(it.pieces, p.slots - slot)};
    kv_partial(partials, p, a.c.heads, a.c.head_dim).note[(int64_t)slot * a.c.heads + head] = n;
}

// Four words of a matrix operand from one word of codes: nibbles 0 and 4, 1 and 5, 2 and 6, 3 and 7, those of even number as u 2^-24, of odd number as u 2^-20
__device__ __forceinline__ half8 kv_operand(uint32_t w)
{
    const uint32_t h = w >> 8;
    uint4 r;
    r.x = w & 0x000f000fu;
    r.y = w & 0x00f000f0u;
    r.z = h & 0x000f000fu;
    r.w = h & 0x00f000f0u;
    return __builtin_bit_cast(half8, r);
}

__device__ __forceinline__ uint32_t kv_half_pair(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{a, b}), half2v));
}

template <bool BF16>
__device__ __forceinline__ float kv_low(uint32_t w) { return BF16 ? __uint_as_float(w << 16) : (float)__builtin_bit_cast(half2v, w)[0]; }
template <bool BF16>
__device__ __forceinline__ float kv_high(uint32_t w) { return BF16 ? __uint_as_float(w & 0xffff0000u) : (float)__builtin_bit_cast(half2v, w)[1]; }

// The larger of m and a magnitude's bits, if that is finite
template <bool BF16>
__device__ __forceinline__ uint32_t kv_finite_max(uint32_t m, uint32_t bits)
{
    return bits < (BF16 ? 0x7f80u : 0x7c00u) ? max(m, bits) : m;
}
// The queries of a lane as operand words: x holds 8 channels to 4 words in their order.  max_across and sum_across fold a value over the lanes that share the row.
template <int N, bool BF16, class Max, class Sum>
__device__ __forceinline__ void kv_queries(const uint32_t (&x)[N], float scale, Max max_across, Sum sum_across, half8 (&q)[N / 4], float &init, float &factor)
{
    uint32_t bits2 = 0, bits;  // of the largest magnitude
#pragma unroll
    for (int i = 0; i < N; ++i) bits2 = kv_fold_max(bits2, x[i] & 0x7fff7fffu);
    bits = max(bits2 & 0xffffu, bits2 >> 16);
    if (bits >= (BF16 ? 0x7f80u : 0x7c00u)) {  // not finite: of those that are
        bits = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) bits = kv_finite_max<BF16>(kv_finite_max<BF16>(bits, x[i] & 0x7fffu), (x[i] >> 16) & 0x7fffu);
    }
    const float top = max_across(kv_scale_value(bits, BF16));
    int e = top > 0.0f ? 11 - (int)((__float_as_uint(top) >> 23) - 126u) : 0;  // top 2^e < 2^11
    e = min(e, BF16 ? 100 : 26);                                             // (rows of the smallest numbers)
    float sum = 0.0f;
    // binary16 numbers are multiplied as they are, by 2^e or 2^(e + 4) in two steps where one factor has no room for it; channels j and j + 4 make a word
    const float first = BF16 ? 1.0f : ldexpf(1.0f, min(e, 11)), second = BF16 ? 1.0f : ldexpf(1.0f, e - min(e, 11));
    const half2v by0 = {(_Float16)first, (_Float16)first}, by1 = {(_Float16)second, (_Float16)second}, by16 = {(_Float16)16.0f, (_Float16)16.0f};
    const float even = ldexpf(1.0f, e + 4), odd = ldexpf(1.0f, e);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        __builtin_amdgcn_sched_barrier(0);  // a few registers at a time
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t a = x[4 * i + j / 2], b = x[4 * i + j / 2 + 2];
            half2v pair;
            if (BF16) {
                const float by = j & 1 ? odd : even;
                pair = __builtin_bit_cast(half2v, kv_half_pair((j & 1 ? kv_high<true>(a) : kv_low<true>(a)) * by, (j & 1 ? kv_high<true>(b) : kv_low<true>(b)) * by));
            } else {
                pair = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(b, a, j & 1 ? 0x07060302u : 0x05040100u)) * by0 * by1;
                if (!(j & 1)) pair *= by16;
            }
            w[j] = __builtin_bit_cast(uint32_t, pair);
            sum = __builtin_amdgcn_fdot2(pair, j & 1 ? half2v{(_Float16)1.0f, (_Float16)1.0f} : half2v{(_Float16)0.0625f, (_Float16)0.0625f}, sum, false);
        }
        q[i] = __builtin_bit_cast(half8, make_uint4(w[0], w[1], w[2], w[3]));
    }
    __builtin_amdgcn_sched_barrier(0);
    init = -7.5f * 0x1p-20f * sum_across(sum);
    // (queries of 2^115 and more: scores beyond any other's all the same.  Neither zero nor infinite: scores of hidden keys are -infinity, those of queries that are zero are zero)
    factor = fminf(fmaxf(ldexpf(scale * 1.44269504088896341f, min(21 - e, 122)), 0x1p-149f), -kLowest);
}

// Pages of 16 keys each: lane i of the result has that of the i-th sixteen of the next steps of a wave (v, v + stride, ...), -1 where there is none
template <int STEP>
__device__ __forceinline__ int kv_page_ids(const KvAttentionArgs &a, const KvItem<STEP> &it, int v, int stride)
{
    const int step = v + kv_lane() / (STEP / 16) * stride;
    if (step >= it.to) return -1;
    const int key = it.key_of(step) + 16 * (kv_lane() % (STEP / 16));
    if (key >= it.s.keys) return -1;
    const int page = a.c.table[it.b * a.c.table_stride + (key >> a.c.page_shift)];
    return page < a.c.pages ? page : -1;
}

// E of a largest scale: s < 2^E.  Held above -80, so that sums of 2^(2 - E) stay in range (scales below 2^-96 lose bits).  Of an E above kMostExponent the rest goes into the value scales
// (kv_rest, a power of two of the row), or weights would be subnormal numbers, which the exponent's instruction does not make.
constexpr int kMostExponent = 64;
__device__ __forceinline__ int kv_rest(int e) { return max(e - kMostExponent, 0); }
// total 2^x + plus for x <= 0.  With bfloat16 scales also where 2^x alone has no room: sums of weights begin between 2^(2 - kMostExponent) and 2^82, and those of a row's tiny values count like
// those of its largest (sums of weights times values that far below the others' do not).
template <bool BF16>
__device__ __forceinline__ float kv_moved(float total, float x, float plus = 0.0f)
{
    if (!BF16) return fmaf(total, __builtin_amdgcn_exp2f(x), plus);
    return fmaf(total * __builtin_amdgcn_exp2f(fminf(x + 100.0f, 0.0f)), __builtin_amdgcn_exp2f(fmaxf(x, -100.0f)), plus);
}
template <bool BF16>
__device__ __forceinline__ int kv_exponent(uint32_t bits) { return BF16 ? max((int)(bits >> 7) - 126, -80) : (int)(bits >> 10) - 14; }
template <bool BF16>
__device__ __forceinline__ uint32_t kv_limit(uint32_t bits) { return bits | (BF16 ? 0x7fu : 0x3ffu); }
#endif

}  // namespace apmm
