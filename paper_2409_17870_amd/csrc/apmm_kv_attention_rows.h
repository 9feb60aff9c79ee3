// Attention of few rows over the four-bit cache (apmm_kv_attention.h): token generation.
//
// A workgroup has 16 rows (the query heads of a key/value head times its new tokens; fewer are there in most calls) and a piece of the keys, its waves take steps of 32 keys
// in turn, each with its own maximum and sums, and meet in LDS at the end.  Matrix instructions 16 x 16 x 32: two for each 32 channels and 16 keys, one for each 16 channels of the result.
// Row i of the key operand is key i of 16, so that a lane's scores are those of keys 4 g to 4 g + 3 of both halves of a step (g = lane / 16).  Each half lies in one page: all loads are a base
// that is the same for the wave plus the lane's offset, which does not change.  A step's loads leave one step ahead (two ahead changed nothing).
//
// Bound by HBM where there is enough to read: 8 sequences of 65536 tokens, 8 key/value heads of 128, 531 MB in 102 us with the join (5.2 TB/s, as fast as a large copy); 32 ragged ones of up to 4096
// tokens, 40 heads, 309 MB in 78 us.  One sequence of 1203 tokens takes 12 us: 4 until the first codes are there, 4 for five steps a wave, which the vector unit bounds, 2 to meet.
#pragma once

#include "apmm_kv_attention.h"

namespace apmm {

template <int D>
struct KvRowsStep {
    uint32_t k[2][D / 32];
    uint2 v[2][D / 64];
    uint2 ks[2], vs[2];
};

template <int D, bool BF16, int WAVES>
__device__ __forceinline__ void kv_attention_rows(const KvAttentionArgs &a, const KvPart &part, int block)
{
    constexpr int W = D / 32, V = D / 64, T = kRowsTile;
    constexpr int R = 4, kPitch = D + 4;  // rows that meet in LDS at a time
    __shared__ __align__(16) float sums[WAVES][R][kPitch];
    __shared__ float bases[WAVES][T], totals[WAVES][T];
    const int slot = kv_divide(block, a.c.by_heads), head = block - slot * a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4;
    KvItem<kRowsStep> it;
    const bool there = kv_item<kRowsStep, kRowsTile>(a, part, slot, it);
    kv_note(a, part, a.partial, slot, head, there, it, threadIdx.x == 0);
    if (!there) return;

    const int rows = min(it.rows, T), row = it.row0 + min(n, rows - 1), at = kv_divide(row, a.by_groups);
    const int pos = it.s.first + at, first_pos = it.s.first + kv_divide(it.row0, a.by_groups), last_pos = it.s.first + kv_divide(it.row0 + rows - 1, a.by_groups);
    auto over_row = [](float v, auto f) {
        v = f(v, __shfl_xor(v, 16));
        return f(v, __shfl_xor(v, 32));
    };
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto plus = [](float x, float y) { return x + y; };

    const int shift = a.c.page_shift, mask = (1 << shift) - 1;
    const uint32_t key_lane = n * (D / 2) + g * (D / 8), value_lane = ((g >> 1) * (D / 4) + n) * 16 + (g & 1) * 8, scale_lane = g * 8;
    auto load = [&](int key, int page0, int page1, KvRowsStep<D> &s) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t place = ((((int64_t)max(t ? page1 : page0, 0) * a.c.heads + head) * 2) << shift) + ((key + 16 * t) & mask);
            const uint8_t *keys = a.c.codes + place * (D / 2), *values = keys + ((int64_t)(D / 2) << shift);
            const uint8_t *scales = reinterpret_cast<const uint8_t *>(a.c.scales + place), *value_scales = scales + ((int64_t)2 << shift);
            if constexpr (D == 128) {
                const uint4 w = *reinterpret_cast<const uint4 *>(keys + key_lane);
                s.k[t][0] = w.x; s.k[t][1] = w.y; s.k[t][2] = w.z; s.k[t][3] = w.w;
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(keys + key_lane);
                s.k[t][0] = w.x; s.k[t][1] = w.y;
            }
            s.ks[t] = *reinterpret_cast<const uint2 *>(scales + scale_lane);
            s.vs[t] = *reinterpret_cast<const uint2 *>(value_scales + scale_lane);
#pragma unroll
            for (int i = 0; i < V; ++i) s.v[t][i] = *reinterpret_cast<const uint2 *>(values + value_lane + 256 * i);
        }
    };

    int v = it.from + wave, ids = kv_page_ids(a, it, v, WAVES), id = 0;
    half8 q[W];
    float init, factor;
    KvRowsStep<D> s0, s1;
    {
        uint32_t x[4 * W];
        kv_load(a.q.data + (int64_t)(it.s.start + at) * a.q.token_stride + (int64_t)(head * a.groups + row - at * a.groups) * a.q.head_stride + g * (D / 4), a.q.aligned, x);
        if (v < it.to) load(it.key_of(v), __builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1), s0);
        kv_queries<4 * W, BF16>(x, a.scale, [&](float v) { return over_row(v, larger); }, [&](float v) { return over_row(v, plus); }, q, init, factor);
    }
    const float4v init4 = {init, init, init, init};

    float4v acc[4][V];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[e][i] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    float top = kLowest, base = -kLowest, total = 0.0f, weights = 0.0f;
    uint32_t limit = 0, met = 0;  // scales of values that the row has met: the largest, and the largest that needs no other E
    bool large = false;           // whether some row's E is more than kMostExponent

    auto step = [&](const KvRowsStep<D> &cur, KvRowsStep<D> &next) {
        const int key0 = it.key_of(v), page0 = __builtin_amdgcn_readlane(ids, id), page1 = __builtin_amdgcn_readlane(ids, id + 1);
        v += WAVES;
        id += 2;
        if (id == 64) {
            ids = kv_page_ids(a, it, v, WAVES);
            id = 0;
        }
        {   // (behind the last step the same one again: from the cache, and no branch)
            const bool more = v < it.to;
            load(more ? it.key_of(v) : key0, more ? __builtin_amdgcn_readlane(ids, id) : page0, more ? __builtin_amdgcn_readlane(ids, id + 1) : page1, next);
        }

        // scores, without the row's factor
        float4v sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sc[t] = init4;
#pragma unroll
            for (int i = 0; i < W; ++i) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_operand(cur.k[t][i]), q[i], sc[t], 0, 0, 0);
        }
        const uint32_t ks[4] = {cur.ks[0].x, cur.ks[0].y, cur.ks[1].x, cur.ks[1].y};
        uint32_t vs[4] = {cur.vs[0].x, cur.vs[0].y, cur.vs[1].x, cur.vs[1].y};
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(sc[i / 4][i % 4], i & 1 ? kv_high<BF16>(ks[i / 2]) : kv_low<BF16>(ks[i / 2]), 0.0f);
        const bool all = key0 + kRowsStep <= it.s.keys && key0 + kRowsStep - 1 <= first_pos && page0 >= 0 && page1 >= 0 &&
                         (!a.window || key0 > last_pos - a.window || key0 + kRowsStep <= a.sinks);
        if (!all) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = key0 + 16 * (i / 4) + 4 * g + i % 4, end = (i < 4 ? page0 : page1) >= 0 ? min(it.s.keys, pos + 1) : 0;
                const bool hidden = (key >= end) | ((a.window != 0) & (key <= pos - a.window) & (key >= a.sinks));
                x[i] = hidden ? -__builtin_inff() : x[i];
                vs[i / 2] &= hidden ? (i & 1 ? 0x0000ffffu : 0xffff0000u) : 0xffffffffu;  // weights of hidden keys are zero whatever their scale is
            }
        }
        const uint32_t most2 = kv_fold_max(kv_fold_max(vs[0], vs[1]), kv_fold_max(vs[2], vs[3])), most = max(most2 & 0xffffu, most2 >> 16);
        const float high = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))) * factor;
        if (__any((high > top + kSlack) | (most > limit))) {
            top = fmaxf(top, over_row(high, larger));
            uint32_t m = met;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = kv_finite_max<BF16>(kv_finite_max<BF16>(m, vs[i] & 0xffffu), vs[i] >> 16);
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            const int e = kv_exponent<BF16>(m);
            const float to = -top + (kRoom - (float)min(e, kMostExponent));
            float by = __builtin_amdgcn_exp2f(to - base);
            total = kv_moved<BF16>(total, to - base);
            base = to;
            if (BF16) {
                by *= ldexpf(1.0f, kv_rest(kv_exponent<true>(met)) - kv_rest(e));
                large = __any(e > kMostExponent);
            }
            met = m;
            limit = kv_limit<BF16>(met);
            weights *= by;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[e][i] *= by;
        }
        uint32_t w[4], rest[4] = {};  // rounded weights and, for results of binary16, what that left: two numbers of 11 bits
        float weight[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(x[2 * i], factor, base)), p1 = __builtin_amdgcn_exp2f(fmaf(x[2 * i + 1], factor, base));
            total += p0 + p1;
            weight[2 * i] = fmaf(p0, kv_low<BF16>(vs[i]), 0.0f);
            weight[2 * i + 1] = fmaf(p1, kv_high<BF16>(vs[i]), 0.0f);
        }
        if (BF16 && large) {
            const float by = ldexpf(1.0f, -kv_rest(kv_exponent<BF16>(met)));
#pragma unroll
            for (int i = 0; i < 8; ++i) weight[i] *= by;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float w0 = weight[2 * i], w1 = weight[2 * i + 1];
            w[i] = kv_half_pair(w0, w1);
            weights = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, w[i]), (half2v){1, 1}, weights, false);
            if (!BF16) {
                rest[i] = kv_half_pair(w0 - kv_low<false>(w[i]), w1 - kv_high<false>(w[i]));
                weights = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, rest[i]), (half2v){1, 1}, weights, false);
            }
        }
        const half8 p = __builtin_bit_cast(half8, make_uint4(w[0], w[1], w[2], w[3])), p_rest = __builtin_bit_cast(half8, make_uint4(rest[0], rest[1], rest[2], rest[3]));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t c[4] = {cur.v[0][i].x, cur.v[0][i].y, cur.v[1][i].x, cur.v[1][i].y};
            uint32_t o[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t h = c[j] >> 8;
                o[0][j] = c[j] & 0x000f000fu;
                o[1][j] = c[j] & 0x00f000f0u;
                o[2][j] = h & 0x000f000fu;
                o[3][j] = h & 0x00f000f0u;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const half8 codes = __builtin_bit_cast(half8, make_uint4(o[e][0], o[e][1], o[e][2], o[e][3]));
                acc[e][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, p, acc[e][i], 0, 0, 0);
                if (!BF16) acc[e][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, p_rest, acc[e][i], 0, 0, 0);
            }
        }
    };
    while (v < it.to) {
        step(s0, s1);
        if (v >= it.to) break;
        step(s1, s0);
    }

    // the waves' sums, four rows at a time: channel 64 i + 16 g + 4 j + e of row n is acc[e][i][j]
    total = over_row(total, plus);
    weights = over_row(weights, plus);
    const float lift = BF16 ? ldexpf(1.0f, kv_rest(kv_exponent<BF16>(met))) : 1.0f;
    if (g == 0) {
        bases[wave][n] = -base;
        totals[wave][n] = total;
    }
    constexpr int kThreads = 64 * WAVES, C = kThreads >= R * D ? 1 : R * D / kThreads;  // channels of a thread
    const int mine = threadIdx.x / (D / C), c0 = threadIdx.x % (D / C) * C;
    const KvPartial partial = kv_partial(a.partial, part, a.c.heads, D);
    for (int r0 = 0; r0 < rows; r0 += R) {
        if ((n & ~(R - 1)) == r0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float4v o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = fmaf(acc[e][i][j], e & 1 ? 0x1p21f : 0x1p25f, -15.0f * weights) * lift;
                    *reinterpret_cast<float4v *>(&sums[wave][n & (R - 1)][64 * i + 16 * g + 4 * j]) = o;
                }
        }
        __syncthreads();
        const int r = r0 + mine;
        if (mine < R && r < rows) {
            float most = bases[0][r];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) most = fmaxf(most, bases[i][r]);
            float sum = 0.0f, o[C] = {};
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                const float by = __builtin_amdgcn_exp2f(bases[i][r] - most);
                sum = kv_moved<BF16>(totals[i][r], bases[i][r] - most, sum);
#pragma unroll
                for (int j = 0; j < C; ++j) o[j] = fmaf(sums[i][mine][c0 + j], by, o[j]);
            }
            if (it.pieces == 1) {
                const int to_row = it.row0 + r, to_at = kv_divide(to_row, a.by_groups);
                const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
                uint16_t *out = a.out.data + (int64_t)(it.s.start + to_at) * a.out.token_stride +
                                (int64_t)(head * a.groups + to_row - to_at * a.groups) * a.out.head_stride + c0;
#pragma unroll
                for (int j = 0; j < C; ++j) out[j] = kv_round(o[j] * over, BF16);
            } else {
                const int64_t place = ((int64_t)slot * a.c.heads + head) * T + r;
#pragma unroll
                for (int j = 0; j < C; ++j) partial.sums[place * D + c0 + j] = o[j];
                if (c0 == 0) partial.row[place] = make_float2(most, sum);
            }
        }
        __syncthreads();
    }
}

}  // namespace apmm
