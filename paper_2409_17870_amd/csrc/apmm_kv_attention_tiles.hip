// Attention of many rows over the four-bit cache (apmm_kv_attention.h): prompts and pieces of prompts.
//
// A workgroup has 128 rows, 32 to each of its four waves, and goes through the keys in steps of 64 with matrix instructions 32 x 32 x 16.  Codes become operands once for all four waves:
// each wave loads a quarter of a step one step ahead, makes its operands and leaves them in LDS, in the order in which lanes take them (no bank is asked twice).  Two buffers, one barrier a step.
#include "apmm_kv_attention.h"

namespace apmm {

namespace {

constexpr int kWaves = 4, kRows = kTilesTile / kWaves;

// 32 keys and values as matrix operands, 64 lanes x 16 bytes each, and their scales
template <int D>
struct Operands {
    uint4 k[D / 16][64];
    uint4 v[2][D / 32][64];
    uint4 ks[4], vs[4];
};

template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves, 2) void kv_attention_tiles_kernel(KvAttentionArgs a, KvPart part)
{
    constexpr int W = D / 16, E = D / 32;  // operands of 32 keys, blocks of 32 channels of the result
    __shared__ Operands<D> shared[2][2];
    const int head = blockIdx.x % a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 31, h = lane >> 5;
    KvItem<kTilesStep> it;
    const int slot = blockIdx.x / a.c.heads;
    const bool there = kv_item(a, part, slot, it);
    kv_note(a, part, slot, head, there, it);
    if (!there) return;

    // what this wave makes ready of each step: keys (waves 0 and 1) or values (2 and 3) of one of its two 32s, with their scales
    const int shift = a.c.page_shift, mask = (1 << shift) - 1, sub = wave & 1;
    const bool values = wave >= 2;
    // operand row 8 i + 4 h' + j of the keys is key 16 h' + 4 i + j; half h of the values' operand s has keys 16 h + 8 s to 16 h + 8 s + 7
    const bool second = values ? h : (n & 4) != 0;
    const uint32_t lane_at = values ? (n & (D / 4 - 1)) * 16 + ((uint32_t)(D / 2) << shift) : (uint32_t)(4 * (n >> 3) + (n & 3)) * (D / 2) + h * (D / 4);
    constexpr int kParts = D == 128 ? 2 : 1;
    uint4 codes[2], scales = {};
    auto load = [&](int key, int page0, int page1) {
        const int64_t place0 = ((((int64_t)max(page0, 0) * a.c.heads + head) * 2) << shift) + (key & mask);
        const int64_t place1 = ((((int64_t)max(page1, 0) * a.c.heads + head) * 2) << shift) + ((key + 16) & mask);
        const uint8_t *at = a.c.codes + (second ? place1 : place0) * (D / 2) + lane_at;
        codes[0] = *reinterpret_cast<const uint4 *>(at);
        if (values) codes[1] = *reinterpret_cast<const uint4 *>(at + D * 4);
        else if (D == 128) codes[1] = *reinterpret_cast<const uint4 *>(at + 16);
        if (lane < 4) scales = *reinterpret_cast<const uint4 *>(a.c.scales + (lane & 2 ? place1 : place0) + (values ? (int64_t)1 << shift : 0) + 8 * (lane & 1));
    };
    auto store = [&](Operands<D> &to) {
        if (values) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                uint32_t c[4] = {codes[s].x, codes[s].y, codes[s].z, codes[s].w};
                if (D == 64) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) c[j] >>= 8 * (n >> 4);  // operand rows 16 and up: channels 4 m + 2 and 4 m + 3
                }
                constexpr uint32_t L = 0x000f000fu, H = 0x00f000f0u;
                to.v[s][0][lane] = make_uint4(c[0] & L, c[1] & L, c[2] & L, c[3] & L);
                to.v[s][1][lane] = make_uint4(c[0] & H, c[1] & H, c[2] & H, c[3] & H);
                if constexpr (D == 128) {
                    to.v[s][2][lane] = make_uint4((c[0] >> 8) & L, (c[1] >> 8) & L, (c[2] >> 8) & L, (c[3] >> 8) & L);
                    to.v[s][3][lane] = make_uint4((c[0] >> 8) & H, (c[1] >> 8) & H, (c[2] >> 8) & H, (c[3] >> 8) & H);
                }
            }
        } else {
#pragma unroll
            for (int s = 0; s < kParts; ++s) {
                const uint32_t c[4] = {codes[s].x, codes[s].y, codes[s].z, codes[s].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) to.k[4 * s + j][lane] = __builtin_bit_cast(uint4, kv_operand(c[j]));
            }
        }
        if (lane < 4) (values ? to.vs : to.ks)[lane] = scales;
    };

    const int row0 = it.row0 + wave * kRows, rows = min(it.rows - wave * kRows, kRows);  // (may be none: such a wave helps the others)
    const int row = row0 + max(min(n, rows - 1), 0), at = min(row / a.groups, it.s.n - 1);
    const int pos = it.s.first + at, first_pos = it.s.first + row0 / a.groups, last_pos = rows > 0 ? it.s.first + (row0 + rows - 1) / a.groups : -1;
    auto over_row = [](float v, auto f) { return f(v, __shfl_xor(v, 32)); };
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto plus = [](float x, float y) { return x + y; };

    int v = it.from, ids = kv_page_ids(a, it, v, 1), next_ids = -1, id = 0;
    half8 q[W];
    float init, factor;
    {
        uint32_t x[4 * W];
        kv_load(a.q.data + (int64_t)(it.s.start + at) * a.q.token_stride + (int64_t)(head * a.groups + row % a.groups) * a.q.head_stride + h * (D / 2), a.q.aligned, x);
        if (v < it.to) {
            load(it.key_of(v) + 32 * sub, __builtin_amdgcn_readlane(ids, 2 * sub), __builtin_amdgcn_readlane(ids, 2 * sub + 1));
            store(shared[0][sub]);
        }
        kv_queries<4 * W, BF16>(x, a.scale, [&](float v) { return over_row(v, larger); }, [&](float v) { return over_row(v, plus); }, q, init, factor);
    }

    float16v acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[e][i] = 0.0f;
    float top = kLowest, base = -kLowest, total = 0.0f, weights = 0.0f;
    uint32_t limit = 0, met = 0;  // largest scale of values: where it is passed, met so far
    bool moved = false;           // the step at hand has moved the maximum (scales that are not finite would do so again)
    bool loaded = false;
    int buffer = 0;

    __syncthreads();
    while (v < it.to) {
        float high, x[2][16];
        uint32_t vs[2][8];
        do {  // steps that leave the maximum where it is; one that does not ends the loop before it has added anything, and is done again
            const int key0 = it.key_of(v);
            if (!loaded && v + 1 < it.to) {
                int after = id + 4;
                if (after == 64) {
                    next_ids = kv_page_ids(a, it, v + 1, 1);
                    after = 0;
                }
                const int from = after ? ids : next_ids;
                load(it.key_of(v + 1) + 32 * sub, __builtin_amdgcn_readlane(from, after + 2 * sub), __builtin_amdgcn_readlane(from, after + 2 * sub + 1));
                loaded = true;
            }
            const uint32_t pages = (uint32_t)(__ballot(ids >= 0) >> id) & 15u;
            const bool all = key0 + kTilesStep <= it.s.keys && key0 + kTilesStep - 1 <= first_pos && pages == 15u &&
                             (!a.window || key0 > last_pos - a.window || key0 + kTilesStep <= a.sinks);
            uint32_t most2 = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const Operands<D> &cur = shared[buffer][t];
                float16v sc;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = init;
#pragma unroll
                for (int i = 0; i < W; ++i) sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, cur.k[i][lane]), q[i], sc, 0, 0, 0);
                const uint4 ks0 = cur.ks[2 * h], ks1 = cur.ks[2 * h + 1], vs0 = cur.vs[2 * h], vs1 = cur.vs[2 * h + 1];
                const uint32_t ks[8] = {ks0.x, ks0.y, ks0.z, ks0.w, ks1.x, ks1.y, ks1.z, ks1.w};
                vs[t][0] = vs0.x; vs[t][1] = vs0.y; vs[t][2] = vs0.z; vs[t][3] = vs0.w; vs[t][4] = vs1.x; vs[t][5] = vs1.y; vs[t][6] = vs1.z; vs[t][7] = vs1.w;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[t][i] = fmaf(sc[i], i & 1 ? kv_high<BF16>(ks[i / 2]) : kv_low<BF16>(ks[i / 2]), 0.0f);
            }
            if (!all) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int end = pages >> (2 * t + h) & 1 ? min(it.s.keys, pos + 1) : 0, first = key0 + 32 * t + 16 * h;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = first + i;
                        const bool hidden = (key >= end) | ((a.window != 0) & (key <= pos - a.window) & (key >= a.sinks));
                        x[t][i] = hidden ? -__builtin_inff() : x[t][i];
                        vs[t][i / 2] &= hidden ? (i & 1 ? 0x0000ffffu : 0xffff0000u) : 0xffffffffu;  // weights of hidden keys are zero whatever their scale is
                    }
                }
            }
            high = x[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int i = 0; i < 8; ++i) most2 = kv_fold_max(most2, vs[t][i]);
#pragma unroll
                for (int i = 0; i < 16; ++i) high = fmaxf(high, x[t][i]);
            }
            const uint32_t most = max(most2 & 0xffffu, most2 >> 16);
            high *= factor;
            if (!moved && __any((high > top + kSlack) | (most > limit))) break;
            moved = false;

#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const Operands<D> &cur = shared[buffer][t];
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(x[t][2 * i], factor, base)), p1 = __builtin_amdgcn_exp2f(fmaf(x[t][2 * i + 1], factor, base));
                    total += p0 + p1;
                    w[i] = kv_half_pair(fmaf(p0, kv_low<BF16>(vs[t][i]), 0.0f), fmaf(p1, kv_high<BF16>(vs[t][i]), 0.0f));
                    weights = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, w[i]), (half2v){1, 1}, weights, false);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const half8 p = __builtin_bit_cast(half8, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, cur.v[i][e][lane]), p, acc[e], 0, 0, 0);
                }
            }
            buffer ^= 1;
            if (loaded) store(shared[buffer][sub]);
            __syncthreads();
            loaded = false;
            ++v;
            id += 4;
            if (id == 64) {
                ids = next_ids;
                id = 0;
            }
        } while (v < it.to);
        if (v >= it.to) break;
        top = fmaxf(top, over_row(high, larger));
        uint32_t m = met;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = kv_finite_max<BF16>(kv_finite_max<BF16>(m, vs[i / 8][i % 8] & 0xffffu), vs[i / 8][i % 8] >> 16);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
        met = m;
        limit = kv_limit<BF16>(met);
        const float to = -top + (kRoom - (float)kv_exponent<BF16>(met));
        const float by = __builtin_amdgcn_exp2f(to - base);
        base = to;
        total *= by;
        weights *= by;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[e][i] *= by;
        moved = true;
    }

    // row n's channels of this lane, 16 at a time: 32 i + 16 h + 4 j + e of acc[e][4 i + j] (64 channels: 32 i + 16 h + 4 j + e of acc[e & 1][4 (i + (e & 2)) + j])
    total = over_row(total, plus);
    weights = over_row(weights, plus);
    if (n >= rows) return;
    const bool whole = it.pieces == 1;
    const float over = whole ? (total == 0.0f ? 0.0f : 1.0f / total) : 1.0f;
    uint16_t *out = a.out.data + (int64_t)(it.s.start + at) * a.out.token_stride + (int64_t)(head * a.groups + row % a.groups) * a.out.head_stride;
    const int64_t place = ((int64_t)slot * a.c.heads + head) * kTilesTile + wave * kRows + n;
    const KvPartial partial = kv_partial(a.partial, part, a.c.heads, D);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        float o[16];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = D == 128 ? acc[e & (E - 1)][4 * i + j] : acc[e & 1][4 * ((i + (e & 2)) & 3) + j];
                o[4 * j + e] = fmaf(x, e & 1 ? 0x1p21f : 0x1p25f, -15.0f * weights) * over;
            }
        const int c0 = 32 * i + 16 * h;
        if (whole) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = kv_round(o[2 * j], BF16) | (uint32_t)kv_round(o[2 * j + 1], BF16) << 16;
            kv_store(out + c0, a.out.aligned, w);
        } else {
#pragma unroll
            for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4v *>(partial.sums + place * D + c0 + j) = float4v{o[j], o[j + 1], o[j + 2], o[j + 3]};
        }
    }
    if (!whole && h == 0) partial.row[place] = make_float2(-base, total);
}

}  // namespace

hipError_t launch_kv_attention_tiles(const KvAttentionArgs &a, const KvPart &part, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)part.slots * a.c.heads)), block(64 * kWaves);
    if (a.c.head_dim == 128) {
        if (a.c.bf16) kv_attention_tiles_kernel<128, true><<<grid, block, 0, stream>>>(a, part);
        else kv_attention_tiles_kernel<128, false><<<grid, block, 0, stream>>>(a, part);
    } else {
        if (a.c.bf16) kv_attention_tiles_kernel<64, true><<<grid, block, 0, stream>>>(a, part);
        else kv_attention_tiles_kernel<64, false><<<grid, block, 0, stream>>>(a, part);
    }
    return hipGetLastError();
}

}  // namespace apmm
