// Attention of many rows over the four-bit cache (apmm_kv_attention.h): prompts and pieces of prompts.
//
// A workgroup has 128 rows, 32 to each of its four waves, which go through the keys by themselves: steps of 32 keys, matrix instructions 32 x 32 x 16, keys and values from memory (L1, L2: the
// waves and the workgroups of a head read the same) into registers one step ahead, no LDS and no barrier.
#include "apmm_kv_attention.h"

namespace apmm {

namespace {

constexpr int kWaves = 4, kRows = kTilesTile / kWaves;

template <int D>
struct Step {
    uint32_t k[D / 16];
    uint4 v[2];
    uint4 ks[2], vs[2];
    int key, page[2];
};

template <int D>
__device__ __forceinline__ void load_step(const KvAttentionArgs &a, int head, int key, int page0, int page1, Step<D> &s)
{
    const int lane = kv_lane(), r = lane & 31, h = lane >> 5, shift = a.c.page_shift, mask = (1 << shift) - 1;
    s.key = key;
    s.page[0] = page0;
    s.page[1] = page1;
    const int64_t block0 = ((int64_t)max(page0, 0) * a.c.heads + head) * 2, block1 = ((int64_t)max(page1, 0) * a.c.heads + head) * 2;
    const int in0 = key & mask, in1 = (key + 16) & mask;
    {   // operand row 8 i + 4 h' + j is key 16 h' + 4 i + j
        const bool second = r & 4;
        const uint8_t *keys = a.c.codes + (((second ? block1 : block0) << shift) + (second ? in1 : in0) + 4 * (r >> 3) + (r & 3)) * (D / 2) + h * (D / 4);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const uint4 w = reinterpret_cast<const uint4 *>(keys)[i];
            s.k[4 * i] = w.x; s.k[4 * i + 1] = w.y; s.k[4 * i + 2] = w.z; s.k[4 * i + 3] = w.w;
        }
    }
    const int64_t place = ((h ? block1 : block0) << shift) + (h ? in1 : in0);
    const uint4 *scales = reinterpret_cast<const uint4 *>(a.c.scales + place), *value_scales = reinterpret_cast<const uint4 *>(a.c.scales + place + ((int64_t)1 << shift));
    const uint4 *values = reinterpret_cast<const uint4 *>(a.c.codes + (place + ((int64_t)1 << shift)) * (D / 2)) + (r & (D / 4 - 1));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        s.ks[i] = scales[i];
        s.vs[i] = value_scales[i];
        s.v[i] = values[i * (D / 4)];
    }
}

template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves, 2) void kv_attention_tiles_kernel(KvAttentionArgs a, KvPlan plan)
{
    constexpr int W = D / 16, E = D / 32;  // words of a lane's key, blocks of 32 channels of the result
    const int head = blockIdx.x % a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 31, h = lane >> 5;
    KvItem it;
    const int slot = blockIdx.x / a.c.heads;
    const bool there = kv_item(a, plan, slot, it);
    kv_note(a, plan, slot, head, there, it);
    if (!there) return;

    const int row0 = it.row0 + wave * kRows, rows = min(it.rows - wave * kRows, kRows);
    if (rows <= 0) return;
    const int row = row0 + min(n, rows - 1), at = row / a.groups;
    const int pos = it.s.first + at, first_pos = it.s.first + row0 / a.groups, last_pos = it.s.first + (row0 + rows - 1) / a.groups;
    auto over_row = [](float v, auto f) { return f(v, __shfl_xor(v, 32)); };
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto plus = [](float x, float y) { return x + y; };

    half8 q[W];
    float init, factor;
    {
        uint32_t x[4 * W];
        kv_load(a.q.data + (int64_t)(it.s.start + at) * a.q.token_stride + (int64_t)(head * a.groups + row % a.groups) * a.q.head_stride + h * (D / 2), a.q.aligned, x);
        kv_queries<4 * W, BF16>(x, a.scale, [&](float v) { return over_row(v, larger); }, [&](float v) { return over_row(v, plus); }, q, init, factor);
    }

    float16v acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[e][i] = 0.0f;
    float top = kLowest, base = -kLowest, total = 0.0f, weights = 0.0f;
    uint32_t limit = 0, met = 0;

    // the steps of this wave: those of the workgroup's that some row of it sees
    auto seen = [&](int key) { return key <= last_pos && (!a.window || key + kKvStep > first_pos - a.window + 1 || key < a.sinks); };
    int to = it.to;
    while (to > it.from && !seen(it.key_of(to - 1))) --to;
    int v = it.from;
    while (v < to && !seen(it.key_of(v))) ++v;
    int ids = kv_page_ids(a, it, v, 1), id = 0;
    Step<D> cur, next;
    if (v < to) load_step<D>(a, head, it.key_of(v), __builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1), cur);
    for (; v < to; ++v, cur = next) {
        id += 2;
        if (id == 64) {
            ids = kv_page_ids(a, it, v + 1, 1);
            id = 0;
        }
        if (v + 1 < to) load_step<D>(a, head, it.key_of(v + 1), __builtin_amdgcn_readlane(ids, id), __builtin_amdgcn_readlane(ids, id + 1), next);

        float16v sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = init;
#pragma unroll
        for (int i = 0; i < W; ++i) sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(kv_operand(cur.k[i]), q[i], sc, 0, 0, 0);
        const uint32_t ks[8] = {cur.ks[0].x, cur.ks[0].y, cur.ks[0].z, cur.ks[0].w, cur.ks[1].x, cur.ks[1].y, cur.ks[1].z, cur.ks[1].w};
        uint32_t vs[8] = {cur.vs[0].x, cur.vs[0].y, cur.vs[0].z, cur.vs[0].w, cur.vs[1].x, cur.vs[1].y, cur.vs[1].z, cur.vs[1].w};
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = fmaf(sc[i], i & 1 ? kv_high<BF16>(ks[i / 2]) : kv_low<BF16>(ks[i / 2]), 0.0f);
        const bool all = cur.key + kKvStep <= it.s.keys && cur.key + kKvStep - 1 <= first_pos && cur.page[0] >= 0 && cur.page[1] >= 0 &&
                         (!a.window || cur.key > last_pos - a.window || cur.key + kKvStep <= a.sinks);
        if (!all) {
            const bool page = (h ? cur.page[1] : cur.page[0]) >= 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = cur.key + 16 * h + i;
                if (!(page && key < it.s.keys && key <= pos && (!a.window || key > pos - a.window || key < a.sinks))) {
                    x[i] = -__builtin_inff();
                    vs[i / 2] &= i & 1 ? 0x0000ffffu : 0xffff0000u;  // weights of hidden keys are zero whatever their scale is
                }
            }
        }
        uint32_t most2 = vs[0];
        float high = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) most2 = kv_fold_max(most2, vs[i]);
        const uint32_t most = max(most2 & 0xffffu, most2 >> 16);
#pragma unroll
        for (int i = 1; i < 16; ++i) high = fmaxf(high, x[i]);
        high *= factor;
        if (__any(high > top + kSlack || most > limit)) {
            top = fmaxf(top, over_row(high, larger));
            uint32_t m = met;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = kv_finite_max<BF16>(kv_finite_max<BF16>(m, vs[i] & 0xffffu), vs[i] >> 16);
#pragma unroll
            for (int d = 1; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
            met = m;
            limit = kv_limit<BF16>(met);
            const float moved = -top + (kRoom - (float)kv_exponent<BF16>(met));
            const float by = __builtin_amdgcn_exp2f(moved - base);
            base = moved;
            total *= by;
            weights *= by;
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[e][i] *= by;
        }
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(x[2 * i], factor, base)), p1 = __builtin_amdgcn_exp2f(fmaf(x[2 * i + 1], factor, base));
            total += p0 + p1;
            w[i] = kv_half_pair(fmaf(p0, kv_low<BF16>(vs[i]), 0.0f), fmaf(p1, kv_high<BF16>(vs[i]), 0.0f));
            weights = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, w[i]), (half2v){1, 1}, weights, false);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const half8 p = __builtin_bit_cast(half8, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
            uint32_t c[4] = {cur.v[i].x, cur.v[i].y, cur.v[i].z, cur.v[i].w};
            uint32_t o[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (D == 64) c[j] >>= 8 * (n >> 4);  // operand rows 16 and up: channels 4 m + 2 and 4 m + 3
                o[0][j] = c[j] & 0x000f000fu;
                o[1][j] = c[j] & 0x00f000f0u;
                o[2][j] = (c[j] >> 8) & 0x000f000fu;
                o[3][j] = (c[j] >> 8) & 0x00f000f0u;
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, make_uint4(o[e][0], o[e][1], o[e][2], o[e][3])), p, acc[e], 0, 0, 0);
        }
    }

    // row n's channels of this lane, 16 at a time: 32 i + 16 h + 4 j + e of acc[e][4 i + j] (64 channels: 32 i + 16 h + 4 j + e of acc[e & 1][4 (i + (e & 2)) + j])
    total = over_row(total, plus);
    weights = over_row(weights, plus);
    if (n >= rows) return;
    const bool whole = it.pieces == 1;
    const float over = whole ? (total == 0.0f ? 0.0f : 1.0f / total) : 1.0f;
    uint16_t *out = a.out.data + (int64_t)(it.s.start + at) * a.out.token_stride + (int64_t)(head * a.groups + row % a.groups) * a.out.head_stride;
    const int64_t place = ((int64_t)it.slot * a.c.heads + head) * kTilesTile + wave * kRows + n;
    const KvPartial partial = kv_partial(a.partial, plan, a.c.heads, D);
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

hipError_t launch_kv_attention_tiles(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)plan.slots * a.c.heads)), block(64 * kWaves);
    if (a.c.head_dim == 128) {
        if (a.c.bf16) kv_attention_tiles_kernel<128, true><<<grid, block, 0, stream>>>(a, plan);
        else kv_attention_tiles_kernel<128, false><<<grid, block, 0, stream>>>(a, plan);
    } else {
        if (a.c.bf16) kv_attention_tiles_kernel<64, true><<<grid, block, 0, stream>>>(a, plan);
        else kv_attention_tiles_kernel<64, false><<<grid, block, 0, stream>>>(a, plan);
    }
    return hipGetLastError();
}

}  // namespace apmm
