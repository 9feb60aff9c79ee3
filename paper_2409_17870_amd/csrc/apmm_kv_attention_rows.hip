// Attention of few rows over the four-bit cache (apmm_kv_attention.h): token generation.
//
// A workgroup has 16 rows (the query heads of a key/value head times its new tokens; fewer are there in most calls) and a piece of the keys, its four waves take steps of 32 keys
// in turn, each with its own maximum and sums, and meet in LDS at the end.  Matrix instructions 16 x 16 x 32: two for each 32 channels and 16 keys, one for each 16 channels of the result.
// A lane loads its parts of keys and values from memory into registers, one step ahead: rows of keys whole, 16 bytes a lane.
#include "apmm_kv_attention.h"

namespace apmm {

namespace {

constexpr int kWaves = 4;

template <int D>
struct Step {
    uint32_t k[2][D / 32];
    uint4 v[D / 64];
    uint4 ks, vs;
    int key, page[2];
};

template <int D>
__device__ __forceinline__ void load_step(const KvAttentionArgs &a, int head, int key, int page0, int page1, Step<D> &s)
{
    const int lane = kv_lane(), r = lane & 15, g = lane >> 4, shift = a.c.page_shift, mask = (1 << shift) - 1;
    s.key = key;
    s.page[0] = page0;
    s.page[1] = page1;
    const int64_t block0 = ((int64_t)max(page0, 0) * a.c.heads + head) * 2, block1 = ((int64_t)max(page1, 0) * a.c.heads + head) * 2;
    const int in0 = key & mask, in1 = (key + 16) & mask;
    {   // operand row 4 g' + j of key tile t is key 8 g' + 4 t + j
        const uint8_t *keys = a.c.codes + (((r < 8 ? block0 : block1) << shift) + (r < 8 ? in0 : in1)) * (D / 2) + (8 * ((r >> 2) & 1) + (r & 3)) * (D / 2) + g * (D / 8);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (D == 128) {
                const uint4 w = *reinterpret_cast<const uint4 *>(keys + 4 * t * (D / 2));
                s.k[t][0] = w.x; s.k[t][1] = w.y; s.k[t][2] = w.z; s.k[t][3] = w.w;
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(keys + 4 * t * (D / 2));
                s.k[t][0] = w.x; s.k[t][1] = w.y;
            }
        }
    }
    const int64_t block = (g < 2 ? block0 : block1) << shift;
    const int in = (g < 2 ? in0 : in1) + 8 * (g & 1);
    const uint16_t *scales = a.c.scales + block + in;
    s.ks = *reinterpret_cast<const uint4 *>(scales);
    s.vs = *reinterpret_cast<const uint4 *>(scales + ((int64_t)1 << shift));
    const uint4 *values = reinterpret_cast<const uint4 *>(a.c.codes + (block + in + ((int64_t)1 << shift)) * (D / 2)) + r;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) s.v[i] = values[16 * i];
}

template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves) void kv_attention_rows_kernel(KvAttentionArgs a, KvPlan plan, int least)
{
    constexpr int W = D / 32, V = D / 64, T = kRowsTile;
    constexpr int kPitch = D + 4;
    __shared__ __align__(16) float sums[kWaves][T][kPitch];
    __shared__ float bases[kWaves][T], totals[kWaves][T];
    const int head = blockIdx.x % a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), n = lane & 15, g = lane >> 4;
    const int piece = kv_piece(a, plan, least);
    KvItem it;
    if (!kv_item(a, plan, piece, blockIdx.x / a.c.heads, it)) return;

    const int rows = min(it.rows, T), row = it.row0 + min(n, rows - 1), at = row / a.groups;
    const int pos = it.s.first + at, first_pos = it.s.first + it.row0 / a.groups, last_pos = it.s.first + (it.row0 + rows - 1) / a.groups;
    auto over_row = [](float v, auto f) {
        v = f(v, __shfl_xor(v, 16));
        return f(v, __shfl_xor(v, 32));
    };
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto plus = [](float x, float y) { return x + y; };

    half8 q[W];
    float init, factor;
    {
        uint32_t x[4 * W];
        kv_load(a.q.data + (int64_t)(it.s.start + at) * a.q.token_stride + (int64_t)(head * a.groups + row % a.groups) * a.q.head_stride + g * (D / 4), a.q.aligned, x);
        kv_queries<4 * W, BF16>(x, a.scale, [&](float v) { return over_row(v, larger); }, [&](float v) { return over_row(v, plus); }, q, init, factor);
    }
    const float4v init4 = {init, init, init, init};

    float4v acc[4][V];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[e][i] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    float top = kLowest, base = -kLowest, total = 0.0f, weights = 0.0f;
    uint32_t limit = 0, met = 0;  // largest scale of values: where it is passed, met so far

    int v = it.from + wave, ids = kv_page_ids(a, it, v, kWaves), id = 0;
    Step<D> cur, next;
    if (v < it.to) load_step<D>(a, head, it.key_of(v), __builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1), cur);
    for (; v < it.to; v += kWaves, cur = next) {
        id += 2;
        if (id == 64) {
            ids = kv_page_ids(a, it, v + kWaves, kWaves);
            id = 0;
        }
        if (v + kWaves < it.to) load_step<D>(a, head, it.key_of(v + kWaves), __builtin_amdgcn_readlane(ids, id), __builtin_amdgcn_readlane(ids, id + 1), next);

        // scores, without the row's factor
        float4v sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sc[t] = init4;
#pragma unroll
            for (int i = 0; i < W; ++i) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_operand(cur.k[t][i]), q[i], sc[t], 0, 0, 0);
        }
        const uint32_t ks[4] = {cur.ks.x, cur.ks.y, cur.ks.z, cur.ks.w};
        uint32_t vs[4] = {cur.vs.x, cur.vs.y, cur.vs.z, cur.vs.w};
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(sc[i / 4][i % 4], i & 1 ? kv_high<BF16>(ks[i / 2]) : kv_low<BF16>(ks[i / 2]), 0.0f);
        const bool all = cur.key + kKvStep <= it.s.keys && cur.key + kKvStep - 1 <= first_pos && cur.page[0] >= 0 && cur.page[1] >= 0 &&
                         (!a.window || cur.key > last_pos - a.window || cur.key + kKvStep <= a.sinks);
        if (!all) {
            const bool page = cur.page[g >> 1] >= 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = cur.key + 8 * g + i;
                if (!(page && key < it.s.keys && key <= pos && (!a.window || key > pos - a.window || key < a.sinks))) {
                    x[i] = -__builtin_inff();
                    vs[i / 2] &= i & 1 ? 0x0000ffffu : 0xffff0000u;  // weights of hidden keys are zero whatever their scale is
                }
            }
        }
        const uint32_t most2 = kv_fold_max(kv_fold_max(vs[0], vs[1]), kv_fold_max(vs[2], vs[3])), most = max(most2 & 0xffffu, most2 >> 16);
        const float high = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))) * factor;
        if (__any(high > top + kSlack || most > limit)) {
            top = fmaxf(top, over_row(high, larger));
            uint32_t m = met;
#pragma unroll
            for (int i = 0; i < 4; ++i) m = kv_finite_max<BF16>(kv_finite_max<BF16>(m, vs[i] & 0xffffu), vs[i] >> 16);
            m = max(m, (uint32_t)__shfl_xor((int)m, 16));
            m = max(m, (uint32_t)__shfl_xor((int)m, 32));
            m = max(m, (uint32_t)__shfl_xor((int)m, 1));
            m = max(m, (uint32_t)__shfl_xor((int)m, 2));
            m = max(m, (uint32_t)__shfl_xor((int)m, 4));
            m = max(m, (uint32_t)__shfl_xor((int)m, 8));  // (rows see different keys where some are hidden)
            met = m;
            limit = kv_limit<BF16>(met);
            const float to = -top + (kRoom - (float)kv_exponent<BF16>(met));
            const float by = __builtin_amdgcn_exp2f(to - base);
            base = to;
            total *= by;
            weights *= by;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[e][i] *= by;
        }
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(x[2 * i], factor, base)), p1 = __builtin_amdgcn_exp2f(fmaf(x[2 * i + 1], factor, base));
            total += p0 + p1;
            w[i] = kv_half_pair(fmaf(p0, kv_low<BF16>(vs[i]), 0.0f), fmaf(p1, kv_high<BF16>(vs[i]), 0.0f));
            weights = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, w[i]), (half2v){1, 1}, weights, false);
        }
        const half8 p = __builtin_bit_cast(half8, make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t c[4] = {cur.v[i].x, cur.v[i].y, cur.v[i].z, cur.v[i].w};
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
            for (int e = 0; e < 4; ++e)
                acc[e][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, make_uint4(o[e][0], o[e][1], o[e][2], o[e][3])), p, acc[e][i], 0, 0, 0);
        }
    }

    // the four waves' sums: channel 64 i + 16 g + 4 j + e of row n is acc[e][i][j]
    total = over_row(total, plus);
    weights = over_row(weights, plus);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float4v o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(acc[e][i][j], e & 1 ? 0x1p21f : 0x1p25f, -15.0f * weights);
            *reinterpret_cast<float4v *>(&sums[wave][n][64 * i + 16 * g + 4 * j]) = o;
        }
    if (g == 0) {
        bases[wave][n] = -base;
        totals[wave][n] = total;
    }
    __syncthreads();
    constexpr int C = D / 16;  // channels of a thread
    const int mine = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * C;
    if (mine >= rows) return;
    float most = bases[0][mine];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) most = fmaxf(most, bases[i][mine]);
    float sum = 0.0f, o[C] = {};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        const float by = __builtin_amdgcn_exp2f(bases[i][mine] - most);
        sum = fmaf(totals[i][mine], by, sum);
#pragma unroll
        for (int j = 0; j < C; ++j) o[j] = fmaf(sums[i][mine][c0 + j], by, o[j]);
    }
    if (it.pieces == 1) {
        const int r = it.row0 + mine;
        const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
        uint32_t w[C / 2];
#pragma unroll
        for (int j = 0; j < C / 2; ++j) w[j] = kv_round(o[2 * j] * over, BF16) | (uint32_t)kv_round(o[2 * j + 1] * over, BF16) << 16;
        kv_store(a.out.data + (int64_t)(it.s.start + r / a.groups) * a.out.token_stride + (int64_t)(head * a.groups + r % a.groups) * a.out.head_stride + c0, a.out.aligned, w);
    } else {
        const int64_t place = ((int64_t)it.slot * a.c.heads + head) * T + mine;
        float *to = a.partial + place * D + c0;
#pragma unroll
        for (int j = 0; j < C; j += 4) *reinterpret_cast<float4v *>(to + j) = float4v{o[j], o[j + 1], o[j + 2], o[j + 3]};
        if (c0 == 0) {
            float *meta = a.partial + (int64_t)plan.slots * a.c.heads * T * D + place * 2;
            meta[0] = most;
            meta[1] = sum;
        }
    }
}

}  // namespace

hipError_t launch_kv_attention_rows(const KvAttentionArgs &a, const KvPlan &plan, int least, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)plan.slots * a.c.heads)), block(64 * kWaves);
    if (a.c.head_dim == 128) {
        if (a.c.bf16) kv_attention_rows_kernel<128, true><<<grid, block, 0, stream>>>(a, plan, least);
        else kv_attention_rows_kernel<128, false><<<grid, block, 0, stream>>>(a, plan, least);
    } else {
        if (a.c.bf16) kv_attention_rows_kernel<64, true><<<grid, block, 0, stream>>>(a, plan, least);
        else kv_attention_rows_kernel<64, false><<<grid, block, 0, stream>>>(a, plan, least);
    }
    return hipGetLastError();
}

}  // namespace apmm
