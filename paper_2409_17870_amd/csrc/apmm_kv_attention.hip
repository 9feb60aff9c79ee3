// How an attention call over the four-bit cache is cut and launched, and the kernel that joins the pieces of rows whose keys were cut.
#include <algorithm>

#include "apmm_kv_attention.h"

namespace apmm {

hipError_t launch_kv_attention_rows(const KvAttentionArgs &a, const KvPlan &plan, int least, hipStream_t stream);
hipError_t launch_kv_attention_tiles(const KvAttentionArgs &a, const KvPlan &plan, int least, hipStream_t stream);

namespace {

constexpr int kWaves = 4;

// One wave for each row that was cut.  The pieces' sums o_i and totals s_i stand for 2^base_i o_i and 2^base_i s_i: the row is sum 2^(base_i - M) o_i / sum 2^(base_i - M) s_i.
template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves) void kv_attention_join_kernel(KvAttentionArgs a, KvPlan plan, int least)
{
    constexpr int C = D / 64;  // channels of a lane
    const int lane = kv_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int query_heads = a.c.heads * a.groups;
    const int64_t unit = (int64_t)blockIdx.x * kWaves + wave;
    const int token = (int)(unit / query_heads), query_head = (int)(unit % query_heads), head = query_head / a.groups;
    if (token >= a.c.tokens) return;
    const int piece = kv_piece(a, plan, least);
    // the token's sequence and the slots before it
    KvSequence s;
    int b = -1, before = 0;
    for (int from = 0; from < a.c.sequences && b < 0; from += 64) {
        const int at = from + lane;
        int count = 0, start = 0, n = 0;
        if (at < a.c.sequences) {
            int tiles, steps;
            s = kv_sequence(a.c, at);
            kv_extent(a, s, plan.tile, tiles, steps);
            count = tiles * kv_pieces(steps, piece);
            start = s.start;
            n = s.n;
        }
        const int to = kv_scan(count);
        const uint64_t here = __ballot(token >= start && token < start + n);
        if (here) {
            const int l = __ffsll((long long)here) - 1;
            b = __builtin_amdgcn_readfirstlane(from + l);
            before += __builtin_amdgcn_readfirstlane(__shfl(to, l) - __shfl(count, l));
        } else {
            before += __builtin_amdgcn_readfirstlane(__shfl(to, 63));
        }
    }
    if (b < 0) return;
    int tiles, steps;
    s = kv_sequence(a.c, b);
    kv_extent(a, s, plan.tile, tiles, steps);
    const int pieces = kv_pieces(steps, piece);
    if (pieces == 1) return;
    const int row = (token - s.start) * a.groups + query_head % a.groups, tile = row / plan.tile;
    const int64_t slot = before + (int64_t)(tiles - 1 - tile) * pieces;
    if (slot < 0 || slot + pieces > plan.slots) return;  // (starts that are not ascending from 0 to tokens)
    const int64_t place = (slot * a.c.heads + head) * plan.tile + row % plan.tile, step = (int64_t)a.c.heads * plan.tile;
    const float *meta = a.partial + (int64_t)plan.slots * a.c.heads * plan.tile * D, *sums = a.partial + lane * C;
    float most = kLowest, total = 0.0f, o[C] = {};
    for (int from = 0; from < pieces; from += 64) {
        const int here = min(pieces - from, 64);
        float base = kLowest, t = 0.0f;
        if (lane < here) {
            const float2 m = *reinterpret_cast<const float2 *>(meta + (place + (from + lane) * step) * 2);
            base = m.x;
            t = m.y;
        }
        float top = base;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        top = fmaxf(top, most);
        const float old = __builtin_amdgcn_exp2f(most - top), by = __builtin_amdgcn_exp2f(base - top);
        most = top;
        float part = t * by;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) part += __shfl_xor(part, d);
        total = fmaf(total, old, part);
#pragma unroll
        for (int j = 0; j < C; ++j) o[j] *= old;
#pragma unroll 4
        for (int i = 0; i < here; ++i) {
            const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), i));
            const float *from_piece = sums + (place + (from + i) * step) * D;
#pragma unroll
            for (int j = 0; j < C; ++j) o[j] = fmaf(from_piece[j], f, o[j]);
        }
    }
    const float over = total == 0.0f ? 0.0f : 1.0f / total;
    uint16_t *out = a.out.data + (int64_t)token * a.out.token_stride + (int64_t)query_head * a.out.head_stride + lane * C;
#pragma unroll
    for (int j = 0; j < C; ++j) out[j] = kv_round(o[j] * over, BF16);
}

// Fewest steps of a piece: one for each wave of the rows kernel, twice
int least_steps(const KvPlan &plan) { return plan.tile == kRowsTile ? 8 : 16; }

}  // namespace

KvPlan kv_plan(int sequences, int64_t tokens, int heads, int groups, int)
{
    KvPlan p;
    const int64_t rows = tokens * groups;
    p.tile = rows <= 32 * (int64_t)sequences ? kRowsTile : kTilesTile;
    const int64_t tiles = std::min(tokens * ((groups + p.tile - 1) / p.tile), rows / p.tile + sequences);
    const int wanted = p.tile == kRowsTile ? 1024 : 512;
    p.target = tiles * heads >= 4 * wanted ? 0 : std::max(wanted / heads, 1);
    p.slots = (int)(tiles + p.target);
    return p;
}

size_t kv_partial_bytes(const KvPlan &plan, int heads, int head_dim)
{
    return plan.target ? (size_t)plan.slots * heads * plan.tile * (head_dim + 2) * sizeof(float) : 0;
}

hipError_t launch_kv_attention(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream)
{
    const int least = least_steps(plan);
    const hipError_t e = plan.tile == kRowsTile ? launch_kv_attention_rows(a, plan, least, stream) : launch_kv_attention_tiles(a, plan, least, stream);
    if (e != hipSuccess || !plan.target) return e;
    const dim3 grid((uint32_t)(((int64_t)a.c.tokens * a.c.heads * a.groups + kWaves - 1) / kWaves)), block(64 * kWaves);
    if (a.c.head_dim == 128) {
        if (a.c.bf16) kv_attention_join_kernel<128, true><<<grid, block, 0, stream>>>(a, plan, least);
        else kv_attention_join_kernel<128, false><<<grid, block, 0, stream>>>(a, plan, least);
    } else {
        if (a.c.bf16) kv_attention_join_kernel<64, true><<<grid, block, 0, stream>>>(a, plan, least);
        else kv_attention_join_kernel<64, false><<<grid, block, 0, stream>>>(a, plan, least);
    }
    return hipGetLastError();
}

}  // namespace apmm
