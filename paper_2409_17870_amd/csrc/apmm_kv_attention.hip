// How an attention call over the four-bit cache is cut and launched, and the kernel that joins the pieces of tiles whose keys were cut.
#include <algorithm>

#include "apmm_kv_attention.h"

namespace apmm {

namespace {

constexpr int kFewRows = 32;  // of a sequence: those go to kv_attention_rows_kernel

// A workgroup looks at one piece and head (blockIdx.x) and 16 rows of its tile (blockIdx.y), and has work where the piece is the first of several.  16 lanes to a row; what is left of
// the 256 for fewer rows shares out the pieces, each with its own running base, and meets in LDS.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(KvAttentionArgs a, KvPart part)
{
    constexpr int C = D / 16;  // channels of a lane
    __shared__ float bases[16][16], totals[16][16];  // by threadIdx.x / 16: share of the pieces, row
    __shared__ __align__(16) float sums[256][C];
    const KvPartial partial = kv_partial(a.partial, part, a.c.heads, D);
    const KvPieceNote note = partial.note[blockIdx.x];
    const int first_row = blockIdx.y * 16, rows = min(note.rows - first_row, 16);
    if (note.pieces == 0 || rows <= 0) return;
    const int row_slots = rows > 8 ? 16 : rows > 4 ? 8 : rows > 2 ? 4 : rows, shares = 16 / row_slots;
    const int group = threadIdx.x >> 4, row = group % row_slots, share = group / row_slots, c0 = (threadIdx.x & 15) * C;
    const int head = blockIdx.x - kv_divide(blockIdx.x, a.by_heads) * a.c.heads;
    float base = kLowest, total = 0.0f, o[C] = {};
    if (row < rows) {
        const int64_t place = (int64_t)blockIdx.x * part.tile + first_row + row, step = (int64_t)a.c.heads * part.tile;
#pragma unroll 4
        for (int i = share; i < note.pieces; i += shares) {
            const int64_t at = place + i * step;
            const float2 r = partial.row[at];
            float x[C];
#pragma unroll
            for (int j = 0; j < C; j += 4) {
                const float4v v = *reinterpret_cast<const float4v *>(partial.sums + at * D + c0 + j);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[j + k] = v[k];
            }
            const float top = fmaxf(base, r.x), old = __builtin_amdgcn_exp2f(base - top), by = __builtin_amdgcn_exp2f(r.x - top);
            base = top;
            total = fmaf(total, old, r.y * by);
#pragma unroll
            for (int j = 0; j < C; ++j) o[j] = fmaf(o[j], old, x[j] * by);
        }
    }
    bases[group][0] = base;
    totals[group][0] = total;
#pragma unroll
    for (int j = 0; j < C; ++j) sums[threadIdx.x][j] = o[j];
    __syncthreads();
    if (share || row >= rows) return;
    for (int i = 1; i < shares; ++i) {
        const int other = group + i * row_slots;
        const float b = bases[other][0], top = fmaxf(base, b), old = __builtin_amdgcn_exp2f(base - top), by = __builtin_amdgcn_exp2f(b - top);
        base = top;
        total = fmaf(total, old, totals[other][0] * by);
#pragma unroll
        for (int j = 0; j < C; ++j) o[j] = fmaf(o[j], old, sums[threadIdx.x + 16 * i * row_slots][j] * by);
    }
    const float over = total == 0.0f ? 0.0f : 1.0f / total;
    uint32_t w[C / 2];
#pragma unroll
    for (int j = 0; j < C / 2; ++j) w[j] = kv_round(o[2 * j] * over, BF16) | (uint32_t)kv_round(o[2 * j + 1] * over, BF16) << 16;
    const int r = note.row0 + first_row + row, at = kv_divide(r, a.by_groups);
    kv_store(a.out.data + (int64_t)(note.start + at) * a.out.token_stride + (int64_t)(head * a.groups + r - at * a.groups) * a.out.head_stride + c0, a.out.aligned, w);
}

}  // namespace

namespace {

// The workgroups of one kernel for sequences of at most `tokens` new tokens in all
void cut(KvPart &p, const KvArgs &c, int groups, int step, int wanted)
{
    const int64_t rows = (int64_t)c.tokens * groups;
    const int64_t tiles = std::min<int64_t>((int64_t)c.tokens * ((groups + p.tile - 1) / p.tile), rows / p.tile + c.sequences);
    const int64_t most_steps = (((int64_t)c.width << c.page_shift) + step - 1) / step;  // of a sequence, as far as the page table goes
    p.target = tiles * c.heads >= 4 * (int64_t)wanted || most_steps <= p.least ? 0 : std::max(wanted / c.heads, 1);
    p.over_target = p.target ? 1.0f / p.target : 0.0f;
    p.slots = (int)(tiles + (p.target ? p.target + 1 : 0));
}

template <int D, bool BF16>
void join(const KvAttentionArgs &a, const KvPart &part, hipStream_t stream)
{
    kv_attention_join_kernel<D, BF16><<<dim3((uint32_t)((int64_t)part.slots * a.c.heads), part.tile / 16), dim3(256), 0, stream>>>(a, part);
}

}  // namespace

KvPlan kv_plan(const KvArgs &c, int groups)
{
    KvPlan p = {};
    const int64_t rows = (int64_t)c.tokens * groups;
    // A sequence's rows are as many as the call's where it is the only one, and no more than one token's where there is no other: else both kernels are launched
    const bool few = rows <= kFewRows || c.tokens <= c.sequences, many = !few && c.sequences == 1;
    if (!many) {
        p.rows.tile = kRowsTile;
        p.rows.to_rows = few ? INT32_MAX : kFewRows;
        const int64_t groups_of = std::min<int64_t>((int64_t)c.sequences, c.tokens) * c.heads * ((std::min<int64_t>(groups, rows) + kRowsTile - 1) / kRowsTile);
        p.rows.waves = groups_of >= 512 ? 4 : 8;
        p.rows.least = 64;
        cut(p.rows, c, groups, kRowsStep, p.rows.waves == 4 ? 2048 : 256);
    }
    if (!few) {
        p.tiles.tile = kTilesTile;
        p.tiles.waves = 4;
        p.tiles.from_rows = many ? 0 : kFewRows + 1;
        p.tiles.to_rows = INT32_MAX;
        p.tiles.least = 16;
        cut(p.tiles, c, groups, kTilesStep, 512);
    }
    return p;
}

size_t kv_partial_bytes(const KvPart &part, int heads, int head_dim)
{
    if (!part.tile || !part.target) return 0;
    const KvPartial p = kv_partial(nullptr, part, heads, head_dim);
    return reinterpret_cast<size_t>(p.note + (int64_t)part.slots * heads);
}

hipError_t launch_kv_attention(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream)
{
    KvAttentionArgs b = a;
    for (const KvPart *part : {&plan.rows, &plan.tiles}) {
        if (!part->tile) continue;
        const hipError_t e = part == &plan.rows ? launch_kv_attention_rows(b, *part, stream) : launch_kv_attention_tiles(b, *part, stream);
        if (e != hipSuccess) return e;
        if (part->target) {
            if (a.c.head_dim == 128) a.c.bf16 ? join<128, true>(b, *part, stream) : join<128, false>(b, *part, stream);
            else a.c.bf16 ? join<64, true>(b, *part, stream) : join<64, false>(b, *part, stream);
            const hipError_t j = hipGetLastError();
            if (j != hipSuccess) return j;
        }
        b.partial += kv_partial_bytes(*part, a.c.heads, a.c.head_dim) / sizeof(float);
    }
    return hipSuccess;
}

}  // namespace apmm
