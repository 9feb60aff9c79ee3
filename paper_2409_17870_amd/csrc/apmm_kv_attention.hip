// How an attention call over the four-bit cache is cut and launched, and the kernel that joins the pieces of tiles whose keys were cut.
#include <algorithm>

#include "apmm_kv_attention.h"

namespace apmm {

namespace {

// Reads what the pieces wrote, 4 (head_dim + 2) bytes a row and piece; a launch of it takes 4 to 7 us, nearly all of it the launch and the notes' way from memory.
// A workgroup looks at one piece and head and 16 rows of its tile, and has work where the piece is the first of several.  16 lanes to a row; what is left of the 256 for fewer rows shares
// out the pieces, each with its own running base, and meets in LDS.  One launch for both kernels' pieces: those of kv_attention_rows_kernel first.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(KvAttentionArgs a, KvPlan plan, int of_rows)
{
    const bool tiles = (int)blockIdx.x >= of_rows;
    const KvPart &part = tiles ? plan.tiles : plan.rows;
    const int in_tile = tiles ? (int)(blockIdx.x - of_rows) % (kTilesTile / 16) : 0, item = tiles ? (int)(blockIdx.x - of_rows) / (kTilesTile / 16) : blockIdx.x;
    constexpr int C = D / 16;  // channels of a lane
    __shared__ float bases[16][16], totals[16][16];  // by threadIdx.x / 16: share of the pieces, row
    __shared__ __align__(16) float sums[256][C];
    const KvPartial partial = kv_partial(a.partial + (tiles ? plan.tiles_partial : 0), part, a.c.heads, D);
    const KvPieceNote note = partial.note[item];
    const int first_row = in_tile * 16, rows = min(note.rows - first_row, 16);
    if (note.pieces == 0 || rows <= 0) return;
    const int row_slots = rows > 8 ? 16 : rows > 4 ? 8 : rows > 2 ? 4 : rows, shares = 16 / row_slots;
    const int group = threadIdx.x >> 4, row = group % row_slots, share = group / row_slots, c0 = (threadIdx.x & 15) * C;
    const int head = item - kv_divide(item, a.c.by_heads) * a.c.heads;
    float base = kLowest, total = 0.0f, o[C] = {};
    if (row < rows) {
        const int64_t place = (int64_t)item * part.tile + first_row + row, step = (int64_t)a.c.heads * part.tile;
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
            total = kv_moved<BF16>(total, base - top, kv_moved<BF16>(r.y, r.x - top));
            base = top;
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
        total = kv_moved<BF16>(total, base - top, kv_moved<BF16>(totals[other][0], b - top));
        base = top;
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

// How many workgroups one kernel has for sequences of at most `tokens` new tokens in all: `tiles` for a head where nothing is cut.  Nothing is where there are `plenty` anyway.
void cut(KvPart &p, const KvArgs &c, int groups, int window, int sinks, int64_t tiles, int step, int wanted, int plenty)
{
    int64_t most_steps = (((int64_t)c.width << c.page_shift) + step - 1) / step;  // of a sequence, as far as the page table goes
    if (window) most_steps = std::min<int64_t>(most_steps, kv_window_steps(window, sinks, (p.tile + groups - 2) / groups, step));
    p.target = tiles * c.heads >= plenty || most_steps <= p.least ? 0 : std::max(wanted / c.heads, 1);
    p.slots = (int)(tiles + (p.target ? p.target + 1 : 0));
}

int64_t join_groups_of_rows(const KvPlan &plan, int heads) { return plan.rows.target ? (int64_t)plan.rows.slots * heads : 0; }
int64_t join_groups(const KvPlan &plan, int heads)
{
    return join_groups_of_rows(plan, heads) + (plan.tiles.target ? (int64_t)plan.tiles.slots * heads * (kTilesTile / 16) : 0);
}

template <int D, bool BF16>
void join(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream)
{
    const int64_t of_rows = join_groups_of_rows(plan, a.c.heads), groups = join_groups(plan, a.c.heads);
    kv_attention_join_kernel<D, BF16><<<dim3((uint32_t)groups), dim3(256), 0, stream>>>(a, plan, (int)of_rows);
}

}  // namespace

KvPlan kv_plan(const KvArgs &c, int groups, int window, int sinks)
{
    KvPlan p = {};
    const int64_t rows = (int64_t)c.tokens * groups, sequences = std::min(c.sequences, c.tokens);  // (with new tokens)
    // A sequence's rows are as many as the call's where it is the only one: else workgroups of both kinds, but where there are no more tokens than sequences.  That is one token of each as a rule; a
    // batch of many slots without new tokens has its few longer ones in tiles of 16 rows then (500 new tokens of 4000 beside 511 empty slots, 8 heads of 8: 146 us, beside 300 112).
    // Few rows of a sequence go to kv_attention_rows: up to 32, where keys are cut for the sake of enough workgroups; where there are enough a tile reads the keys of 17 to 32 rows once, not twice
    // (20 new ones of 1000 tokens, 32 heads: 8 sequences 18 us with 32 as the border, 28 with 16, 12 27 and 28, 16 33 and 28, 40 74 and 50; 7 tokens of 4 query heads, 8 heads, sequences of 2000:
    // 48 44 and 45, 64 52 and 48; 30 rows of one of 56000: 36 and 48.  Longer contexts cross earlier: 30 rows of 2 sequences of 8000, 32 heads, 52 and 36)
    const int few_rows = sequences * c.heads >= 512 ? 16 : 32;
    const bool few = rows <= few_rows || c.tokens <= c.sequences, many = !few && c.sequences == 1;
    auto tiles = [&](int tile) { return std::min(c.tokens * (int64_t)((groups + tile - 1) / tile), rows / tile + sequences); };
    if (!many) {
        p.rows.tile = kRowsTile;
        p.rows.to_rows = few ? INT32_MAX : few_rows;
        const int64_t most = std::min(tiles(kRowsTile), few ? INT64_MAX : sequences * (few_rows / kRowsTile));
        const int64_t groups_of = sequences * c.heads * ((std::min<int64_t>(groups, rows) + kRowsTile - 1) / kRowsTile);
        p.rows.waves = !few || groups_of >= 512 ? 4 : 8;
        // Few workgroups (less than two for each compute unit): eight waves, one workgroup to a unit at a time, pieces for one round.  Else four waves, three workgroups to a unit.
        // (8 x 65536 tokens, 8 heads: 102 us in one round of 256, 106 in 512; 32 sequences of up to 4096, 40 heads: 73 us with 2048 wanted, 75 with 768 and 77 with 1536.)  Shorter
        // pieces do not pay for the join: 1203 tokens uncut 11 us, in pieces of 32 steps 15.  Beside tiles, which take longer, there is time for longer ones.
        p.rows.least = !few ? 128 : p.rows.waves == 4 ? 64 : 48;
        const int wanted = p.rows.waves == 4 ? 2048 : 256;
        cut(p.rows, c, groups, window, sinks, most, kRowsStep, wanted, 4 * wanted);
    }
    if (!few) {
        p.tiles.tile = kTilesTile;
        p.tiles.from_rows = many ? 0 : few_rows + 1;
        p.tiles.to_rows = INT32_MAX;
        // Two workgroups of two tiles to a compute unit at a time.  A piece costs its beginning (5 us) and 32 KiB written and read, so no more of them than fit at once, 1024: with twice as many a
        // batch of 5 pieces of prompts took 5 % longer and a prompt of 2048 tokens 20 %, with three quarters the batch 10 %.  Pieces of 32 steps at least: 1000 tokens 36 us, with 16 46.
        // How many are enough without cutting.  Tiles of one sequence are enough where more than one workgroup of two comes to a compute unit; from there on cutting is the join's 4 to 7 us more
        // (prompts of 4096 tokens: 520 tiles 93 us uncut and 71 cut, 585 90 and 94, 2080 151 and 158; 500 new tokens of 8000: 512 170 and 156, 528 235 and 240).  Those of several sequences may be
        // few long ones among short ones (60 prompts of 64 tokens and 64 new ones of 8000, 3904 tiles: 188 us uncut, 71 cut), which cutting loses 2 to 5 % for where all are alike (8 pieces of 500
        // behind 4000 tokens: 269 and 276); the line is there for the workspace, 136 MB at 4096 tiles of 128 channels.  A window of up to 80 steps bounds what the long ones cost (window 2048: 2 pieces
        // of 1000, 1016 tiles, 80 us uncut and 85 cut; 14 prompts of 64 and 64 new of 9000, 960 tiles, 53 and 36; window 4096: 150 and 154, 96 and 39).
        p.tiles.least = 32;
        // Two workgroups run on each of the 256 compute units at a time, and the second set comes to them in the order of the first: shortest of these first, each unit gets one long and one
        // short pair of tiles and all are done with both at about the same time (2048 tokens of 32 heads: 72.9 us without, 69.5 so; 4096: 199 and 191; from 8192 on no difference).
        p.tiles.turn = many ? 512 / c.heads : 0;
        const bool short_window = window && kv_window_steps(window, sinks, (kTilesTile + groups - 2) / groups, kTilesStep) <= 80;
        cut(p.tiles, c, groups, window, sinks, tiles(kTilesTile), kTilesStep, 1024, many ? 576 : short_window ? 896 : 4096);
    }
    p.tiles_partial = (int64_t)(kv_partial_bytes(p.rows, c.heads, c.head_dim) / sizeof(float));
    return p;
}

size_t kv_partial_bytes(const KvPart &part, int heads, int head_dim)
{
    if (!part.tile || !part.target) return 0;
    const KvPartial p = kv_partial(nullptr, part, heads, head_dim);
    return reinterpret_cast<size_t>(p.note + (int64_t)part.slots * heads);
}

int64_t kv_attention_items(const KvPlan &plan, int heads)
{
    const int64_t rows = plan.rows.tile ? (int64_t)plan.rows.slots * heads : 0;
    const int64_t first = plan.tiles.tile ? (kv_tiles_groups(plan.tiles, heads) + rows) * 256 : rows * 64 * plan.rows.waves;
    return std::max(first, join_groups(plan, heads) * 256);
}

hipError_t launch_kv_attention(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream)
{
    const hipError_t e = plan.tiles.tile ? launch_kv_attention_tiles(a, plan, stream) : launch_kv_attention_rows(a, plan.rows, stream);
    if (e != hipSuccess) return e;
    if (plan.rows.target || plan.tiles.target) {
        if (a.c.head_dim == 128) a.c.bf16 ? join<128, true>(a, plan, stream) : join<128, false>(a, plan, stream);
        else a.c.bf16 ? join<64, true>(a, plan, stream) : join<64, false>(a, plan, stream);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace apmm
