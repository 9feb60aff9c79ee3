// Attention of many rows over the four-bit cache (apmm_kv_attention.h): prompts and pieces of prompts.
//
// A workgroup has two tiles of 64 rows of a head, 32 rows to each of its four waves, which go through the keys by themselves in steps of 32 with matrix instructions 32 x 32 x 16: codes come
// from memory (L1 and L2: the waves and the workgroups of a head read the same) into registers and become operands there, no barrier anywhere.  (One tile of 128 rows leaves two waves idle
// where a sequence has 33 to 64: 30 sequences of 4000 tokens with 50 new ones, 32 heads, 280 us in place of 200; long prompts take the same time.  Workgroups of one tile of 64: 5 % longer.)  Only the scales, which lanes need sixteen of, go through a little LDS of the wave.
// (Operands made once for the workgroup and shared through LDS save three quarters of the unpacking, and lost more than that in barriers: 280 us where this takes 190.)
//
// What bounds it is the vector unit, then the power of the card: of a step's about 200 instructions 80 unpack codes and 96 are the weights of 16 keys a lane (product with the key's scale and
// exponent in one, power, sum, product with the value's scale and rounding, sum of the rounded ones), beside 16 matrix instructions that take half as long.  Hence
//   - the factor of a query's row is the same for the 32 of a wave in nearly all calls and goes into the keys' scales, one product a lane instead of one a key and row;
//   - a step that has no hidden keys does not look for the maximum of its scores: its sums tell afterwards whether a weight was too large for the running maximum.
// Every other step (the first, those at the diagonal and at the window's edge, those whose sums are too large, all of a wave whose queries differ by 2^10, all behind a value scale of 2^64) goes
// the general way.
// 16384 tokens of 32 heads of 128, binary16: 2.26 ms, 972 TFLOP/s; 4096 tokens: 191 us, 720 TFLOP/s (the vector units issue for 65 % of the kernel, for 76 % of the time that a compute unit
// has work; the rest is the uneven end).  8192-cubed products of a library reach 1194 TFLOP/s here.
#include "apmm_kv_attention_rows.h"

namespace apmm {

namespace {

constexpr int kWaves = 4, kRows = 32, kTileWaves = kTilesTile / kRows;

// SMALL: pages of 16 keys, two to a step
template <int D, bool BF16, bool SMALL>
__device__ __forceinline__ void kv_attention_tiles(const KvAttentionArgs &a, const KvPart &part, float *partials, int block_id)
{
    constexpr int W = D / 16, E = D / 32;  // words of a lane's key, blocks of 32 channels of the result
    __shared__ __align__(16) float scales[kWaves][64];  // of a step: keys, values
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tile_wave = wave % kTileWaves, lane = kv_lane(), n = lane & 31, h = lane >> 5;
    const int at_block = kv_divide(block_id, a.c.by_heads), slot = at_block * (kWaves / kTileWaves) + wave / kTileWaves, head = block_id - at_block * a.c.heads;
    if (slot >= part.slots) return;
    KvItem<kTilesStep> it;
    const bool there = kv_item<kTilesStep, kTilesTile>(a, part, slot, it);
    kv_note(a, part, partials, slot, head, there, it, tile_wave == 0 && lane == 0);
    if (!there) return;

    const int row0 = it.row0 + tile_wave * kRows, rows = min(it.rows - tile_wave * kRows, kRows);
    if (rows <= 0) return;
    const int row = row0 + min(n, rows - 1), at = kv_divide(row, a.by_groups);
    const int pos = it.s.first + at, first_pos = it.s.first + kv_divide(row0, a.by_groups), last_pos = it.s.first + kv_divide(row0 + rows - 1, a.by_groups);
    auto over_row = [](float v, auto f) { return f(v, __shfl_xor(v, 32)); };
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto plus = [](float x, float y) { return x + y; };

    // the steps of this wave: those of the workgroup's up to its last query (a workgroup's window begins with its first wave: the others' steps before theirs are few)
    const int ends = last_pos < 0 ? 0 : last_pos / kTilesStep + 1;
    const int to = min(it.to, ends <= it.sink_steps ? ends : max(ends - it.gap, it.sink_steps));
    int t = it.from;

    // Where a step's codes and scales are.  Operand row 8 i + 4 h' + j of the keys is key 16 h' + 4 i + j; half h of the values' operand s has keys 16 h + 8 s to 16 h + 8 s + 7.
    const int shift = a.c.page_shift, mask = (1 << shift) - 1;
    const int64_t page_scales = (int64_t)a.c.heads << (shift + 2), page_codes = page_scales / 4 * D;  // bytes of a page (a scale is 2 for D / 2 of codes)
    const uint8_t *const codes_head = a.c.codes + (((int64_t)head * D) << shift), *const scales_head = reinterpret_cast<const uint8_t *>(a.c.scales) + ((int64_t)head << (shift + 2));
    const bool key_half = n & 4;
    const uint32_t key_lane = (uint32_t)(4 * (n >> 3) + (n & 3) + (!SMALL && key_half ? 16 : 0)) * (D / 2) + h * (D / 4);
    const uint32_t value_lane = (uint32_t)(n & (D / 4 - 1)) * 16 + ((uint32_t)(D / 2) << shift) + (!SMALL ? h * 8 * D : 0);
    const uint32_t scale_lane = ((uint32_t)(lane & (SMALL ? 15 : 31)) + (h ? 1u << shift : 0u)) * 2;
    struct Place {
        const uint8_t *codes, *scales;
        int64_t codes_on, scales_on;  // in small pages: from there to the second half of the step
    };
    auto place_of = [&](int t, int ids, int i) {  // lanes 2 i and 2 i + 1 of ids are its pages
        Place p = {};
        const int key = it.key_of(t), page = max(__builtin_amdgcn_readlane(ids, 2 * i), 0), in = key & mask;
        p.codes = codes_head + page * page_codes + in * (D / 2);
        p.scales = scales_head + page * page_scales + in * 2;
        if (SMALL) {
            const int page1 = max(__builtin_amdgcn_readlane(ids, 2 * i + 1), 0), in1 = (key + 16) & mask;
            p.codes_on = (page1 - page) * page_codes + (in1 - in) * (D / 2);
            p.scales_on = (page1 - page) * page_scales + (in1 - in) * 2;
        }
        return p;
    };
    auto load_keys = [&](const Place &p, uint4 (&k)[D / 64]) {
        const uint8_t *from = p.codes + (SMALL && key_half ? p.codes_on : 0) + key_lane;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) k[i] = reinterpret_cast<const uint4 *>(from)[i];
    };
    auto load_values = [&](const Place &p, uint4 (&v)[2]) {
        const uint8_t *from = p.codes + (SMALL && h ? p.codes_on : 0) + value_lane;
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const uint4 *>(from + i * (D * 4));
    };
    auto load_scales = [&](const Place &p) -> uint32_t { return *reinterpret_cast<const uint16_t *>(p.scales + (SMALL && (lane & 16) ? p.scales_on : 0) + scale_lane); };
    // Wherever a step begins, keys, scales and values have been asked for in this order: the wait for the keys is none for the values
    auto in_order = [] { __builtin_amdgcn_sched_barrier(0); };
    // Pages of steps t to t + 31, and whether one of their keys has none
    auto pages_from = [&](int t, bool &bad) {
        const int ids = kv_page_ids(a, it, t, 1), step = t + (lane >> 1);
        bad = __any(ids < 0 && step < it.to && it.key_of(step) + 16 * (lane & 1) < it.s.keys);
        return ids;
    };

    // The rows of a wave share the factor of its largest query unless some row's are so small (2^-10 of that) that they would lose bits of it
    bool one_factor;
    half8 q[W];
    float init, factor;
    uint4 k[D / 64] = {}, v[2] = {};  // of step t, on their way
    uint32_t scale = 0;
    int ids;              // pages of the 32 steps behind `block`
    int block = t;
    const int begin = t;
    bool bad, bad_before; // whether keys of those, of the 32 up to `block`, have none
    {
        uint32_t x[4 * W];
        kv_load(a.q.data + (int64_t)(it.s.start + at) * a.q.token_stride + (int64_t)(head * a.groups + row - at * a.groups) * a.q.head_stride + h * (D / 2), a.q.aligned, x);
        const Place here = place_of(t, pages_from(t, bad_before), 0);
        ids = pages_from(t + 1, bad);
        if (t < to) {
            load_keys(here, k);
            in_order();
            scale = load_scales(here);
            in_order();
            load_values(here, v);
            in_order();
        }
        kv_queries<4 * W, BF16>(x, a.scale, [&](float v) {
            v = over_row(v, larger);
            float all = v;
#pragma unroll
            for (int i = 1; i < 32; i *= 2) all = fmaxf(all, __shfl_xor(all, i));
            one_factor = !__any(v > 0.0f && v < 0x1p-10f * all);
            return one_factor ? all : v;
        }, [&](float v) { return over_row(v, plus); }, q, init, factor);
    }

    const float scale_by = h ? 1.0f : factor;  // of the scale that a lane loads: a key's or a value's

    float16v acc[E], init16;
#pragma unroll
    for (int i = 0; i < 16; ++i) init16[i] = init;
    asm volatile("" : "+v"(init16));  // stays in registers: made anew it would be 16 moves a step
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[e][i] = 0.0f;
    float top = kLowest, base = -kLowest, total = 0.0f, weights = 0.0f;
    float met = 0.0f, limit = 0.0f, most = 0.0f;  // largest scale of values that the row has met, the power of two above it; largest sum that a step may add

    bool large = false;  // whether some row's E is more than kMostExponent
    auto exponent_of = [](float s) { return max((int)(__float_as_uint(s) >> 23) - 126, -80); };  // E: 2^E above s, from -80 (sums of 2^(2 - E) stay in range; scales below 2^-96 lose bits)

    auto scores = [&]() {
        float16v s = init16;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint4 x = k[i / 4];
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kv_operand(i % 4 == 0 ? x.x : i % 4 == 1 ? x.y : i % 4 == 2 ? x.z : x.w), q[i], s, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        return s;
    };
    auto add = [&](const uint32_t (&w)[8]) {
#pragma unroll
        for (int i = 0; i < 2 * E; ++i) {
            const int j = i / E, e = i % E;
            uint32_t c[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (D == 64) c[x] >>= 8 * (n >> 4);  // operand rows 16 and up: channels 4 m + 2 and 4 m + 3
                if (e & 2) c[x] >>= 8;
                c[x] &= e & 1 ? 0x00f000f0u : 0x000f000fu;
            }
            acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, make_uint4(c[0], c[1], c[2], c[3])),
                                                            __builtin_bit_cast(half8, make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3])), acc[e], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto weigh = [&](int i, float x0, float by0, float x1, float by1, const float (&vs)[16], uint32_t (&w)[8], float &sum, float &weight_sum) {  // two keys
        const float p0 = __builtin_amdgcn_exp2f(fmaf(x0, by0, base)), p1 = __builtin_amdgcn_exp2f(fmaf(x1, by1, base));
        sum += p0 + p1;
        const half2v pair = {(_Float16)(p0 * vs[2 * i]), (_Float16)(p1 * vs[2 * i + 1])};
        w[i] = __builtin_bit_cast(uint32_t, pair);
        weight_sum = __builtin_amdgcn_fdot2(pair, (half2v){1, 1}, weight_sum, false);
    };
    auto take_scales = [&](float own, float (&ks)[16], float (&vs)[16]) {
        scales[wave][lane] = own;
        kv_wave_fence();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4v x = *reinterpret_cast<const float4v *>(&scales[wave][16 * h + 4 * i]), y = *reinterpret_cast<const float4v *>(&scales[wave][32 + 16 * h + 4 * i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                ks[4 * i + j] = x[j];
                vs[4 * i + j] = y[j];
            }
        }
        kv_wave_fence();
    };
    // Steps from t on that every row of the wave sees all keys of, as far as the places of keys go
    auto plain_until = [&]() {
        const int key0 = it.key_of(t);
        if (key0 + 32 > it.s.keys || key0 + 31 > first_pos || t == begin) return t;
        if (a.window && key0 <= last_pos - a.window) return min(min(it.sink_steps, a.sinks / 32), it.s.keys / 32);  // (the last of these may end behind the page table)
        return min(it.s.keys, first_pos + 1) / 32 - it.gap;
    };

    while (t < to) {
        if (t == block + 32) {
            block = t;
            bad_before = bad;
            ids = pages_from(t + 1, bad);
        }
        const int stop = __builtin_amdgcn_readfirstlane(bad || bad_before || !one_factor || large ? t : min(min(plain_until(), block + 32), to));
        bool again = false;
        if (t < stop) __builtin_amdgcn_s_waitcnt(0x0f70);  // nothing under way here, so that in the loop only its own loads are waited for, and each where it is needed
        while (t < stop && !again) {
            float ks[16], vs[16];
            const float own = kv_scale_value(scale, BF16) * scale_by;
            take_scales(own, ks, vs);
            const float16v s = scores();
            const Place next = place_of(min(t + 1, to - 1), ids, max(min(t + 1, to - 1) - block - 1, 0));
            load_keys(next, k);
            in_order();
            scale = load_scales(next);
            in_order();
            float sum = 0.0f, weight_sum = 0.0f;
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) weigh(i, s[2 * i], ks[2 * i], s[2 * i + 1], ks[2 * i + 1], vs, w, sum, weight_sum);
            again = __any((sum > most) | (weight_sum > 60000.0f) | (own > -kLowest));
            if (!again) {
                total += sum;
                weights += weight_sum;
                add(w);
            }
            load_values(next, v);
            in_order();
            ++t;
        }
        if (again) {  // back to the step
            --t;
            const Place here = place_of(t, t == block ? kv_page_ids(a, it, t, 1) : ids, t == block ? 0 : t - block - 1);
            load_keys(here, k);
            in_order();
            scale = load_scales(here);
            in_order();
            load_values(here, v);
            in_order();
        } else if (t == to || t == block + 32) {
            continue;
        }
        // step t in general
        float ks[16], vs[16];
        take_scales(kv_scale_value(scale, BF16), ks, vs);
        const float16v s = scores();
        const Place next = place_of(min(t + 1, to - 1), ids, max(min(t + 1, to - 1) - block - 1, 0));
        load_keys(next, k);
        in_order();
        scale = load_scales(next);
        in_order();
        const int first = it.key_of(t) + 16 * h;
        int end = min(it.s.keys, pos + 1);
        if ((bad || bad_before) && first < it.s.keys) {
            const int page = a.c.table[it.b * a.c.table_stride + (first >> shift)];
            if (page < 0 || page >= a.c.pages) end = 0;
        }
        float x[16], high = -__builtin_inff(), largest = met;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int key = first + i;
            const bool hidden = (key >= end) | ((a.window != 0) & (key <= pos - a.window) & (key >= a.sinks));
            x[i] = hidden ? -__builtin_inff() : s[i] * ks[i];
            vs[i] = hidden ? 0.0f : vs[i];  // weights of hidden keys are zero whatever their scale is
            high = fmaxf(high, x[i]);
            largest = fmaxf(largest, vs[i] <= -kLowest ? vs[i] : 0.0f);
        }
        high *= factor;
        if (__any((high > top + kSlack) | (largest > limit))) {
            top = fmaxf(top, over_row(high, larger));
            const int before = kv_rest(exponent_of(met));
            met = over_row(largest, larger);
            const int e = exponent_of(met);
            limit = ldexpf(1.0f, e);
            const float moved = -top + (kRoom - (float)min(e, kMostExponent));
            float by = __builtin_amdgcn_exp2f(moved - base);
            total = kv_moved<BF16>(total, moved - base);
            base = moved;
            most = ldexpf(1.0f, (int)(kRoom + kSlack) - min(e, kMostExponent));
            if (BF16) {
                by *= ldexpf(1.0f, before - kv_rest(e));
                large = __any(e > kMostExponent);
            }
            weights *= by;
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[e][i] *= by;
        }
        if (BF16 && large) {
            const float by = ldexpf(1.0f, -kv_rest(exponent_of(met)));
#pragma unroll
            for (int i = 0; i < 16; ++i) vs[i] *= by;
        }
        float sum = 0.0f, weight_sum = 0.0f;
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) weigh(i, x[2 * i], factor, x[2 * i + 1], factor, vs, w, sum, weight_sum);
        total += sum;
        weights += weight_sum;
        add(w);
        load_values(next, v);
        in_order();
        ++t;
    }

    // row n's channels of this lane, 16 at a time: 32 i + 16 h + 4 j + e of acc[e][4 i + j] (64 channels: 32 i + 16 h + 4 j + e of acc[e & 1][4 (i + (e & 2)) + j])
    total = over_row(total, plus);
    weights = over_row(weights, plus);
    if (n >= rows) return;
    const bool whole = it.pieces == 1;
    const float over = whole ? (total == 0.0f ? 0.0f : 1.0f / total) : 1.0f, lift = BF16 ? ldexpf(1.0f, kv_rest(exponent_of(met))) : 1.0f;
    uint16_t *out = a.out.data + (int64_t)(it.s.start + at) * a.out.token_stride + (int64_t)(head * a.groups + row - at * a.groups) * a.out.head_stride;
    const int64_t place = ((int64_t)slot * a.c.heads + head) * kTilesTile + tile_wave * kRows + n;
    const KvPartial partial = kv_partial(partials, part, a.c.heads, D);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        float o[16];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = D == 128 ? acc[e & (E - 1)][4 * i + j] : acc[e & 1][4 * ((i + (e & 2)) & 3) + j];
                o[4 * j + e] = fmaf(x, e & 1 ? 0x1p21f : 0x1p25f, -15.0f * weights) * lift * over;
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

// Workgroups of both kinds in one launch: those of tiles first, which take long; those of sequences with few rows come in where the others leave room (two launches one after the other took
// 15 us more of a batch of 5 pieces of prompts and 19 sequences with a new token each, 3000 tokens at most).
template <int D, bool BF16, bool SMALL>
__global__ __launch_bounds__(64 * kWaves, 2) void kv_attention_tiles_kernel(KvAttentionArgs a, KvPlan plan, int of_tiles)
{
    if ((int)blockIdx.x < of_tiles) kv_attention_tiles<D, BF16, SMALL>(a, plan.tiles, a.partial + plan.tiles_partial, blockIdx.x);
    else kv_attention_rows<D, BF16, kWaves>(a, plan.rows, blockIdx.x - of_tiles);
}

template <int D, bool BF16>
void launch(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream)
{
    static_assert(kWaves / kTileWaves == 2 && kWaves == 4, "two tiles to a workgroup of 256 lanes");
    const int of_tiles = (int)kv_tiles_groups(plan.tiles, a.c.heads), of_rows = plan.rows.tile ? plan.rows.slots * a.c.heads : 0;
    const dim3 grid((uint32_t)(of_tiles + of_rows)), block(64 * kWaves);
    if (a.c.page_shift == 4) kv_attention_tiles_kernel<D, BF16, true><<<grid, block, 0, stream>>>(a, plan, of_tiles);
    else kv_attention_tiles_kernel<D, BF16, false><<<grid, block, 0, stream>>>(a, plan, of_tiles);
}

}  // namespace

hipError_t launch_kv_attention_tiles(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream)
{
    if (a.c.head_dim == 128) a.c.bf16 ? launch<128, true>(a, plan, stream) : launch<128, false>(a, plan, stream);
    else a.c.bf16 ? launch<64, true>(a, plan, stream) : launch<64, false>(a, plan, stream);
    return hipGetLastError();
}

}  // namespace apmm
