// What the kernels that write rows into the four-bit key/value cache and read them share: the eights of positions that waves take, and the quantisation of a row.
//
// A row x (head_dim numbers of a token and head) becomes s = max |x| / 15 rounded to its type and codes u = clamp(floor(x / (2 s)) + 8, 0, 15): the nearest odd
// multiple 2 u - 15 of s, ties upward, as apmm_quantize_pack_activations has it.
#pragma once
#include <algorithm>
#include <type_traits>

#include "apmm_kv.h"

namespace apmm {

// The most eights that `tokens` new ones can touch: n tokens of a sequence lie in n of them at most, and in (n + 14) / 8
inline int64_t kv_eights(const KvArgs &c) { return std::min<int64_t>(c.tokens, c.tokens / 8 + 2 * (int64_t)c.sequences); }

#ifdef __HIPCC__
struct Eight {  // of one wave
    KvSequence s;
    int first, in_page;        // position of its first token (a multiple of eight, may be negative), its place in the page
    int page;                  // -1: none
    bool is_new;               // this lane's token is one of the call's
    bool whole;                // all eight are
};

// Eight `eight` of the call; false: there are fewer
__device__ __forceinline__ bool find_eight(const KvArgs &c, int eight, Eight &e)
{
    int b, rest;
    auto count = [&](int at) {
        const KvSequence s = kv_sequence(c, at);
        return s.n ? ((s.first + s.n - 1) >> 3) - (s.first >> 3) + 1 : 0;
    };
    if (!kv_find(c.sequences, eight, b, rest, count)) return false;
    e.s = kv_sequence(c, b);
    e.first = ((e.s.first >> 3) + rest) * 8;
    e.page = e.first >= 0 && e.first < e.s.keys ? c.table[b * c.table_stride + (e.first >> c.page_shift)] : -1;
    if (e.page >= c.pages) e.page = -1;
    e.in_page = e.first & ((1 << c.page_shift) - 1);
    const int at = e.first + (kv_lane() >> 3), end = e.s.first + e.s.n;
    e.is_new = at >= e.s.first && at < end;
    e.whole = e.first >= e.s.first && e.first + 8 <= end;
    return true;
}

// A lane's channels: eight that follow each other, and with head_dim 128 eight more 64 behind them, so that eight lanes move 128 bytes at a time
template <int N>
__device__ __forceinline__ void load_row(const uint16_t *row, bool aligned, int part, uint32_t (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        uint32_t w[4];
        kv_load(row + 64 * i + 8 * part, aligned, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = w[j];
    }
}
template <int N>
__device__ __forceinline__ void store_row(uint16_t *row, bool aligned, int part, const uint32_t (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint32_t w[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
        kv_store(row + 64 * i + 8 * part, aligned, w);
    }
}

// The i-th four of a lane's channels among all of them
__device__ __forceinline__ int four_of(int part, int i) { return i / 2 * 16 + part * 2 + (i & 1); }

// Largest of the eight lanes of a token
__device__ __forceinline__ uint32_t max_over_eight(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));   // lanes 1, 0, 3, 2 of four
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));   // lanes 2, 3, 0, 1
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));  // eight lanes mirrored
}

__device__ __forceinline__ int floor_of(float x)
{
    int i;
    asm("v_cvt_flr_i32_f32 %0, %1" : "=v"(i) : "v"(x));  // (0 for NaN)
    return i;
}

// Scale bits and the codes of a lane's channels, eight to a word, channel order from the low bits
template <int N, bool BF16>
__device__ __forceinline__ uint32_t quantise(const uint32_t (&x)[N], uint32_t (&u)[N / 4])
{
    uint32_t top2 = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top2 = kv_fold_max(top2, x[i] & 0x7fff7fffu);  // |x| orders like its bit pattern
    const uint32_t top = max_over_eight(max(top2 & 0xffffu, top2 >> 16));
    constexpr uint32_t kInfinity = BF16 ? 0x7f80u : 0x7c00u;
    uint32_t scale = kv_round(kv_scale_value(top, BF16) / 15.0f, BF16);
    if (top >= kInfinity) scale = kInfinity | (kInfinity >> 1);  // a number that is not finite: no scale, the row reads back as NaN
    const float s = kv_scale_value(scale, BF16);
    const bool small = s < (BF16 ? 0x1p-64f : 0x1p-18f);  // 1 / s could leave the range, or s has been rounded by so much that |t| passes 8
    const bool large = BF16 && s > 0x1p15f;               // the smallest numbers could become zero
    const float by = BF16 && small ? 0x1p64f : 1.0f, r = 0.5f / (s * by);
    // t = x / (2 s) up to 2^-23 of itself.  What is not an integer is 2^-12 from every one but zero (numbers of 11 bits and |t| <= 8, or a few bits and |t| <= 12), so moving t up by
    // 2^-21 |t| gives the floor of the exact quotient.  Codes less 8, which the sum puts on all eight of a word.
    auto codes = [&](auto general) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            uint32_t w = 0x88888888u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t bits = j & 1 ? x[4 * i + j / 2] >> 16 : x[4 * i + j / 2] & 0xffffu;
                const float v = kv_scale_value(bits, BF16), t = (general ? v * by : v) * r;
                int code = floor_of(fmaf(fabsf(t), 0x1p-21f, t));
                if (general) {
                    code = min(max(code, -8), 7);
                    if (BF16 && t == 0.0f && v < 0.0f) code = -1;
                }
                w += (uint32_t)code << (4 * j);
            }
            u[i] = s > 0.0f ? w : 0x88888888u;  // (no scale, or one that rounds to zero: every code is that of +1)
        }
    };
    if (__any(small || large)) codes(std::true_type());
    else codes(std::false_type());
    return scale;
}

// The rows of an eight of tokens of one head, as codes, into the cache.  `turn`: D / 4 * 8 pieces of LDS of the wave's.
template <int D>
__device__ __forceinline__ void write_codes(const KvArgs &c, const Eight &e, int head, const uint32_t (&uk)[D / 64], uint32_t sk, const uint32_t (&uv)[D / 64], uint32_t sv, kv_u16 *t)
{
    constexpr int P = D / 32;  // 16-bit pieces of a lane
    const int lane = kv_lane(), token = lane >> 3, part = lane & 7;
    const int64_t block = ((int64_t)e.page * c.heads + head) * 2;
    uint16_t *scales = c.scales + (block << c.page_shift) + e.in_page;
    uint8_t *keys = c.codes + (block << c.page_shift) * (D / 2) + (int64_t)e.in_page * (D / 2);
    uint16_t *values = reinterpret_cast<uint16_t *>(keys + ((int64_t)(D / 2) << c.page_shift));  // (an eight of tokens has its place at the same byte)
    if (e.is_new) {
        uint32_t *to = reinterpret_cast<uint32_t *>(keys + token * (D / 2)) + part;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) to[8 * i] = uk[i];
        if (part == 0) {
            scales[token] = (uint16_t)sk;
            scales[((int64_t)1 << c.page_shift) + token] = (uint16_t)sv;
        }
    }
    if (e.whole) {
#pragma unroll
        for (int i = 0; i < P; ++i) t[four_of(part, i) * 8 + token] = (uint16_t)(uv[i / 2] >> (16 * (i & 1)));
        kv_wave_fence();
        if constexpr (P == 4) reinterpret_cast<uint2 *>(values)[lane] = reinterpret_cast<const uint2 *>(t)[lane];
        else reinterpret_cast<uint32_t *>(values)[lane] = reinterpret_cast<const uint32_t *>(t)[lane];
        kv_wave_fence();  // (the next head's go to the same place)
    } else if (e.is_new) {
#pragma unroll
        for (int i = 0; i < P; ++i) values[four_of(part, i) * 8 + token] = (uint16_t)(uv[i / 2] >> (16 * (i & 1)));
    }
}

#endif

}  // namespace apmm
