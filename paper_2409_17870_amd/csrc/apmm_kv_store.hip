// Writing the four-bit key/value cache and reading it back.
//
// A row x (head_dim numbers of a token and head) becomes s = max |x| / 15 rounded to its type and codes u = clamp(floor(x / (2 s)) + 8, 0, 15): the nearest odd
// multiple 2 u - 15 of s, ties upward, as apmm_quantize_pack_activations has it.
//
// One wave takes the up to eight tokens of an aligned eight of positions, one head (or two of 64 channels), keys and values: eight lanes to a token.  The eight tokens of
// a channel are neighbours in the cache's values, so they are turned in LDS and written whole (an eight that is not all new is written in pieces of 16 bits, what is there
// of earlier tokens stays).  Bound by HBM: 4 bytes a channel in or out,
// one and a bit in the cache.  Reading 16384 tokens of 32 heads of 128: 338 MB in 61 us, 5.5 TB/s (a large copy: 5.1); writing 2048 of 40 heads: 53 MB in 13 us, some 4 of them the launch and
// the way from lengths and pages to the first row.  (Two pieces of 16 bytes to a lane side by side, in place of 128 bytes to eight lanes, took 75 us of the first.)
#include <algorithm>
#include <type_traits>

#include "apmm_kv.h"

namespace apmm {

namespace {

constexpr int kWaves = 4;
// Heads of a wave: two of 64 channels where there is enough for two rounds of waves, or finding its eight costs as much as moving it (3 sequences of 37000 tokens, 16 heads of 64, read
// back: 147 us with one, 120 with two; pieces of 333 tokens and single ones of 23 sequences, 8 heads: 4.2 and 4.7)
constexpr int kManyUnits = 16384;
template <int D>
__device__ __forceinline__ int heads_of_wave(const KvArgs &c) { return D == 64 ? c.per_wave : 1; }

struct Eight {  // of one wave
    KvSequence s;
    int head, first, in_page;  // the first of its heads; position of its first token (a multiple of eight, may be negative), its place in the page
    int page;                  // -1: none
    bool is_new;               // this lane's token is one of the call's
    bool whole;                // all eight are
};

// false: nothing for this wave.  (by_heads is that of the heads' groups of `per`, 1 or 2)
__device__ __forceinline__ bool find_eight(const KvArgs &c, int per, Eight &e)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = blockIdx.x * kWaves + wave, eight = kv_divide(unit, c.by_heads);  // (fewer than 2^26 units, kv_store_items)
    e.head = (unit - eight * (per == 1 ? c.heads : (c.heads + 1) >> 1)) * per;
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

template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves) void kv_write_kernel(KvArgs c, KvTensor k, KvTensor v)
{
    constexpr int N = D / 16;  // words of a lane's channels, two to a word
    constexpr int P = D / 32;  // 16-bit pieces of a lane
    __shared__ __align__(16) kv_u16 turn[kWaves][D / 4 * 8];
    Eight e;
    const int per = heads_of_wave<D>(c);
    if (!find_eight(c, per, e) || e.page < 0) return;
    const int lane = kv_lane(), token = lane >> 3, part = lane & 7;
    const int64_t row = e.s.start + (e.is_new ? e.first + token - e.s.first : 0);  // (a lane without one reads the first)
    for (int head = e.head; head < min(e.head + per, c.heads); ++head) {
        uint32_t xk[N], xv[N];
        load_row(k.data + row * k.token_stride + head * k.head_stride, k.aligned, part, xk);
        load_row(v.data + row * v.token_stride + head * v.head_stride, v.aligned, part, xv);
        uint32_t uk[N / 4], uv[N / 4];
        const uint32_t sk = quantise<N, BF16>(xk, uk), sv = quantise<N, BF16>(xv, uv);

        const int64_t block = ((int64_t)e.page * c.heads + head) * 2;
        uint16_t *scales = c.scales + (block << c.page_shift) + e.in_page;
        uint8_t *keys = c.codes + (block << c.page_shift) * (D / 2) + (int64_t)e.in_page * (D / 2);
        uint16_t *values = reinterpret_cast<uint16_t *>(keys + ((int64_t)(D / 2) << c.page_shift));  // (an eight of tokens has its place at the same byte)
        if (e.is_new) {
            uint32_t *to = reinterpret_cast<uint32_t *>(keys + token * (D / 2)) + part;
#pragma unroll
            for (int i = 0; i < N / 4; ++i) to[8 * i] = uk[i];
            if (part == 0) {
                scales[token] = (uint16_t)sk;
                scales[((int64_t)1 << c.page_shift) + token] = (uint16_t)sv;
            }
        }
        if (e.whole) {
            kv_u16 *t = turn[threadIdx.x >> 6];
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
}

// What codes u (eight to a word, from the low bits) stand for: (2 u - 15) s, exact in 32 bits, rounded once.  A product beyond the largest finite number becomes that: 15 s may
// round past the number that s came from.
template <int N, bool BF16>
__device__ __forceinline__ void values_of(const uint32_t (&u)[N / 4], uint32_t scale, uint32_t (&x)[N])
{
    constexpr float kTop = BF16 ? 0x1.fep127f : 65504.0f;
    const float s = kv_scale_value(scale, BF16), s2 = 2.0f * s, s15 = -15.0f * s;
    const bool odd_case = !(fabsf(s15) < kTop);
    float f[2 * N];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint32_t lo = u[i] & 0x0f0f0f0fu, hi = (u[i] >> 4) & 0x0f0f0f0fu;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = (float)((lo >> (8 * j)) & 0xffu), b = (float)((hi >> (8 * j)) & 0xffu);
            f[8 * i + 2 * j] = fmaf(a, s2, s15);
            f[8 * i + 2 * j + 1] = fmaf(b, s2, s15);
            if (odd_case) {
                const float va = (2.0f * a - 15.0f) * s, vb = (2.0f * b - 15.0f) * s;
                f[8 * i + 2 * j] = va != va ? va : fminf(fmaxf(va, -kTop), kTop);
                f[8 * i + 2 * j + 1] = vb != vb ? vb : fminf(fmaxf(vb, -kTop), kTop);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = kv_round(f[2 * i], BF16) | (uint32_t)kv_round(f[2 * i + 1], BF16) << 16;
}

template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves) void kv_read_kernel(KvArgs c, KvTensor k, KvTensor v)
{
    constexpr int N = D / 16;
    __shared__ __align__(16) kv_u16 turn[kWaves][D / 4 * 8];
    Eight e;
    const int per = heads_of_wave<D>(c);
    if (!find_eight(c, per, e)) return;
    const int lane = kv_lane(), token = lane >> 3, part = lane & 7;
    const bool there = e.page >= 0;
    for (int head = e.head; head < min(e.head + per, c.heads); ++head) {
        const int64_t block = ((int64_t)(there ? e.page : 0) * c.heads + head) * 2;
        const uint16_t *scales = c.scales + (block << c.page_shift) + e.in_page;
        const uint8_t *keys = c.codes + (block << c.page_shift) * (D / 2) + (int64_t)e.in_page * (D / 2);
        const uint8_t *values = keys + ((int64_t)(D / 2) << c.page_shift);
        kv_u16 *t = turn[threadIdx.x >> 6];
        uint32_t uk[N / 4], uv[N / 4], xk[N], xv[N];
        const uint32_t *from = reinterpret_cast<const uint32_t *>(keys + token * (D / 2)) + part;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) uk[i] = from[8 * i];
        if constexpr (N == 8) reinterpret_cast<uint2 *>(t)[lane] = reinterpret_cast<const uint2 *>(values)[lane];
        else reinterpret_cast<uint32_t *>(t)[lane] = reinterpret_cast<const uint32_t *>(values)[lane];
        const uint32_t sk = scales[token], sv = scales[((int64_t)1 << c.page_shift) + token];
        kv_wave_fence();
#pragma unroll
        for (int i = 0; i < N / 4; ++i) uv[i] = t[four_of(part, 2 * i) * 8 + token] | (uint32_t)t[four_of(part, 2 * i + 1) * 8 + token] << 16;
        kv_wave_fence();
        values_of<N, BF16>(uk, sk, xk);
        values_of<N, BF16>(uv, sv, xv);
        if (!there) {  // a position before the first token, or without a page: zeros
#pragma unroll
            for (int i = 0; i < N; ++i) xk[i] = xv[i] = 0;
        }
        if (!e.is_new) continue;
        const int64_t row = e.s.start + e.first + token - e.s.first;
        store_row(k.data + row * k.token_stride + head * k.head_stride, k.aligned, part, xk);
        store_row(v.data + row * v.token_stride + head * v.head_stride, v.aligned, part, xv);
    }
}

// Waves for the most eights that `tokens` new ones can touch: n tokens of a sequence lie in n of them at most, and in (n + 14) / 8
int64_t eights(const KvArgs &c) { return std::min<int64_t>(c.tokens, c.tokens / 8 + 2 * (int64_t)c.sequences); }

int heads_of_a_wave(const KvArgs &c) { return c.head_dim == 64 && eights(c) * c.heads >= kManyUnits ? 2 : 1; }
int64_t workgroups(const KvArgs &c)
{
    const int per_wave = heads_of_a_wave(c);
    return (eights(c) * ((c.heads + per_wave - 1) / per_wave) + kWaves - 1) / kWaves;
}

template <int D, bool BF16>
hipError_t launch(bool write, const KvArgs &c, const KvTensor &k, const KvTensor &v, hipStream_t stream)
{
    KvArgs a = c;
    a.per_wave = heads_of_a_wave(c);
    a.by_heads = kv_divisor((c.heads + a.per_wave - 1) / a.per_wave);
    const int64_t groups = workgroups(c);
    if (write) kv_write_kernel<D, BF16><<<dim3((uint32_t)groups), dim3(64 * kWaves), 0, stream>>>(a, k, v);
    else kv_read_kernel<D, BF16><<<dim3((uint32_t)groups), dim3(64 * kWaves), 0, stream>>>(a, k, v);
    return hipGetLastError();
}

hipError_t launch(bool write, const KvArgs &c, const KvTensor &k, const KvTensor &v, hipStream_t stream)
{
    if (c.head_dim == 128) return c.bf16 ? launch<128, true>(write, c, k, v, stream) : launch<128, false>(write, c, k, v, stream);
    return c.bf16 ? launch<64, true>(write, c, k, v, stream) : launch<64, false>(write, c, k, v, stream);
}

}  // namespace

int64_t kv_store_items(const KvArgs &c) { return workgroups(c) * 64 * kWaves; }
hipError_t launch_kv_write(const KvArgs &c, const KvTensor &k, const KvTensor &v, hipStream_t stream) { return launch(true, c, k, v, stream); }
hipError_t launch_kv_read(const KvArgs &c, const KvTensor &k, const KvTensor &v, hipStream_t stream) { return launch(false, c, k, v, stream); }

}  // namespace apmm
