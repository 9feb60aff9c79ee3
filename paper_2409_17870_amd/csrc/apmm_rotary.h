// Rotary positions: what the kernel that turns rows and the one that turns them on their way into the four-bit cache share (the public ABI is include/apmm.h).
//
//   (a, b) of a pair becomes (g (a cos t - b sin t), g (b cos t + a sin t)), t = position times the pair's frequency
//
// The angle is a product in 64 bits, taken as turns less the whole ones: positions of 2^31 leave it off by 2^-24 of a turn at most, 32 bits would be off by many turns.  Cosine and sine are made in
// 64 bits too and go on as two numbers of 32; a sum is made of numbers of 32 and of what its products and steps leave, as far as that can decide its rounding to the rows' type: the result is the pair's of 64
// bits, rounded to 32, then to 16 (none of 537 million differed; of sums, products, cosines and sines of 32 bits alone one in 6300 of binary16, one in 39000 of bfloat16).
#pragma once
#include "apmm_kv.h"

namespace apmm {

struct RotaryArgs {
    const double *frequencies;  // radians a position
    const int32_t *positions;   // of each row; null: a token's place in its sequence
    int pairs;
    bool interleaved;
    float magnitude, sign;      // sign: -1 turns back
};

struct RotaryRows {
    KvTensor x, out;
    RotaryArgs r;
    int64_t tokens;
    int heads, head_dim, tokens_of_group;
    bool bf16;
    uint64_t by_items;          // what kv_divide divides by a head's pieces with
    int items;                  // pieces of a head: eights of channels, or pairs and single channels
    bool eights;
};

struct KvRotaryArgs {
    KvArgs c;
    KvTensor q, q_out, k, v;
    RotaryArgs r;
    int q_heads;
    int per_wave, blocks;       // heads of a wave, workgroups of an eight of tokens
    uint64_t by_blocks;
};

hipError_t launch_rotary(const RotaryRows &a, hipStream_t stream);
int64_t kv_rotary_items(const KvArgs &c, int q_heads);
hipError_t launch_kv_write_rotary(const KvRotaryArgs &a, hipStream_t stream);

#ifdef __HIPCC__
// Cosine and sine of a pair at a position, times the magnitude, made in 64 bits, as numbers of 32 and what these leave: Taylor's series over an eighth of a turn to either side, whose next terms are below 2^-45
__device__ __forceinline__ float4 rotary_turn(const RotaryArgs &r, int position, int pair)
{
    constexpr double kPerRadian = 0.15915494309189535, kPerRadianLow = -9.839338337591243e-18, kRadians = 6.283185307179586;  // 1 / (2 pi) in two parts
    // turns less the whole ones with one rounding of what is left.  (As the product less the whole ones, and the product's rounding after it, the compiler would take the first of these in one step and the rounding twice.)
    const double t = (double)position * r.frequencies[pair], rest = fma(t, kPerRadianLow, fma(t, kPerRadian, -rint(t * kPerRadian)));
    const double quarter = rint(4.0 * rest), x = (rest - 0.25 * quarter) * kRadians, y = x * x;
    double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
    s = fma(s, y, -1.0 / 39916800.0);
    s = fma(s, y, 1.0 / 362880.0);
    s = fma(s, y, -1.0 / 5040.0);
    s = fma(s, y, 1.0 / 120.0);
    s = fma(s, y, -1.0 / 6.0);
    s = fma(s * y, x, x);
    c = fma(c, y, 1.0 / 479001600.0);
    c = fma(c, y, -1.0 / 3628800.0);
    c = fma(c, y, 1.0 / 40320.0);
    c = fma(c, y, -1.0 / 720.0);
    c = fma(c, y, 1.0 / 24.0);
    c = fma(c, y, -0.5);
    c = fma(c, y, 1.0);
    const int q = (int)quarter & 3;
    const double cosine = q & 1 ? s : c, sine = q & 1 ? c : s;
    const double cs = (q == 1 || q == 2 ? -cosine : cosine) * r.magnitude, sn = (q & 2 ? -sine : sine) * (r.magnitude * r.sign);
    const float c1 = (float)cs, s1 = (float)sn;
    return make_float4(c1, s1, (float)(cs - (double)c1), (float)(sn - (double)s1));
}
// One of a pair: `other` comes with the sign that the sine has for it.  What the product and the rounding of cosine and sine to 32 bits have left goes in as a sum of its own, so that the result is off by two roundings
// of 32 bits, and by 2^-47 of the larger product, which is less wherever no more than 20 bits of the pair cancel.
__device__ __forceinline__ float rotary_sum(float x, float other, const float4 &t)
{
#pragma clang fp contract(off)
    const float p = other * t.y, sum = fmaf(x, t.x, p), all = sum + fmaf(x, t.z, fmaf(other, t.w, fmaf(other, t.y, -p)));
    return all == all ? all : sum;  // (what infinities leave is an infinity of either sign or no number)
}
// The same with what every step leaves: the sum rounded to 32 bits once (NaN where a product has no place in 32 bits)
__device__ __forceinline__ float rotary_all(float x, float other, const float4 &t)
{
#pragma clang fp contract(off)
    const float q = x * t.x, p = other * t.y, sum = q + p, b = sum - q;
    return sum + (((q - (sum - b)) + (p - b)) + ((fmaf(x, t.x, -q) + fmaf(other, t.y, -p)) + fmaf(x, t.z, other * t.w)));
}
template <bool BF16>
__device__ __forceinline__ float rotary_exact(float x, float other, const float4 &t, float v)
{
    float all = rotary_all(x, other, t);
    if (BF16 && all != all)  // the sum of such products may have a place, and does as products of numbers 2^128 times smaller
        all = rotary_all(x * 0x1p-64f, other * 0x1p-64f, make_float4(t.x * 0x1p-64f, t.y * 0x1p-64f, t.z * 0x1p-64f, t.w * 0x1p-64f)) * 0x1p64f * 0x1p64f;
    return all == all ? all : v;
}
// Rounding in the sum decides the one to 16 bits where the number is so near the middle between two of those: one in 1600 (binary16) or 13000.  Keys are quantised behind this, where a number rounded the other way may
// cost a code.  Below 2^-14 binary16 numbers are equally far apart, and the middles not at one place of the bits: any of these is near (rows of
// zeros, as batches are filled up with, would take a fifth longer if they were).  So is, of
// bfloat16, whose largest numbers are those of 32 bits, what has become infinite on the way.
template <bool BF16>
__device__ __forceinline__ bool rotary_near(float v)
{
    constexpr uint32_t kHalf = BF16 ? 0x8000 : 0x1000;
    return (((__float_as_uint(v) - (kHalf - 2)) & (2 * kHalf - 1)) <= 4) | (BF16 ? !(fabsf(v) < __builtin_inff()) : fabsf(fabsf(v) - 0x1p-15f) < 0x1p-15f);  // (zeros, and what is less than 2^-40 and will be one, are not)
}
// Each number is made again by its own nearness alone, here and where both of a pair are a lane's: so all kernels have the same.
template <bool BF16>
__device__ __forceinline__ float rotary_one(float x, float other, const float4 &t)
{
    float v = rotary_sum(x, other, t);
    if (rotary_near<BF16>(v)) v = rotary_exact<BF16>(x, other, t, v);
    return v;
}
// (a, b) turned
template <bool BF16>
__device__ __forceinline__ void rotary_both(float &a, float &b, const float4 &t)
{
    float first = rotary_sum(a, -b, t), second = rotary_sum(b, a, t);
    const bool near_first = rotary_near<BF16>(first), near_second = rotary_near<BF16>(second);
    if (near_first | near_second) {
        const float first_exact = rotary_exact<BF16>(a, -b, t, first), second_exact = rotary_exact<BF16>(b, a, t, second);
        first = near_first ? first_exact : first;
        second = near_second ? second_exact : second;
    }
    a = first;
    b = second;
}

// A token's cosines and sines in LDS: pair p in row p % 8 or p % 4, as many rows as an eight of channels has pairs with (8) or within (4) it, so that lanes with an eight each read places that follow each other
template <bool INTERLEAVED>
struct RotaryTurns {
    static constexpr int kShift = INTERLEAVED ? 2 : 3;
    float4 *at;
    int stride;
    __device__ __forceinline__ float4 &operator[](int pair) const { return at[(pair & ((1 << kShift) - 1)) * stride + (pair >> kShift)]; }
};

__device__ __forceinline__ uint32_t rotary_pair(float a, float b, bool bf16) { return kv_round(a, bf16) | (uint32_t)kv_round(b, bf16) << 16; }

// Eight channels from c0 on of the row that begins at `row`, w their words
template <bool BF16, bool INTERLEAVED>
__device__ __forceinline__ void rotary_eight(const uint16_t *row, bool aligned, int c0, uint32_t (&w)[4], const RotaryTurns<INTERLEAVED> &t, int pairs)
{
    if (c0 >= 2 * pairs) return;
    if (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pair = c0 / 2 + i;
            if (pair >= pairs) break;
            const float4 cs = t[pair];
            float a = kv_scale_value(w[i] & 0xffffu, BF16), b = kv_scale_value(w[i] >> 16, BF16);
            rotary_both<BF16>(a, b, cs);
            w[i] = rotary_pair(a, b, BF16);
        }
        return;
    }
    uint32_t other[4];
    if (pairs % 8 == 0) {
        kv_load(row + (c0 < pairs ? c0 + pairs : c0 - pairs), aligned, other);
        const int p0 = c0 < pairs ? c0 : c0 - pairs;
        const float by = c0 < pairs ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 c1 = t[p0 + 2 * i], c2 = t[p0 + 2 * i + 1];
            w[i] = rotary_pair(rotary_one<BF16>(kv_scale_value(w[i] & 0xffffu, BF16), by * kv_scale_value(other[i] & 0xffffu, BF16), c1),
                               rotary_one<BF16>(kv_scale_value(w[i] >> 16, BF16), by * kv_scale_value(other[i] >> 16, BF16), c2), BF16);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = c0 + i;
        if (c >= 2 * pairs) break;
        const float4 cs = t[c < pairs ? c : c - pairs];
        const float x = kv_scale_value(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu, BF16), y = kv_scale_value(row[c < pairs ? c + pairs : c - pairs], BF16);
        const uint32_t bits = kv_round(rotary_one<BF16>(x, c < pairs ? -y : y, cs), BF16);
        w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | bits << 16 : (w[i / 2] & 0xffff0000u) | bits;
    }
}
#endif

}  // namespace apmm
