// Rotary positions: what the kernel that turns rows and the one that turns them on their way into the four-bit cache share (the public ABI is include/apmm.h).
//
//   (a, b) of a pair becomes (g (a cos t - b sin t), g (b cos t + a sin t)), t = position times the pair's frequency
//
// The angle is a product in 64 bits, taken as turns less the whole ones: positions of 2^31 leave it off by 2^-24 of a turn at most, 32 bits would be off by many turns.  Sums and products of the turn
// itself are of 32 bits, rounded once to the rows' type.
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
// Cosine and sine of a pair at a position, times the magnitude
__device__ __forceinline__ float2 rotary_turn(const RotaryArgs &r, int position, int pair)
{
    const double turns = (double)position * (r.frequencies[pair] * 0.15915494309189533577), rest = turns - rint(turns);
    // (what 32 bits leave of the angle goes in as the sums' first order: keys are quantised behind this, where an error may cost a code)
    const float near = (float)rest, left = 6.283185307f * (float)(rest - (double)near);
    float s, c;
    sincospif(2.0f * near, &s, &c);
    return make_float2(fmaf(-left, s, c) * r.magnitude, fmaf(left, c, s) * (r.magnitude * r.sign));
}
// One of a pair: `other` comes with the sign that the sine has for it.  (Always in this form, so that rows come out the same wherever they are turned.)
__device__ __forceinline__ float rotary_one(float x, float other, float cosine, float sine) { return fmaf(x, cosine, other * sine); }

__device__ __forceinline__ uint32_t rotary_pair(float a, float b, bool bf16) { return kv_round(a, bf16) | (uint32_t)kv_round(b, bf16) << 16; }

// Eight channels from c0 on of the row that begins at `row`, w their words; t: the token's cosines and sines by pair
template <bool BF16>
__device__ __forceinline__ void rotary_eight(const uint16_t *row, bool aligned, int c0, uint32_t (&w)[4], const float2 *t, int pairs, bool interleaved)
{
    if (c0 >= 2 * pairs) return;
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pair = c0 / 2 + i;
            if (pair >= pairs) break;
            const float2 cs = t[pair];
            const float a = kv_scale_value(w[i] & 0xffffu, BF16), b = kv_scale_value(w[i] >> 16, BF16);
            w[i] = rotary_pair(rotary_one(a, -b, cs.x, cs.y), rotary_one(b, a, cs.x, cs.y), BF16);
        }
        return;
    }
    uint32_t other[4];
    if (pairs % 8 == 0) {
        kv_load(row + (c0 < pairs ? c0 + pairs : c0 - pairs), aligned, other);
        const float2 *at = t + (c0 < pairs ? c0 : c0 - pairs);
        const float by = c0 < pairs ? -1.0f : 1.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 c1 = at[2 * i], c2 = at[2 * i + 1];
            w[i] = rotary_pair(rotary_one(kv_scale_value(w[i] & 0xffffu, BF16), by * kv_scale_value(other[i] & 0xffffu, BF16), c1.x, c1.y),
                               rotary_one(kv_scale_value(w[i] >> 16, BF16), by * kv_scale_value(other[i] >> 16, BF16), c2.x, c2.y), BF16);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = c0 + i;
        if (c >= 2 * pairs) break;
        const float2 cs = t[c < pairs ? c : c - pairs];
        const float x = kv_scale_value(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu, BF16), y = kv_scale_value(row[c < pairs ? c + pairs : c - pairs], BF16);
        const uint32_t bits = kv_round(rotary_one(x, c < pairs ? -y : y, cs.x, cs.y), BF16);
        w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | bits << 16 : (w[i / 2] & 0xffff0000u) | bits;
    }
}
#endif

}  // namespace apmm
