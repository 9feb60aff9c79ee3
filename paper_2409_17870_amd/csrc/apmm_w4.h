// Products of 16-bit activations with four-bit weights and group scales: the packed form and the launchers (the public ABI is include/apmm.h).
//
//   y[m][n] = sum_k x[m][k] (2 u[n][k] - 15) s[n][k / group]
//
// Packed form: channels in tiles of 16, inputs in blocks of 128, both padded.
//   codes   [tile][block][lane][4 words]: lane l has channel l % 16 and, in word j, inputs 32 j + 8 (l / 16) to + 7 of the block: its part of the matrix unit's operand of 32 inputs.  A wave
//           takes a block with one load of 1 KiB.  Where in its word a code lies goes by the type of the activations (w4_word): so that few operations make the odd integer 2 u - 15 of that type.
//   scales  [tile][group][16] of the activations' type
// Padded codes meet activations that are zero, padded scales are zero.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace apmm {

constexpr int64_t kW4MostRows = 1 << 20;
constexpr int kW4Tile = 16, kW4Block = 128, kW4BlockBytes = kW4Tile * kW4Block / 2;

struct W4Shape {
    int64_t N, K;
    int group;
    int64_t tiles() const { return (N + kW4Tile - 1) / kW4Tile; }
    int64_t blocks() const { return (K + kW4Block - 1) / kW4Block; }
    int64_t groups() const { return blocks() * (kW4Block / group); }
    int64_t code_bytes() const { return tiles() * blocks() * kW4BlockBytes; }
    int64_t bytes() const { return code_bytes() + tiles() * groups() * kW4Tile * 2; }
};

struct W4Args {
    const uint16_t *x;
    const uint8_t *packed;
    uint16_t *y;
    float *partial;
    int64_t x_stride, y_stride;  // elements between rows
    int64_t code_bytes;          // where the scales begin
    int M, N, K, blocks;
};

hipError_t launch_w4_pack(const uint8_t *codes, const uint16_t *scales, const W4Shape &s, bool bf16, uint8_t *packed, hipStream_t stream);

// Which kernel a call takes, by its sizes
struct W4Rule {
    bool tiles;     // w4_tiles_kernel: blocks of 32 tokens, shares of the inputs; else w4_rows_kernel: tiles of 16 channels, waves
    int t, shares;
    int c, waves;
};
W4Rule w4_rule(int64_t M, int64_t N, int64_t blocks);
int64_t w4_items(int64_t M, int64_t N, const W4Rule &r);  // of the largest launch
// Of the workspace that the inputs' shares take
__host__ __device__ inline int64_t w4_partial_stride(int64_t N) { return (N + 3) / 4 * 4; }
inline int64_t w4_partial_bytes(int64_t M, int64_t N, const W4Rule &r) { return r.shares > 1 ? r.shares * M * w4_partial_stride(N) * 4 : 0; }
hipError_t launch_w4_gemm(const W4Args &a, const W4Rule &r, int group, bool bf16, hipStream_t stream);
hipError_t launch_w4_tiles(const W4Args &a, const W4Rule &r, int group, bool bf16, hipStream_t stream);

#ifdef __HIPCC__
// Word of eight codes.
//   binary16  Code 2 e + i (e = 0 to 3, i = 0, 1) in bits 16 i + 4 e + 1 to 16 i + 4 e + 4, the last one's highest bit in bit 0.  In bits 1 to 4 of a half whose upper bits are those of 1024 it
//             makes 1024 + 2 u, in bits 5 to 8 under those of 64 64 + 2 u: one operation for each pair, one that takes off 1039 or 79, one rotation for the second half of the word.
//   bfloat16  has eight significant bits and no packed sum: a magnitude's byte comes out of a table of eight, m = (|2 u - 15| - 1) / 2 of code b in bits 8 b to 8 b + 2, of code 4 + b in bits
//             8 b + 4 to 8 b + 6, the signs in bits 8 b + 7 and 8 b + 3.
template <bool BF16>
__device__ __forceinline__ uint32_t w4_word(const uint32_t (&u)[8])
{
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (BF16) {
            const uint32_t m = u[i] >= 8 ? u[i] - 8 : 7 - u[i], sign = u[i] >= 8 ? 0 : 1;
            const int b = 8 * (i & 3);
            w |= i < 4 ? m << b | sign << (b + 7) : m << (b + 4) | sign << (b + 3);
        } else {
            const int at = 16 * (i & 1) + 4 * (i >> 1) + 1;
            w |= u[i] << at | (at > 28 ? u[i] >> (32 - at) : 0);
        }
    }
    return w;
}

template <bool BF16> struct W4Type { typedef _Float16 Eight __attribute__((ext_vector_type(8))); };
template <> struct W4Type<true> { typedef __bf16 Eight __attribute__((ext_vector_type(8))); };

__device__ __forceinline__ uint32_t w4_and_or(uint32_t x, uint32_t mask, uint32_t bits)
{
    uint32_t r;  // (in one instruction with one of the two in a scalar register; of two literals the compiler makes two)
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "s"(mask), "v"(bits));
    return r;
}

// The eight odd integers of a word as an operand
template <bool BF16>
__device__ __forceinline__ typename W4Type<BF16>::Eight w4_operand(uint32_t w)
{
    uint32_t r[4];
    if (BF16) {
        // the upper and lower bytes of 1, 3, ..., 15 as bfloat16 numbers
        constexpr uint32_t kHigh0 = 0x4040403fu, kHigh1 = 0x41414141u, kLow0 = 0xe0a04080u, kLow1 = 0x70503010u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t m = (i ? w >> 4 : w) & 0x07070707u, sign = (i ? w << 4 : w) & 0x80808080u;
            const uint32_t high = __builtin_amdgcn_perm(kHigh1, kHigh0, m) | sign, low = __builtin_amdgcn_perm(kLow1, kLow0, m);
            r[2 * i] = __builtin_amdgcn_perm(high, low, 0x05010400u);
            r[2 * i + 1] = __builtin_amdgcn_perm(high, low, 0x07030602u);
        }
    } else {
        typedef _Float16 half2v __attribute__((ext_vector_type(2)));
        const uint32_t v = __builtin_amdgcn_alignbit(w, w, 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t from = i < 2 ? w : v, pair = i & 1 ? w4_and_or(from, 0x01e001e0u, 0x54005400u) : w4_and_or(from, 0x001e001eu, 0x64006400u);
            const half2v less = i & 1 ? half2v{(_Float16)-79.0f, (_Float16)-79.0f} : half2v{(_Float16)-1039.0f, (_Float16)-1039.0f};
            r[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, pair) + less);
        }
    }
    return __builtin_bit_cast(typename W4Type<BF16>::Eight, make_uint4(r[0], r[1], r[2], r[3]));
}

// Eight numbers of a row at any address, zeros behind K
template <class Eight>
__device__ __forceinline__ Eight w4_row_eight(const uint16_t *row, int k, int K)
{
    uint4 w = make_uint4(0, 0, 0, 0);
    if (k + 8 <= K) {
        __builtin_memcpy(&w, row + k, 16);
    } else if (k < K) {
        uint32_t p[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < K) p[i / 2] |= (uint32_t)row[k + i] << (16 * (i & 1));
        w = make_uint4(p[0], p[1], p[2], p[3]);
    }
    return __builtin_bit_cast(Eight, w);
}

template <bool BF16>
__device__ __forceinline__ float w4_scale(uint16_t s) { return BF16 ? __uint_as_float((uint32_t)s << 16) : (float)__builtin_bit_cast(_Float16, s); }
template <bool BF16>
__device__ __forceinline__ uint16_t w4_round(float x) { return BF16 ? __builtin_bit_cast(uint16_t, (__bf16)x) : __builtin_bit_cast(uint16_t, (_Float16)x); }
#endif

}  // namespace apmm
