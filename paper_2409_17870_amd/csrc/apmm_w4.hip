// Four-bit weights with group scales times 16-bit activations (apmm_w4.h): packing, and the kernels for few and for many tokens.
//
// The codes' odd integers are exact in both types and so are their products with the activations in 32 bits; a group's sum is multiplied with its scale in 32 bits, results are rounded once.
#include <type_traits>

#include "apmm_w4.h"

namespace apmm {

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

// A lane makes a word.  Bound by HBM: a byte a code in, half a byte out.
template <bool BF16>
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t *codes, const uint16_t *scales, int64_t N, int64_t K, int64_t tiles, int64_t blocks, int group, int64_t groups_in, uint8_t *packed)
{
    const int64_t words = tiles * blocks * 256, per_block = kW4Block / group;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < words; at += (int64_t)gridDim.x * 256) {
        const int64_t unit = at >> 8, tile = unit / blocks, block = unit - tile * blocks;
        const int lane = (int)(at >> 2) & 63, j = (int)at & 3;
        const int64_t n = tile * kW4Tile + (lane & 15), k0 = block * kW4Block + 32 * j + 8 * (lane >> 4);
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = n < N && k0 + i < K ? codes[n * K + k0 + i] & 15u : 0u;
        reinterpret_cast<uint32_t *>(packed)[at] = w4_word<BF16>(u);
    }
    uint16_t *to = reinterpret_cast<uint16_t *>(packed + words * 4);
    const int64_t groups = blocks * per_block, all = tiles * groups * kW4Tile;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t unit = at / kW4Tile, tile = unit / groups, g = unit - tile * groups, n = tile * kW4Tile + at % kW4Tile;
        to[at] = n < N && g < groups_in ? scales[n * groups_in + g] : (uint16_t)0;
    }
}

// Eight numbers of a row at any address, zeros behind K
template <class Eight>
__device__ __forceinline__ Eight row_eight(const uint16_t *row, int k, int K)
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
__device__ __forceinline__ float4v multiply(typename W4Type<BF16>::Eight a, typename W4Type<BF16>::Eight b, float4v c)
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Few tokens: a workgroup has a tile of 16 channels and 16 T tokens, its waves take blocks of 128 inputs in turn and meet in LDS.
template <bool BF16, int GROUP, int T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void w4_rows_kernel(W4Args a)
{
    typedef typename W4Type<BF16>::Eight Eight;
    constexpr int kGroups = kW4Block / GROUP, kSteps = GROUP / 32;  // groups of a block, matrix instructions of a group
    __shared__ float4v sums[WAVES][T][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int tile = blockIdx.x, row0 = blockIdx.y * 16 * T;
    const uint8_t *codes = a.packed + (int64_t)tile * a.blocks * kW4BlockBytes + lane * 16;
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(a.packed + a.code_bytes) + (int64_t)tile * a.blocks * kGroups * kW4Tile + n;
    const uint16_t *rows[T];
#pragma unroll
    for (int t = 0; t < T; ++t) rows[t] = a.x + min(row0 + 16 * t + n, a.M - 1) * a.x_stride;  // (a row that there is not has results that are not written)

    float4v acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t) acc[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = wave; b < a.blocks; b += WAVES) {
        const uint4 w = *reinterpret_cast<const uint4 *>(codes + (int64_t)b * kW4BlockBytes);
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
        uint16_t s[kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) s[i] = scales[((int64_t)b * kGroups + i) * kW4Tile];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            float4v part[T];
#pragma unroll
            for (int t = 0; t < T; ++t) part[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = i * kSteps; j < (i + 1) * kSteps; ++j) {
                const Eight c = w4_operand<BF16>(words[j]);
#pragma unroll
                for (int t = 0; t < T; ++t) part[t] = multiply<BF16>(row_eight<Eight>(rows[t], b * kW4Block + 32 * j + 8 * g, a.K), c, part[t]);
            }
            const float by = w4_scale<BF16>(s[i]);
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[t][r] = fmaf(part[t][r], by, acc[t][r]);
        }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < T; t += WAVES) {
        float4v all = sums[0][t][lane];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) all += sums[i][t][lane];
        const int channel = tile * kW4Tile + n;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = row0 + 16 * t + 4 * g + r;
            if (row < a.M && channel < a.N) a.y[row * a.y_stride + channel] = w4_round<BF16>(all[r]);
        }
    }
}

template <bool BF16, int GROUP>
void launch(const W4Args &a, hipStream_t stream)
{
    const uint32_t tiles = (uint32_t)((a.N + kW4Tile - 1) / kW4Tile);
    if (a.M <= 16) w4_rows_kernel<BF16, GROUP, 1, 8><<<dim3(tiles), dim3(512), 0, stream>>>(a);
    else w4_rows_kernel<BF16, GROUP, 4, 4><<<dim3(tiles, (uint32_t)((a.M + 63) / 64)), dim3(256), 0, stream>>>(a);
}

}  // namespace

hipError_t launch_w4_pack(const uint8_t *codes, const uint16_t *scales, const W4Shape &s, bool bf16, uint8_t *packed, hipStream_t stream)
{
    const int64_t words = s.code_bytes() / 4;
    const uint32_t groups = (uint32_t)(words / 256 < 16384 ? words / 256 : 16384);
    const int64_t groups_in = (s.K + s.group - 1) / s.group;
    if (bf16) w4_pack_kernel<true><<<dim3(groups), dim3(256), 0, stream>>>(codes, scales, s.N, s.K, s.tiles(), s.blocks(), s.group, groups_in, packed);
    else w4_pack_kernel<false><<<dim3(groups), dim3(256), 0, stream>>>(codes, scales, s.N, s.K, s.tiles(), s.blocks(), s.group, groups_in, packed);
    return hipGetLastError();
}

int64_t w4_items(const W4Args &a) { return (int64_t)((a.N + kW4Tile - 1) / kW4Tile) * (a.M <= 16 ? 512 : (a.M + 63) / 64 * 256); }

hipError_t launch_w4_gemm(const W4Args &a, int group, bool bf16, hipStream_t stream)
{
    auto go = [&](auto b) {
        constexpr bool B = decltype(b)::value;
        if (group == 32) launch<B, 32>(a, stream);
        else if (group == 64) launch<B, 64>(a, stream);
        else launch<B, 128>(a, stream);
    };
    if (bf16) go(std::true_type());
    else go(std::false_type());
    return hipGetLastError();
}

}  // namespace apmm
