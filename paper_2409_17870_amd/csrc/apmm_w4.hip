// Four-bit weights with group scales times 16-bit activations (apmm_w4.h): packing, the kernel for few tokens, and which kernel a call takes.
//
// The codes' odd integers are exact in both types and so are their products with the activations in 32 bits; a group's sum is multiplied with its scale in 32 bits, results are rounded once.
#include <algorithm>
#include <type_traits>

#include "apmm_w4.h"

namespace apmm {

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));

// A lane makes a word.  4096 x 4096 32 us, 11008 x 4096 85, 5119 x 13800 96: 0.8 to 1.1 TB/s of the byte a code that comes in and the half that goes out, a fifth of what a copy reaches, since codes come one load a
// byte.  A model's weights are packed once.
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

template <bool BF16>
__device__ __forceinline__ float4v multiply(typename W4Type<BF16>::Eight a, typename W4Type<BF16>::Eight b, float4v c)
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Up to 32 tokens.  A workgroup has 16 C channels and 16 T tokens, its waves take blocks of 128 inputs in turn, the next block's weights and activations on their way while one is multiplied, and meet in LDS.
// Activations come from the caches into each wave's registers: they are no two waves' of a workgroup.  Bound by HBM and the way there: one token of 11008 x 4096 23 MB in 8.0 us, of 4096 x 4096 in 4.3 as
// called; at sixteen tokens by the activations beside it, which every workgroup reads (9.7 us).
template <bool BF16, int GROUP, int T, int C>
struct Block {
    typedef typename W4Type<BF16>::Eight Eight;
    uint4 w[C];
    uint16_t s[C][kW4Block / GROUP];
    Eight x[T][4];
};

template <bool BF16, int GROUP, int T, int C, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void w4_rows_kernel(W4Args a)
{
    typedef typename W4Type<BF16>::Eight Eight;
    typedef Block<BF16, GROUP, T, C> Block;
    constexpr int kGroups = kW4Block / GROUP, kSteps = GROUP / 32;  // groups of a block, matrix instructions of a group
    __shared__ float sums[WAVES][T * C][256];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int tiles = (a.N + kW4Tile - 1) / kW4Tile, tile0 = blockIdx.x * C, row0 = blockIdx.y * 16 * T;
    const uint8_t *codes[C];
    const uint16_t *scales[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t tile = min(tile0 + c, tiles - 1);
        codes[c] = a.packed + tile * a.blocks * kW4BlockBytes + lane * 16;
        scales[c] = reinterpret_cast<const uint16_t *>(a.packed + a.code_bytes) + tile * a.blocks * kGroups * kW4Tile + n;
    }
    const uint16_t *rows[T];
    bool there[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        there[t] = row0 + 16 * t + n < a.M;
        rows[t] = a.x + (there[t] ? row0 + 16 * t + n : 0) * a.x_stride + 8 * g;
    }
    auto load = [&](int b, Block &to) {
#pragma unroll
        for (int c = 0; c < C; ++c) to.w[c] = *reinterpret_cast<const uint4 *>(codes[c] + (int64_t)b * kW4BlockBytes);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kGroups; ++i) to.s[c][i] = scales[c][((int64_t)b * kGroups + i) * kW4Tile];
        const int K = (b + 1) * kW4Block <= a.K ? INT32_MAX : a.K - 8 * g;  // (the last block's may end in it)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                to.x[t][j] = __builtin_bit_cast(Eight, make_uint4(0, 0, 0, 0));
                if (there[t]) to.x[t][j] = w4_row_eight<Eight>(rows[t], b * kW4Block + 32 * j, K);
            }
    };

    float4v acc[T][C];
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int c = 0; c < C; ++c) acc[t][c] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](const Block &x) {
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint32_t words[4] = {x.w[c].x, x.w[c].y, x.w[c].z, x.w[c].w};
                float4v part[T];
#pragma unroll
                for (int t = 0; t < T; ++t) part[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = i * kSteps; j < (i + 1) * kSteps; ++j) {
                    const Eight w = w4_operand<BF16>(words[j]);
#pragma unroll
                    for (int t = 0; t < T; ++t) part[t] = multiply<BF16>(x.x[t][j], w, part[t]);
                }
                const float by = w4_scale<BF16>(x.s[c][i]);
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[t][c][r] = fmaf(part[t][r], by, acc[t][c][r]);
            }
        }
    };
    Block one, other;
    int b = wave;
    if (b < a.blocks) load(b, one);
    while (b < a.blocks) {
        if (b + WAVES < a.blocks) load(b + WAVES, other);
        add(one);
        b += WAVES;
        if (b >= a.blocks) break;
        if (b + WAVES < a.blocks) load(b + WAVES, one);
        add(other);
        b += WAVES;
    }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int c = 0; c < C; ++c) *reinterpret_cast<float4v *>(&sums[wave][t * C + c][4 * lane]) = acc[t][c];
    __syncthreads();
    const int left = min(a.M - row0, 16 * T);
    for (int i = threadIdx.x; i < left * 16 * C; i += 64 * WAVES) {
        const int row = i / (16 * C), c = i % (16 * C) / 16, column = i % 16, channel = (tile0 + c) * kW4Tile + column;
        const int at = (row % 16 / 4 * 16 + column) * 4 + row % 4;
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) all += sums[w][row / 16 * C + c][at];
        if (channel < a.N) a.y[(row0 + row) * a.y_stride + channel] = w4_round<BF16>(all);
    }
}

template <bool BF16, int GROUP>
void launch(const W4Args &a, const W4Rule &r, hipStream_t stream)
{
    const dim3 grid((uint32_t)((a.N + kW4Tile * r.c - 1) / (kW4Tile * r.c)), (uint32_t)((a.M + 16 * r.t - 1) / (16 * r.t)));
    if (r.t == 2) {
        if (r.c == 3) w4_rows_kernel<BF16, GROUP, 2, 3, 8><<<grid, dim3(512), 0, stream>>>(a);
        else if (r.c == 2) w4_rows_kernel<BF16, GROUP, 2, 2, 8><<<grid, dim3(512), 0, stream>>>(a);
        else w4_rows_kernel<BF16, GROUP, 2, 1, 8><<<grid, dim3(512), 0, stream>>>(a);
    } else if (r.c == 3 && r.waves == 16) w4_rows_kernel<BF16, GROUP, 1, 3, 16><<<grid, dim3(1024), 0, stream>>>(a);
    else if (r.c == 3) w4_rows_kernel<BF16, GROUP, 1, 3, 8><<<grid, dim3(512), 0, stream>>>(a);
    else if (r.c == 2 && r.waves == 16) w4_rows_kernel<BF16, GROUP, 1, 2, 16><<<grid, dim3(1024), 0, stream>>>(a);
    else if (r.c == 2) w4_rows_kernel<BF16, GROUP, 1, 2, 8><<<grid, dim3(512), 0, stream>>>(a);
    else if (r.waves == 16) w4_rows_kernel<BF16, GROUP, 1, 1, 16><<<grid, dim3(1024), 0, stream>>>(a);
    else w4_rows_kernel<BF16, GROUP, 1, 1, 8><<<grid, dim3(512), 0, stream>>>(a);
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

// Up to sixteen tokens: w4_rows_kernel.  As many tiles of channels to a workgroup, up to three, as leave the compute unit that has most with the fewest, and of equals the most, since every workgroup reads all
// activations (one and sixteen tokens, with one, two and three: 688 tiles of 4096 inputs 9.0, 9.4, 8.0 and 14.8, 12.5, 9.7 us; 320 of 13824 16.7, 15.5, 19.4 and 30.4, 19.5, 23.1; 256 of 4096 4.3, 5.4, 6.8 and 6.2,
// 6.9, 8.2; 1376 of 4096 15.3, 13.4, 13.3 and 27.0, 17.4, 16.3; four are never the least).  Sixteen waves where each then has four blocks and more (256 tiles of 11008 inputs 10.1 and 8.3 us, of 4096 inputs no difference).
// The same kernel with two blocks of tokens for up to 32, where the inputs and the compute units' tiles are few (17 and 32 tokens, this and w4_tiles_kernel: 11008 x 4096 11.5, 13.6 and 15.1, 16.9 us; 4096 x 4096 7.2, 9.8
// and 9.4, 10.6; 11008 x 2048 7.1, 8.4 and 11.0, 12.6; but 4096 x 6144 10.2, 14.1 and 11.0, 12.1, 22016 x 4096 20.9, 25.0 and 20.9, 22.2).
//
// More: w4_tiles_kernel, with the tokens and shares that promise the least time.  A workgroup takes 0.45 + 0.2 T us a block where it is alone on its compute unit and 0.3 + 0.17 T for each on it where there
// are more, its launch and the way to the first block are the same for all; shares cost a launch of 3.5 us and their sums' way out and in.  (77 x 5119 x 13800 in shares of 4: 39 us, 8: 34, 12: 30; 128 x 4096 x
// 4096 whole 46 us, in shares of 4 23, 8 23, 12 25; 512 x 4096 x 11008 whole 127, in 2 73, 4 63, 8 75; 1024 x 11008 x 4096 whole 114, in 2 138.)
W4Rule w4_rule(int64_t M, int64_t N, int64_t blocks)
{
    W4Rule r = {false, 1, 1, 1, 8};
    const int64_t tiles = (N + kW4Tile - 1) / kW4Tile;
    int64_t tiles_on_unit = INT64_MAX;
    for (int c = 1; c <= 3; ++c) {
        const int64_t n = ((tiles + c - 1) / c + 255) / 256 * c;
        if (n <= tiles_on_unit) {
            tiles_on_unit = n;
            r.c = c;
        }
    }
    if (M <= 16 || (M <= 32 && blocks <= 32 && tiles_on_unit <= 3)) {
        r.t = M <= 16 ? 1 : 2;
        r.waves = M <= 16 && blocks >= 64 ? 16 : 8;
        return r;
    }
    r.tiles = true;
    float least = 0.0f;
    for (int t = 1; t <= 4; ++t) {
        if (t < 4 && M > 96 * t) continue;  // (small tiles for many tokens)
        const int64_t groups = (M + 32 * t - 1) / (32 * t) * ((N + 127) / 128);
        for (int shares = 1; shares <= 16 && (shares == 1 || shares * 2 <= blocks); ++shares) {
            const int64_t on_unit = (groups * shares + 255) / 256;
            const float block = std::max(0.45f + 0.2f * t, (0.3f + 0.17f * t) * (float)on_unit);
            const float us = (float)((blocks + shares - 1) / shares) * block + (shares > 1 ? 3.5f + (float)(shares * M * N) * 2e-6f : 0.0f);
            if (least == 0.0f || us < least) {
                least = us;
                r.t = t;
                r.shares = shares;
            }
        }
    }
    return r;
}

int64_t w4_items(int64_t M, int64_t N, const W4Rule &r)
{
    if (!r.tiles) return (N + kW4Tile * r.c - 1) / (kW4Tile * r.c) * 64 * r.waves;
    const int64_t first = (M + 32 * r.t - 1) / (32 * r.t) * ((N + 127) / 128) * r.shares * 256;
    return r.shares > 1 ? std::max(first, M * w4_partial_stride(N) / 4 + 256) : first;
}

hipError_t launch_w4_gemm(const W4Args &a, const W4Rule &r, int group, bool bf16, hipStream_t stream)
{
    if (r.tiles) return launch_w4_tiles(a, r, group, bf16, stream);
    auto go = [&](auto b) {
        constexpr bool B = decltype(b)::value;
        if (group == 32) launch<B, 32>(a, r, stream);
        else if (group == 64) launch<B, 64>(a, r, stream);
        else launch<B, 128>(a, r, stream);
    };
    if (bf16) go(std::true_type());
    else go(std::false_type());
    return hipGetLastError();
}

}  // namespace apmm
