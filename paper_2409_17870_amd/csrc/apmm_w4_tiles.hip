// Four-bit weights with group scales times 16-bit activations (apmm_w4.h), more tokens than few.
//
// A workgroup has 128 channels, 32 to each of its four waves (or pairs of waves), 32 T tokens and a share of the inputs.  Activations of 128 inputs at a time go through LDS, straight from memory, the next blocks on their way
// while one is used; a wave's weights come into registers as codes and become operands there: no two waves unpack the same.  Where there are few tiles the inputs are cut in shares, whose sums of 32 bits
// meet in a second launch.
// A group's sum is multiplied with its scale in 32 bits, one instruction for each result and group.  (With weights times scales rounded to 16 bits it is none, a wave has registers for 64 channels, and
// 2048 x 11008 x 4096 took 190 us where this form then took 205, at 1.4 times the error of an exact product's rounding; groups of 32 inputs 205 and 260.)
//
// What bounds many tokens: LDS, which gives every wave all of the block's activations, 128 bytes a clock at the full rate of the matrix unit, and beside it the vector unit (unpacking 43 % (bfloat16) or 28 %
// (binary16) of the matrix unit's time at T = 4, the groups' products 25, 50 or 100 %): two workgroups on a compute unit, so that one's vector instructions run under the other's products.
// 2048 x 11008 x 4096 takes 197 us, 937 TFLOP/s, where calls follow each other (240 in the first twenty after a pause).  (A wave with 64 channels, which halves what is read from LDS, took 207 to 260, with two waves to a vector unit or one: it is not LDS alone.)
// What bounds a few: a workgroup's way from its first load to its first product (5 us with launch and join), then 0.45 + 0.2 T us a block for one workgroup to a compute unit.
#include <type_traits>

#include "apmm_w4.h"

namespace apmm {

namespace {

typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kChannels = 32;  // channels of a wave

template <bool BF16>
__device__ __forceinline__ float16v multiply(typename W4Type<BF16>::Eight a, typename W4Type<BF16>::Eight b, float16v c)
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// 1 KiB from memory to LDS, lane l's 16 bytes at base + voff to lds + 16 l.  By hand: behind the builtin the compiler waits for every such load before any LDS read that it cannot tell apart from it.
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t voff, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
// All but this wave's last N loads have arrived and what it asked of LDS is done; then the same of every wave
template <int N>
__device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

// Blocks of activations in LDS: the one in use and those on their way.  As many as leave room for two workgroups on a compute unit (three of one block of tokens).
constexpr int ring_of(int t) { return t == 1 ? 6 : t == 2 ? 4 : t == 3 ? 3 : 2; }

// Two waves to the same channels, half of a block's inputs each, where the groups' products keep a wave busy between matrix instructions (groups of 32, with and without: 77 x 5119 x 13800 34 and 41 us, 96 x 11008 x 4096
// 29 and 35, 64 x 5119 x 13800 26 and 31; groups of 64 31 and 36, 27 and 31, 25 and 28; of 128 no difference; one block of tokens 17 and 16 us; four, and rows at any address, have no registers for it)
constexpr int halves_of(int group, int t, bool direct) { return direct && group < 128 && (t == 2 || t == 3) ? 2 : 1; }

// DIRECT: rows of x begin at multiples of 16 bytes and a tile's lie within 2^31 bytes
template <bool BF16, int GROUP, int T, bool DIRECT>
__global__ __launch_bounds__(64 * kWaves * halves_of(GROUP, T, DIRECT), 2 * halves_of(GROUP, T, DIRECT)) void w4_tiles_kernel(W4Args a, int tiles_m, int shares)
{
    typedef typename W4Type<BF16>::Eight Eight;
    constexpr int H = halves_of(GROUP, T, DIRECT), kPart = kW4Block / H;  // inputs of a block that a wave multiplies
    constexpr int kGroups = kPart / GROUP, kTokens = 32 * T, kSteps = GROUP / 16, R = ring_of(T);
    constexpr int kRows = 2 * T / H, kLoads = kRows + 2 + kGroups;  // of a wave for a block: activations, codes, scales
    __shared__ uint4 rows[R][kTokens * 16];      // [token][eight of inputs, its number xor token % 16]
    const int any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = any_wave % kWaves, half = any_wave / kWaves, lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    // a die's workgroups (every eighth) take work that follows each other: the shares of a tile, then the tiles of the same channels, whose weights meet in its L2
    const int all = gridDim.x, id = all % 8 == 0 ? (int)(blockIdx.x % 8) * (all / 8) + (int)(blockIdx.x / 8) : (int)blockIdx.x;
    const int tile = id / shares, share = id - tile * shares, tn = tile / tiles_m, tm = tile - tn * tiles_m, m0 = tm * kTokens, n0 = (tn * kWaves + wave) * kChannels;
    const int first = (int)((int64_t)a.blocks * share / shares), last = (int)((int64_t)a.blocks * (share + 1) / shares);

    const int last_tile = (a.N + kW4Tile - 1) / kW4Tile - 1;
    const int64_t packed_tile = min((n0 + n) / kW4Tile, last_tile);  // (channels behind the last: results that are not written)
    const uint8_t *codes = a.packed + packed_tile * a.blocks * kW4BlockBytes + ((n & 15) + 16 * h) * 16 + half * 8;
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(a.packed + a.code_bytes) + (packed_tile * a.blocks * H + half) * kGroups * kW4Tile + (n & 15);
    uint32_t from[DIRECT ? kRows : 1];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4 *)&rows[0][0];
    const uint16_t *x0 = a.x + m0 * a.x_stride;
    if (DIRECT) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int token = 4 * (any_wave * kRows + i) + (lane >> 4), eight = (lane & 15) ^ (token & 15);
            from[i] = (uint32_t)(min(token, a.M - 1 - m0) * (int)a.x_stride * 2 + eight * 16);
        }
    }
    auto stage = [&](int b, int to) {
        if (DIRECT && (b + 1) * kW4Block <= a.K) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) load_to_lds(x0 + b * kW4Block, from[i], lds0 + (uint32_t)(to * kTokens * 256 + (any_wave * kRows + i) * 1024));
        } else {
            for (int i = threadIdx.x; i < kTokens * 16; i += 64 * kWaves * H) {
                const int token = i >> 4, eight = (i & 15) ^ (token & 15);
                rows[to][i] = w4_row_eight<uint4>(x0 + min(token, a.M - 1 - m0) * a.x_stride, b * kW4Block + eight * 8, a.K);
            }
        }
    };
    typedef typename std::conditional<H == 1, uint4, uint2>::type Codes;
    struct Weights {
        Codes w[2];
        uint16_t s[kGroups];
    } weights[R];
    auto load_weights = [&](int b, Weights &to) {
#pragma unroll
        for (int i = 0; i < 2; ++i) to.w[i] = *reinterpret_cast<const Codes *>(codes + (int64_t)b * kW4BlockBytes + i * 512);
#pragma unroll
        for (int i = 0; i < kGroups; ++i) to.s[i] = scales[((int64_t)b * H * kGroups + i) * kW4Tile];
    };

    float16v acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[t][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < R - 1; ++i)
        if (first + i < last) {
            load_weights(first + i, weights[i]);
            stage(first + i, i);
        }
    auto block = [&](int b, auto place) {  // place: of the block in the ring
        constexpr int at = decltype(place)::value;
        // behind this block's loads there are those of R - 2 others, each as many (a last block that ends within has its rows waited for as they are loaded), or fewer at the end
        if (b + R - 2 < last) wait_and_meet<(R - 2) * kLoads>();
        else wait_and_meet<0>();
        uint32_t words[8 / H];  // of sixteen inputs each, this lane's half of them
#pragma unroll
        for (int i = 0; i < 8 / H; ++i) words[i] = reinterpret_cast<const uint32_t *>(&weights[at].w[i & 1])[i >> 1];
        float scales_of[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) scales_of[g] = w4_scale<BF16>(weights[at].s[g]);
        // taken here, before the next loads are begun: a first use behind them would be waited for with all of them, since the compiler cannot tell how many they are (256 x 11008 x 4096 44 us in place of 51, 2048 196 in
        // place of 205)
#pragma unroll
        for (int i = 0; i < 8 / H; ++i) asm volatile("" : "+v"(words[i]));
#pragma unroll
        for (int g = 0; g < kGroups; ++g) asm volatile("" : "+v"(scales_of[g]));
        if (b + R - 1 < last) {
            load_weights(b + R - 1, weights[(at + R - 1) % R]);
            stage(b + R - 1, (at + R - 1) % R);
        }
        const uint4 *here = &rows[at][n * 16];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            Eight w[kSteps];
#pragma unroll
            for (int k = 0; k < kSteps; ++k) w[k] = w4_operand<BF16>(words[g * kSteps + k]);
            const float scale = scales_of[g];
#pragma unroll
            for (int t = 0; t < T; ++t) {
                float16v part;
#pragma unroll
                for (int i = 0; i < 16; ++i) part[i] = 0.0f;
#pragma unroll
                for (int k = 0; k < kSteps; ++k)
                    part = multiply<BF16>(__builtin_bit_cast(Eight, here[t * 32 * 16 + ((kPart / 8 * half + 2 * (g * kSteps + k) + h) ^ (n & 15))]), w[k], part);
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][i] = fmaf(part[i], scale, acc[t][i]);
                if (GROUP < 128 && T > 2) __builtin_amdgcn_sched_barrier(0);  // (the compiler would begin sums of all groups at a time, for which there are no registers)
            }
#pragma unroll
            for (int t = 0; t < T; ++t) asm volatile("" : "+v"(acc[t]));  // (nor are these products put off to the end of the loop)
        }
    };
    for (int b = first; b < last; b += R) {
        block(b, std::integral_constant<int, 0>());
        if (b + 1 < last) block(b + 1, std::integral_constant<int, 1>());
        if (R > 2 && b + 2 < last) block(b + 2, std::integral_constant<int, 2 % R>());
        if (R > 3 && b + 3 < last) block(b + 3, std::integral_constant<int, 3 % R>());
        if (R > 4 && b + 4 < last) block(b + 4, std::integral_constant<int, 4 % R>());
        if (R > 5 && b + 5 < last) block(b + 5, std::integral_constant<int, 5 % R>());
    }
    if (H > 1) {  // the halves meet in the place of the activations
        float4 *const meet = reinterpret_cast<float4 *>(&rows[0][0]) + wave * T * 4 * 64 + lane;
        static_assert(kWaves * 4 * 64 <= R * 32 * 16, "");
        __syncthreads();
        if (half) {
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) meet[(t * 4 + i) * 64] = make_float4(acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]);
        }
        __syncthreads();
        if (half) return;
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 x = meet[(t * 4 + i) * 64];
                acc[t][4 * i] += x.x; acc[t][4 * i + 1] += x.y; acc[t][4 * i + 2] += x.z; acc[t][4 * i + 3] += x.w;
            }
    }
    const int64_t stride = w4_partial_stride(a.N);
    float *partial = a.partial + share * a.M * stride;
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = m0 + 32 * t + 8 * (i / 4) + 4 * h + i % 4, channel = n0 + n;
            if (row >= a.M || channel >= a.N) continue;
            if (shares > 1) partial[row * stride + channel] = acc[t][i];
            else a.y[row * a.y_stride + channel] = w4_round<BF16>(acc[t][i]);
        }
}

// Sums of the shares of the inputs, four channels to a lane
template <bool BF16>
__global__ __launch_bounds__(256) void w4_join_kernel(W4Args a, int shares)
{
    const int64_t stride = w4_partial_stride(a.N), quads = stride / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = i / quads;
    const int channel = (int)(i - row * quads) * 4;
    if (row >= a.M) return;
    float4 all = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float *at = a.partial + row * stride + channel;
#pragma unroll 4
    for (int s = 0; s < shares; ++s) {
        const float4 x = *reinterpret_cast<const float4 *>(at + (int64_t)s * a.M * stride);
        all.x += x.x; all.y += x.y; all.z += x.z; all.w += x.w;  // (behind the last channel: what lies there, not written)
    }
    const float v[4] = {all.x, all.y, all.z, all.w};
    uint16_t *y = a.y + row * a.y_stride + channel;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (channel + c < a.N) y[c] = w4_round<BF16>(v[c]);
}

template <bool BF16, int GROUP, int T>
void launch(const W4Args &a, const W4Rule &r, hipStream_t stream)
{
    const bool direct = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && a.x_stride % 8 == 0 && a.x_stride < (1 << 22);
    const int tiles_m = (a.M + 32 * T - 1) / (32 * T), tiles_n = (a.N + kWaves * kChannels - 1) / (kWaves * kChannels);
    const dim3 grid((uint32_t)((int64_t)tiles_m * tiles_n * r.shares)), block(64 * kWaves * halves_of(GROUP, T, true)), one(64 * kWaves);
    if (direct) w4_tiles_kernel<BF16, GROUP, T, true><<<grid, block, 0, stream>>>(a, tiles_m, r.shares);
    else w4_tiles_kernel<BF16, GROUP, T, false><<<grid, one, 0, stream>>>(a, tiles_m, r.shares);
    if (r.shares > 1) w4_join_kernel<BF16><<<dim3((uint32_t)((a.M * (w4_partial_stride(a.N) / 4) + 255) / 256)), dim3(256), 0, stream>>>(a, r.shares);
}

template <bool BF16, int GROUP>
void launch(const W4Args &a, const W4Rule &r, hipStream_t stream)
{
    if (r.t == 1) launch<BF16, GROUP, 1>(a, r, stream);
    else if (r.t == 2) launch<BF16, GROUP, 2>(a, r, stream);
    else if (r.t == 3) launch<BF16, GROUP, 3>(a, r, stream);
    else launch<BF16, GROUP, 4>(a, r, stream);
}

}  // namespace

hipError_t launch_w4_tiles(const W4Args &a, const W4Rule &r, int group, bool bf16, hipStream_t stream)
{
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
