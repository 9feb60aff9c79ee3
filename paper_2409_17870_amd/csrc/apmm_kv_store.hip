// Writing the four-bit key/value cache and reading it back.
//
// One wave takes the up to eight tokens of an aligned eight of positions, one head (or two of 64 channels), keys and values: eight lanes to a token.  The eight tokens of
// a channel are neighbours in the cache's values, so they are turned in LDS and written whole (an eight that is not all new is written in pieces of 16 bits, what is there
// of earlier tokens stays).  Bound by HBM: 4 bytes a channel in or out,
// one and a bit in the cache.  Reading 16384 tokens of 32 heads of 128: 338 MB in 61 us, 5.5 TB/s (a large copy: 5.1); writing 2048 of 40 heads: 53 MB in 13 us, some 4 of them the launch and
// the way from lengths and pages to the first row.  (Two pieces of 16 bytes to a lane side by side, in place of 128 bytes to eight lanes, took 75 us of the first.)
#include "apmm_kv_store.h"

namespace apmm {

namespace {

constexpr int kWaves = 4;
// Heads of a wave: two of 64 channels where there is enough for two rounds of waves, or finding its eight costs as much as moving it (3 sequences of 37000 tokens, 16 heads of 64, read
// back: 147 us with one, 120 with two; pieces of 333 tokens and single ones of 23 sequences, 8 heads: 4.2 and 4.7)
constexpr int kManyUnits = 16384;
template <int D>
__device__ __forceinline__ int heads_of_wave(const KvArgs &c) { return D == 64 ? c.per_wave : 1; }
// The eight of a wave, and the first of its heads (by_heads is that of the heads' groups of `per`, 1 or 2)
__device__ __forceinline__ int eight_of_wave(const KvArgs &c, int per, int &head)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = blockIdx.x * kWaves + wave, eight = kv_divide(unit, c.by_heads);  // (fewer than 2^26 units, kv_store_items)
    head = (unit - eight * (per == 1 ? c.heads : (c.heads + 1) >> 1)) * per;
    return eight;
}

template <int D, bool BF16>
__global__ __launch_bounds__(64 * kWaves) void kv_write_kernel(KvArgs c, KvTensor k, KvTensor v)
{
    constexpr int N = D / 16;  // words of a lane's channels, two to a word
    __shared__ __align__(16) kv_u16 turn[kWaves][D / 4 * 8];
    Eight e;
    const int per = heads_of_wave<D>(c);
    int first;
    if (!find_eight(c, eight_of_wave(c, per, first), e) || e.page < 0) return;
    const int lane = kv_lane(), token = lane >> 3, part = lane & 7;
    const int64_t row = e.s.start + (e.is_new ? e.first + token - e.s.first : 0);  // (a lane without one reads the first)
    for (int head = first; head < min(first + per, c.heads); ++head) {
        uint32_t xk[N], xv[N];
        load_row(k.data + row * k.token_stride + head * k.head_stride, k.aligned, part, xk);
        load_row(v.data + row * v.token_stride + head * v.head_stride, v.aligned, part, xv);
        uint32_t uk[N / 4], uv[N / 4];
        const uint32_t sk = quantise<N, BF16>(xk, uk), sv = quantise<N, BF16>(xv, uv);

        write_codes<D>(c, e, head, uk, sk, uv, sv, turn[threadIdx.x >> 6]);
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
    int first;
    if (!find_eight(c, eight_of_wave(c, per, first), e)) return;
    const int lane = kv_lane(), token = lane >> 3, part = lane & 7;
    const bool there = e.page >= 0;
    for (int head = first; head < min(first + per, c.heads); ++head) {
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

int heads_of_a_wave(const KvArgs &c) { return c.head_dim == 64 && kv_eights(c) * c.heads >= kManyUnits ? 2 : 1; }
int64_t workgroups(const KvArgs &c)
{
    const int per_wave = heads_of_a_wave(c);
    return (kv_eights(c) * ((c.heads + per_wave - 1) / per_wave) + kWaves - 1) / kWaves;
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
