// host_wave's header with what the sources of rotary positions, of the cache's budget and of the products with four-bit weights use beside it: launches of two dimensions, additions in LDS, counts of bits, matrix
// instructions of bfloat16, loads to LDS that arrive where they are waited for.
#pragma once
#define dim3 host_wave_dim3
#include "../../host_wave/hip/hip_runtime.h"
#undef dim3
#undef blockIdx

struct dim3 {
    uint32_t x, y;
    dim3(uint32_t x, uint32_t y = 1) : x(x), y(y) {}
};
struct float4 { float x, y, z, w; };
inline float4 make_float4(float x, float y, float z, float w) { return {x, y, z, w}; }

namespace host_layers {

inline dim3 block(0), grid(0);

inline void launch(dim3 groups, dim3 threads, const std::function<void()> &f)
{
    grid = groups;
    for (block.y = 0; block.y < groups.y; ++block.y)
        for (block.x = 0; block.x < groups.x; ++block.x) host_wave::run_block((int)threads.x, f);
}

}  // namespace host_layers

#define blockIdx host_layers::block
#define gridDim host_layers::grid
inline int64_t min(int64_t a, int b) { return b < a ? b : a; }
inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
inline uint32_t atomicAdd(uint32_t *p, uint32_t v) { const uint32_t was = *p; *p += v; return was; }
inline uint32_t host_mbcnt_lo(uint32_t mask, uint32_t v) { const int l = host_wave::lane(); return v + __builtin_popcount(l >= 32 ? mask : mask & ((1u << l) - 1)); }
inline uint32_t host_mbcnt_hi(uint32_t mask, uint32_t v) { const int l = host_wave::lane(); return l <= 32 ? v : v + __builtin_popcount(mask & ((1u << (l - 32)) - 1)); }
#define __builtin_amdgcn_mbcnt_lo host_mbcnt_lo
#define __builtin_amdgcn_mbcnt_hi host_mbcnt_hi

// ---------------------------------------------------------------- products
namespace host_layers {

typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));

inline float bf16_value(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
struct Bf16Operands { uint16_t a[8], b[8]; };
template <int SIDE, int K, class Acc>  // as host_wave::mfma
Acc mfma_bf16(bf8_t a, bf8_t b, Acc c)
{
    Bf16Operands mine;
    std::memcpy(mine.a, &a, 16);
    std::memcpy(mine.b, &b, 16);
    const auto all = host_wave::exchange(mine);
    constexpr int N = sizeof(Acc) / sizeof(float);
    const int l = host_wave::lane();
    for (int i = 0; i < N; ++i) {
        const int row = SIDE == 16 ? 4 * (l / 16) + i : 8 * (i / 4) + 4 * (l / 32) + i % 4;
        float s = c[i];
        for (int g = 0; g < K / 8; ++g) {
            const Bf16Operands x = all[g * SIDE + row], y = all[g * SIDE + l % SIDE];
            for (int k = 0; k < 8; ++k) s += bf16_value(x.a[k]) * bf16_value(y.b[k]);
        }
        c[i] = s;
    }
    return c;
}
inline host_wave::float4_t mfma16_bf16(bf8_t a, bf8_t b, host_wave::float4_t c, int, int, int) { return mfma_bf16<16, 32>(a, b, c); }
inline host_wave::float16_t mfma32_bf16(bf8_t a, bf8_t b, host_wave::float16_t c, int, int, int) { return mfma_bf16<32, 16>(a, b, c); }

// The loads of each lane's wave that are on their way, oldest first.  One without `to` is the compiler's own, which arrives by itself and counts here alone.
struct OnItsWay {
    uint4 *to;
    const void *from;
};
inline std::vector<std::vector<OnItsWay>> on_their_way(1024);
inline char *lds;
inline size_t lds_bytes;

inline std::vector<OnItsWay> &mine() { return on_their_way[host_wave::current]; }
inline uint32_t lds_begins(void *at, size_t bytes)
{
    lds = static_cast<char *>(at);
    lds_bytes = bytes;
    mine().clear();  // (a lane's first steps)
    return 0;
}
inline void issued(int n)
{
    for (int i = 0; i < n; ++i) mine().push_back({nullptr, nullptr});
}
inline void load_to_lds(uint32_t to, uint32_t from, const void *base)
{
    const size_t at = to + 16 * (size_t)host_wave::lane();
    if (at + 16 > lds_bytes) std::fprintf(stderr, "host_layers: a load behind the LDS that there is\n"), std::abort();
    volatile const char *touched = static_cast<const char *>(base) + from;
    (void)touched[0];
    (void)touched[15];
    mine().push_back({reinterpret_cast<uint4 *>(lds + at), static_cast<const char *>(base) + from});
}
inline void arrive(int but)
{
    auto &all = mine();
    const size_t n = all.size() > (size_t)but ? all.size() - but : 0;
    for (size_t i = 0; i < n; ++i)
        if (all[i].to) std::memcpy(all[i].to, all[i].from, 16);
    all.erase(all.begin(), all.begin() + n);
}

}  // namespace host_layers

#define __builtin_amdgcn_mfma_f32_16x16x32_bf16 host_layers::mfma16_bf16
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16 host_layers::mfma32_bf16
inline uint32_t host_alignbit(uint32_t high, uint32_t low, uint32_t by) { return (uint32_t)(((uint64_t)high << 32 | low) >> (by & 31)); }
#define __builtin_amdgcn_alignbit host_alignbit
