// host_wave's header with what the sources of rotary positions and of the cache's budget use beside it: launches of two dimensions, additions in LDS, counts of bits, sines of half turns.
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
inline void sincospif(float x, float *s, float *c)
{
    const double t = std::remainder((double)x, 2.0) * 3.14159265358979323846;
    *s = (float)std::sin(t);
    *c = (float)std::cos(t);
}
inline uint32_t host_mbcnt_lo(uint32_t mask, uint32_t v) { const int l = host_wave::lane(); return v + __builtin_popcount(l >= 32 ? mask : mask & ((1u << l) - 1)); }
inline uint32_t host_mbcnt_hi(uint32_t mask, uint32_t v) { const int l = host_wave::lane(); return l <= 32 ? v : v + __builtin_popcount(mask & ((1u << (l - 32)) - 1)); }
#define __builtin_amdgcn_mbcnt_lo host_mbcnt_lo
#define __builtin_amdgcn_mbcnt_hi host_mbcnt_hi
