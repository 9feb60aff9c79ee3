// Device code on the host, for tests: the lanes of a workgroup are contexts of one thread that take turns, and change places wherever a wave exchanges something (moves between lanes,
// ballots, matrix instructions, wave fences) or the workgroup meets at a barrier.  Between two such places one lane runs after the other, so that an exchange through LDS without a fence
// reads what was there before.  Covers what the key/value cache's sources use; matrix instructions of gfx950, 64 lanes to a wave.
#pragma once
#include <csetjmp>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <vector>

#include <sys/mman.h>
#include <ucontext.h>

#define __HIPCC__ 1
#define __host__
#define __device__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define __align__(n) __attribute__((aligned(n)))

struct uint2 { uint32_t x, y; };
struct uint4 { uint32_t x, y, z, w; };
struct float2 { float x, y; };
inline uint2 make_uint2(uint32_t x, uint32_t y) { return {x, y}; }
inline uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return {x, y, z, w}; }
inline float2 make_float2(float x, float y) { return {x, y}; }
struct dim3 {
    uint32_t x;
    dim3(uint32_t n) : x(n) {}
};
typedef void *hipStream_t;
typedef int hipError_t;
constexpr hipError_t hipSuccess = 0;
inline hipError_t hipGetLastError() { return hipSuccess; }

#define WAVE_MIN_MAX(T)                               \
    inline T min(T a, T b) { return b < a ? b : a; } \
    inline T max(T a, T b) { return a < b ? b : a; }
WAVE_MIN_MAX(int)
WAVE_MIN_MAX(uint32_t)
WAVE_MIN_MAX(int64_t)

namespace host_wave {

struct Words { uint32_t w[8]; };  // what a lane gives
enum Wait { kReady, kWave, kBlock, kDone };
struct Lane {
    jmp_buf at;
    ucontext_t begin;
    char *stack = nullptr;
    bool begun;
    Wait wait;
    int turn;
    Words given[2];
    dim3 thread{0};
};
constexpr size_t kStack = 512 << 10;

inline std::vector<Lane> lanes;
inline int current;
inline dim3 block{0};
inline jmp_buf scheduler;
inline const std::function<void()> *body;

inline Lane &self() { return lanes[current]; }
inline void wait(Wait for_what)
{
    self().wait = for_what;
    if (_setjmp(self().at) == 0) _longjmp(scheduler, 1);
}
// Gives `mine` and returns what lane l of this wave gave
template <class T>
struct Given {
    const Lane *wave;
    int turn;
    T operator[](int l) const
    {
        T v;
        std::memcpy(&v, wave[l].given[turn].w, sizeof(T));
        return v;
    }
    bool there(int l) const { return wave[l].wait != kDone; }
};
template <class T>
Given<T> exchange(const T &mine)
{
    static_assert(sizeof(T) <= sizeof(Words), "");
    Lane &me = self();
    const int turn = me.turn;
    std::memcpy(me.given[turn].w, &mine, sizeof(T));
    me.turn ^= 1;
    wait(kWave);
    return {&lanes[current & ~63], turn};
}
inline int lane() { return current & 63; }

inline void run()
{
    (*body)();
    wait(kDone);
    std::abort();
}
inline void resume(int i)
{
    current = i;
    Lane &l = lanes[i];
    if (_setjmp(scheduler)) return;
    if (l.begun) _longjmp(l.at, 1);
    l.begun = true;
    setcontext(&l.begin);
}
inline void run_block(int threads, const std::function<void()> &f)
{
    body = &f;
    if ((int)lanes.size() < threads) lanes.resize(threads);
    for (int i = 0; i < threads; ++i) {
        Lane &l = lanes[i];
        if (!l.stack) l.stack = static_cast<char *>(mmap(nullptr, kStack, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
        getcontext(&l.begin);
        l.begin.uc_stack.ss_sp = l.stack;
        l.begin.uc_stack.ss_size = kStack;
        l.begin.uc_link = nullptr;
        makecontext(&l.begin, run, 0);
        l.begun = false;
        l.wait = kReady;
        l.turn = 0;
        l.thread.x = i;
    }
    for (int left = threads; left;) {
        left = 0;
        int at_barrier = 0;
        for (int w = 0; w < threads; w += 64) {
            bool ready = true;
            while (ready) {  // this wave, until it waits for others
                int waiting = 0;
                ready = false;
                for (int i = w; i < w + 64 && i < threads; ++i)
                    if (lanes[i].wait == kReady) resume(i);
                for (int i = w; i < w + 64 && i < threads; ++i) waiting += lanes[i].wait == kBlock;
                for (int i = w; i < w + 64 && i < threads; ++i)
                    if (lanes[i].wait == kWave) {
                        if (waiting) std::fprintf(stderr, "host_wave: lanes of a wave wait in different places\n"), std::abort();
                        lanes[i].wait = kReady;
                        ready = true;
                    }
            }
        }
        for (int i = 0; i < threads; ++i) left += lanes[i].wait != kDone, at_barrier += lanes[i].wait == kBlock;
        if (at_barrier != left) std::fprintf(stderr, "host_wave: a barrier that not all reach\n"), std::abort();
        for (int i = 0; i < threads; ++i)
            if (lanes[i].wait == kBlock) lanes[i].wait = kReady;
    }
}
inline void launch(dim3 grid, dim3 threads, const std::function<void()> &f)
{
    for (uint32_t b = 0; b < grid.x; ++b) {
        block.x = b;
        run_block((int)threads.x, f);
    }
}

// -------------------------------------------------------------------- moves
template <class T>
T shfl_xor(T v, int d) { return exchange(v)[lane() ^ d]; }
inline uint64_t ballot(bool p)
{
    const auto all = exchange((int)p);
    uint64_t m = 0;
    for (int i = 0; i < 64; ++i)
        if (all.there(i) && all[i]) m |= 1ull << i;
    return m;
}
inline int readlane(int v, int l)
{
    if (l < 0 || l > 63) std::fprintf(stderr, "host_wave: lane %d of a wave is read\n", l), std::abort();
    return exchange(v)[l];
}
inline int update_dpp(int old, int v, int ctrl, int row_mask, int bank_mask, bool zero)
{
    const auto all = exchange(v);
    const int l = lane();
    if (!(row_mask >> (l / 16) & 1) || !(bank_mask >> (l % 16 / 4) & 1)) return old;
    int from = -1;
    if (ctrl < 0x100) from = (l & ~3) | (ctrl >> (2 * (l & 3)) & 3);              // any order of four
    else if (ctrl > 0x110 && ctrl < 0x120) from = l % 16 >= (ctrl & 15) ? l - (ctrl & 15) : -1;
    else if (ctrl == 0x140) from = l ^ 15;                                        // sixteen mirrored
    else if (ctrl == 0x141) from = l ^ 7;                                         // eight mirrored
    else if (ctrl == 0x142) from = l >= 16 ? (l & ~15) - 1 : -1;
    else if (ctrl == 0x143) from = l >= 32 ? 31 : -1;
    else std::abort();
    return from < 0 ? (zero ? 0 : old) : all[from];
}
inline uint32_t perm(uint32_t high, uint32_t low, uint32_t select)
{
    const uint64_t both = (uint64_t)high << 32 | low;
    uint32_t r = 0;
    for (int i = 0; i < 4; ++i) r |= (uint32_t)(both >> (8 * (select >> (8 * i) & 7)) & 0xff) << (8 * i);
    return r;
}

// --------------------------------------------------------------- arithmetic
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));

inline float exp2_of(float x)
{
    const float r = exp2f(x);
    return r < 0x1p-126f ? 0.0f : r;  // v_exp_f32 has no subnormal results
}
inline float fdot2(half2_t a, half2_t b, float c, bool) { return (float)a[0] * (float)b[0] + (float)a[1] * (float)b[1] + c; }
struct Operands { _Float16 a[8], b[8]; };
static_assert(sizeof(Operands) == sizeof(Words), "");
template <int SIDE, int K, int N>  // a: SIDE x K, b: K x SIDE; N results a lane
inline void mfma(half8_t a, half8_t b, float (&acc)[N])
{
    Operands mine;
    for (int i = 0; i < 8; ++i) mine.a[i] = a[i], mine.b[i] = b[i];
    exchange(mine);
    const Lane *wave = &lanes[current & ~63];
    const int turn = self().turn ^ 1, l = lane(), col = l % SIDE;
    auto operands = [&](int i) { return reinterpret_cast<const Operands *>(wave[i].given[turn].w); };
    for (int i = 0; i < N; ++i) {
        const int row = SIDE == 16 ? 4 * (l / 16) + i : 8 * (i / 4) + 4 * (l / 32) + i % 4;
        float s = acc[i];
        for (int g = 0; g < K / 8; ++g) {
            const Operands *x = operands(g * SIDE + row), *y = operands(g * SIDE + col);
            for (int k = 0; k < 8; ++k) s += (float)x->a[k] * (float)y->b[k];
        }
        acc[i] = s;
    }
}
inline float4_t mfma16(half8_t a, half8_t b, float4_t c, int, int, int)
{
    float acc[4];
    for (int i = 0; i < 4; ++i) acc[i] = c[i];
    mfma<16, 32>(a, b, acc);
    for (int i = 0; i < 4; ++i) c[i] = acc[i];
    return c;
}
inline float16_t mfma32(half8_t a, half8_t b, float16_t c, int, int, int)
{
    float acc[16];
    for (int i = 0; i < 16; ++i) acc[i] = c[i];
    mfma<32, 16>(a, b, acc);
    for (int i = 0; i < 16; ++i) c[i] = acc[i];
    return c;
}

}  // namespace host_wave

#define threadIdx (host_wave::self().thread)
#define blockIdx (host_wave::block)
inline void __syncthreads() { host_wave::wait(host_wave::kBlock); }
template <class T>
T __shfl_xor(T v, int d) { return host_wave::shfl_xor(v, d); }
inline uint64_t __ballot(bool p) { return host_wave::ballot(p); }
inline bool __any(bool p) { return host_wave::ballot(p) != 0; }
inline int __ffsll(long long v) { return __builtin_ffsll(v); }
inline float __uint_as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
inline uint32_t __float_as_uint(float v) { return __builtin_bit_cast(uint32_t, v); }
#define __builtin_amdgcn_readlane host_wave::readlane
#define __builtin_amdgcn_readfirstlane(v) host_wave::readlane((int)(v), 0)
#define __builtin_amdgcn_update_dpp host_wave::update_dpp
#define __builtin_amdgcn_perm host_wave::perm
#define __builtin_amdgcn_exp2f host_wave::exp2_of
#define __builtin_amdgcn_fdot2 host_wave::fdot2
#define __builtin_amdgcn_mfma_f32_16x16x32_f16 host_wave::mfma16
#define __builtin_amdgcn_mfma_f32_32x32x16_f16 host_wave::mfma32
#define __builtin_amdgcn_fence(...) host_wave::wait(host_wave::kWave)
#define __builtin_amdgcn_sched_barrier(...) ((void)0)
#define __builtin_amdgcn_s_waitcnt(...) ((void)0)
