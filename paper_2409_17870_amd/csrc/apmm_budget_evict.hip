// Keeping the heaviest tokens of the four-bit cache: which of a sequence and head stay (radix selection of the budget-th largest weight, ties to the lower place), and the copy to other pages.
#include <algorithm>

#include "apmm_budget.h"

namespace apmm {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kDigits = 2048;  // 11 bits at a time: 11, 11 and 10

// Weights as numbers that order like them: 0 for a token without a page (which never stays), 1 for NaN and tokens without a weight, the largest for those that stay whatever their weight
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 1;
    const uint32_t u = __float_as_uint(w + 0.0f);  // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Tokens {
    const KvEvictArgs &a;
    const float *w;
    const int32_t *table;
    int keys, length;
    __device__ __forceinline__ uint32_t operator()(int t) const
    {
        if (t >= keys) return 0;
        const int page = table[t >> a.c.page_shift];
        if (page < 0 || page >= a.c.pages) return 0;
        if (t < a.sinks || t >= length - a.recent) return 0xffffffffu;
        return t < a.w.capacity ? order_of(w[t]) : 1u;
    }
};

// A workgroup to a sequence and head.  Three passes find the budget-th largest number, digit by digit from the highest; then each wave takes a stretch of tokens, counts those that stay, and after the
// counts have met writes them in their order.
__global__ __launch_bounds__(kThreads) void kv_select_kernel(KvEvictArgs a)
{
    __shared__ uint32_t digits[kDigits];
    __shared__ int above[kWaves], equal[kWaves];
    __shared__ uint32_t found_digit, found_rest;
    const int b = blockIdx.x, head = blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane();
    const int length = min(max(a.c.lengths[b], 0), kKvMost), keys = (int)min((int64_t)length, (int64_t)a.c.width << a.c.page_shift);
    const Tokens order = {a, a.w.data + b * a.w.sequence_stride + head * a.w.head_stride, a.c.table + b * a.c.table_stride, keys, length};
    uint32_t least = 0, rest = (uint32_t)a.budget;  // what the digits so far say; how many are wanted of those that begin with them
    bool all = false;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        const uint32_t mask = (1u << bits) - 1, upper = pass == 0 ? 0 : ~0u << (shift + bits);
        for (int i = threadIdx.x; i < kDigits; i += kThreads) digits[i] = 0;
        if (threadIdx.x == 0) found_digit = 0xffffffffu;
        __syncthreads();
        for (int t = threadIdx.x; t < keys; t += kThreads) {
            const uint32_t v = order(t);
            if (v && (v & upper) == (least & upper)) atomicAdd(&digits[v >> shift & mask], 1u);
        }
        __syncthreads();
        if (wave == 0) {  // from the highest digit down: each lane has 32 that follow each other
            uint32_t own = 0;
            const int high = kDigits - 1 - 32 * lane;
            for (int i = 0; i < 32; ++i) own += digits[high - i];
            uint32_t before = (uint32_t)kv_scan((int)own) - own;
            if (before < rest && before + own >= rest) {
                for (int i = 0; i < 32; ++i) {
                    const uint32_t n = digits[high - i];
                    if (before + n >= rest) {
                        found_digit = (uint32_t)(high - i);
                        found_rest = rest - before;
                        break;
                    }
                    before += n;
                }
            }
        }
        __syncthreads();
        if (found_digit == 0xffffffffu) {  // fewer than the budget (pass 0): all stay
            all = true;
            break;
        }
        least |= found_digit << shift;
        rest = found_rest;
        __syncthreads();
    }
    if (all) {
        least = 0;  // all above it
        rest = 0;
    }
    const int stretch = ((keys + kThreads - 1) / kThreads) * 64, from = min(wave * stretch, keys), to = min(from + stretch, keys);
    int n_above = 0, n_equal = 0;
    for (int t = from + lane; t < to; t += 64) {
        const uint32_t v = order(t);
        n_above += v > least;
        n_equal += v == least;
    }
    n_above = __builtin_amdgcn_readlane(kv_scan(n_above), 63);
    n_equal = __builtin_amdgcn_readlane(kv_scan(n_equal), 63);
    if (lane == 0) {
        above[wave] = n_above;
        equal[wave] = n_equal;
    }
    __syncthreads();
    int equal_before = 0, place = 0, kept = 0, equals_so_far = 0;
    for (int i = 0; i < kWaves; ++i) {
        if (i == wave) {
            place = kept;
            equal_before = equals_so_far;
        }
        kept += above[i] + min(equal[i], max((int)rest - equals_so_far, 0));
        equals_so_far += equal[i];
    }
    int32_t *kept_to = a.kept + ((int64_t)b * a.c.heads + head) * a.budget;
    float *weights_to = a.to_weights + ((int64_t)b * a.c.heads + head) * a.budget;
    for (int t0 = from; t0 < to; t0 += 64) {
        const int t = t0 + lane;
        const uint32_t v = t < to ? order(t) : 0u;
        const bool is_equal = t < to && v == least;
        const uint64_t equals = __ballot(is_equal);
        const bool stays = (t < to && v > least) || (is_equal && equal_before + (int)__popcll(equals & ((1ull << lane) - 1)) < (int)rest);
        const uint64_t staying = __ballot(stays);
        if (stays) {
            const int at = place + (int)__popcll(staying & ((1ull << lane) - 1));
            kept_to[at] = t;
            weights_to[at] = t < a.w.capacity ? order.w[t] : 0.0f;
        }
        place += (int)__popcll(staying);
        equal_before += (int)__popcll(equals);
    }
    for (int i = kept + (int)threadIdx.x; i < a.budget; i += kThreads) {
        kept_to[i] = -1;
        weights_to[i] = 0.0f;
    }
    if (head == 0 && threadIdx.x == 0) a.to_lengths[b] = kept;
}

constexpr int kMoveWaves = 4;

// A wave has eight places of the new pages that follow each other, of a head, eight lanes to a token.  (The values of a token lie 16 bits a line of 16 bytes: lines are read for a token alone.)
template <int D>
__global__ __launch_bounds__(64 * kMoveWaves) void kv_move_kernel(KvEvictArgs a, uint64_t by_heads, int eights, int64_t units)
{
    constexpr int P = D / 32;
    __shared__ __align__(16) kv_u16 turn[kMoveWaves][D / 4 * 8];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane(), token = lane >> 3, part = lane & 7;
    const int64_t unit = (int64_t)blockIdx.x * kMoveWaves + wave;
    if (unit >= units) return;
    const int seq_eight = kv_divide((int)unit, by_heads), head = (int)unit - seq_eight * a.c.heads, b = seq_eight / eights, first = (seq_eight - b * eights) * 8;
    const int kept = a.to_lengths[b], shift = a.c.page_shift, mask = (1 << shift) - 1;
    if (first >= kept || (first >> shift) >= a.to_width) return;
    const int to_page = a.to_table[b * a.to_stride + (first >> shift)];
    if (to_page < 0 || to_page >= a.c.pages) return;
    const bool there = first + token < kept, whole = first + 8 <= kept;
    const int from = a.kept[((int64_t)b * a.c.heads + head) * a.budget + (there ? first + token : first)];
    const int page = a.c.table[b * a.c.table_stride + (from >> shift)];
    const int64_t block = ((int64_t)page * a.c.heads + head) * 2, to_block = ((int64_t)to_page * a.c.heads + head) * 2, half = (int64_t)(D / 2) << shift;
    const uint8_t *keys = a.c.codes + (block << shift) * (D / 2) + (int64_t)(from & mask) * (D / 2);
    const uint16_t *values = reinterpret_cast<const uint16_t *>(a.c.codes + (block << shift) * (D / 2) + half + (int64_t)(from & mask & ~7) * (D / 2)) + (from & 7);
    const uint16_t *scales = a.c.scales + (block << shift) + (from & mask);
    uint32_t k[P / 2];
    uint16_t v[P], s = 0;
#pragma unroll
    for (int i = 0; i < P / 2; ++i) k[i] = reinterpret_cast<const uint32_t *>(keys)[part * (P / 2) + i];
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = values[(part * P + i) * 8];
    if (part < 2) s = scales[part ? (int64_t)1 << shift : 0];
    uint8_t *to_keys = a.c.codes + (to_block << shift) * (D / 2) + (int64_t)(first & mask) * (D / 2);
    uint16_t *to_values = reinterpret_cast<uint16_t *>(to_keys + half), *to_scales = a.c.scales + (to_block << shift) + (first & mask);
    if (there) {
#pragma unroll
        for (int i = 0; i < P / 2; ++i) reinterpret_cast<uint32_t *>(to_keys + token * (D / 2))[part * (P / 2) + i] = k[i];
        if (part < 2) to_scales[(part ? (int64_t)1 << shift : 0) + token] = s;
    }
    if (whole) {
        kv_u16 *t = turn[wave];
#pragma unroll
        for (int i = 0; i < P; ++i) t[(part * P + i) * 8 + token] = v[i];
        kv_wave_fence();
        if constexpr (P == 4) reinterpret_cast<uint2 *>(to_values)[lane] = reinterpret_cast<const uint2 *>(t)[lane];
        else reinterpret_cast<uint32_t *>(to_values)[lane] = reinterpret_cast<const uint32_t *>(t)[lane];
    } else if (there) {
#pragma unroll
        for (int i = 0; i < P; ++i) to_values[(part * P + i) * 8 + token] = v[i];
    }
}

int64_t move_units(const KvEvictArgs &a) { return (int64_t)a.c.sequences * ((a.budget + 7) / 8) * a.c.heads; }

}  // namespace

int64_t kv_evict_items(const KvEvictArgs &a)
{
    return std::max<int64_t>((move_units(a) + kMoveWaves - 1) / kMoveWaves * 64 * kMoveWaves, (int64_t)a.c.sequences * a.c.heads * kThreads);
}

hipError_t launch_kv_evict(const KvEvictArgs &a, hipStream_t stream)
{
    kv_select_kernel<<<dim3((uint32_t)a.c.sequences, (uint32_t)a.c.heads), dim3(kThreads), 0, stream>>>(a);
    const int64_t units = move_units(a);
    const dim3 grid((uint32_t)((units + kMoveWaves - 1) / kMoveWaves)), block(64 * kMoveWaves);
    if (a.c.head_dim == 128) kv_move_kernel<128><<<grid, block, 0, stream>>>(a, kv_divisor(a.c.heads), (a.budget + 7) / 8, units);
    else kv_move_kernel<64><<<grid, block, 0, stream>>>(a, kv_divisor(a.c.heads), (a.budget + 7) / 8, units);
    return hipGetLastError();
}

}  // namespace apmm
