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
    const float *w;
    const int32_t *table;
    int64_t pages, capacity;
    int keys, shift, sinks, recent_from;
    // of any t from 0 on where there is a token (no branch: tokens behind the last are looked at in the last one's place)
    __device__ __forceinline__ uint32_t operator()(int t) const
    {
        const int at = min(t, keys - 1), page = table[at >> shift];
        const uint32_t held = t < sinks || t >= recent_from ? 0xffffffffu : order_of(w[min((int64_t)at, capacity - 1)]);
        return t >= keys || page < 0 || page >= pages ? 0u : held != 0xffffffffu && t >= capacity ? 1u : held;
    }
};

// Of N waves' numbers those of the waves before this one, summed
template <int N>
__device__ __forceinline__ uint32_t sum_before(const uint32_t (&of_waves)[N], int wave)
{
    const int lane = kv_lane();
    return (uint32_t)__builtin_amdgcn_readlane(kv_scan(lane < wave ? (int)of_waves[min(lane, N - 1)] : 0), 63);
}

// Numbers of tokens begin + 64 i + lane, zeros from `to` on
template <int N>
__device__ __forceinline__ void read_tokens(const Tokens &order, int begin, int to, uint32_t (&v)[N])
{
    // tokens that all have a weight and a page are read as they lie
    const int lane = kv_lane(), end = min(begin + 64 * N, to), last = end - begin - 1;
    bool plain = last >= 0 && end <= order.capacity;
    if (plain) {
        const float *w = order.w + begin;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __float_as_uint(w[min(64 * i + lane, last)]);
        for (int page = (begin >> order.shift) + lane; page <= (end - 1) >> order.shift; page += 64) plain &= order.table[page] >= 0 && order.table[page] < order.pages;
    }
    if (__ballot(!plain) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 64 * i + lane <= last ? order_of(__uint_as_float(v[i])) : 0u;
        if (begin < order.sinks || end > order.recent_from) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int t = begin + 64 * i + lane;
                v[i] = t < end && (t < order.sinks || t >= order.recent_from) ? 0xffffffffu : v[i];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0;
            if (64 * i <= last) v[i] = 64 * i + lane <= last ? order(begin + 64 * i + lane) : 0u;
            if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);  // (eight on their way at a time: of more there are no registers)
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ Tokens tokens_of(const KvEvictArgs &a, int b, int head)
{
    const int length = min(max(a.c.lengths[b], 0), kKvMost), keys = (int)min((int64_t)length, (int64_t)a.c.width << a.c.page_shift);
    return {a.w.data + b * a.w.sequence_stride + head * a.w.head_stride, a.c.table + b * a.c.table_stride, a.c.pages, a.w.capacity, keys, a.c.page_shift, a.sinks, length - a.recent};
}

// A workgroup to a sequence and head, each of its waves has a stretch of tokens.  Three passes find the budget-th largest number, digit by digit from the highest; then each wave counts those of its stretch that
// stay, and after the counts have met writes their places in order, whose weights are fetched at the end by all.  Sequences of up to 1024 HELD tokens, as far as the table goes, are read once and held in registers, the second half of 64 to a
// lane in LDS.  Bound by the instructions of the one compute unit that has a sequence and head: 65001 tokens take 81 000 cycles, 18 000 to read them, 36 000 for the three passes, 8 000 to count and 19 000 to write.
// Tried and slower, of as many cycles: every token read with its own checks (55 000 to read), a weight fetched as its place is written (48 000 to write), counts of all lanes in one (19 500 for the first pass, 16 500
// so), the end of a stretch asked for at every token (18 000 more in all).
template <int HELD>
__global__ __launch_bounds__(kThreads) void kv_select_kernel(KvEvictArgs a)
{
    __shared__ __align__(16) uint32_t digits[kDigits][2];  // (by even and odd lanes: fewer meet in one)
    __shared__ uint32_t totals[kWaves];
    __shared__ int above[kWaves], equal[kWaves];
    __shared__ uint32_t found_digit, found_rest;
    const int b = kv_divide(blockIdx.x, a.c.by_heads), head = blockIdx.x - b * a.c.heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane();
    const Tokens order = tokens_of(a, b, head);
    const int keys = order.keys, stretch = ((keys + kThreads - 1) / kThreads) * 64, own_from = min(wave * stretch, keys), to = min(own_from + stretch, keys);
    constexpr int kInRegisters = HELD < 32 ? HELD : 32;
    uint32_t held[kInRegisters];
    __shared__ uint32_t more[HELD > 32 ? HELD - 32 : 1][kThreads];
    constexpr int kBatch = HELD < 16 ? HELD : 16;
#pragma unroll
    for (int first = 0; first < HELD; first += kBatch) {
        uint32_t v[kBatch];
        read_tokens(order, min(own_from + 64 * first, to), to, v);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (first + i < 32) held[first + i < 32 ? first + i : 0] = v[i];
            else more[first + i < 32 ? 0 : first + i - 32][threadIdx.x] = v[i];
        }
    }
    // f(token, number) of this lane's tokens, sixty-four to a wave at a time
    auto each = [&](auto f) {
        int from = own_from, lane = kv_lane();
        asm volatile("" : "+s"(from), "+v"(lane));  // (places and borders of 64 tokens are not kept from one pass for the next: for those there are no registers)
        constexpr int kOnce = HELD < 8 ? HELD : 8;
#pragma unroll
        for (int first = 0; first < HELD; first += kOnce) {
            if (from + 64 * first < to) {  // (behind `to` numbers are zero)
#pragma unroll
                for (int i = first; i < first + kOnce; ++i) f(from + 64 * i + lane, i < 32 ? held[i < 32 ? i : 0] : more[i < 32 ? 0 : i - 32][threadIdx.x]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    uint32_t least = 0, rest = (uint32_t)a.budget;  // what the digits so far say; how many are wanted of those that begin with them
    bool all = false;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        const uint32_t mask = (1u << bits) - 1, upper = pass == 0 ? 0 : ~0u << (shift + bits);
        reinterpret_cast<uint4 *>(digits)[threadIdx.x] = make_uint4(0, 0, 0, 0);
        static_assert(sizeof(digits) == kThreads * sizeof(uint4), "");
        if (threadIdx.x == 0) found_digit = 0xffffffffu;
        __syncthreads();
        each([&](int, uint32_t v) {
            if (v && (v & upper) == (least & upper)) atomicAdd(&digits[v >> shift & mask][lane & 1], 1u);
        });
        __syncthreads();
        // from the highest digit down, two to a lane
        const uint4 both = reinterpret_cast<const uint4 *>(digits)[kThreads - 1 - threadIdx.x];
        const uint32_t high = both.z + both.w, low = both.x + both.y;
        const uint32_t up_to = (uint32_t)kv_scan((int)(high + low));
        if (lane == 63) totals[wave] = up_to;
        __syncthreads();
        const uint32_t before = up_to - high - low + sum_before(totals, wave);
        if (before < rest && before + high + low >= rest) {
            const bool first = before + high >= rest;
            found_digit = kDigits - 1 - 2 * threadIdx.x - (first ? 0 : 1);
            found_rest = rest - before - (first ? 0 : high);
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
    int n_above = 0, n_equal = 0;
    each([&](int t, uint32_t v) {
        n_above += v > least;
        n_equal += t < to && v == least;
    });
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
    auto put = [&](int t, bool stays) {
        const uint64_t staying = __ballot(stays);
        if (stays) kept_to[place + __builtin_amdgcn_mbcnt_hi((uint32_t)(staying >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)staying, 0))] = t;
        place += (int)__popcll(staying);
    };
    const int equals_left = (int)rest - equal_before;  // of this stretch's tokens of the least number, so many stay
    if (equals_left <= 0 || equals_left >= equal[wave]) {
        const uint32_t over = equals_left <= 0 ? least : least - 1;  // (equals_left > 0: least > 0)
        each([&](int t, uint32_t v) { put(t, v > over); });
    } else {
        each([&](int t, uint32_t v) {
            const bool is_equal = t < to && v == least;
            const uint64_t equals = __ballot(is_equal);
            put(t, v > least || (is_equal && equal_before + (int)__popcll(equals & ((1ull << lane) - 1)) < (int)rest));
            equal_before += (int)__popcll(equals);
        });
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.budget; i += kThreads) {
        const int t = i < kept ? kept_to[i] : -1;
        if (t < 0) kept_to[i] = -1;
        weights_to[i] = t >= 0 && t < a.w.capacity ? order.w[t] : 0.0f;
    }
    if (head == 0 && threadIdx.x == 0) a.to_lengths[b] = kept;
}

// The same by many workgroups: a part of a sequence's tokens to each, in chunks of kChunk, a launch for each digit.  Counts of a digit meet in memory by additions of whole numbers, whose order changes nothing; each
// workgroup finds the digits before its own again.  Six launches, bound by what each has to wait for in turn: lengths, pages, weights, counts.
constexpr int kPartThreads = 256, kPartWaves = 4, kPartHeld = 16, kChunk = kPartThreads * kPartHeld, kMostParts = 256;

struct Counts {  // of a sequence and head
    uint32_t digits[3][kDigits];
};
struct Tally {   // of a part: tokens above the least number that stays, and tokens that have it
    int above, equal;
};

__global__ __launch_bounds__(kPartThreads) void kv_clear_kernel(uint32_t *at, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kPartThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kPartThreads) at[i] = 0;
}

struct Least {
    uint32_t number, rest;  // the digits found; how many are wanted of the tokens that have them
    bool all;               // fewer tokens than the budget: all stay
};
// By all lanes of a workgroup, from the highest digit down, eight to a lane
template <int PASSES>
__device__ __forceinline__ Least find_least(const Counts *counts, uint32_t budget)
{
    __shared__ uint32_t totals[kPartWaves], digit, left;
    const int wave = threadIdx.x >> 6, lane = kv_lane();
    Least l = {0, budget, false};
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        const uint4 *at = reinterpret_cast<const uint4 *>(counts->digits[pass] + kDigits - 8 - 8 * (int)threadIdx.x);
        const uint4 low = at[0], high = at[1];
        const uint32_t n[8] = {high.w, high.z, high.y, high.x, low.w, low.z, low.y, low.x};
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += n[i];
        const uint32_t up_to = (uint32_t)kv_scan((int)sum);
        if (lane == 63) totals[wave] = up_to;
        if (threadIdx.x == 0) digit = 0xffffffffu;
        __syncthreads();
        uint32_t before = up_to - sum + sum_before(totals, wave);
        if (before < l.rest && before + sum >= l.rest) {
            int i = 0;
            while (before + n[i] < l.rest) before += n[i++];
            digit = kDigits - 1 - 8 * threadIdx.x - i;
            left = l.rest - before;
        }
        __syncthreads();
        if (digit == 0xffffffffu) {  // (in the first pass, and for all workgroups of the sequence and head alike)
            l = {0, 0, true};
            return l;
        }
        l.number |= digit << (pass == 0 ? 21 : pass == 1 ? 10 : 0);
        l.rest = left;
        __syncthreads();
    }
    return l;
}

struct Part {
    int unit, part, b, head;  // unit: sequence and head
    __device__ __forceinline__ Part(const KvEvictArgs &a, const KvEvictParts &p)
    {
        unit = kv_divide(blockIdx.x, p.by_parts);
        part = blockIdx.x - unit * p.parts;
        b = kv_divide(unit, a.c.by_heads);
        head = unit - b * a.c.heads;
    }
};

template <int PASS>
__global__ __launch_bounds__(kPartThreads) void kv_count_kernel(KvEvictArgs a, KvEvictParts p)
{
    __shared__ uint32_t digits[kDigits];
    const Part at(a, p);
    const Tokens order = tokens_of(a, at.b, at.head);
    const int from = (int)min((int64_t)at.part * p.chunks * kChunk, (int64_t)order.keys), to = (int)min((int64_t)from + (int64_t)p.chunks * kChunk, (int64_t)order.keys);
    if (from >= to) return;
    Counts *counts = static_cast<Counts *>(p.counts) + at.unit;
    const Least l = find_least<PASS>(counts, (uint32_t)a.budget);
    if (l.all) return;
    for (int i = threadIdx.x; i < kDigits; i += kPartThreads) digits[i] = 0;
    __syncthreads();
    constexpr int shift = PASS == 0 ? 21 : PASS == 1 ? 10 : 0, bits = PASS == 2 ? 10 : 11;
    constexpr uint32_t mask = (1u << bits) - 1, upper = PASS == 0 ? 0 : ~0u << (shift + bits);
    for (int begin = from + (int)(threadIdx.x >> 6) * 64 * kPartHeld; begin < to; begin += kChunk) {
        uint32_t v[kPartHeld];
        read_tokens(order, begin, to, v);
#pragma unroll
        for (int i = 0; i < kPartHeld; ++i)
            if (v[i] && (v[i] & upper) == (l.number & upper)) atomicAdd(&digits[v[i] >> shift & mask], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kDigits; i += kPartThreads)
        if (digits[i]) atomicAdd(&counts->digits[PASS][i], digits[i]);
}

// Tokens of a chunk's stretch of a wave above l.number, and of it
__device__ __forceinline__ Tally tally_of(const uint32_t (&v)[kPartHeld], int begin, int to, const Least &l)
{
    Tally t = {0, 0};
#pragma unroll
    for (int i = 0; i < kPartHeld; ++i) {
        t.above += v[i] > l.number;
        t.equal += begin + 64 * i + kv_lane() < to && v[i] == l.number;
    }
    return {__builtin_amdgcn_readlane(kv_scan(t.above), 63), __builtin_amdgcn_readlane(kv_scan(t.equal), 63)};
}

__global__ __launch_bounds__(kPartThreads) void kv_tally_kernel(KvEvictArgs a, KvEvictParts p)
{
    __shared__ Tally waves[kPartWaves];
    const Part at(a, p);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Tokens order = tokens_of(a, at.b, at.head);
    const int from = (int)min((int64_t)at.part * p.chunks * kChunk, (int64_t)order.keys), to = (int)min((int64_t)from + (int64_t)p.chunks * kChunk, (int64_t)order.keys);
    const Least l = find_least<3>(static_cast<const Counts *>(p.counts) + at.unit, (uint32_t)a.budget);
    Tally sum = {0, 0};
    for (int begin = from + wave * 64 * kPartHeld; begin < to; begin += kChunk) {
        uint32_t v[kPartHeld];
        read_tokens(order, begin, to, v);
        const Tally t = tally_of(v, begin, to, l);
        sum.above += t.above;
        sum.equal += t.equal;
    }
    if (kv_lane() == 0) waves[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kPartWaves; ++i) {
            sum.above += waves[i].above;
            sum.equal += waves[i].equal;
        }
        static_cast<Tally *>(p.tallies)[(int64_t)at.unit * p.parts + at.part] = sum;
    }
}

__global__ __launch_bounds__(kPartThreads) void kv_keep_kernel(KvEvictArgs a, KvEvictParts p)
{
    __shared__ Tally waves[kPartWaves], before_of[kPartWaves], all_of[kPartWaves];
    const Part at(a, p);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = kv_lane();
    const Tokens order = tokens_of(a, at.b, at.head);
    const int from = (int)min((int64_t)at.part * p.chunks * kChunk, (int64_t)order.keys), to = (int)min((int64_t)from + (int64_t)p.chunks * kChunk, (int64_t)order.keys);
    const Least l = find_least<3>(static_cast<const Counts *>(p.counts) + at.unit, (uint32_t)a.budget);
    static_assert(kMostParts <= kPartThreads, "a part to a lane");
    Tally mine = {0, 0};
    if ((int)threadIdx.x < p.parts) mine = static_cast<const Tally *>(p.tallies)[(int64_t)at.unit * p.parts + threadIdx.x];
    const bool earlier = (int)threadIdx.x < at.part;
    const Tally some = {__builtin_amdgcn_readlane(kv_scan(earlier ? mine.above : 0), 63), __builtin_amdgcn_readlane(kv_scan(earlier ? mine.equal : 0), 63)};
    const Tally whole = {__builtin_amdgcn_readlane(kv_scan(mine.above), 63), __builtin_amdgcn_readlane(kv_scan(mine.equal), 63)};
    if (lane == 0) {
        before_of[wave] = some;
        all_of[wave] = whole;
    }
    __syncthreads();
    int above = 0, equals = 0, all_above = 0, all_equal = 0;  // before this part; of all
    for (int i = 0; i < kPartWaves; ++i) {
        above += before_of[i].above;
        equals += before_of[i].equal;
        all_above += all_of[i].above;
        all_equal += all_of[i].equal;
    }
    const int rest = (int)l.rest, kept = all_above + min(all_equal, rest), first = above + min(equals, rest);
    int32_t *kept_to = a.kept + (int64_t)at.unit * a.budget;
    float *weights_to = a.to_weights + (int64_t)at.unit * a.budget;
    for (int chunk = from; chunk < to; chunk += kChunk) {  // (the same for all waves)
        const int begin = min(chunk + wave * 64 * kPartHeld, to);
        uint32_t v[kPartHeld];
        read_tokens(order, begin, to, v);
        const Tally t = tally_of(v, begin, to, l);
        __syncthreads();
        if (lane == 0) waves[wave] = t;
        __syncthreads();
        int a0 = above, e0 = equals;
        for (int i = 0; i < kPartWaves; ++i) {
            if (i < wave) {
                a0 += waves[i].above;
                e0 += waves[i].equal;
            }
            above += waves[i].above;
            equals += waves[i].equal;
        }
        int place = a0 + min(e0, rest);
#pragma unroll
        for (int i = 0; i < kPartHeld; ++i) {
            const int token = begin + 64 * i + lane;
            const bool is_equal = token < to && v[i] == l.number;
            const uint64_t same = __ballot(is_equal), below = (1ull << lane) - 1;
            const bool stays = v[i] > l.number || (is_equal && e0 + (int)__popcll(same & below) < rest);
            const uint64_t staying = __ballot(stays);
            if (stays) kept_to[place + (int)__popcll(staying & below)] = token;
            place += (int)__popcll(staying);
            e0 += (int)__popcll(same);
        }
    }
    __syncthreads();
    for (int i = first + (int)threadIdx.x; i < above + min(equals, rest); i += kPartThreads) {
        const int t = kept_to[i];
        weights_to[i] = t < a.w.capacity ? order.w[t] : 0.0f;
    }
    for (int64_t i = kept + (int64_t)at.part * kPartThreads + threadIdx.x; i < a.budget; i += (int64_t)p.parts * kPartThreads) {
        kept_to[i] = -1;
        weights_to[i] = 0.0f;
    }
    if (at.head == 0 && at.part == 0 && threadIdx.x == 0) a.to_lengths[at.b] = kept;
}

constexpr int kMoveWaves = 4;

// A wave has eight places of the new pages that follow each other, of a head, eight lanes to a token.  (The values of a token lie 16 bits a line of 16 bytes: lines are read for a token alone.)
// Bound by these scattered reads: 24 sequences of which 1000 tokens stay, 8 heads of 64, 11 us; 4096 of 65001 tokens, 8 heads of 128, 7.
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

// Many workgroups to a sequence and head where its weights do not fit into one's registers and LDS.  By the page table's width, since the host does not know lengths: short sequences under a table that wide pay for
// six launches (24 of up to 2300 tokens, 8 heads of 64, 69 us in place of 19; one of 2300 40 and 11; 8 of up to 16000 58 and 31).  (Tokens of 8 heads, with the copy and the read back: 130000 51 us, a million 82; 20000, 33000 and 65000 would take 49 to
// 51, and take 33, 39 and 49 with one workgroup.)
KvEvictParts kv_evict_parts(const KvArgs &c)
{
    KvEvictParts p = {};
    const int64_t most = std::min<int64_t>((int64_t)c.width << c.page_shift, kKvMost), units = (int64_t)c.sequences * c.heads;  // tokens of a sequence, as far as the page table goes
    if (most <= 64 * kThreads) return p;
    const int64_t chunks = (most + kChunk - 1) / kChunk, parts = std::min<int64_t>(kMostParts, std::max<int64_t>(1, ((int64_t)1 << 23) / units));
    p.chunks = (int)((chunks + parts - 1) / parts);
    p.parts = (int)((chunks + p.chunks - 1) / p.chunks);
    p.by_parts = kv_divisor(p.parts);
    p.counts_bytes = (size_t)units * sizeof(Counts);
    p.bytes = p.counts_bytes + (size_t)units * p.parts * sizeof(Tally);
    return p;
}

int64_t kv_evict_items(const KvEvictArgs &a, const KvEvictParts &p)
{
    const int64_t units = (int64_t)a.c.sequences * a.c.heads;
    return std::max<int64_t>((move_units(a) + kMoveWaves - 1) / kMoveWaves * 64 * kMoveWaves, p.parts ? units * p.parts * kPartThreads : units * kThreads);
}

hipError_t launch_kv_evict(const KvEvictArgs &a, const KvEvictParts &p, hipStream_t stream)
{
    const int64_t most = (int64_t)a.c.width << a.c.page_shift, units = (int64_t)a.c.sequences * a.c.heads;
    if (p.parts) {
        const int64_t words = (int64_t)(p.counts_bytes / 4);
        const dim3 groups((uint32_t)(units * p.parts)), block(kPartThreads), clear((uint32_t)std::min<int64_t>((words + kPartThreads - 1) / kPartThreads, 4096));
        kv_clear_kernel<<<clear, block, 0, stream>>>(static_cast<uint32_t *>(p.counts), words);
        kv_count_kernel<0><<<groups, block, 0, stream>>>(a, p);
        kv_count_kernel<1><<<groups, block, 0, stream>>>(a, p);
        kv_count_kernel<2><<<groups, block, 0, stream>>>(a, p);
        kv_tally_kernel<<<groups, block, 0, stream>>>(a, p);
        kv_keep_kernel<<<groups, block, 0, stream>>>(a, p);
    } else {
        const dim3 groups((uint32_t)units), block(kThreads);
        if (most <= 4 * kThreads) kv_select_kernel<4><<<groups, block, 0, stream>>>(a);
        else if (most <= 16 * kThreads) kv_select_kernel<16><<<groups, block, 0, stream>>>(a);
        else kv_select_kernel<64><<<groups, block, 0, stream>>>(a);
    }
    const int64_t places = move_units(a);
    const dim3 grid((uint32_t)((places + kMoveWaves - 1) / kMoveWaves)), four(64 * kMoveWaves);
    if (a.c.head_dim == 128) kv_move_kernel<128><<<grid, four, 0, stream>>>(a, kv_divisor(a.c.heads), (a.budget + 7) / 8, places);
    else kv_move_kernel<64><<<grid, four, 0, stream>>>(a, kv_divisor(a.c.heads), (a.budget + 7) / 8, places);
    return hipGetLastError();
}

}  // namespace apmm
