// Rotary positions (apmm_rotary.h): rows turned where they lie or into other ones, and queries, keys and values turned and written into the four-bit cache in one launch.
#include <algorithm>
#include <type_traits>

#include "apmm_kv_store.h"
#include "apmm_rotary.h"

namespace apmm {

namespace {

constexpr int kThreads = 256;
constexpr int kTurns = 512;  // cosines and sines that a workgroup holds: of one token, or of several that have 256 with those that fill up a row of RotaryTurns

// A workgroup has some tokens (those whose cosines and sines it holds) and a share of their heads.  A piece is what one lane reads and writes: both partners of its pairs are its own, so rows may be
// turned where they lie.  Bound by HBM: 8192 tokens of 64 heads of 128, 268 MB, 49 us on the device (5.5 TB/s; 3 to 4 less without the second look at numbers near a middle, 105 with all sums of 64 bits); 8 tokens of 40 heads 3.5, the launch and positions -> frequencies -> rows.
template <bool BF16, bool INTERLEAVED, bool EIGHTS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryRows a)
{
    __shared__ float4 turns[kTurns];
    const int pairs = a.r.pairs, all = a.heads * a.items, shift = RotaryTurns<INTERLEAVED>::kShift, stride = (pairs + (1 << shift) - 1) >> shift;
    for (int64_t first = (int64_t)blockIdx.x * a.tokens_of_group; first < a.tokens; first += (int64_t)gridDim.x * a.tokens_of_group) {
        const int tokens = (int)min((int64_t)a.tokens_of_group, a.tokens - first);
        __syncthreads();
        for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) {
            const int token = i / pairs;
            RotaryTurns<INTERLEAVED>{turns + (token * stride << shift), stride}[i - token * pairs] = rotary_turn(a.r, a.r.positions[first + token], i - token * pairs);
        }
        __syncthreads();
        for (int token = 0; token < tokens; ++token) {
            const uint16_t *x = a.x.data + (first + token) * a.x.token_stride;
            uint16_t *out = a.out.data + (first + token) * a.out.token_stride;
            const RotaryTurns<INTERLEAVED> t = {turns + (token * stride << shift), stride};
            for (int i = blockIdx.y * kThreads + threadIdx.x; i < all; i += gridDim.y * kThreads) {
                const int head = kv_divide(i, a.by_items), piece = i - head * a.items;
                const uint16_t *from = x + head * a.x.head_stride;
                uint16_t *to = out + head * a.out.head_stride;
                if (EIGHTS) {
                    // interleaved: the i-th eight of channels.  Halves: the i-th eight of first ones with that of second ones, behind these the eights that are not turned.
                    const int of_pairs = INTERLEAVED ? pairs / 4 : pairs / 8;
                    uint32_t w[4];
                    if (piece >= of_pairs) {
                        const int c0 = 2 * pairs + (piece - of_pairs) * 8;
                        kv_load(from + c0, true, w);
                        kv_store(to + c0, true, w);
                    } else if (INTERLEAVED) {
                        kv_load(from + piece * 8, true, w);
                        rotary_eight<BF16, INTERLEAVED>(from, true, piece * 8, w, t, pairs);
                        kv_store(to + piece * 8, true, w);
                    } else {
                        uint32_t v[4];
                        kv_load(from + piece * 8, true, w);
                        kv_load(from + piece * 8 + pairs, true, v);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float4 c1 = t[piece * 8 + 2 * j], c2 = t[piece * 8 + 2 * j + 1];
                            float a1 = kv_scale_value(w[j] & 0xffffu, BF16), a2 = kv_scale_value(w[j] >> 16, BF16), b1 = kv_scale_value(v[j] & 0xffffu, BF16), b2 = kv_scale_value(v[j] >> 16, BF16);
                            rotary_both<BF16>(a1, b1, c1);
                            rotary_both<BF16>(a2, b2, c2);
                            w[j] = rotary_pair(a1, a2, BF16);
                            v[j] = rotary_pair(b1, b2, BF16);
                        }
                        kv_store(to + piece * 8, true, w);
                        kv_store(to + piece * 8 + pairs, true, v);
                    }
                } else if (piece >= pairs) {
                    to[pairs + piece] = from[pairs + piece];
                } else {
                    const int c1 = INTERLEAVED ? 2 * piece : piece, c2 = INTERLEAVED ? c1 + 1 : piece + pairs;
                    const float4 cs = t[piece];
                    float x1 = kv_scale_value(from[c1], BF16), x2 = kv_scale_value(from[c2], BF16);
                    rotary_both<BF16>(x1, x2, cs);
                    to[c1] = kv_round(x1, BF16);
                    to[c2] = kv_round(x2, BF16);
                }
            }
        }
    }
}

constexpr int kWaves = 4;

// A workgroup has the up to eight tokens of an aligned eight of positions, as kv_write_kernel's waves have, and `per_wave` heads to each wave: those of keys and values first, then those of queries.
// It makes the eight's cosines and sines once.  Four heads to a wave where there are many: 13 sequences of up to 1500 new tokens, 32 heads of 128, 184 MB read and written in 57 us (both forms of pairs in one
// kernel, which has no registers for a fourth wave, 11 more; two heads to a wave, or eight, 3 and 5 more); 32 single tokens of 8 and 32 heads 7.7, of which the way from lengths to pages to a partly filled eight is the longer part.
template <int D, bool BF16, bool INTERLEAVED>
__global__ __launch_bounds__(64 * kWaves) void kv_rotary_write_kernel(KvRotaryArgs a)
{
    constexpr int N = D / 16;
    __shared__ __align__(16) kv_u16 turn[kWaves][D / 4 * 8];
    __shared__ float4 turns[8 * 64];  // (eight tokens)
    const int eight = kv_divide(blockIdx.x, a.by_blocks), block = blockIdx.x - eight * a.blocks, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Eight e;
    if (!find_eight(a.c, eight, e)) return;  // (all waves of the workgroup alike)
    const int lane = kv_lane(), token = lane >> 3, part = lane & 7, pairs = a.r.pairs, all = a.c.heads + a.q_heads;
    const int64_t row = e.s.start + (e.is_new ? e.first + token - e.s.first : 0);  // (a lane without one reads the first)
    auto head_of = [&](int i) { return (block * a.per_wave + i) * kWaves + wave; };
    auto first_row = [&](int head) { return head < a.c.heads ? a.k.data + row * a.k.token_stride + head * a.k.head_stride : a.q.data + row * a.q.token_stride + (head - a.c.heads) * a.q.head_stride; };
    auto load = [&](int head, uint32_t (&x)[N], uint32_t (&y)[N]) {  // a query, or a key and a value
        if (head >= all || (head < a.c.heads && e.page < 0)) return;
        load_row(first_row(head), head < a.c.heads ? a.k.aligned : a.q.aligned, part, x);
        if (head < a.c.heads) load_row(a.v.data + row * a.v.token_stride + head * a.v.head_stride, a.v.aligned, part, y);
    };
    auto turns_of = [&](int t) { return RotaryTurns<INTERLEAVED>{turns + t * (INTERLEAVED ? 16 : 8), INTERLEAVED ? 128 : 64}; };
    uint32_t x[N], y[N];
    load(head_of(0), x, y);  // (on their way while the cosines and sines are made)
    for (int i = threadIdx.x; i < 8 * pairs; i += 64 * kWaves) {
        const int t = i / pairs, place = e.first + t;
        if (place < e.s.first || place >= e.s.first + e.s.n) continue;
        turns_of(t)[i - t * pairs] = rotary_turn(a.r, a.r.positions ? a.r.positions[e.s.start + place - e.s.first] : place, i - t * pairs);
    }
    __syncthreads();
    const RotaryTurns<INTERLEAVED> of_token = turns_of(token);
    auto turned = [&](const uint16_t *from, bool aligned) {
        if (D == 128 && !INTERLEAVED && pairs == 64) {  // both partners are this lane's
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int second = D == 128 ? 4 + j : j;
                const float4 c1 = of_token[8 * part + 2 * j], c2 = of_token[8 * part + 2 * j + 1];
                float a1 = kv_scale_value(x[j] & 0xffffu, BF16), a2 = kv_scale_value(x[j] >> 16, BF16), b1 = kv_scale_value(x[second] & 0xffffu, BF16), b2 = kv_scale_value(x[second] >> 16, BF16);
                rotary_both<BF16>(a1, b1, c1);
                rotary_both<BF16>(a2, b2, c2);
                x[j] = rotary_pair(a1, a2, BF16);
                x[second] = rotary_pair(b1, b2, BF16);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            uint32_t w[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
            rotary_eight<BF16, INTERLEAVED>(from, aligned, 64 * i + 8 * part, w, of_token, pairs);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[4 * i + j] = w[j];
        }
    };
    for (int i = 0; i < a.per_wave; ++i) {
        const int head = head_of(i);
        if (head >= all) break;
        if (i) load(head, x, y);
        if (head >= a.c.heads) {
            turned(first_row(head), a.q.aligned);
            if (e.is_new) store_row(a.q_out.data + row * a.q_out.token_stride + (head - a.c.heads) * a.q_out.head_stride, a.q_out.aligned, part, x);
        } else if (e.page >= 0) {
            uint32_t uk[N / 4], uv[N / 4];
            turned(first_row(head), a.k.aligned);
            const uint32_t sk = quantise<N, BF16>(x, uk), sv = quantise<N, BF16>(y, uv);
            write_codes<D>(a.c, e, head, uk, sk, uv, sv, turn[wave]);
        }
    }
}

template <class Go>
void forms(bool bf16, bool interleaved, const Go &go)
{
    if (bf16) interleaved ? go(std::true_type(), std::true_type()) : go(std::true_type(), std::false_type());
    else interleaved ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
}

int heads_of_a_wave(const KvArgs &c, int q_heads)
{
    return kv_eights(c) * (c.heads + q_heads) >= 16384 ? 4 : 1;
}
int blocks_of_an_eight(const KvArgs &c, int q_heads)
{
    const int of_block = kWaves * heads_of_a_wave(c, q_heads);
    return (c.heads + q_heads + of_block - 1) / of_block;
}

}  // namespace

hipError_t launch_rotary(const RotaryRows &in, hipStream_t stream)
{
    RotaryRows a = in;
    const int pairs = a.r.pairs, rest = a.head_dim - 2 * pairs;
    const bool copies = a.x.data != a.out.data;  // else what is not turned stays as it is
    a.eights = a.x.aligned && a.out.aligned && pairs % (a.r.interleaved ? 4 : 8) == 0 && rest % 8 == 0;
    a.items = a.eights ? pairs / (a.r.interleaved ? 4 : 8) + (copies ? rest / 8 : 0) : pairs + (copies ? rest : 0);
    a.by_items = kv_divisor(a.items);
    const int64_t pieces = (int64_t)a.heads * a.items;
    // as many tokens to a workgroup as give its lanes a cosine and sine each, where there are workgroups enough without
    const int most = std::max(1, kThreads / ((pairs + 7) / 8 * 8));
    a.tokens_of_group = (int)std::max<int64_t>(1, std::min<int64_t>(most, a.tokens / 1024));
    const int64_t groups = std::min<int64_t>((a.tokens + a.tokens_of_group - 1) / a.tokens_of_group, 1 << 20);
    const int64_t shares = std::max<int64_t>(1, std::min<int64_t>((pieces + kThreads - 1) / kThreads, 2048 / groups));
    const dim3 grid((uint32_t)groups, (uint32_t)shares), block(kThreads);
    auto go = [&](auto bf16, auto interleaved) {
        constexpr bool B = decltype(bf16)::value, I = decltype(interleaved)::value;
        if (a.eights) rotary_kernel<B, I, true><<<grid, block, 0, stream>>>(a);
        else rotary_kernel<B, I, false><<<grid, block, 0, stream>>>(a);
    };
    forms(a.bf16, a.r.interleaved, go);
    return hipGetLastError();
}

int64_t kv_rotary_items(const KvArgs &c, int q_heads) { return kv_eights(c) * blocks_of_an_eight(c, q_heads) * 64 * kWaves; }

hipError_t launch_kv_write_rotary(const KvRotaryArgs &in, hipStream_t stream)
{
    KvRotaryArgs a = in;
    a.per_wave = heads_of_a_wave(a.c, a.q_heads);
    a.blocks = blocks_of_an_eight(a.c, a.q_heads);
    a.by_blocks = kv_divisor(a.blocks);
    const dim3 grid((uint32_t)(kv_eights(a.c) * a.blocks)), block(64 * kWaves);
    auto go = [&](auto bf16, auto interleaved) {
        constexpr bool B = decltype(bf16)::value, I = decltype(interleaved)::value;
        if (a.c.head_dim == 128) kv_rotary_write_kernel<128, B, I><<<grid, block, 0, stream>>>(a);
        else kv_rotary_write_kernel<64, B, I><<<grid, block, 0, stream>>>(a);
    };
    forms(a.c.bf16, a.r.interleaved, go);
    return hipGetLastError();
}

}  // namespace apmm
