// The four-bit key/value cache: its layout, the batch that a call works on, and the launchers of its kernels (the public ABI is include/apmm.h).
//
// codes:  [page][head][2][page tokens * head_dim / 2 bytes], keys then values
//   keys    token by token, channel c in the low (even c) or high (odd c) four bits of byte c / 2: a lane of the matrix unit's operand K takes 8
//           channels of one token, one word, and gets them as binary16 pairs (c, c + 4) with one AND each (kv_operand)
//   values  by eights of tokens; of one, for each m the channels 4 m to 4 m + 3 of the eight tokens, 16 bits a token: a lane of the operand V^T takes
//           8 tokens of one channel, and a word of two tokens gives the pairs of four channels the same way
// scales: [page][head][2][page tokens] of the type of the tensors
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace apmm {

constexpr int kKvMost = 1 << 30;  // tokens, positions, window

struct KvArgs {
    uint8_t *codes;
    uint16_t *scales;
    const int32_t *table;    // sequences x table_stride, the first `width` of a row are pages
    const int32_t *lengths;  // tokens of each sequence
    const int32_t *starts;   // sequences + 1, or null: one new token a sequence
    int64_t pages, table_stride;
    int sequences, tokens, width, heads, page_shift, head_dim;
    bool bf16;
    uint64_t by_heads;       // what kv_divide divides by heads with
    int per_wave;            // writing and reading: heads of a wave
};

struct KvTensor {  // rows of head_dim contiguous elements
    uint16_t *data;
    int64_t token_stride, head_stride;  // elements
    bool aligned;                       // every row starts at a multiple of 16 bytes
};

struct KvAttentionArgs {
    KvArgs c;
    KvTensor q, out;
    int groups;        // query heads to a key/value head
    uint64_t by_groups;  // what kv_divide divides by groups with
    int window, sinks; // window 0: none
    float scale;
    float *partial;    // results of pieces of sequences: see KvPlan
};

// How the work of an attention call is cut.  Rows are the queries of the heads that share a key/value head; a kernel takes the sequences with `from_rows` to `to_rows` of them, `tile` rows
// to a tile.  The keys that a tile sees are cut in pieces of at least `least` steps so that there are about `target` workgroups for each key/value head whatever the lengths
// are, which the host does not know.
struct KvPart {
    int tile;    // rows of a workgroup; 0: the kernel is not launched
    int waves;   // of a workgroup of kv_attention_rows_kernel
    int target;  // 0: nothing is cut
    int least;
    int slots;   // most pieces there can be
    int turn;    // of a sequence's tiles, longest first, the second `turn` come in reverse order; 0: none
    int from_rows, to_rows;
};
struct KvPlan {
    KvPart rows, tiles;     // kv_attention_rows_kernel's, kv_attention_tiles_kernel's
    int64_t tiles_partial;  // where the latter's pieces begin in the workspace
};
KvPlan kv_plan(const KvArgs &c, int groups, int window, int sinks);
size_t kv_partial_bytes(const KvPart &part, int heads, int head_dim);  // of the workspace that pieces take

// Work items of the largest launch of a call; there may be fewer than 2^32
constexpr int64_t kKvMostItems = UINT32_MAX;
int64_t kv_store_items(const KvArgs &c);
int64_t kv_attention_items(const KvPlan &plan, int heads);

hipError_t launch_kv_write(const KvArgs &c, const KvTensor &k, const KvTensor &v, hipStream_t stream);
hipError_t launch_kv_read(const KvArgs &c, const KvTensor &k, const KvTensor &v, hipStream_t stream);
hipError_t launch_kv_attention(const KvAttentionArgs &a, const KvPlan &plan, hipStream_t stream);

// x / d as (x m) >> 63 with m = 2^63 / d, rounded up: exact for 0 <= x < 2^31 and d <= 1024, since x (m - 2^63 / d) < 2^31 is less than 2^63 / 1024
inline uint64_t kv_divisor(int d) { return ((1ull << 63) + d - 1) / d; }

#ifdef __HIPCC__
typedef uint16_t __attribute__((may_alias)) kv_u16;  // what is written in these and read in words, or the other way round
typedef uint32_t __attribute__((may_alias)) kv_u32;

// (the high half of 2 x m, a product of up to 95 bits; 2 x is one of 32)
__device__ __forceinline__ int kv_divide(int x, uint64_t m)
{
    const uint64_t y = 2u * (uint32_t)x;
    return (int)((y * (m >> 32) + ((y * (uint32_t)m) >> 32)) >> 32);
}

// Place of lane `lane` within its wave of a workgroup of whole waves
__device__ __forceinline__ int kv_lane() { return threadIdx.x & 63; }

// What lanes of a wave have written to LDS before this the others read behind it, and the other way round.  No instruction: a wave's LDS accesses are done in their order, which is
// kept by the compiler only where it is told that one lane's are another's.
__device__ __forceinline__ void kv_wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }

// A sequence of the batch.  Whatever lies in lengths and starts, rows start .. start + n - 1 are rows of the tensors and keys below `keys` have a place in the table.
struct KvSequence {
    int start, n;  // new tokens
    int first;     // position of the first new token; may be negative
    int keys;
};
__device__ __forceinline__ KvSequence kv_sequence(const KvArgs &c, int b)
{
    KvSequence s;
    int end;
    if (c.starts) {
        s.start = min(max(c.starts[b], 0), c.tokens);
        end = min(max(c.starts[b + 1], s.start), c.tokens);
    } else {
        s.start = b;
        end = b + 1;
    }
    s.n = end - s.start;
    const int length = min(max(c.lengths[b], 0), kKvMost);
    s.first = length - s.n;
    s.keys = (int)min((int64_t)length, (int64_t)c.width << c.page_shift);
    return s;
}

// Sum over the lanes up to this one, by moves within the vector unit
__device__ __forceinline__ int kv_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // one to four lanes up within sixteen
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // the last of sixteen to the next sixteen, of 32 to the next 32
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
    return v;
}

// The sequence that has unit `unit` where sequence b has count(b) of them, and the unit's number within it; false: there are fewer.  All lanes take part, all get the same.
template <class Count>
__device__ __forceinline__ bool kv_find(int sequences, int unit, int &b, int &rest, Count count)
{
    int before = 0;
    for (int base = 0; base < sequences; base += 64) {
        const int at = base + kv_lane();
        const int n = at < sequences ? count(at) : 0;
        const int to = before + kv_scan(n);
        const uint64_t past = __ballot(to > unit);
        if (past) {
            const int l = __ffsll((long long)past) - 1;
            b = base + l;
            rest = unit - (__builtin_amdgcn_readlane(to, l) - __builtin_amdgcn_readlane(n, l));
            return true;
        }
        before = __builtin_amdgcn_readlane(to, 63);
    }
    return false;
}

// The larger of two 16-bit numbers each
__device__ __forceinline__ uint32_t kv_fold_max(uint32_t m, uint32_t w)
{
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, m), __builtin_bit_cast(us2, w)));
}

__device__ __forceinline__ float kv_scale_value(uint32_t bits, bool bf16)
{
    if (bf16) return __uint_as_float(bits << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

__device__ __forceinline__ uint16_t kv_round(float x, bool bf16)
{
    if (bf16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// Words of a row's 16-bit elements, two at a time; rows that are not aligned element by element
template <int N>
__device__ __forceinline__ void kv_load(const uint16_t *src, bool aligned, uint32_t (&w)[N])
{
    if (aligned) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 x = *reinterpret_cast<const uint4 *>(src + 2 * i);
            w[i] = x.x; w[i + 1] = x.y; w[i + 2] = x.z; w[i + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = src[2 * i] | (uint32_t)src[2 * i + 1] << 16;
    }
}
template <int N>
__device__ __forceinline__ void kv_store(uint16_t *dst, bool aligned, const uint32_t (&w)[N])
{
    if (aligned) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4) *reinterpret_cast<uint4 *>(dst + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        } else {
            static_assert(N % 2 == 0, "pairs of words");
#pragma unroll
            for (int i = 0; i < N; i += 2) *reinterpret_cast<uint2 *>(dst + 2 * i) = make_uint2(w[i], w[i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            dst[2 * i] = (uint16_t)w[i];
            dst[2 * i + 1] = (uint16_t)(w[i] >> 16);
        }
    }
}
#endif

}  // namespace apmm
