// C ABI of rotary positions and of what keeps the four-bit key/value cache within a budget (include/apmm.h): argument checks and launches.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "apmm_budget.h"
#include "apmm_kv_checks.h"
#include "apmm_rotary.h"

namespace {

using apmm::aligned;
using apmm::check_batch;
using apmm::check_sizes;
using apmm::check_tensor;
using apmm::fail;
using apmm::fail_hip;

apmm_status check_rotation(const apmm_rotation *r, int head_dim, apmm::RotaryArgs &a)
{
    if (!r) return fail(APMM_ERR_INVALID_ARG, "rotary: no rotation");
    if (r->pairs < 1 || 2 * r->pairs > head_dim) return fail(APMM_ERR_INVALID_ARG, "rotary: pairs must be from 1 to head_dim / 2");
    if (!r->frequencies || !aligned(r->frequencies, 8)) return fail(APMM_ERR_INVALID_ARG, "rotary: null or misaligned frequencies");
    if (!(r->magnitude > 0.0f) || !std::isfinite(r->magnitude)) return fail(APMM_ERR_INVALID_ARG, "rotary: magnitude must be positive and finite");
    a.frequencies = r->frequencies;
    a.pairs = (int)r->pairs;
    a.interleaved = r->interleaved != 0;
    a.magnitude = r->magnitude;
    a.sign = 1.0f;
    return APMM_OK;
}

// `sequences`: of a call that writes them, whose rows must not overlap; else 0
apmm_status check_weights(const apmm_kv_cache *cache, const float *weights, int64_t sequence_stride, int64_t head_stride, int64_t capacity, int sequences, apmm::KvWeights &w)
{
    if (capacity < 1 || sequence_stride < 0 || head_stride < 0) return fail(APMM_ERR_INVALID_ARG, "kv: weights need capacity >= 1 and strides >= 0");
    if (capacity > ((int64_t)1 << 46) || sequence_stride > ((int64_t)1 << 46) || head_stride > ((int64_t)1 << 46)) return fail(APMM_ERR_UNSUPPORTED, "kv: capacity or a stride of weights > 2^46");
    // the shorter stride holds a row, the longer one all rows of the shorter; a stride of one sequence or head counts for nothing
    const int64_t s = sequences > 1 ? sequence_stride : INT64_MAX, h = cache->kv_heads > 1 ? head_stride : INT64_MAX;
    const int64_t inner = std::min(s, h), outer = std::max(s, h), rows = s < h ? sequences : cache->kv_heads;
    if (sequences && (inner < capacity || (outer != INT64_MAX && outer < (rows - 1) * inner + capacity))) return fail(APMM_ERR_INVALID_ARG, "kv: weights' rows overlap");
    if (!weights || !aligned(weights, 4)) return fail(APMM_ERR_INVALID_ARG, "kv: null or misaligned weights");
    w.data = const_cast<float *>(weights);
    w.sequence_stride = sequence_stride;
    w.head_stride = head_stride;
    w.capacity = capacity;
    return APMM_OK;
}

// Rows, places and sizes of the statistics' plan
apmm_status check_weighing(const apmm_kv_cache *cache, const apmm_kv_batch *batch, const apmm::KvArgs &a, int q_heads, int window, int sinks, apmm::KvWeightsPlan &plan)
{
    if (q_heads < 1 || q_heads % cache->kv_heads) return fail(APMM_ERR_INVALID_ARG, "kv_weights: q_heads must be a multiple of kv_heads");
    const int groups = q_heads / cache->kv_heads;
    if (groups > 1024 || (batch->tokens + batch->sequences) * q_heads > INT32_MAX / 4)
        return fail(APMM_ERR_UNSUPPORTED, "kv_weights: more than 1024 query heads to a key/value head, or tokens * q_heads is more than one launch takes");
    if (apmm::kv_weights_blocks(a) > INT32_MAX / 2) return fail(APMM_ERR_UNSUPPORTED, "kv_weights: sequences * table_width * page_size is 2^38 or more");
    plan = apmm::kv_weights_plan(a, groups, window, sinks);
    if (apmm::kv_weights_items(plan, a.heads) > apmm::kKvMostItems) return fail(APMM_ERR_UNSUPPORTED, "kv_weights: tokens * q_heads is more than one launch takes");
    return APMM_OK;
}

}  // namespace

extern "C" {

apmm_status apmm_rotary(int64_t tokens, int heads, int head_dim, int dtype, const void *x, int64_t x_token_stride, int64_t x_head_stride, const int32_t *positions, const apmm_rotation *rotation,
                        int inverse, void *out, int64_t out_token_stride, int64_t out_head_stride, void *stream)
{
    if (tokens < 0 || heads < 0 || head_dim < 1 || (dtype != APMM_F16 && dtype != APMM_BF16)) return fail(APMM_ERR_INVALID_ARG, "rotary: tokens < 0, heads < 0, head_dim < 1, or an unknown dtype");
    if (tokens > apmm::kKvMost || heads > 65536 || head_dim > 1024) return fail(APMM_ERR_UNSUPPORTED, "rotary: more than 2^30 tokens, 65536 heads or 1024 channels");
    apmm::RotaryRows a;
    apmm_status st = check_rotation(rotation, head_dim, a.r);
    if (st != APMM_OK || tokens == 0 || heads == 0) return st;
    if ((st = check_tensor(x, x_token_stride, x_head_stride, a.x)) != APMM_OK || (st = check_tensor(out, out_token_stride, out_head_stride, a.out)) != APMM_OK) return st;
    if (x == out && (x_token_stride != out_token_stride || x_head_stride != out_head_stride)) return fail(APMM_ERR_INVALID_ARG, "rotary: rows that are turned where they lie must have one set of strides");
    if (!positions || !aligned(positions, 4)) return fail(APMM_ERR_INVALID_ARG, "rotary: null or misaligned positions");
    a.r.positions = positions;
    if (inverse) a.r.sign = -1.0f;
    a.tokens = tokens;
    a.heads = heads;
    a.head_dim = head_dim;
    a.bf16 = dtype == APMM_BF16;
    const hipError_t e = apmm::launch_rotary(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_rotary");
}

apmm_status apmm_kv_write_rotary(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads, const int32_t *positions, const apmm_rotation *rotation,
                                 const void *q, int64_t q_token_stride, int64_t q_head_stride, void *q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
                                 const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride, int64_t v_head_stride, void *stream)
{
    apmm::KvRotaryArgs a = {};
    bool empty;
    apmm_status st = check_batch(cache, batch, a.c, empty);
    if (st != APMM_OK) return st;
    if (q_heads < 0) return fail(APMM_ERR_INVALID_ARG, "kv_write_rotary: q_heads < 0");
    if (q_heads > 2048) return fail(APMM_ERR_UNSUPPORTED, "kv_write_rotary: more than 2048 query heads");
    if ((st = check_rotation(rotation, cache->head_dim, a.r)) != APMM_OK || empty) return st;
    if (!aligned(positions, 4)) return fail(APMM_ERR_INVALID_ARG, "kv_write_rotary: misaligned positions");
    if ((st = check_tensor(k, k_token_stride, k_head_stride, a.k)) != APMM_OK || (st = check_tensor(v, v_token_stride, v_head_stride, a.v)) != APMM_OK) return st;
    if (q_heads) {
        if ((st = check_tensor(q, q_token_stride, q_head_stride, a.q)) != APMM_OK || (st = check_tensor(q_out, q_out_token_stride, q_out_head_stride, a.q_out)) != APMM_OK) return st;
        if (q == q_out && (q_token_stride != q_out_token_stride || q_head_stride != q_out_head_stride))
            return fail(APMM_ERR_INVALID_ARG, "kv_write_rotary: queries that are turned where they lie must have one set of strides");
        if (q_out == k || q_out == v) return fail(APMM_ERR_INVALID_ARG, "kv_write_rotary: q_out must be neither k nor v");
    }
    a.q_heads = q_heads;
    a.r.positions = positions;
    if (apmm::kv_rotary_items(a.c, q_heads) > apmm::kKvMostItems) return fail(APMM_ERR_UNSUPPORTED, "kv_write_rotary: tokens * heads is more than one launch takes");
    const hipError_t e = apmm::launch_kv_write_rotary(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_kv_write_rotary");
}

// (without a window and with starts: under one and without them as much is needed or less)
size_t apmm_kv_weights_workspace_bytes(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads)
{
    static const int32_t any = 0;
    apmm::KvArgs a;
    apmm::KvWeightsPlan plan;
    if (check_sizes(cache, batch, a) != APMM_OK || batch->sequences == 0 || batch->tokens == 0) return 0;
    a.starts = &any;
    if (check_weighing(cache, batch, a, q_heads, 0, 0, plan) != APMM_OK) return 0;
    return apmm::kv_weights_bytes(plan);
}

apmm_status apmm_kv_weights(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads, const void *q, int64_t q_token_stride, int64_t q_head_stride,
                            float *weights, int64_t weights_sequence_stride, int64_t weights_head_stride, int64_t capacity, float decay, float scale, int64_t window, int64_t sinks,
                            void *workspace, size_t workspace_bytes, void *stream)
{
    apmm::KvAttentionArgs a = {};
    apmm::KvWeights w;
    apmm::KvWeightsPlan plan;
    bool empty;
    apmm_status st = check_batch(cache, batch, a.c, empty);
    if (st != APMM_OK) return st;
    if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(APMM_ERR_INVALID_ARG, "kv_weights: scale must be positive and finite");
    if (!(decay >= 0.0f) || !std::isfinite(decay)) return fail(APMM_ERR_INVALID_ARG, "kv_weights: decay must be finite and not negative");
    if (window < 0 || sinks < 0) return fail(APMM_ERR_INVALID_ARG, "kv_weights: window < 0 or sinks < 0");
    if (window > apmm::kKvMost || sinks > apmm::kKvMost) return fail(APMM_ERR_UNSUPPORTED, "kv_weights: window or sinks > 2^30");
    if ((st = check_weighing(cache, batch, a.c, q_heads, (int)window, (int)sinks, plan)) != APMM_OK || empty) return st;
    if ((st = check_tensor(q, q_token_stride, q_head_stride, a.q)) != APMM_OK || (st = check_weights(cache, weights, weights_sequence_stride, weights_head_stride, capacity, batch->sequences, w)) != APMM_OK) return st;
    const size_t need = apmm::kv_weights_bytes(plan);
    if (!workspace || workspace_bytes < need) return fail(APMM_ERR_WORKSPACE, "kv_weights: needs a workspace of apmm_kv_weights_workspace_bytes() bytes");
    if (!aligned(workspace, 16)) return fail(APMM_ERR_INVALID_ARG, "kv_weights: workspace must be 16-byte aligned");
    a.groups = q_heads / cache->kv_heads;
    a.by_groups = apmm::kv_divisor(a.groups);
    a.window = (int)window;
    a.sinks = window ? (int)sinks : 0;
    a.scale = scale;
    a.partial = static_cast<float *>(workspace);
    const hipError_t e = apmm::launch_kv_weights(a, w, decay, plan, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_kv_weights");
}

size_t apmm_kv_evict_workspace_bytes(const apmm_kv_cache *cache, int sequences, int64_t table_width)
{
    apmm::KvArgs a;
    const apmm_kv_batch batch = {sequences, sequences, nullptr, nullptr, nullptr, table_width, table_width};
    if (check_sizes(cache, &batch, a) != APMM_OK || sequences == 0) return 0;
    return apmm::kv_evict_parts(a).bytes;
}

apmm_status apmm_kv_evict(const apmm_kv_cache *cache, int sequences, const int32_t *lengths, const int32_t *page_table, int64_t table_stride, int64_t table_width,
                          const float *weights, int64_t weights_sequence_stride, int64_t weights_head_stride, int64_t capacity, int64_t budget, int64_t sinks, int64_t recent,
                          const int32_t *to_table, int64_t to_stride, int64_t to_width, int32_t *to_lengths, int32_t *kept, float *to_weights, void *workspace, size_t workspace_bytes, void *stream)
{
    apmm::KvEvictArgs a = {};
    bool empty;
    const apmm_kv_batch batch = {sequences, sequences, lengths, nullptr, page_table, table_stride, table_width};
    apmm_status st = check_batch(cache, &batch, a.c, empty);
    if (st != APMM_OK) return st;
    if (budget < 1 || sinks < 0 || recent < 0 || sinks > budget || recent > budget - sinks) return fail(APMM_ERR_INVALID_ARG, "kv_evict: budget < 1, or sinks and recent that are negative or more than it");
    if (budget > apmm::kKvMost) return fail(APMM_ERR_UNSUPPORTED, "kv_evict: budget > 2^30");
    if (to_width < 1 || to_stride < to_width) return fail(APMM_ERR_INVALID_ARG, "kv_evict: to_width < 1 or to_stride < to_width");
    if (to_width > (1 << 26)) return fail(APMM_ERR_UNSUPPORTED, "kv_evict: to_width > 2^26");
    if (empty) return APMM_OK;
    if ((st = check_weights(cache, weights, weights_sequence_stride, weights_head_stride, capacity, 0, a.w)) != APMM_OK) return st;
    if (!to_table || !to_lengths || !kept || !to_weights) return fail(APMM_ERR_INVALID_ARG, "kv_evict: null pointer");
    if (!aligned(to_table, 4) || !aligned(to_lengths, 4) || !aligned(kept, 4) || !aligned(to_weights, 4)) return fail(APMM_ERR_INVALID_ARG, "kv_evict: misaligned pointer");
    if (to_weights == weights) return fail(APMM_ERR_INVALID_ARG, "kv_evict: to_weights must not be weights");
    if (to_lengths == lengths) return fail(APMM_ERR_INVALID_ARG, "kv_evict: to_lengths must not be lengths");
    a.to_table = to_table;
    a.to_stride = to_stride;
    a.to_width = (int)to_width;
    a.budget = (int)budget;
    a.sinks = (int)sinks;
    a.recent = (int)recent;
    a.kept = kept;
    a.to_lengths = to_lengths;
    a.to_weights = to_weights;
    apmm::KvEvictParts parts = apmm::kv_evict_parts(a.c);
    if (apmm::kv_evict_items(a, parts) > apmm::kKvMostItems) return fail(APMM_ERR_UNSUPPORTED, "kv_evict: sequences * kv_heads * budget is more than one launch takes");
    if (parts.parts) {
        if (!workspace || workspace_bytes < parts.bytes) return fail(APMM_ERR_WORKSPACE, "kv_evict: needs a workspace of apmm_kv_evict_workspace_bytes() bytes");
        if (!aligned(workspace, 16)) return fail(APMM_ERR_INVALID_ARG, "kv_evict: workspace must be 16-byte aligned");
        parts.counts = workspace;
        parts.tallies = static_cast<uint8_t *>(workspace) + parts.counts_bytes;
    }
    const hipError_t e = apmm::launch_kv_evict(a, parts, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_kv_evict");
}

}  // extern "C"
