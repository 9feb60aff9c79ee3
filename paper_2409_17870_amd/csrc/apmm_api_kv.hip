// C ABI of the four-bit key/value cache and attention over it (include/apmm.h): argument checks and launches.
#include <cmath>

#include "apmm_kv_checks.h"

namespace {

using apmm::aligned;
using apmm::check_batch;
using apmm::check_sizes;
using apmm::check_tensor;
using apmm::fail;
using apmm::fail_hip;

apmm_status check_pair(const apmm_kv_cache *cache, const apmm_kv_batch *batch, const void *k, int64_t kt, int64_t kh, const void *v, int64_t vt, int64_t vh,
                       apmm::KvArgs &a, apmm::KvTensor &tk, apmm::KvTensor &tv, bool &empty)
{
    apmm_status st = check_batch(cache, batch, a, empty);
    if (st != APMM_OK || empty) return st;
    if ((st = check_tensor(k, kt, kh, tk)) != APMM_OK || (st = check_tensor(v, vt, vh, tv)) != APMM_OK) return st;
    if (apmm::kv_store_items(a) > apmm::kKvMostItems) return fail(APMM_ERR_UNSUPPORTED, "kv: tokens * kv_heads is more than one launch takes");
    return APMM_OK;
}

apmm_status check_heads(const apmm_kv_cache *cache, const apmm_kv_batch *batch, const apmm::KvArgs &a, int q_heads, int window, int sinks, apmm::KvPlan &plan)
{
    if (q_heads < 1 || q_heads % cache->kv_heads) return fail(APMM_ERR_INVALID_ARG, "kv_attention: q_heads must be a multiple of kv_heads");
    const int groups = q_heads / cache->kv_heads;
    if (groups > 1024 || (batch->tokens + batch->sequences) * q_heads > INT32_MAX / 4)
        return fail(APMM_ERR_UNSUPPORTED, "kv_attention: more than 1024 query heads to a key/value head, or tokens * q_heads is more than one launch takes");
    plan = apmm::kv_plan(a, groups, window, sinks);
    if (apmm::kv_attention_items(plan, a.heads) > apmm::kKvMostItems) return fail(APMM_ERR_UNSUPPORTED, "kv_attention: tokens * q_heads is more than one launch takes");
    return APMM_OK;
}

size_t partial_bytes(const apmm::KvPlan &plan, const apmm::KvArgs &a)
{
    return apmm::kv_partial_bytes(plan.rows, a.heads, a.head_dim) + apmm::kv_partial_bytes(plan.tiles, a.heads, a.head_dim);
}

}  // namespace

extern "C" {

apmm_status apmm_kv_write(const apmm_kv_cache *cache, const apmm_kv_batch *batch, const void *k, int64_t k_token_stride, int64_t k_head_stride,
                          const void *v, int64_t v_token_stride, int64_t v_head_stride, void *stream)
{
    apmm::KvArgs a;
    apmm::KvTensor tk, tv;
    bool empty;
    const apmm_status st = check_pair(cache, batch, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, a, tk, tv, empty);
    if (st != APMM_OK || empty) return st;
    const hipError_t e = apmm::launch_kv_write(a, tk, tv, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_kv_write");
}

apmm_status apmm_kv_read(const apmm_kv_cache *cache, const apmm_kv_batch *batch, void *k, int64_t k_token_stride, int64_t k_head_stride,
                         void *v, int64_t v_token_stride, int64_t v_head_stride, void *stream)
{
    apmm::KvArgs a;
    apmm::KvTensor tk, tv;
    bool empty;
    const apmm_status st = check_pair(cache, batch, k, k_token_stride, k_head_stride, v, v_token_stride, v_head_stride, a, tk, tv, empty);
    if (st != APMM_OK || empty) return st;
    const hipError_t e = apmm::launch_kv_read(a, tk, tv, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_kv_read");
}

// (without a window: under one as much is needed or less)
size_t apmm_kv_attention_workspace_bytes(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads)
{
    apmm::KvArgs a;
    apmm::KvPlan plan;
    if (check_sizes(cache, batch, a) != APMM_OK || batch->sequences == 0 || batch->tokens == 0 || check_heads(cache, batch, a, q_heads, 0, 0, plan) != APMM_OK) return 0;
    return partial_bytes(plan, a);
}

apmm_status apmm_kv_attention(const apmm_kv_cache *cache, const apmm_kv_batch *batch, int q_heads, const void *q, int64_t q_token_stride,
                              int64_t q_head_stride, void *out, int64_t out_token_stride, int64_t out_head_stride, float scale, int64_t window,
                              int64_t sinks, void *workspace, size_t workspace_bytes, void *stream)
{
    apmm::KvAttentionArgs a;
    apmm::KvPlan plan;
    bool empty;
    apmm_status st = check_batch(cache, batch, a.c, empty);
    if (st != APMM_OK) return st;
    if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(APMM_ERR_INVALID_ARG, "kv_attention: scale must be positive and finite");
    if (window < 0 || sinks < 0) return fail(APMM_ERR_INVALID_ARG, "kv_attention: window < 0 or sinks < 0");
    if (window > apmm::kKvMost || sinks > apmm::kKvMost) return fail(APMM_ERR_UNSUPPORTED, "kv_attention: window or sinks > 2^30");
    if ((st = check_heads(cache, batch, a.c, q_heads, (int)window, (int)sinks, plan)) != APMM_OK || empty) return st;
    if ((st = check_tensor(q, q_token_stride, q_head_stride, a.q)) != APMM_OK || (st = check_tensor(out, out_token_stride, out_head_stride, a.out)) != APMM_OK) return st;
    const size_t need = partial_bytes(plan, a.c);
    if (need && (!workspace || workspace_bytes < need)) return fail(APMM_ERR_WORKSPACE, "kv_attention: needs a workspace of apmm_kv_attention_workspace_bytes() bytes");
    if (need && !aligned(workspace, 16)) return fail(APMM_ERR_INVALID_ARG, "kv_attention: workspace must be 16-byte aligned");
    a.groups = q_heads / cache->kv_heads;
    a.by_groups = apmm::kv_divisor(a.groups);
    a.window = (int)window;
    a.sinks = window ? (int)sinks : 0;
    a.scale = scale;
    a.partial = static_cast<float *>(workspace);
    const hipError_t e = apmm::launch_kv_attention(a, plan, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_kv_attention");
}

}  // extern "C"
