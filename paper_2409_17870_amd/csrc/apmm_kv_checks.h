// Checks of the arguments that the entry points on the four-bit key/value cache share (include/apmm.h).
#pragma once
#include "../../include/apmm.h"
#include "apmm_api.h"
#include "apmm_kv.h"

namespace apmm {

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Sizes alone, without the pointers
inline apmm_status check_sizes(const apmm_kv_cache *c, const apmm_kv_batch *b, KvArgs &a)
{
    if (!c || !b) return fail(APMM_ERR_INVALID_ARG, "kv: no cache or no batch");
    if (c->pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1 || (c->dtype != APMM_F16 && c->dtype != APMM_BF16))
        return fail(APMM_ERR_INVALID_ARG, "kv: pages, page_size, kv_heads or head_dim < 1, or an unknown dtype");
    if (c->page_size < 16 || c->page_size > (1 << 20) || (c->page_size & (c->page_size - 1)))
        return fail(APMM_ERR_UNSUPPORTED, "kv: page_size must be a power of two from 16 to 1048576");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(APMM_ERR_UNSUPPORTED, "kv: head_dim must be 64 or 128");
    if (c->kv_heads > 1024 || c->pages > INT32_MAX) return fail(APMM_ERR_UNSUPPORTED, "kv: more than 1024 key/value heads or 2^31 - 1 pages");
    if (b->sequences < 0 || b->tokens < 0) return fail(APMM_ERR_INVALID_ARG, "kv: sequences < 0 or tokens < 0");
    if (b->sequences > 65536 || b->tokens > kKvMost) return fail(APMM_ERR_UNSUPPORTED, "kv: more than 65536 sequences or 2^30 tokens");
    if (b->table_width < 1 || b->table_stride < b->table_width) return fail(APMM_ERR_INVALID_ARG, "kv: table_width < 1 or table_stride < table_width");
    if (b->table_width > (1 << 26)) return fail(APMM_ERR_UNSUPPORTED, "kv: table_width > 2^26");
    a.codes = static_cast<uint8_t *>(c->codes);
    a.scales = static_cast<uint16_t *>(c->scales);
    a.table = b->page_table;
    a.lengths = b->lengths;
    a.starts = b->starts;
    a.pages = c->pages;
    a.table_stride = b->table_stride;
    a.sequences = b->sequences;
    a.tokens = (int)b->tokens;
    a.width = (int)b->table_width;
    a.heads = c->kv_heads;
    a.page_shift = __builtin_ctz((unsigned)c->page_size);
    a.head_dim = c->head_dim;
    a.bf16 = c->dtype == APMM_BF16;
    a.by_heads = kv_divisor(c->kv_heads);
    return APMM_OK;
}

// `empty`: no sequence or no token, nothing to launch
inline apmm_status check_batch(const apmm_kv_cache *c, const apmm_kv_batch *b, KvArgs &a, bool &empty)
{
    const apmm_status st = check_sizes(c, b, a);
    if (st != APMM_OK) return st;
    empty = b->sequences == 0 || b->tokens == 0;
    if (empty) return APMM_OK;
    if (!b->starts && b->tokens != b->sequences) return fail(APMM_ERR_INVALID_ARG, "kv: without starts there is one token a sequence");
    if (!c->codes || !c->scales || !b->lengths || !b->page_table) return fail(APMM_ERR_INVALID_ARG, "kv: null pointer in the cache or the batch");
    if (!aligned(c->codes, 16) || !aligned(c->scales, 16)) return fail(APMM_ERR_INVALID_ARG, "kv: codes and scales must be 16-byte aligned");
    if (!aligned(b->lengths, 4) || !aligned(b->starts, 4) || !aligned(b->page_table, 4)) return fail(APMM_ERR_INVALID_ARG, "kv: misaligned lengths, starts or page_table");
    return APMM_OK;
}

inline apmm_status check_tensor(const void *p, int64_t token_stride, int64_t head_stride, KvTensor &t)
{
    if (!p || !aligned(p, 2)) return fail(APMM_ERR_INVALID_ARG, "kv: null or misaligned tensor");
    t.data = static_cast<uint16_t *>(const_cast<void *>(p));
    t.token_stride = token_stride;
    t.head_stride = head_stride;
    t.aligned = aligned(p, 16) && token_stride % 8 == 0 && head_stride % 8 == 0;
    return APMM_OK;
}

}  // namespace apmm
