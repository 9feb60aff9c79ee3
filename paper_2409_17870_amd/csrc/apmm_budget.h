// Keeping the four-bit cache within a budget: what attention gives each cached token, and the tokens that stay (the public ABI is include/apmm.h).
#pragma once
#include "apmm_kv_attention.h"

namespace apmm {

struct KvWeights {  // sequences x heads x capacity numbers
    float *data;
    int64_t sequence_stride, head_stride, capacity;
};

// How a call of kv_weights is cut: sequences of few rows, those of many, each with pieces of the keys for the first pass (KvPart).  The workspace has few's pieces, its scores where they are kept, many's pieces, and many's rows as operands with their factors.
struct KvWeightsPlan {
    KvPart few, many;              // tile 0: none of these
    size_t few_bytes, many_bytes;  // of the workspace that pieces take
    int64_t score_stride;          // few's scores, from one row to the next, and what they take of the workspace; 0: they are made twice
    size_t score_bytes;
    int64_t row_tiles;             // of 16 rows, of a head, whose operands and factors are in it
    size_t rows_bytes;
    int64_t units;                 // workgroups of many's second pass, for a head
    int key_tiles;                 // of 16 keys, of a wave of it
};
KvWeightsPlan kv_weights_plan(const KvArgs &c, int groups, int window, int sinks);
int64_t kv_weights_blocks(const KvArgs &c);
size_t kv_weights_bytes(const KvWeightsPlan &plan);
int64_t kv_weights_items(const KvWeightsPlan &plan, int heads);
hipError_t launch_kv_weights(const KvAttentionArgs &a, const KvWeights &w, float decay, const KvWeightsPlan &plan, hipStream_t stream);

struct KvEvictArgs {
    KvArgs c;
    KvWeights w;
    const int32_t *to_table;
    int64_t to_stride;
    int to_width;
    int budget, sinks, recent;
    int32_t *kept, *to_lengths;  // sequences x heads x budget; sequences
    float *to_weights;           // sequences x heads x budget
};
// Many workgroups to a sequence and head, each with `chunks` of its tokens; parts 0: one.  The workspace has their counts and, behind these, what each part has to give.
struct KvEvictParts {
    int parts, chunks;
    uint64_t by_parts;  // what kv_divide divides by parts with
    size_t counts_bytes, bytes;
    void *counts, *tallies;
};
KvEvictParts kv_evict_parts(const KvArgs &c);
int64_t kv_evict_items(const KvEvictArgs &a, const KvEvictParts &p);
hipError_t launch_kv_evict(const KvEvictArgs &a, const KvEvictParts &p, hipStream_t stream);

}  // namespace apmm
