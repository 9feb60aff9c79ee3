// Keeping the four-bit cache within a budget: what attention gives each cached token, and the tokens that stay (the public ABI is include/apmm.h).
#pragma once
#include "apmm_kv_attention.h"

namespace apmm {

struct KvWeights {  // sequences x heads x capacity numbers
    float *data;
    int64_t sequence_stride, head_stride, capacity;
};

// What kv_weights' statistics of rows are cut into: the plan's one part (KvPart), and where in the workspace the rows' base and factor lie
struct KvWeightsPlan {
    KvPart part;
    int row_tiles;        // tiles of 16 rows that a wave of the statistics has at a time: 1 or 4
    int64_t rows;         // tokens * q_heads
    size_t pieces_bytes;  // of the workspace that pieces take, in front of the rows'
    int64_t groups;       // workgroups of the sums
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
int64_t kv_evict_items(const KvEvictArgs &a);
hipError_t launch_kv_evict(const KvEvictArgs &a, hipStream_t stream);

}  // namespace apmm
