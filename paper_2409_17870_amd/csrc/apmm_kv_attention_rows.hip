// Attention over the four-bit cache where every sequence has few rows (apmm_kv_attention_rows.h).
#include "apmm_kv_attention_rows.h"

namespace apmm {

namespace {

template <int D, bool BF16, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 ? 3 : 2) void kv_attention_rows_kernel(KvAttentionArgs a, KvPart part)
{
    kv_attention_rows<D, BF16, WAVES>(a, part, blockIdx.x);
}

template <int WAVES>
void launch(const KvAttentionArgs &a, const KvPart &part, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)part.slots * a.c.heads)), block(64 * WAVES);
    if (a.c.head_dim == 128) {
        if (a.c.bf16) kv_attention_rows_kernel<128, true, WAVES><<<grid, block, 0, stream>>>(a, part);
        else kv_attention_rows_kernel<128, false, WAVES><<<grid, block, 0, stream>>>(a, part);
    } else {
        if (a.c.bf16) kv_attention_rows_kernel<64, true, WAVES><<<grid, block, 0, stream>>>(a, part);
        else kv_attention_rows_kernel<64, false, WAVES><<<grid, block, 0, stream>>>(a, part);
    }
}

}  // namespace

hipError_t launch_kv_attention_rows(const KvAttentionArgs &a, const KvPart &part, hipStream_t stream)
{
    if (part.waves == 4) launch<4>(a, part, stream);
    else launch<8>(a, part, stream);
    return hipGetLastError();
}

}  // namespace apmm
