// C ABI of the products with four-bit weights and group scales (include/apmm.h): argument checks and launches.
#include "../../include/apmm.h"
#include "apmm_api.h"
#include "apmm_w4.h"

namespace {

using apmm::fail;
using apmm::fail_hip;

constexpr int64_t kMost = 1 << 24;  // channels and inputs: codes and scales stay below 2^50 bytes, a tile's below 2^31

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

apmm_status check_sizes(int64_t N, int64_t K, int group)
{
    if (N < 0 || K < 1) return fail(APMM_ERR_INVALID_ARG, "w4: N < 0 or K < 1");
    if (group != 32 && group != 64 && group != 128) return fail(group < 1 ? APMM_ERR_INVALID_ARG : APMM_ERR_UNSUPPORTED, "w4: group must be 32, 64 or 128");
    if (N > kMost || K > kMost) return fail(APMM_ERR_UNSUPPORTED, "w4: more than 2^24 channels or inputs");
    return APMM_OK;
}

bool known(int dtype) { return dtype == APMM_F16 || dtype == APMM_BF16; }

}  // namespace

extern "C" {

size_t apmm_w4_packed_bytes(int64_t N, int64_t K, int group)
{
    if (check_sizes(N, K, group) != APMM_OK) return 0;
    return (size_t)apmm::W4Shape{N, K, group}.bytes();
}

apmm_status apmm_w4_pack(const uint8_t *codes, const void *scales, int64_t N, int64_t K, int group, int dtype, void *packed, void *stream)
{
    const apmm_status st = check_sizes(N, K, group);
    if (st != APMM_OK) return st;
    if (!known(dtype)) return fail(APMM_ERR_INVALID_ARG, "w4: unknown dtype");
    if (N == 0) return APMM_OK;
    if (!codes || !scales || !packed) return fail(APMM_ERR_INVALID_ARG, "w4: null pointer");
    if (!aligned(scales, 2) || !aligned(packed, 16)) return fail(APMM_ERR_INVALID_ARG, "w4: scales must be 2-byte, packed weights 16-byte aligned");
    const hipError_t e = apmm::launch_w4_pack(codes, static_cast<const uint16_t *>(scales), apmm::W4Shape{N, K, group}, dtype == APMM_BF16, static_cast<uint8_t *>(packed), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_w4_pack");
}

size_t apmm_w4_workspace_bytes(int64_t M, int64_t N, int64_t K, int group)
{
    if (check_sizes(N, K, group) != APMM_OK || M < 1 || N == 0 || M > apmm::kW4MostRows) return 0;
    return (size_t)apmm::w4_partial_bytes(M, N, apmm::w4_rule(M, N, apmm::W4Shape{N, K, group}.blocks()));
}

apmm_status apmm_w4_gemm(int64_t M, int64_t N, int64_t K, int group, int dtype, const void *x, int64_t x_stride, const void *packed, void *y, int64_t y_stride,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    const apmm_status st = check_sizes(N, K, group);
    if (st != APMM_OK) return st;
    if (M < 0 || !known(dtype)) return fail(APMM_ERR_INVALID_ARG, "w4: M < 0, or an unknown dtype");
    if (M > apmm::kW4MostRows) return fail(APMM_ERR_UNSUPPORTED, "w4: more than 2^20 tokens");
    if (M == 0 || N == 0) return APMM_OK;
    if (!x || !packed || !y) return fail(APMM_ERR_INVALID_ARG, "w4: null pointer");
    if (!aligned(x, 2) || !aligned(y, 2) || !aligned(packed, 16)) return fail(APMM_ERR_INVALID_ARG, "w4: x and y must be 2-byte, packed weights 16-byte aligned");
    if (x == y) return fail(APMM_ERR_INVALID_ARG, "w4: y must not be x, which other workgroups still read");
    if (M > 1 && (x_stride < 0 || y_stride < N)) return fail(APMM_ERR_INVALID_ARG, "w4: x_stride < 0, or rows of y that overlap");
    const apmm::W4Shape s = {N, K, group};
    const apmm::W4Rule r = apmm::w4_rule(M, N, s.blocks());
    if (apmm::w4_items(M, N, r) >= ((int64_t)1 << 32)) return fail(APMM_ERR_UNSUPPORTED, "w4: M * N is more than one launch takes");
    const size_t need = (size_t)apmm::w4_partial_bytes(M, N, r);
    if (need && (!workspace || workspace_bytes < need)) return fail(APMM_ERR_WORKSPACE, "w4: needs a workspace of apmm_w4_workspace_bytes() bytes");
    if (need && !aligned(workspace, 16)) return fail(APMM_ERR_INVALID_ARG, "w4: workspace must be 16-byte aligned");
    apmm::W4Args a;
    a.x = static_cast<const uint16_t *>(x);
    a.packed = static_cast<const uint8_t *>(packed);
    a.y = static_cast<uint16_t *>(y);
    a.partial = static_cast<float *>(workspace);
    a.x_stride = M > 1 ? x_stride : 0;
    a.y_stride = M > 1 ? y_stride : 0;
    a.code_bytes = s.code_bytes();
    a.M = (int)M;
    a.N = (int)N;
    a.K = (int)K;
    a.blocks = (int)s.blocks();
    const hipError_t e = apmm::launch_w4_gemm(a, r, group, dtype == APMM_BF16, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APMM_OK : fail_hip(e, "apmm_w4_gemm");
}

}  // extern "C"
