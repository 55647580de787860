// C ABI of what surrounds a layer's products (include/mxfp4.h: mxfp4_rms_norm, mxfp4_w4a8_gemm, mxfp4_lora): argument checks and
// launches.  As everywhere in the library, the work goes to the caller's stream, and nothing here synchronises, allocates or frees
// device memory.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "layer.h"
#include "../../include/mxfp4.h"

namespace mxfp4 {

static bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

static int launched(hipError_t e, const char* what) { return e == hipSuccess ? MXFP4_OK : hip_fail(e, what); }

// A BF16 tensor read and written in pieces of eight elements.
static int check_rows(const void* p, int64_t ld, int64_t k, const char* what)
{
    if (ld < k)
        return fail(MXFP4_ERR_SHAPE, "%s: row stride %lld is less than %lld", what, (long long)ld, (long long)k);
    if (!aligned(p, 16) || ld % 8)
        return fail(MXFP4_ERR_ALIGN, "%s must be 16-byte aligned with a row stride that is a multiple of 8", what);
    return MXFP4_OK;
}

constexpr int64_t kMostRows = 0x7FFFFF00, kMostStride = 1 << 23;     // (64 rows are within reach of a 31-bit offset)

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

int mxfp4_rms_norm(const void* x_bf16, int64_t M, int64_t K, int64_t ldx, const void* residual_bf16, int64_t ldr,
                   const void* weight_bf16, float eps, void* sum_bf16, int64_t lds, void* y_bf16, int64_t ldy, void* q8,
                   void* scales_e8m0, void* stream)
{
    begin_call();
    if (M < 0 || M > kMostRows || K < 8 || K % 8 || K > MXFP4_MAX_K)
        return fail(MXFP4_ERR_SHAPE, "M=%lld or K=%lld out of range (K a multiple of 8, at most %d)", (long long)M, (long long)K, MXFP4_MAX_K);
    if (!(eps >= 0.f) || !isfinite(eps))
        return fail(MXFP4_ERR_ARG, "eps must be a finite number, not negative");
    if (M == 0)
        return MXFP4_OK;
    if (!x_bf16)
        return fail(MXFP4_ERR_NULL, "x is NULL");
    if (q8 && K % 32)
        return fail(MXFP4_ERR_SHAPE, "K=%lld must be a multiple of 32 for 8-bit blocks", (long long)K);
    if (!q8 != !scales_e8m0 || (!y_bf16 && !q8))
        return fail(MXFP4_ERR_NULL, "y, or q8 and scales together, must be given");
    if (sum_bf16 && !residual_bf16)
        return fail(MXFP4_ERR_ARG, "a sum without a residual");
    int rc;
    if ((rc = check_rows(x_bf16, ldx, K, "x")) || (residual_bf16 && (rc = check_rows(residual_bf16, ldr, K, "residual"))) ||
        (sum_bf16 && (rc = check_rows(sum_bf16, lds, K, "sum"))) || (y_bf16 && (rc = check_rows(y_bf16, ldy, K, "y"))))
        return rc;
    // in place of an input, but not of other rows of it than the row that is read
    auto crosses = [&](const void* out, int64_t ld) {
        return out && M > 1 && ((out == x_bf16 && ld != ldx) || (out == residual_bf16 && ld != ldr));
    };
    if (crosses(sum_bf16, lds) || crosses(y_bf16, ldy) || (sum_bf16 && sum_bf16 == y_bf16))
        return fail(MXFP4_ERR_ARG, "sum or y is an input with another row stride, or both are the same");
    if (!aligned(weight_bf16, 16) || !aligned(q8, 8))
        return fail(MXFP4_ERR_ALIGN, "weight must be 16-byte aligned, q8 8-byte");
    NormArgs a = {};
    a.x = static_cast<const uint16_t*>(x_bf16);
    a.r = static_cast<const uint16_t*>(residual_bf16);
    a.w = static_cast<const uint16_t*>(weight_bf16);
    a.sum = static_cast<uint16_t*>(sum_bf16);
    a.y = static_cast<uint16_t*>(y_bf16);
    a.q8 = static_cast<uint8_t*>(q8);
    a.s = static_cast<uint8_t*>(scales_e8m0);
    a.ldx = ldx;
    a.ldr = ldr;
    a.lds = lds;
    a.ldy = ldy;
    a.m = (int)M;
    a.k = (int)K;
    a.eps = eps;
    return launched(launch_rms_norm(a, static_cast<hipStream_t>(stream)), "norm launch");
}

int mxfp4_w4a8_gemm(const void* x_e4m3, const void* x_scales_e8m0, int64_t M, const void* q_packed, const void* scales_e8m0, int64_t N,
                    int64_t K, const void* bias_bf16, int act, const void* residual_bf16, int64_t ldr, void* y_bf16, int64_t ldy,
                    void* stream)
{
    begin_call();
    if (act != MXFP4_ACT_NONE && act != MXFP4_ACT_SWIGLU)
        return fail(MXFP4_ERR_ARG, "unknown act %d", act);
    if (M < 1 || M > kMostRows || N < 1 || N > kMostRows || K < 32 || K % 32 || K > MXFP4_MAX_K)
        return fail(MXFP4_ERR_SHAPE, "M=%lld, N=%lld or K=%lld out of range (K a multiple of 32, at most %d)", (long long)M, (long long)N,
                    (long long)K, MXFP4_MAX_K);
    if (act == MXFP4_ACT_SWIGLU && N % 2)
        return fail(MXFP4_ERR_SHAPE, "N=%lld must be even with the gate", (long long)N);
    if (!x_e4m3 || !x_scales_e8m0 || !q_packed || !scales_e8m0 || !y_bf16)
        return fail(MXFP4_ERR_NULL, "x, its scales, q, its scales or y is NULL");
    const int64_t C = act == MXFP4_ACT_SWIGLU ? N / 2 : N;
    if (ldy < C || (residual_bf16 && ldr < C))
        return fail(MXFP4_ERR_SHAPE, "ldy=%lld or ldr=%lld is less than %lld", (long long)ldy, (long long)ldr, (long long)C);
    if (M > 1 && residual_bf16 == y_bf16 && ldr != ldy)
        return fail(MXFP4_ERR_ARG, "residual is y with another row stride");
    if (!aligned(x_e4m3, 16) || !aligned(q_packed, 16) || !aligned(x_scales_e8m0, 4) || !aligned(scales_e8m0, 4) || !aligned(bias_bf16, 2) ||
        !aligned(residual_bf16, 2) || !aligned(y_bf16, 2))
        return fail(MXFP4_ERR_ALIGN, "x and q must be 16-byte aligned, the scales 4-byte, bias, residual and y 2-byte");
    DeviceInfo dev;
    const int rc = device_info(&dev);
    if (rc)
        return rc;
    A8Args a = {};
    a.x = static_cast<const uint8_t*>(x_e4m3);
    a.xs = static_cast<const uint8_t*>(x_scales_e8m0);
    a.q = static_cast<const uint8_t*>(q_packed);
    a.s = static_cast<const uint8_t*>(scales_e8m0);
    a.y = static_cast<uint16_t*>(y_bf16);
    a.ldy = ldy;
    a.ldr = ldr;
    a.epi = {static_cast<const uint16_t*>(bias_bf16), static_cast<const uint16_t*>(residual_bf16), 0, act};
    a.m = (int)M;
    a.n = (int)N;
    a.k = (int)K;
    return launched(launch_w4a8(a, dev, static_cast<hipStream_t>(stream)), "8-bit product launch");
}

static bool lora_sizes(int64_t M, int64_t K, int64_t R)
{
    return M >= 0 && M <= kMostRows && K >= 8 && K % 8 == 0 && K <= MXFP4_MAX_K && R >= 8 && R % 8 == 0 && R <= 128;
}

size_t mxfp4_lora_workspace_bytes(int64_t M, int64_t K, int64_t R)
{
    return lora_sizes(M, K, R) && M ? lora_workspace(M, K, R) : 0;
}

int mxfp4_lora(const void* x_bf16, int64_t M, int64_t ldx, const void* a_bf16, const void* b_bf16, int64_t adapters, int64_t R, int64_t N,
               int64_t K, const int32_t* ids, const float* scales_f32, const void* base_bf16, int64_t ldb, void* y_bf16, int64_t ldy,
               void* workspace, size_t workspace_bytes, void* stream)
{
    begin_call();
    if (!lora_sizes(M, K, R) || N < 8 || N % 8 || N > kMostRows)
        return fail(MXFP4_ERR_SHAPE, "M=%lld, N=%lld, K=%lld or R=%lld out of range (N, K, R multiples of 8, K at most %d, R at most 128)",
                    (long long)M, (long long)N, (long long)K, (long long)R, MXFP4_MAX_K);
    if (adapters < 1 || adapters > kMostAdapters)
        return fail(MXFP4_ERR_SHAPE, "adapters=%lld out of range (at most %d)", (long long)adapters, kMostAdapters);
    if (M == 0)
        return MXFP4_OK;
    if (!x_bf16 || !a_bf16 || !b_bf16 || !ids || !y_bf16)
        return fail(MXFP4_ERR_NULL, "x, a, b, ids or y is NULL");
    int rc;
    if ((rc = check_rows(x_bf16, ldx, K, "x")) || (base_bf16 && (rc = check_rows(base_bf16, ldb, N, "base"))) ||
        (rc = check_rows(y_bf16, ldy, N, "y")))
        return rc;
    const int64_t most = ldx > ldy ? ldx : ldy;
    if (most > kMostStride || (base_bf16 && ldb > kMostStride))
        return fail(MXFP4_ERR_SHAPE, "a row stride of %lld is more than %lld", (long long)(most > kMostStride ? most : ldb), (long long)kMostStride);
    if (base_bf16 == y_bf16 && ldb != ldy)
        return fail(MXFP4_ERR_ARG, "base is y with another row stride");
    if (!aligned(a_bf16, 16) || !aligned(b_bf16, 16) || !aligned(ids, 4) || !aligned(scales_f32, 4) || !aligned(workspace, 16))
        return fail(MXFP4_ERR_ALIGN, "a, b and workspace must be 16-byte aligned, ids and scales 4-byte");
    const size_t need = mxfp4_lora_workspace_bytes(M, K, R);
    if (!workspace || workspace_bytes < need)
        return fail(MXFP4_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    DeviceInfo dev;
    if ((rc = device_info(&dev)))
        return rc;
    LoraArgs a = {};
    a.x = static_cast<const uint16_t*>(x_bf16);
    a.a = static_cast<const uint16_t*>(a_bf16);
    a.b = static_cast<const uint16_t*>(b_bf16);
    a.ids = ids;
    a.scales = scales_f32;
    a.base = static_cast<const uint16_t*>(base_bf16);
    a.y = static_cast<uint16_t*>(y_bf16);
    a.part = static_cast<float*>(workspace);
    a.ldx = ldx;
    a.ldb = base_bf16 ? ldb : 0;
    a.ldy = ldy;
    a.m = (int)M;
    a.n = (int)N;
    a.k = (int)K;
    a.r = (int)R;
    a.adapters = (int)adapters;
    return launched(launch_lora(a, dev, static_cast<hipStream_t>(stream)), "adapter launch");
}

}  // extern "C"
