// Host side of grouped four-bit integers: argument checks and launches.  As the other word-table operators: no handle, no device memory
// of its own, nothing that waits.
#include <hip/hip_runtime.h>

#include <cmath>

#include "group_kernels.h"
#include "operands.h"

using namespace same::host;
using same::fail_without_handle;

namespace {

template <class TI, class TO>
void product_launch(const same::GroupProductArgs& p, int group_log2, hipStream_t st)
{
    const int64_t tiles = ((p.rows_a + 15) / 16) * ((p.rows_b + 15) / 16);
    const dim3 grid((unsigned)at_most((tiles + 3) / 4, kMaxGroups));
    switch (group_log2) {
        case 5:  hipLaunchKernelGGL((same::group_product_kernel<TI, TO, 5>), grid, dim3(256), 0, st, p); break;
        case 6:  hipLaunchKernelGGL((same::group_product_kernel<TI, TO, 6>), grid, dim3(256), 0, st, p); break;
        default: hipLaunchKernelGGL((same::group_product_kernel<TI, TO, 7>), grid, dim3(256), 0, st, p); break;
    }
}

template <class TI>
void product_to(const same::GroupProductArgs& p, int group_log2, int32_t type, hipStream_t st)
{
    switch (type) {
        case SAME_LDA_FLOAT:  return product_launch<TI, float>(p, group_log2, st);
        case SAME_LDA_BFLOAT: return product_launch<TI, __bf16>(p, group_log2, st);
        default:              return product_launch<TI, _Float16>(p, group_log2, st);
    }
}

}  // namespace

extern "C" {

int same_lda_group_size(int64_t rows, int32_t width, int32_t group, size_t* code_bytes, size_t* scale_bytes)
{
    if (!code_bytes || !scale_bytes) return fail_without_handle(SAME_LDA_EINVAL, "group_size: code_bytes or scale_bytes is null");
    if (rows < 0 || rows >= (int64_t)1 << 31 || width < 1 || width > SAME_LDA_WIDTH_MAX || !is_grouped(group))
        return fail_without_handle(SAME_LDA_EINVAL, "group_size: bad shape %lld x %d in groups of %d", (long long)rows, width, group);
    *code_bytes = (size_t)rows * (size_t)same::micro_code_pitch(width);
    *scale_bytes = (size_t)rows * (size_t)same::group_scale_pitch(width, __builtin_ctz((unsigned)group));
    return SAME_LDA_OK;
}

int same_lda_group_quantize(const same_lda_rows* x, const same_lda_rows* group_out, void* hip_stream)
{
    int rc = check_rows("group_quantize", "x", x, kNumbers);
    if (!rc) rc = check_rows("group_quantize", "group_out", group_out, kGrouped);
    if (rc) return rc;
    if (x->rows != group_out->rows || x->width != group_out->width)
        return fail_without_handle(SAME_LDA_EINVAL, "group_quantize: %lld x %d into %lld x %d", (long long)x->rows, x->width, (long long)group_out->rows, group_out->width);
    if (x->rows == 0) return SAME_LDA_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const same::GroupQuantizeArgs a = {x->data, x->rows, x->stride, x->width, __builtin_ctz((unsigned)group_out->type), static_cast<uint32_t*>(group_out->data),
                                       reinterpret_cast<uint32_t*>(group_out->scales)};
    const int64_t pieces = x->rows * same::micro_groups(x->width) * 16;
    const dim3 grid((unsigned)at_most((pieces + 255) / 256, kMaxGroups));
    switch (x->type) {
        case SAME_LDA_FLOAT:  hipLaunchKernelGGL(same::group_quantize_kernel<float>, grid, dim3(256), 0, st, a); break;
        case SAME_LDA_BFLOAT: hipLaunchKernelGGL(same::group_quantize_kernel<__bf16>, grid, dim3(256), 0, st, a); break;
        default:              hipLaunchKernelGGL(same::group_quantize_kernel<_Float16>, grid, dim3(256), 0, st, a); break;
    }
    return launched("group_quantize");
}

int same_lda_group_product(const same_lda_rows* a, const same_lda_rows* b, float scale, const same_lda_rows* out, void* hip_stream)
{
    int rc = check_rows("group_product", "a", a, kNumbers);
    if (!rc) rc = check_rows("group_product", "b", b, kGrouped);
    if (rc) return rc;
    if (a->width != b->width) return fail_without_handle(SAME_LDA_EINVAL, "group_product: rows of %d and of %d elements", a->width, b->width);
    if (b->rows == 0) return SAME_LDA_OK;                                                  // no columns: out is not looked at
    if ((rc = check_rows("group_product", "out", out, kNumbers, INT32_MAX))) return rc;
    if (out->rows != a->rows || out->width != b->rows)
        return fail_without_handle(SAME_LDA_EINVAL, "group_product: %lld rows by %lld rows do not give %lld x %d", (long long)a->rows, (long long)b->rows,
                                   (long long)out->rows, out->width);
    if (!std::isfinite(scale)) return fail_without_handle(SAME_LDA_EINVAL, "group_product: the scale must be finite");
    if (a->rows == 0) return SAME_LDA_OK;
    const int group_log2 = __builtin_ctz((unsigned)b->type);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const same::GroupProductArgs p = {a->data, a->rows, a->stride, a->width, static_cast<const uint8_t*>(b->data), b->scales, b->rows,
                                      same::micro_code_pitch(b->width), same::group_scale_pitch(b->width, group_log2), scale, out->data, out->stride};
    switch (a->type) {
        case SAME_LDA_FLOAT:  product_to<float>(p, group_log2, out->type, st); break;
        case SAME_LDA_BFLOAT: product_to<__bf16>(p, group_log2, out->type, st); break;
        default:              product_to<_Float16>(p, group_log2, out->type, st); break;
    }
    return launched("group_product");
}

}  // extern "C"
