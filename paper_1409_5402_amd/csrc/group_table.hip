// Host side of grouped four-bit integers: argument checks and launches.  As the other word-table operators: no handle, no device memory
// of its own, nothing that waits.
#include <hip/hip_runtime.h>

#include <cmath>

#include "group_kernels.h"
#include "operands.h"

using namespace same::host;
using same::fail_without_handle;

namespace {

constexpr int64_t kRowsOfA = (int64_t)1 << 24, kRowsOfB = (int64_t)1 << 28;

template <class TI, int P, bool kStack, int kGroupLog2, int KB>
void product_few(same::GroupProductArgs& p, int blocks, hipStream_t st)
{
    int kw = 1;
    while (kw * KB < blocks) kw *= 2;                                    // at most 8
    p.waves_per_row = kw;
    const int waves = kw < 4 ? 4 : kw, streams = waves / kw;
    const int64_t turns = ((p.rows_b + 15) / 16 + streams - 1) / streams;
    hipLaunchKernelGGL((same::group_product_few_kernel<TI, P, kStack, kGroupLog2, KB>), dim3((unsigned)at_most(turns, kComputeUnits * 8 / waves)), dim3(64 * waves), 0, st, p);
}

template <class TI, int P, bool kStack, int kGroupLog2>
void product_few_by_width(same::GroupProductArgs& p, int blocks, hipStream_t st)
{
    if (blocks == 1) product_few<TI, P, kStack, kGroupLog2, 1>(p, blocks, st);
    else if (blocks <= 2 || blocks == 16) product_few<TI, P, kStack, kGroupLog2, 2>(p, blocks, st);
    else product_few<TI, P, kStack, kGroupLog2, 4>(p, blocks, st);
}

template <class TI, int kGroupLog2, int MT, int NT, int WK>
void product_tiles(const same::GroupProductArgs& p, hipStream_t st)
{
    const int64_t across = 16 * NT * (4 / WK), tiles_a = (p.rows_a + 16 * MT - 1) / (16 * MT), tiles_b = ((p.rows_b + across - 1) / across + 7) / 8 * 8;
    hipLaunchKernelGGL((same::group_product_kernel<TI, kGroupLog2, MT, NT, WK>), dim3((unsigned)(tiles_a * tiles_b)), dim3(256), 0, st, p);
}

template <class TI, int kGroupLog2>
void product_launch(same::GroupProductArgs& p, hipStream_t st)
{
    const int blocks = (p.width + 127) / 128;
    if (p.rows_a <= 16 && blocks <= 32) {
        if constexpr (sizeof(TI) == 4) return p.rows_a <= 4 ? product_few_by_width<TI, 1, true, kGroupLog2>(p, blocks, st) : product_few_by_width<TI, 3, false, kGroupLog2>(p, blocks, st);
        else return product_few_by_width<TI, 1, false, kGroupLog2>(p, blocks, st);
    }
    constexpr int kTall = sizeof(TI) == 4 ? 2 : 4;                       // of 16 rows of a
    if (p.rows_a <= 16)      product_tiles<TI, kGroupLog2, 1, 2, 4>(p, st);
    else if (p.rows_a <= 32) product_tiles<TI, kGroupLog2, 2, 2, sizeof(TI) == 4 ? 2 : 4>(p, st);
    else                     product_tiles<TI, kGroupLog2, kTall, 4, 1>(p, st);
}

template <class TI>
void product_to(same::GroupProductArgs& p, int group_log2, hipStream_t st)
{
    switch (group_log2) {
        case 5:  return product_launch<TI, 5>(p, st);
        case 6:  return product_launch<TI, 6>(p, st);
        default: return product_launch<TI, 7>(p, st);
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
    // slices of either operand: grids stay below 2^32 threads (the output's size bounds the tiles)
    for (int64_t i = 0; i < a->rows; i += kRowsOfA)
        for (int64_t j = 0; j < b->rows; j += kRowsOfB) {
            same::GroupProductArgs p = {};
            p.rows_a = at_most(a->rows - i, kRowsOfA);
            p.rows_b = at_most(b->rows - j, kRowsOfB);
            p.a = static_cast<const char*>(a->data) + i * a->stride * element_bytes(a->type);
            p.stride_a = a->stride;
            p.width = a->width;
            p.type_out = out->type;
            p.pitch = same::micro_code_pitch(b->width);
            p.scale_pitch = same::group_scale_pitch(b->width, group_log2);
            p.codes = static_cast<const uint8_t*>(b->data) + j * p.pitch;
            p.scales = b->scales + j * p.scale_pitch;
            p.scale = scale;
            p.out = static_cast<char*>(out->data) + (i * out->stride + j) * element_bytes(out->type);
            p.out_stride = out->stride;
            switch (a->type) {
                case SAME_LDA_FLOAT:  product_to<float>(p, group_log2, st); break;
                case SAME_LDA_BFLOAT: product_to<__bf16>(p, group_log2, st); break;
                default:              product_to<_Float16>(p, group_log2, st); break;
            }
        }
    return launched("group_product");
}

}  // extern "C"
