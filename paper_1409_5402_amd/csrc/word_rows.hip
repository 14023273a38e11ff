// Host side of dropout, of the lookup with dropout and of rows of tables in grouped integers.  As the other word-table operators:
// no handle, no device memory of its own, nothing that waits.
#include <hip/hip_runtime.h>

#include <cmath>

#include "rows_call.h"
#include "rows_kernel.h"

namespace same {
namespace host {

int check_drop(const char* call, const same_lda_drop* drop, float* scale, Drop* d)
{
    if (!drop) return fail_without_handle(SAME_LDA_EINVAL, "%s: drop is null", call);
    if (!(drop->p >= 0.0 && drop->p <= 1.0)) return fail_without_handle(SAME_LDA_EINVAL, "%s: the probability %g is not in [0, 1]", call, drop->p);
    if (drop->step >> 56) return fail_without_handle(SAME_LDA_EINVAL, "%s: the step is not in [0, 2^56)", call);
    if ((uintptr_t)drop->step_at % 8) return fail_without_handle(SAME_LDA_EINVAL, "%s: the step in device memory is not aligned to its size", call);
    if (!std::isfinite(*scale)) return fail_without_handle(SAME_LDA_EINVAL, "%s: the scale must be finite", call);
    const double keep = std::nearbyint((1.0 - drop->p) * 4294967296.0), factor = drop->p < 1.0 ? (double)*scale / (1.0 - drop->p) : 0.0;
    if (!std::isfinite((float)factor)) return fail_without_handle(SAME_LDA_EINVAL, "%s: the scale %g / (1 - %g) is beyond binary32", call, (double)*scale, drop->p);
    const uint64_t border = (uint64_t)keep;
    *scale = (float)factor;
    const uint32_t keep_hi = border >> 32 ? 0xFFFFu : (uint32_t)(border >> 16);              // all of them: every half up to 65,535, and there every other
    *d = {(uint32_t)drop->seed, (uint32_t)(drop->seed >> 32), drop->step, drop->step_at, keep_hi, (uint32_t)(border - ((uint64_t)keep_hi << 16))};
    return SAME_LDA_OK;
}

namespace {

constexpr int64_t kRounds = 8;                                           // workgroups of a launch for each that a compute unit holds

template <class TI, class TO>
int rows_launch(const char* call, RowsArgs& a, bool drop, hipStream_t st)
{
    const int64_t groups = at_most((a.n * a.chunks + kChunksAtOnce - 1) / kChunksAtOnce, kComputeUnits * 8 * kRounds);
    const int64_t step = groups * kChunksAtOnce;
    a.step_rows = (int32_t)(step / a.chunks);
    a.step_chunks = (int32_t)(step % a.chunks);
    const dim3 grid((unsigned)groups);
    if (drop) hipLaunchKernelGGL((rows_kernel<TI, TO, true>), grid, dim3(256), 0, st, a);
    else if constexpr (__is_same(TI, GroupCode)) hipLaunchKernelGGL((rows_kernel<TI, TO, false>), grid, dim3(256), 0, st, a);
    return launched(call);
}

template <class TI>
int rows_to(const char* call, RowsArgs& a, bool drop, int32_t type, hipStream_t st)
{
    switch (type) {
        case SAME_LDA_FLOAT:  return rows_launch<TI, float>(call, a, drop, st);
        case SAME_LDA_BFLOAT: return rows_launch<TI, __bf16>(call, a, drop, st);
        default:              return rows_launch<TI, _Float16>(call, a, drop, st);
    }
}

}  // namespace

int rows_call(const char* call, const same_lda_rows* table, const void* tokens, int32_t token_bytes, float scale, const Drop* drop, const same_lda_rows* out,
              void* hip_stream)
{
    if (out->rows == 0) return SAME_LDA_OK;
    const int form = form_of(table->type), group_log2 = form == kGrouped ? __builtin_ctz((unsigned)table->type) : 0;
    RowsArgs a = {};
    a.table = table->data;
    a.scales = table->scales;
    a.rows = table->rows;
    a.stride = form == kNumbers ? table->stride : micro_code_pitch(table->width);
    a.scale_pitch = form == kGrouped ? group_scale_pitch(table->width, group_log2) : 0;
    a.group_log2 = group_log2;
    a.tokens = {tokens, token_bytes == 8};
    a.n = out->rows;
    a.factor = scale;
    a.out = out->data;
    a.out_stride = out->stride;
    a.width = out->width;
    a.chunks = (out->width + 7) / 8;
    a.inverse = 1.0f / (float)a.chunks;
    if (drop) a.drop = *drop;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    switch (table->type) {
        case SAME_LDA_FLOAT:  return rows_to<float>(call, a, drop, out->type, st);
        case SAME_LDA_BFLOAT: return rows_to<__bf16>(call, a, drop, out->type, st);
        case SAME_LDA_HALF:   return rows_to<_Float16>(call, a, drop, out->type, st);
        case SAME_LDA_MICRO:  return rows_to<MicroCode>(call, a, drop, out->type, st);
        default:              return rows_to<GroupCode>(call, a, drop, out->type, st);
    }
}

}  // namespace host
}  // namespace same

using namespace same::host;

extern "C" {

int same_lda_dropout(const same_lda_rows* x, const same_lda_drop* drop, const same_lda_rows* out, void* hip_stream)
{
    int rc = check_rows("dropout", "x", x, kNumbers);
    if (!rc) rc = check_rows("dropout", "out", out, kNumbers);
    if (rc) return rc;
    if (x->rows != out->rows || x->width != out->width)
        return same::fail_without_handle(SAME_LDA_EINVAL, "dropout: %lld x %d into %lld x %d", (long long)x->rows, x->width, (long long)out->rows, out->width);
    same::Drop d;
    float scale = 1.0f;
    if ((rc = check_drop("dropout", drop, &scale, &d))) return rc;
    return rows_call("dropout", x, nullptr, 8, scale, &d, out, hip_stream);
}

int same_lda_embed_dropout(const same_lda_rows* table, const void* tokens, int32_t token_bytes, float scale, const same_lda_drop* drop, const same_lda_rows* out,
                           void* hip_stream)
{
    int rc = check_rows("embed_dropout", "table", table, kNumbers | kMicro | kGrouped);
    if (!rc) rc = check_rows("embed_dropout", "out", out, kNumbers);
    if (!rc) rc = check_tokens("embed_dropout", tokens, token_bytes, out->rows);
    if (rc) return rc;
    if (table->width != out->width) return same::fail_without_handle(SAME_LDA_EINVAL, "embed_dropout: rows of %d and of %d elements", table->width, out->width);
    if (!tokens && out->rows != table->rows)
        return same::fail_without_handle(SAME_LDA_EINVAL, "embed_dropout: without tokens all %lld rows are written, not %lld", (long long)table->rows, (long long)out->rows);
    same::Drop d;
    if ((rc = check_drop("embed_dropout", drop, &scale, &d))) return rc;
    return rows_call("embed_dropout", table, tokens, token_bytes, scale, &d, out, hip_stream);
}

}  // extern "C"
