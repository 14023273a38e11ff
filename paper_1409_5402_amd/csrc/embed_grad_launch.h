// Launches of the gradient's sums, with and without dropout in the lookup: compiled in two sources.
#pragma once
#include <hip/hip_runtime.h>

#include "embed_grad_kernels.h"
#include "operands.h"

namespace same {
namespace host {

constexpr int kFewerTokens = 8192;                                   // most tokens of the smaller of the kernels that take few

inline const char* grad_call_name(bool drop) { return drop ? "embed_dropout_grad" : "embed_grad"; }     // in messages

template <class TI, class TO, int V, bool kDrop>
int grad_launch(GradArgs& a, hipStream_t st)
{
    a.chunks = a.width / V;
    a.lanes_log2 = lanes_log2_for(a.chunks);
    const int64_t per = (int64_t)256 >> a.lanes_log2;
    const unsigned across = (unsigned)((a.chunks + (1 << a.lanes_log2) - 1) >> a.lanes_log2);
    const int64_t most = kMaxGroups / across;                        // across <= SAME_LDA_WIDTH_MAX / 64
    if (!a.start) {                                                  // few tokens
        // 512 workgroups, for each reads the whole list; more where a workgroup's words would be more than fit.  A compute unit holds two
        // of them up to 8192 tokens and V < 8; otherwise (some 100 registers, or 114 KB of LDS) one, and the grid runs in two rounds
        if (a.lanes_log2 < 2) a.lanes_log2 = 2;                      // 256 groups at most, and words
        const int64_t groups = (int64_t)1024 >> a.lanes_log2;
        a.unit_log2 = 0;
        while (a.unit_log2 < 5 && ((int64_t)a.width * (int64_t)sizeof(TO) << a.unit_log2) < 128) ++a.unit_log2;
        const int64_t units = ((a.rows - 1) >> a.unit_log2) + 1, most_units = kFewWords >> a.unit_log2;
        int64_t workgroups = at_most((a.rows + groups - 1) / groups, 2 * kComputeUnits / across > 1 ? 2 * kComputeUnits / across : 1);
        workgroups = workgroups < (units + most_units - 1) / most_units ? (units + most_units - 1) / most_units : workgroups;
        a.words = (int32_t)((units + workgroups - 1) / workgroups << a.unit_log2);
        if (a.n <= kFewerTokens) hipLaunchKernelGGL((embed_grad_few_kernel<TI, TO, V, kFewerTokens / 1024, kDrop>), dim3((unsigned)workgroups, across), dim3(1024), 0, st, a);
        else                     hipLaunchKernelGGL((embed_grad_few_kernel<TI, TO, V, kFewTokens / 1024, kDrop>), dim3((unsigned)workgroups, across), dim3(1024), 0, st, a);
        return launched(grad_call_name(kDrop));
    }
    const dim3 grid((unsigned)at_most((a.ranges + a.rows + per - 1) / per, most), across);
    if (a.lanes_log2 < 4) hipLaunchKernelGGL((embed_grad_kernel<TI, TO, V, true, kDrop>), grid, dim3(256), 0, st, a);
    else                  hipLaunchKernelGGL((embed_grad_kernel<TI, TO, V, false, kDrop>), grid, dim3(256), 0, st, a);
    if (a.lanes_log2 > kJoinLanesLog2) a.lanes_log2 = kJoinLanesLog2;
    const int64_t items = (int64_t)1024 >> a.lanes_log2;             // ranges of a workgroup
    const unsigned columns = (unsigned)((a.chunks + (1 << a.lanes_log2) - 1) >> a.lanes_log2), deep = (columns + 65534) / 65535;   // 65,535 of them side by side
    hipLaunchKernelGGL((embed_grad_join_kernel<TO, V>), dim3((unsigned)((a.ranges + items - 1) / items), (columns + deep - 1) / deep, deep), dim3(1024), 0, st, a);
    return launched(grad_call_name(kDrop));
}

template <class TI, class TO, bool kDrop>
int grad_by_width(GradArgs& a, const same_lda_rows* grad, const same_lda_rows* out, hipStream_t st)
{
    constexpr int kWide = sizeof(TI) == 4 && sizeof(TO) == 4 ? 4 : 8;
    if (chunks_fit(grad, kWide) && chunks_fit(out, kWide)) return grad_launch<TI, TO, kWide, kDrop>(a, st);
    if (chunks_fit(grad, 2) && chunks_fit(out, 2)) return grad_launch<TI, TO, 2, kDrop>(a, st);
    return grad_launch<TI, TO, 1, kDrop>(a, st);
}

template <class TI, bool kDrop>
int grad_to(GradArgs& a, const same_lda_rows* grad, const same_lda_rows* out, hipStream_t st)
{
    switch (out->type) {
        case SAME_LDA_FLOAT:  return grad_by_width<TI, float, kDrop>(a, grad, out, st);
        case SAME_LDA_BFLOAT: return grad_by_width<TI, __bf16, kDrop>(a, grad, out, st);
        default:              return grad_by_width<TI, _Float16, kDrop>(a, grad, out, st);
    }
}

// The sums for gradients of one type after a lookup with dropout: a source each, they take longest to compile.
__attribute__((visibility("hidden"))) int grad_sums_dropout_float(GradArgs& a, const same_lda_rows* grad, const same_lda_rows* table_grad, hipStream_t st);
__attribute__((visibility("hidden"))) int grad_sums_dropout_bfloat(GradArgs& a, const same_lda_rows* grad, const same_lda_rows* table_grad, hipStream_t st);
__attribute__((visibility("hidden"))) int grad_sums_dropout_half(GradArgs& a, const same_lda_rows* grad, const same_lda_rows* table_grad, hipStream_t st);

}  // namespace host
}  // namespace same
