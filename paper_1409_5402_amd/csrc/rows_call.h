// Calls that the sources of the word-table operators share.
#pragma once
#include "dropout.h"
#include "operands.h"

namespace same {
namespace host {

// A call's dropout as the kernels take it; the scale becomes that of the elements that are kept, scale / (1 - p) rounded once.
__attribute__((visibility("hidden"))) int check_drop(const char* call, const same_lda_drop* drop, float* scale, Drop* d);

// Lookup with dropout (or without: null) and out of tables in grouped integers; tokens null: the rows in order.  Operands are checked.
__attribute__((visibility("hidden"))) int rows_call(const char* call, const same_lda_rows* table, const void* tokens, int32_t token_bytes, float scale, const Drop* drop,
                                                    const same_lda_rows* out, void* hip_stream);

// A matrix of zeros.
__attribute__((visibility("hidden"))) int rows_of_zeros(const char* call, const same_lda_rows* out, hipStream_t st);

}  // namespace host
}  // namespace same
