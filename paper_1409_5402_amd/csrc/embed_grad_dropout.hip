// The gradient's sums for a lookup with dropout.
#include "embed_grad_launch.h"

namespace same {
namespace host {

int grad_sums_dropout(GradArgs& a, const same_lda_rows* grad, const same_lda_rows* table_grad, hipStream_t st) { return grad_sums<true>(a, grad, table_grad, st); }

}  // namespace host
}  // namespace same
