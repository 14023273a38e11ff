#include "embed_grad_launch.h"

int same::host::grad_sums_dropout_float(GradArgs& a, const same_lda_rows* grad, const same_lda_rows* table_grad, hipStream_t st)
{
    return grad_to<float, true>(a, grad, table_grad, st);
}
