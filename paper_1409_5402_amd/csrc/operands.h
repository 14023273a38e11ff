// Host side of the word-table operators: checks of operands and what launches are sized by.
#pragma once
#include "../../include/same_lda.h"

#include <hip/hip_runtime.h>

#include "errors.h"

namespace same {
namespace host {

// What an operand may be.
constexpr int kNumbers = 1, kMicro = 2, kGrouped = 4;

inline int element_bytes(int32_t type) { return type == SAME_LDA_FLOAT ? 4 : 2; }
inline bool is_grouped(int32_t type) { return type == SAME_LDA_GROUPS_OF_32 || type == SAME_LDA_GROUPS_OF_64 || type == SAME_LDA_GROUPS_OF_128; }
inline int form_of(int32_t type)
{
    return type == SAME_LDA_FLOAT || type == SAME_LDA_BFLOAT || type == SAME_LDA_HALF ? kNumbers : type == SAME_LDA_MICRO ? kMicro : is_grouped(type) ? kGrouped : 0;
}

// Shape, type and alignment of one operand.
inline int check_rows(const char* call, const char* name, const same_lda_rows* m, int allowed, int32_t width_max = SAME_LDA_WIDTH_MAX)
{
    if (!m) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s is null", call, name);
    const int form = form_of(m->type);
    if (!form) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s has the unknown type %d", call, name, m->type);
    if (!(form & allowed)) {
        const bool only = (allowed & (allowed - 1)) == 0 && allowed != kNumbers;
        return fail_without_handle(SAME_LDA_EINVAL, "%s: %s %s be %s", call, name, only ? "must" : "must not", (only ? allowed : form) == kMicro ? "microscaled" : "grouped");
    }
    if (m->rows < 0 || m->rows >= (int64_t)1 << 31) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s has %lld rows, not in [0, 2^31)", call, name, (long long)m->rows);
    if (m->width < 1 || m->width > width_max)
        return fail_without_handle(SAME_LDA_EINVAL, "%s: rows of %s hold %d elements, not in [1, %d]", call, name, m->width, width_max);
    const bool numbers = form == kNumbers;
    if (numbers && m->rows > 1 && m->stride < m->width)
        return fail_without_handle(SAME_LDA_EINVAL, "%s: the stride %lld of %s is less than its width %d", call, (long long)m->stride, name, m->width);
    if (numbers && m->rows > 1 && m->stride > ((int64_t)1 << 62) / 8 / m->rows)
        return fail_without_handle(SAME_LDA_EINVAL, "%s: the stride %lld of %s is too large", call, (long long)m->stride, name);
    if (m->rows == 0) return SAME_LDA_OK;
    if (!m->data || (!numbers && !m->scales)) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s has no data", call, name);
    const uintptr_t align = numbers ? (uintptr_t)element_bytes(m->type) : 16;
    if ((uintptr_t)m->data % align || (!numbers && (uintptr_t)m->scales % 4))
        return fail_without_handle(SAME_LDA_EINVAL, "%s: %s is not aligned (elements to their size, codes to 16 bytes, scales to 4)", call, name);
    return SAME_LDA_OK;
}

inline int check_tokens(const char* call, const void* tokens, int32_t token_bytes, int64_t n)
{
    if (token_bytes != 4 && token_bytes != 8) return fail_without_handle(SAME_LDA_EINVAL, "%s: tokens have %d bytes, not 4 or 8", call, token_bytes);
    if ((uintptr_t)tokens % token_bytes) return fail_without_handle(SAME_LDA_EINVAL, "%s: tokens are not aligned to their size", call);
    if (n < 0 || n >= (int64_t)1 << 31) return fail_without_handle(SAME_LDA_EINVAL, "%s: %lld tokens, not in [0, 2^31)", call, (long long)n);
    return SAME_LDA_OK;
}

inline int launched(const char* call)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SAME_LDA_OK : fail_without_handle(SAME_LDA_EHIP, "%s: %s", call, hipGetErrorString(e));
}

// Whether chunks of v elements of every row are aligned to their size (16 bytes at most).
inline bool chunks_fit(const same_lda_rows* m, int v)
{
    if (form_of(m->type) != kNumbers) return true;
    const int64_t bytes = (int64_t)v * element_bytes(m->type);
    const int64_t align = bytes < 16 ? bytes : 16;
    return m->width % v == 0 && (uintptr_t)m->data % align == 0 && (m->rows < 2 || m->stride * element_bytes(m->type) % align == 0);
}

// Lanes that share a row of so many chunks: the power of two from 1 to 64 that leaves the fewest idle.
inline int lanes_log2_for(int64_t chunks)
{
    int l = 0;
    while (l < 6 && ((int64_t)1 << l) < chunks) ++l;
    return l;
}

inline int64_t at_most(int64_t n, int64_t most) { return n < most ? n : most; }

constexpr int64_t kComputeUnits = 256;
constexpr int64_t kMaxGroups = (int64_t)1 << 22;     // workgroups of a launch (256 threads each: below 2^32 threads)

}  // namespace host
}  // namespace same
