// Host side of the gradient of a word table: argument checks, workspace and launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "embed_grad_launch.h"
#include "operands.h"
#include "rows_call.h"
#include "token_sort.h"

using namespace same::host;
using same::fail_without_handle;

namespace {

// Workspace of the gradient, in this order; every part starts at a multiple of 256 bytes.
struct GradSpace {
    size_t sorted[2], hist, total, start, partial, bytes;
    uint32_t tiles;
    int64_t ranges;
    int passes, bits;
    bool small_tiles;
};

constexpr int kTileRows = 16, kSmallTileRows = 4;                    // rows of 256 tokens in a tile of the sort
constexpr int64_t kSmallTiles = 1 << 22;                             // up to this many tokens the tiles are small

// One launch without a sort (us, sorted after it):
//   up to 8192 tokens     8192 into 30,000 x 1024 bf16 35, 53; into 2000 x 1024 f32 31, 36; into a million words x 16 f32 59, 58
//   up to 16,384 tokens   where rows of the gradient are short (into 2000 x 64 f32 26, 37; into 30,000 x 1024 bf16 59, 57; into 2000 x
//                         1024 f32, where the most frequent word keeps one compute unit busy, 63, 40); beyond 2^18 words not of 512 bytes
//                         and less, for a compute unit takes one workgroup of 256 words at a time then, each reads the whole list,
//                         and writing such rows does not hide it (f32, into 200,000 x 16 40, 45; 400,000 x 16 66, 55; 400,000 x
//                         128 89, 80; 400,000 x 192 116, 129; a million x 16 143, 61)
// and a grid below 2^32 threads: 1024 for every 256 words begun, and every 64 chunks of a row.
constexpr int64_t kScannedWords = 1 << 18;
// With dropout the workgroup of a frequent word has the choice for all its rows to make as well, so beyond 4096 tokens only short rows, or rows of
// tables of many words, go in one launch, and beyond 8192 only both (us, sorted after it: 4096 into 30,000 x 1024 bf16 57, 64, 8192 91, 72; 8000
// into 2000 x 128 f32 36, 53, x 256 54, 39; 8000 into 100,000 x 256 f16 52, 79, 16,000 88, 78; 16,000 into 2000 x 50 f32 48, 45, into 100,000 x
// 64 39, 64).
constexpr int64_t kDroppedTokens = 4096;
bool few_tokens(int64_t n, int64_t rows, const same_lda_rows* grad, bool drop)
{
    if (drop && n > kDroppedTokens) {
        const bool many = rows > 4 * n;
        if (n > kFewerTokens ? !(many && grad->width <= 64) : !(many || grad->width <= 128)) return false;
    }
    const int64_t row_bytes = (int64_t)grad->width * element_bytes(grad->type);
    const bool more = row_bytes <= 2048 && (rows <= kScannedWords || row_bytes > 512);
    return n <= (more ? same::kFewTokens : kFewerTokens) && (rows + 256) * ((grad->width + 63) / 64) < (int64_t)1 << 30;
}

GradSpace grad_space(const same_lda_rows* grad, int64_t rows, bool drop)
{
    const int64_t n = grad->rows, width = grad->width;
    GradSpace s = {};
    if (n == 0 || few_tokens(n, rows, grad, drop)) return s;
    size_t at = 0;
    const auto part = [&at](size_t bytes) { const size_t here = at; at += (bytes + 255) & ~(size_t)255; return here; };
    int bits = 1;
    while (((int64_t)1 << bits) <= rows) ++bits;                     // words 0 .. rows - 1, and rows for padding
    s.passes = (bits + same::kDigitBits - 1) / same::kDigitBits;
    s.bits = (bits + s.passes - 1) / s.passes;
    s.small_tiles = n <= kSmallTiles;
    const int64_t tile = 256 * (s.small_tiles ? kSmallTileRows : kTileRows);
    s.tiles = (uint32_t)(((n + tile - 1) / tile + 3) & ~(int64_t)3);        // four counts in one load
    s.ranges = (n + same::kLongRun - 1) / same::kLongRun;
    for (int i = 0; i < 2; ++i) s.sorted[i] = part((size_t)n * sizeof(same::Placed));
    s.hist = part(((size_t)s.tiles << s.bits) * 4);
    s.total = part(sizeof(uint32_t) << s.bits);
    s.start = part(((size_t)rows + 1) * 4);
    s.partial = part((size_t)s.ranges * 2 * (size_t)width * 4);
    s.bytes = at;
    return s;
}

template <int R>
void sort_pass(const same::GradArgs& a, const GradSpace& s, int64_t n, int pass, uint32_t* hist, uint32_t* total, same::Placed* to, hipStream_t st)
{
    const int shift = pass * s.bits;
    hipLaunchKernelGGL(same::token_histogram<R>, dim3(s.tiles), dim3(256), 0, st, a.tokens, a.rows, a.sorted, n, shift, s.bits, s.tiles, hist);
    if (s.tiles <= same::kFewTiles) {
        hipLaunchKernelGGL((same::token_place<R, true>), dim3(s.tiles), dim3(256), 0, st, a.tokens, a.rows, a.sorted, n, shift, s.bits, s.tiles, hist, total, to);
        return;
    }
    hipLaunchKernelGGL(same::token_offsets, dim3(1u << s.bits), dim3(256), 0, st, hist, s.tiles, total);
    hipLaunchKernelGGL((same::token_place<R, false>), dim3(s.tiles), dim3(256), 0, st, a.tokens, a.rows, a.sorted, n, shift, s.bits, s.tiles, hist, total, to);
}

int check_grad(const char* call, const same_lda_rows* grad, const same_lda_rows* table_grad)
{
    int rc = check_rows(call, "grad", grad, kNumbers);
    if (!rc) rc = check_rows(call, "table_grad", table_grad, kNumbers);
    if (!rc && grad->width != table_grad->width)
        rc = fail_without_handle(SAME_LDA_EINVAL, "%s: rows of %d and of %d elements", call, grad->width, table_grad->width);
    return rc;
}

int workspace_of(const same_lda_rows* grad, const same_lda_rows* table_grad, bool drop, size_t* bytes)
{
    const char* const call = grad_call_name(drop);
    if (!bytes) return fail_without_handle(SAME_LDA_EINVAL, "%s: bytes is null", call);
    const int rc = check_grad(call, grad, table_grad);
    if (rc) return rc;
    *bytes = grad_space(grad, table_grad->rows, drop).bytes;
    return SAME_LDA_OK;
}

// `drop`: that of the lookup, or null
int grad_call(const same_lda_rows* grad, const void* tokens, int32_t token_bytes, float scale, const same::Drop* drop, int32_t accumulate,
              const same_lda_rows* table_grad, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    const char* const call = grad_call_name(drop);
    int rc = check_grad(call, grad, table_grad);
    if (!rc) rc = check_tokens(call, tokens, token_bytes, grad->rows);
    if (rc) return rc;
    if (!tokens && grad->rows > 0) return fail_without_handle(SAME_LDA_EINVAL, "%s: tokens is null", call);
    if (!std::isfinite(scale)) return fail_without_handle(SAME_LDA_EINVAL, "%s: the scale must be finite", call);
    const int64_t n = grad->rows, rows = table_grad->rows;
    const GradSpace s = grad_space(grad, rows, drop);
    if (rows == 0 || (n == 0 && accumulate)) return SAME_LDA_OK;
    if (s.bytes > 0 && (!workspace || workspace_bytes < s.bytes || (uintptr_t)workspace % 16))
        return fail_without_handle(SAME_LDA_EINVAL, "%s: needs %zu bytes of workspace aligned to 16 (got %zu)", call, s.bytes, workspace ? workspace_bytes : (size_t)0);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (n == 0) return rows_of_zeros(call, table_grad, st);
    char* const w = static_cast<char*>(workspace);
    same::GradArgs a = {grad->data, grad->stride, nullptr, nullptr, rows, scale, accumulate, table_grad->data, table_grad->stride,
                        nullptr, s.ranges, grad->width, 0, 0, {tokens, token_bytes == 8}, (int32_t)n, 0, 0, drop ? *drop : same::Drop{}};
    if (!few_tokens(n, rows, grad, drop)) {
        uint32_t* const hist = reinterpret_cast<uint32_t*>(w + s.hist);
        uint32_t* const total = reinterpret_cast<uint32_t*>(w + s.total);
        int32_t* const start = reinterpret_cast<int32_t*>(w + s.start);
        for (int i = 0; i < s.passes; ++i) {
            same::Placed* const to = reinterpret_cast<same::Placed*>(w + s.sorted[i & 1]);
            if (s.small_tiles) sort_pass<kSmallTileRows>(a, s, n, i, hist, total, to, st);
            else               sort_pass<kTileRows>(a, s, n, i, hist, total, to, st);
            a.sorted = to;
        }
        if (rows > 4 * n) hipLaunchKernelGGL(same::word_runs_sparse, dim3((unsigned)((rows + 256) / 256)), dim3(256), 0, st, a.sorted, n, rows, start);
        else              hipLaunchKernelGGL(same::word_runs, dim3((unsigned)((n + 256) / 256)), dim3(256), 0, st, a.sorted, n, rows, start);
        if ((rc = launched(call))) return rc;
        a.start = start;
        a.partial = reinterpret_cast<float*>(w + s.partial);
    }
    switch (grad->type) {
        case SAME_LDA_FLOAT:  return drop ? grad_sums_dropout_float(a, grad, table_grad, st) : grad_to<float, false>(a, grad, table_grad, st);
        case SAME_LDA_BFLOAT: return drop ? grad_sums_dropout_bfloat(a, grad, table_grad, st) : grad_to<__bf16, false>(a, grad, table_grad, st);
        default:              return drop ? grad_sums_dropout_half(a, grad, table_grad, st) : grad_to<_Float16, false>(a, grad, table_grad, st);
    }
}

}  // namespace

extern "C" {

int same_lda_embed_grad_workspace(const same_lda_rows* grad, const same_lda_rows* table_grad, size_t* bytes) { return workspace_of(grad, table_grad, false, bytes); }

int same_lda_embed_dropout_grad_workspace(const same_lda_rows* grad, const same_lda_rows* table_grad, size_t* bytes)
{
    return workspace_of(grad, table_grad, true, bytes);
}

int same_lda_embed_grad(const same_lda_rows* grad, const void* tokens, int32_t token_bytes, float scale, int32_t accumulate,
                        const same_lda_rows* table_grad, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    return grad_call(grad, tokens, token_bytes, scale, nullptr, accumulate, table_grad, workspace, workspace_bytes, hip_stream);
}

int same_lda_embed_dropout_grad(const same_lda_rows* grad, const void* tokens, int32_t token_bytes, float scale, const same_lda_drop* drop, int32_t accumulate,
                                const same_lda_rows* table_grad, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    same::Drop d;
    const int rc = check_drop("embed_dropout_grad", drop, &scale, &d);
    return rc ? rc : grad_call(grad, tokens, token_bytes, scale, &d, accumulate, table_grad, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
