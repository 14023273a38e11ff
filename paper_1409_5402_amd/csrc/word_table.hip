// Host side of the word-table operators: argument checks and launches.  No handle, no device memory of its own, nothing
// that waits: every call only enqueues kernels, so all of them can be captured into a graph.
#include "../../include/same_lda.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "embed_kernels.h"
#include "errors.h"
#include "micro_kernels.h"

namespace {

using same::fail_without_handle;

int element_bytes(int32_t type) { return type == SAME_LDA_FLOAT ? 4 : 2; }
bool is_float_type(int32_t type) { return type == SAME_LDA_FLOAT || type == SAME_LDA_BFLOAT || type == SAME_LDA_HALF; }

// Shape, type and alignment of one operand.  `micro`: whether it is in four bits (-1: either).
int check_rows(const char* call, const char* name, const same_lda_rows* m, int micro, int32_t width_max = SAME_LDA_WIDTH_MAX)
{
    if (!m) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s is null", call, name);
    if (m->type != SAME_LDA_MICRO && !is_float_type(m->type)) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s has the unknown type %d", call, name, m->type);
    if (micro >= 0 && (m->type == SAME_LDA_MICRO) != (micro == 1))
        return fail_without_handle(SAME_LDA_EINVAL, "%s: %s %s be microscaled", call, name, micro ? "must" : "must not");
    if (m->rows < 0 || m->rows >= (int64_t)1 << 31) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s has %lld rows, not in [0, 2^31)", call, name, (long long)m->rows);
    if (m->width < 1 || m->width > width_max)
        return fail_without_handle(SAME_LDA_EINVAL, "%s: rows of %s hold %d elements, not in [1, %d]", call, name, m->width, width_max);
    if (m->type != SAME_LDA_MICRO && m->rows > 1 && m->stride < m->width)
        return fail_without_handle(SAME_LDA_EINVAL, "%s: the stride %lld of %s is less than its width %d", call, (long long)m->stride, name, m->width);
    if (m->type != SAME_LDA_MICRO && m->rows > 1 && m->stride > ((int64_t)1 << 62) / 8 / m->rows)
        return fail_without_handle(SAME_LDA_EINVAL, "%s: the stride %lld of %s is too large", call, (long long)m->stride, name);
    if (m->rows == 0) return SAME_LDA_OK;
    if (!m->data || (m->type == SAME_LDA_MICRO && !m->scales)) return fail_without_handle(SAME_LDA_EINVAL, "%s: %s has no data", call, name);
    const uintptr_t align = m->type == SAME_LDA_MICRO ? 16 : (uintptr_t)element_bytes(m->type);
    if ((uintptr_t)m->data % align || (m->type == SAME_LDA_MICRO && (uintptr_t)m->scales % 4))
        return fail_without_handle(SAME_LDA_EINVAL, "%s: %s is not aligned (elements to their size, codes to 16 bytes, scales to 4)", call, name);
    return SAME_LDA_OK;
}

int check_tokens(const char* call, const void* tokens, int32_t token_bytes, int64_t n)
{
    if (token_bytes != 4 && token_bytes != 8) return fail_without_handle(SAME_LDA_EINVAL, "%s: tokens have %d bytes, not 4 or 8", call, token_bytes);
    if ((uintptr_t)tokens % token_bytes) return fail_without_handle(SAME_LDA_EINVAL, "%s: tokens are not aligned to their size", call);
    if (n < 0 || n >= (int64_t)1 << 31) return fail_without_handle(SAME_LDA_EINVAL, "%s: %lld tokens, not in [0, 2^31)", call, (long long)n);
    return SAME_LDA_OK;
}

int launched(const char* call)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SAME_LDA_OK : fail_without_handle(SAME_LDA_EHIP, "%s: %s", call, hipGetErrorString(e));
}

// Whether chunks of v elements of every row are aligned to their size (16 bytes at most).
bool chunks_fit(const same_lda_rows* m, int v)
{
    if (m->type == SAME_LDA_MICRO) return true;
    const int64_t bytes = (int64_t)v * element_bytes(m->type);
    const int64_t align = bytes < 16 ? bytes : 16;
    return m->width % v == 0 && (uintptr_t)m->data % align == 0 && (m->rows < 2 || m->stride * element_bytes(m->type) % align == 0);
}

// Lanes that share a row of so many chunks: the power of two from 1 to 64 that leaves the fewest idle.
int lanes_log2_for(int64_t chunks)
{
    int l = 0;
    while (l < 6 && ((int64_t)1 << l) < chunks) ++l;
    return l;
}

int64_t at_most(int64_t n, int64_t most) { return n < most ? n : most; }

constexpr int64_t kComputeUnits = 256;
constexpr int64_t kMaxGroups = (int64_t)1 << 22;     // workgroups of a launch (256 threads each: below 2^32 threads)

template <class TI, class TO, int V>
int embed_launch(const char* call, same::EmbedArgs& a, int32_t width, hipStream_t st)
{
    a.chunks = width / V;
    a.lanes_log2 = lanes_log2_for(a.chunks);
    const int64_t per = (int64_t)256 >> a.lanes_log2;
    const int64_t groups = at_most(a.n > 2 * per * kComputeUnits ? (a.n + 2 * per - 1) / (2 * per) : (a.n + per - 1) / per, kMaxGroups);   // two tokens in turn where they are many
    hipLaunchKernelGGL((same::embed_kernel<TI, TO, V>), dim3((unsigned)groups), dim3(256), 0, st, a);
    return launched(call);
}

// The widest chunks that both sides are aligned for: 16 bytes of the narrower type, two elements, or one.
template <class TI, class TO>
int embed_by_width(const char* call, same::EmbedArgs& a, const same_lda_rows* table, const same_lda_rows* out, hipStream_t st)
{
    constexpr int kWide = sizeof(TI) == 4 && sizeof(TO) == 4 ? 4 : 8;
    if (out->width % kWide == 0 && chunks_fit(table, kWide) && chunks_fit(out, kWide)) return embed_launch<TI, TO, kWide>(call, a, out->width, st);
    if (out->width % 2 == 0 && chunks_fit(table, 2) && chunks_fit(out, 2)) return embed_launch<TI, TO, 2>(call, a, out->width, st);
    return embed_launch<TI, TO, 1>(call, a, out->width, st);
}

template <class TI>
int embed_to(const char* call, same::EmbedArgs& a, const same_lda_rows* table, const same_lda_rows* out, hipStream_t st)
{
    switch (out->type) {
        case SAME_LDA_FLOAT:  return embed_by_width<TI, float>(call, a, table, out, st);
        case SAME_LDA_BFLOAT: return embed_by_width<TI, __bf16>(call, a, table, out, st);
        default:              return embed_by_width<TI, _Float16>(call, a, table, out, st);
    }
}

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
constexpr int kFewerTokens = 8192;
constexpr int64_t kScannedWords = 1 << 18;
bool few_tokens(int64_t n, int64_t rows, const same_lda_rows* grad)
{
    const int64_t row_bytes = (int64_t)grad->width * element_bytes(grad->type);
    const bool more = row_bytes <= 2048 && (rows <= kScannedWords || row_bytes > 512);
    return n <= (more ? same::kFewTokens : kFewerTokens) && (rows + 256) * ((grad->width + 63) / 64) < (int64_t)1 << 30;
}

GradSpace grad_space(const same_lda_rows* grad, int64_t rows)
{
    const int64_t n = grad->rows, width = grad->width;
    GradSpace s = {};
    if (n == 0 || few_tokens(n, rows, grad)) return s;
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

template <class TI, class TO, int V>
int grad_launch(same::GradArgs& a, hipStream_t st)
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
        const int64_t units = ((a.rows - 1) >> a.unit_log2) + 1, most_units = same::kFewWords >> a.unit_log2;
        int64_t workgroups = at_most((a.rows + groups - 1) / groups, 2 * kComputeUnits / across > 1 ? 2 * kComputeUnits / across : 1);
        workgroups = workgroups < (units + most_units - 1) / most_units ? (units + most_units - 1) / most_units : workgroups;
        a.words = (int32_t)((units + workgroups - 1) / workgroups << a.unit_log2);
        if (a.n <= kFewerTokens) hipLaunchKernelGGL((same::embed_grad_few_kernel<TI, TO, V, kFewerTokens / 1024>), dim3((unsigned)workgroups, across), dim3(1024), 0, st, a);
        else                     hipLaunchKernelGGL((same::embed_grad_few_kernel<TI, TO, V, same::kFewTokens / 1024>), dim3((unsigned)workgroups, across), dim3(1024), 0, st, a);
        return launched("embed_grad");
    }
    const dim3 grid((unsigned)at_most((a.ranges + a.rows + per - 1) / per, most), across);
    if (a.lanes_log2 < 4) hipLaunchKernelGGL((same::embed_grad_kernel<TI, TO, V, true>), grid, dim3(256), 0, st, a);
    else                  hipLaunchKernelGGL((same::embed_grad_kernel<TI, TO, V, false>), grid, dim3(256), 0, st, a);
    if (a.lanes_log2 > same::kJoinLanesLog2) a.lanes_log2 = same::kJoinLanesLog2;
    const int64_t items = (int64_t)1024 >> a.lanes_log2;             // ranges of a workgroup
    const unsigned columns = (unsigned)((a.chunks + (1 << a.lanes_log2) - 1) >> a.lanes_log2), deep = (columns + 65534) / 65535;   // 65,535 of them side by side
    hipLaunchKernelGGL((same::embed_grad_join_kernel<TO, V>), dim3((unsigned)((a.ranges + items - 1) / items), (columns + deep - 1) / deep, deep), dim3(1024), 0, st, a);
    return launched("embed_grad");
}

template <class TI, class TO>
int grad_by_width(same::GradArgs& a, const same_lda_rows* grad, const same_lda_rows* out, hipStream_t st)
{
    constexpr int kWide = sizeof(TI) == 4 && sizeof(TO) == 4 ? 4 : 8;
    if (chunks_fit(grad, kWide) && chunks_fit(out, kWide)) return grad_launch<TI, TO, kWide>(a, st);
    if (chunks_fit(grad, 2) && chunks_fit(out, 2)) return grad_launch<TI, TO, 2>(a, st);
    return grad_launch<TI, TO, 1>(a, st);
}

template <class TI>
int grad_to(same::GradArgs& a, const same_lda_rows* grad, const same_lda_rows* out, hipStream_t st)
{
    switch (out->type) {
        case SAME_LDA_FLOAT:  return grad_by_width<TI, float>(a, grad, out, st);
        case SAME_LDA_BFLOAT: return grad_by_width<TI, __bf16>(a, grad, out, st);
        default:              return grad_by_width<TI, _Float16>(a, grad, out, st);
    }
}

int check_grad(const same_lda_rows* grad, const same_lda_rows* table_grad)
{
    int rc = check_rows("embed_grad", "grad", grad, 0);
    if (!rc) rc = check_rows("embed_grad", "table_grad", table_grad, 0);
    if (!rc && grad->width != table_grad->width)
        rc = fail_without_handle(SAME_LDA_EINVAL, "embed_grad: rows of %d and of %d elements", grad->width, table_grad->width);
    return rc;
}

template <class TO, int FM, int FN, int WM, int WN, int kStages, int kScaleGroups>
void product_tiles(same::ProductArgs& p, hipStream_t st)
{
    p.tiles_a = (p.rows_a + 32 * FM * WM - 1) / (32 * FM * WM);
    p.tiles_b = (p.rows_b + 32 * FN * WN - 1) / (32 * FN * WN);
    hipLaunchKernelGGL((same::micro_product_kernel<TO, FM, FN, WM, WN, kStages, kScaleGroups>), dim3((unsigned)(p.tiles_a * p.tiles_b)), dim3(64 * WM * WN), 0, st, p);
}

template <class TO, int MF, int RF, int KW, class TI>
void product_few(same::ProductArgs& p, hipStream_t st)
{
    p.tiles_b = (p.rows_b + 16 * RF - 1) / (16 * RF);
    hipLaunchKernelGGL((same::micro_product_few_kernel<TO, MF, RF, KW, TI>), dim3((unsigned)at_most((p.tiles_b + 4 / KW - 1) / (4 / KW), kMaxGroups)), dim3(256), 0, st, p);
}

// Of rows of ten groups and more the four waves of a workgroup take a part each (1 x 60,000 x 1280: whole rows per wave 9.7 us, a quarter
// 10.7; 16 rows 13.5, 11.9; 16 x 20,000 7.7, 6.4; with eight and nine groups a part is too short: 1 x 100,000 x 1024 11.8, 17;
// 16 x 60,000 x 1152 8.7, 9.9; up to 4096 rows it is the shorter wait all the same, 17 x 3000 x 1024 4.1, 4.8).  16 rows of the
// table per wave, or 64 where that still leaves 512 workgroups (16 x 50,000 x 4096: 27, with 16 rows 32; 16 x 20,000 x 4096: with 16
// rows 14.5, 15.3; a single row would do better with 16 everywhere, 1 x 50,000 x 4096 21, 25).
template <class TO, int MF, class TI = void>
void product_few_by_shape(same::ProductArgs& p, hipStream_t st)
{
    if (p.groups < (p.rows_b > 4096 ? 10 : 8)) product_few<TO, MF, 1, 1, TI>(p, st);
    else if (p.rows_b < 64 * 512)              product_few<TO, MF, 1, 4, TI>(p, st);
    else                                       product_few<TO, MF, 4, 4, TI>(p, st);
}

// Rows of numbers, rounded in the call: one launch in place of two (32 x 2000 x 256: 7.2 us, 15.1, as calls).  Beyond 16 rows they are short, and not
// shared out.
template <class TO, class TI>
void product_rounded(same::ProductArgs& p, hipStream_t st)
{
    if (p.rows_a <= 16)      product_few_by_shape<TO, 1, TI>(p, st);
    else if (p.rows_a <= 32) product_few<TO, 2, 1, 1, TI>(p, st);
    else                     product_few<TO, 4, 1, 1, TI>(p, st);
}

// Which kernel (us at rows of a x rows of b x width, the first number the chosen one's):
//   up to 16 rows of a          straight from memory; above, tiles, but up to 32 rows of a by a table of up to 8192 longer rows (17 x 8000 x
//                               4096: 8.2, tiles 10.6; 32 x 8000 x 4096: 9.8, 10.5; 32 x 12,000 x 4096: tiles 11.0, 13.5; 32 x 20,000 x
//                               1024: tiles 6.3, 10.1; 32 x 100,000 x 256: tiles 7.0, 10.1), 16,384 of four groups (17 x 12,000 x 512:
//                               4.0, 4.8; 32 x 20,000 x 512: tiles 5.1, 5.8), or any number of three, for which there are only tiles
//                               of 128 rows (17 x 180,000 x 384: 13, 27)
//   rows of one or two groups   a single stage, four workgroups per compute unit; tiles of 64 x 64 where those of 128 x 128 are few (here
//                               of 64, then of 128: 100 x 131,072 x 256 13, 16; 2048 x 28,672 x 256, at 3584, 39, 40; 128 x 524,288 x 256,
//                               at 4096, 79, 73; to 16 bits, where rows of 64 are half as long: at 1536 2000 x 12,288 x 256 16, 17 and 2048 x
//                               12,288 x 256 14, 13; at 2048 100 x 262,144 x 256 19, 23 and 2048 x 16,384 x 256 18, 15; at 4096 2000 x
//                               32,768 x 256 33, 30: full tiles of 128 would pay from half as many on)
//   256 x 256                   from 256 such tiles on (4096 x 16,384 x 1024: 58, tiles of 128 85; 2048 x 4096 x 4096, 128 tiles: 33,
//                               tiles of 128 27) for more than 640 rows of a (16-bit sums, 700 x 100,000 x 1024: 70, 80; 600 x 70,000 x
//                               1024: tiles of 128 47, 56; 17 x 70,000 x 4096: 72, of 64 32) of eight groups and more (4096 x 8192 x 1024
//                               30, 34; of seven the same, of four 22, 24)
//   64 x 64                     up to 64 rows of a, and up to 160 tiles of 128 x 128 (512 x 4096 x 4096: 13.9, 16.5; 1024 x 4096 x 4096: 27, 18;
//                               64 x 70,000 x 4096: 31, 45; 64 x 600,000 x 128, a single stage: 20, 35)
constexpr int64_t kRowsAtOnce = (int64_t)1 << 28;

template <class TO>
void product_to(same::ProductArgs& p, int32_t type_a, hipStream_t st)
{
    switch (type_a) {
        case SAME_LDA_FLOAT:  return product_rounded<TO, float>(p, st);
        case SAME_LDA_BFLOAT: return product_rounded<TO, __bf16>(p, st);
        case SAME_LDA_HALF:   return product_rounded<TO, _Float16>(p, st);
    }
    if (p.rows_a <= 16) return product_few_by_shape<TO, 1>(p, st);
    if (p.rows_a <= 32 && (p.groups == 3 || (p.groups > 3 && p.rows_b <= (p.groups == 4 ? 16384 : 8192)))) return product_few_by_shape<TO, 2>(p, st);
    const int64_t tiles = ((p.rows_a + 127) / 128) * ((p.rows_b + 127) / 128);
    const int64_t large = ((p.rows_a + 255) / 256) * ((p.rows_b + 255) / 256);
    if (p.groups <= 2) {
        if (p.rows_a <= 64 || tiles <= (sizeof(TO) == 4 ? 4096 : 2048)) product_tiles<TO, 1, 1, 2, 2, 1, 2>(p, st);
        else product_tiles<TO, 2, 2, 2, 2, 1, 2>(p, st);
    } else if (p.groups == 3) {
        product_tiles<TO, 2, 2, 2, 2, 2, 2>(p, st);
    } else if (p.rows_a > 640 && large >= 256 && p.groups >= 8) {
        product_tiles<TO, 4, 2, 2, 4, 2, 4>(p, st);
    } else if (p.rows_a <= 64 || tiles <= 160) {
        product_tiles<TO, 1, 1, 2, 2, 2, 8>(p, st);
    } else {
        product_tiles<TO, 2, 2, 2, 2, 2, 4>(p, st);
    }
}

}  // namespace

extern "C" {

int same_lda_embed(const same_lda_rows* table, const void* tokens, int32_t token_bytes, float scale, const same_lda_rows* out, void* hip_stream)
{
    int rc = check_rows("embed", "table", table, -1);
    if (!rc) rc = check_rows("embed", "out", out, 0);
    if (!rc) rc = check_tokens("embed", tokens, token_bytes, out->rows);
    if (rc) return rc;
    if (table->width != out->width) return fail_without_handle(SAME_LDA_EINVAL, "embed: rows of %d and of %d elements", table->width, out->width);
    if (!tokens && out->rows != table->rows)
        return fail_without_handle(SAME_LDA_EINVAL, "embed: without tokens all %lld rows are written, not %lld", (long long)table->rows, (long long)out->rows);
    if (!std::isfinite(scale)) return fail_without_handle(SAME_LDA_EINVAL, "embed: the scale must be finite");
    if (out->rows == 0) return SAME_LDA_OK;
    const bool micro = table->type == SAME_LDA_MICRO;
    same::EmbedArgs a = {table->data, table->scales, table->rows, micro ? same::micro_code_pitch(table->width) : table->stride, {tokens, token_bytes == 8},
                         out->rows, scale, out->data, out->stride, 0, 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    switch (table->type) {
        case SAME_LDA_FLOAT:  return embed_to<float>("embed", a, table, out, st);
        case SAME_LDA_BFLOAT: return embed_to<__bf16>("embed", a, table, out, st);
        case SAME_LDA_HALF:   return embed_to<_Float16>("embed", a, table, out, st);
        default:              return embed_to<uint8_t>("embed", a, table, out, st);
    }
}

int same_lda_embed_grad_workspace(const same_lda_rows* grad, const same_lda_rows* table_grad, size_t* bytes)
{
    if (!bytes) return fail_without_handle(SAME_LDA_EINVAL, "embed_grad: bytes is null");
    const int rc = check_grad(grad, table_grad);
    if (rc) return rc;
    *bytes = grad_space(grad, table_grad->rows).bytes;
    return SAME_LDA_OK;
}

int same_lda_embed_grad(const same_lda_rows* grad, const void* tokens, int32_t token_bytes, float scale, int32_t accumulate,
                        const same_lda_rows* table_grad, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_grad(grad, table_grad);
    if (!rc) rc = check_tokens("embed_grad", tokens, token_bytes, grad->rows);
    if (rc) return rc;
    if (!tokens && grad->rows > 0) return fail_without_handle(SAME_LDA_EINVAL, "embed_grad: tokens is null");
    if (!std::isfinite(scale)) return fail_without_handle(SAME_LDA_EINVAL, "embed_grad: the scale must be finite");
    const int64_t n = grad->rows, rows = table_grad->rows;
    const GradSpace s = grad_space(grad, rows);
    if (rows == 0 || (n == 0 && accumulate)) return SAME_LDA_OK;
    if (s.bytes > 0 && (!workspace || workspace_bytes < s.bytes || (uintptr_t)workspace % 16))
        return fail_without_handle(SAME_LDA_EINVAL, "embed_grad: needs %zu bytes of workspace aligned to 16 (got %zu)", s.bytes, workspace ? workspace_bytes : (size_t)0);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (n == 0) {                                                    // a table of zeros: the lookup of rows that no table holds
        const same_lda_rows none = {nullptr, nullptr, 0, 0, table_grad->width, SAME_LDA_FLOAT};
        same::EmbedArgs zeros = {nullptr, nullptr, 0, 0, {nullptr, 0}, rows, 1.0f, table_grad->data, table_grad->stride, 0, 0};
        return embed_to<float>("embed_grad", zeros, &none, table_grad, st);
    }
    char* const w = static_cast<char*>(workspace);
    same::GradArgs a = {grad->data, grad->stride, nullptr, nullptr, rows, scale, accumulate, table_grad->data, table_grad->stride,
                        nullptr, s.ranges, grad->width, 0, 0, {tokens, token_bytes == 8}, (int32_t)n, 0, 0};
    if (!few_tokens(n, rows, grad)) {
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
        if ((rc = launched("embed_grad"))) return rc;
        a.start = start;
        a.partial = reinterpret_cast<float*>(w + s.partial);
    }
    switch (grad->type) {
        case SAME_LDA_FLOAT:  return grad_to<float>(a, grad, table_grad, st);
        case SAME_LDA_BFLOAT: return grad_to<__bf16>(a, grad, table_grad, st);
        default:              return grad_to<_Float16>(a, grad, table_grad, st);
    }
}

int same_lda_micro_size(int64_t rows, int32_t width, size_t* code_bytes, size_t* scale_bytes)
{
    if (!code_bytes || !scale_bytes) return fail_without_handle(SAME_LDA_EINVAL, "micro_size: code_bytes or scale_bytes is null");
    if (rows < 0 || rows >= (int64_t)1 << 31 || width < 1 || width > SAME_LDA_WIDTH_MAX)
        return fail_without_handle(SAME_LDA_EINVAL, "micro_size: bad shape %lld x %d", (long long)rows, width);
    *code_bytes = (size_t)rows * (size_t)same::micro_code_pitch(width);
    *scale_bytes = (size_t)rows * (size_t)same::micro_scale_pitch(width);
    return SAME_LDA_OK;
}

int same_lda_micro_quantize(const same_lda_rows* x, const same_lda_rows* micro_out, void* hip_stream)
{
    int rc = check_rows("micro_quantize", "x", x, 0);
    if (!rc) rc = check_rows("micro_quantize", "micro_out", micro_out, 1);
    if (rc) return rc;
    if (x->rows != micro_out->rows || x->width != micro_out->width)
        return fail_without_handle(SAME_LDA_EINVAL, "micro_quantize: %lld x %d into %lld x %d", (long long)x->rows, x->width, (long long)micro_out->rows, micro_out->width);
    if (x->rows == 0) return SAME_LDA_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const same_lda_rows whole = {x->data, nullptr, x->rows, x->stride, 8, x->type};       // alignment of rows, whatever their width
    const same::QuantizeArgs a = {x->data, x->rows, x->stride, x->width, chunks_fit(&whole, 8), static_cast<uint8_t*>(micro_out->data), micro_out->scales};
    const int64_t pieces = x->rows * same::micro_groups(x->width) * 16;
    const dim3 grid((unsigned)at_most((pieces + 255) / 256, kMaxGroups));
    switch (x->type) {
        case SAME_LDA_FLOAT:  hipLaunchKernelGGL(same::micro_quantize_kernel<float>, grid, dim3(256), 0, st, a); break;
        case SAME_LDA_BFLOAT: hipLaunchKernelGGL(same::micro_quantize_kernel<__bf16>, grid, dim3(256), 0, st, a); break;
        default:              hipLaunchKernelGGL(same::micro_quantize_kernel<_Float16>, grid, dim3(256), 0, st, a); break;
    }
    return launched("micro_quantize");
}

int same_lda_micro_product(const same_lda_rows* a, const same_lda_rows* b, float scale, const same_lda_rows* out, void* hip_stream)
{
    int rc = check_rows("micro_product", "a", a, -1);
    if (!rc) rc = check_rows("micro_product", "b", b, 1);
    if (rc) return rc;
    if (a->width != b->width) return fail_without_handle(SAME_LDA_EINVAL, "micro_product: rows of %d and of %d elements", a->width, b->width);
    if (b->rows == 0) return SAME_LDA_OK;                                                  // no columns: out is not looked at
    if ((rc = check_rows("micro_product", "out", out, 0, INT32_MAX))) return rc;
    if (out->rows != a->rows || out->width != b->rows)
        return fail_without_handle(SAME_LDA_EINVAL, "micro_product: %lld rows by %lld rows do not give %lld x %d", (long long)a->rows, (long long)b->rows,
                                   (long long)out->rows, out->width);
    if (!std::isfinite(scale)) return fail_without_handle(SAME_LDA_EINVAL, "micro_product: the scale must be finite");
    if (a->type != SAME_LDA_MICRO && (a->rows > SAME_LDA_ROUND_ROWS || a->rows * a->width > SAME_LDA_ROUND_MAX))
        return fail_without_handle(SAME_LDA_EINVAL, "micro_product: a must be microscaled beyond %d rows or %d elements (got %lld x %d)", SAME_LDA_ROUND_ROWS,
                                   SAME_LDA_ROUND_MAX, (long long)a->rows, a->width);
    static_assert(SAME_LDA_ROUND_MAX == same::kRoundMost && SAME_LDA_ROUND_ROWS == same::kRoundRows, "");
    if (a->rows == 0) return SAME_LDA_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const same_lda_rows whole = {a->data, nullptr, a->rows, a->stride, 8, a->type};                                      // alignment of rows, whatever their width
    const same_lda_rows strip = {out->data, nullptr, out->rows, out->stride, 16 / element_bytes(out->type), out->type};
    const int64_t pitch_a = a->type == SAME_LDA_MICRO ? same::micro_code_pitch(a->width) : 0, pitch_b = same::micro_code_pitch(b->width);
    // at most 2^28 rows of either operand in a launch: grids stay below 2^32 threads (the output's size bounds the tiles)
    for (int64_t i = 0; i < a->rows; i += kRowsAtOnce)
        for (int64_t j = 0; j < b->rows; j += kRowsAtOnce) {
            same::ProductArgs p = {};
            p.a = static_cast<const uint8_t*>(a->data) + i * pitch_a;                                                    // (a matrix of numbers: i = 0)
            p.a_scales = a->scales + i * (pitch_a / 16);
            p.b = static_cast<const uint8_t*>(b->data) + j * pitch_b;
            p.b_scales = b->scales + j * (pitch_b / 16);
            p.rows_a = at_most(a->rows - i, kRowsAtOnce);
            p.rows_b = at_most(b->rows - j, kRowsAtOnce);
            p.groups = (int32_t)same::micro_groups(a->width);
            p.scale = scale;
            p.out = static_cast<char*>(out->data) + (i * out->stride + j) * element_bytes(out->type);
            p.out_stride = out->stride;
            p.wide = chunks_fit(&strip, strip.width);
            p.stride_a = a->stride;
            p.width = a->width;
            p.wide_a = chunks_fit(&whole, 8);
            switch (out->type) {
                case SAME_LDA_FLOAT:  product_to<float>(p, a->type, st); break;
                case SAME_LDA_BFLOAT: product_to<__bf16>(p, a->type, st); break;
                default:              product_to<_Float16>(p, a->type, st); break;
            }
        }
    return launched("micro_product");
}

}  // extern "C"
