// Host side of the word-table operators: argument checks and launches.  No handle, no device memory of its own, nothing
// that waits: every call only enqueues kernels, so all of them can be captured into a graph.
#include "../../include/same_lda.h"

#include <hip/hip_runtime.h>

#include <cmath>

#include "embed_kernels.h"
#include "micro_kernels.h"
#include "operands.h"
#include "rows_call.h"

namespace {

using namespace same::host;
using same::fail_without_handle;

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

// the lookup of rows that no table holds
int same::host::rows_of_zeros(const char* call, const same_lda_rows* out, hipStream_t st)
{
    const same_lda_rows none = {nullptr, nullptr, 0, 0, out->width, SAME_LDA_FLOAT};
    same::EmbedArgs zeros = {nullptr, nullptr, 0, 0, {nullptr, 0}, out->rows, 1.0f, out->data, out->stride, 0, 0};
    return embed_to<float>(call, zeros, &none, out, st);
}

extern "C" {

int same_lda_embed(const same_lda_rows* table, const void* tokens, int32_t token_bytes, float scale, const same_lda_rows* out, void* hip_stream)
{
    int rc = check_rows("embed", "table", table, kNumbers | kMicro | kGrouped);
    if (!rc) rc = check_rows("embed", "out", out, kNumbers);
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
        case SAME_LDA_MICRO:  return embed_to<uint8_t>("embed", a, table, out, st);
        default:              return same::host::rows_call("embed", table, tokens, token_bytes, scale, nullptr, out, hip_stream);
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
    int rc = check_rows("micro_quantize", "x", x, kNumbers);
    if (!rc) rc = check_rows("micro_quantize", "micro_out", micro_out, kMicro);
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
    int rc = check_rows("micro_product", "a", a, kNumbers | kMicro);
    if (!rc) rc = check_rows("micro_product", "b", b, kMicro);
    if (rc) return rc;
    if (a->width != b->width) return fail_without_handle(SAME_LDA_EINVAL, "micro_product: rows of %d and of %d elements", a->width, b->width);
    if (b->rows == 0) return SAME_LDA_OK;                                                  // no columns: out is not looked at
    if ((rc = check_rows("micro_product", "out", out, kNumbers, INT32_MAX))) return rc;
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
