// Host side of grouped four-bit integers: argument checks and launches.  As the other word-table operators: no handle, no device memory
// of its own, nothing that waits.
#include <hip/hip_runtime.h>

#include <cmath>

#include "group_kernels.h"
#include "operands.h"

using namespace same::host;
using same::fail_without_handle;

namespace {

// Rows of either operand in a launch: grids stay below 2^32 threads (the output's size bounds the tiles), and what rows of a are laid down in
// below 256 MB or 4096 rows.
constexpr int64_t kRowsOfB = (int64_t)1 << 28;
int64_t filled_blocks(int64_t width) { return (same::micro_groups(width) + 3) / 4 * 4; }     // for up to four waves that share a row
int64_t rows_of_a(const same_lda_rows* a)
{
    const int64_t most = ((int64_t)1 << 28) / (filled_blocks(a->width) * 128 * (a->type == SAME_LDA_FLOAT ? 6 : 2)) / 128 * 128;
    return most < 4096 ? 4096 : most > ((int64_t)1 << 24) ? (int64_t)1 << 24 : most;
}


// One launch of the kernel that keeps 16 rows of a in registers, or two in tiles: there up to 16 rows, and more while they and the rows of b make no
// more than so many products of 16 x 16 x 128, for which the table is read again for every 16 (us in one and in two, bf16: 64 x 1000 x 1000 3.9,
// 9.2; 32 x 4096 x 4096 11.5, 16.0; 512 x 2000 x 500 9.7, 10.0; 64 x 30,000 x 256 9.3, 8.5; 64 x 4096 x 4096 15.9, 16.5; 512 x 4000 x 300 14.5, 9.3;
// 100 x 8000 x 2000 30, 17; and the second launch and its workspace cost the host 4 to 5).
constexpr int64_t kFewProducts = 16384;
bool few_rows(const same_lda_rows* a, const same_lda_rows* b)
{
    const int64_t blocks = same::micro_groups(a->width);
    return blocks <= 32 && (a->rows <= 16 || (a->rows + 15) / 16 * ((b->rows + 15) / 16) * blocks <= kFewProducts);
}

// Workspace of the rows of a, laid down for tiles of up to 128 rows, of their sums and, in binary32, of the inverses of their powers of two.
struct RowsSpace {
    size_t operands, sums, bytes;
};

RowsSpace rows_space(const same_lda_rows* a, const same_lda_rows* b)
{
    if (few_rows(a, b)) return {0, 0, 0};
    const size_t tiles = (size_t)((at_most(a->rows, rows_of_a(a)) + 127) / 128 * 8), filled = (size_t)filled_blocks(a->width);
    const size_t operands = tiles * filled * 4 * (a->type == SAME_LDA_FLOAT ? 3 : 1) * 1024;
    const size_t sums = tiles * filled * 4 * 16 * sizeof(float);
    return {operands, sums, operands + sums + (a->type == SAME_LDA_FLOAT ? tiles * 16 * sizeof(float) : 0)};
}

// Where rows of a are laid down.
struct Laid {
    same::v4u32* operands;
    float *sums, *inverse;
};

template <class TI, int P, bool kStack, int kGroupLog2, int KB>
void product_few(same::GroupProductArgs& p, int blocks, hipStream_t st)
{
    int kw = 1;
    while (kw * KB < blocks) kw *= 2;                                    // at most 8
    p.waves_per_row = kw;
    const int waves = kw < 4 ? 4 : kw, streams = waves / kw;
    const int64_t turns = ((p.rows_b + 15) / 16 + streams - 1) / streams;
    const int64_t across = (p.rows_a + 15) / 16, most = (kComputeUnits * 8 / waves + across - 1) / across;
    hipLaunchKernelGGL((same::group_product_few_kernel<TI, P, kStack, kGroupLog2, KB>), dim3((unsigned)at_most(turns, most), (unsigned)across), dim3(64 * waves), 0, st, p);
}

// Up to two blocks of a row in a wave while eight waves hold the row (us with 1, 2 and 4 of them: 1 x 100,000 x 128 bf16 4.8, 6.5, 10.1;
// x 256 7.7, 6.3, 9.6; x 1024 19.3, 16.5, 18.5; 16 x 50,021 x 2048 f32 22.7, 22.8, 35.5).  Two waves per SIMD: with three or four of these
// 1 x 50,021 x 2048 bf16 takes 21 and 18 us for 16, its rows of a being fetched by more workgroups.
template <class TI, int P, bool kStack, int kGroupLog2>
void product_few_by_width(same::GroupProductArgs& p, int blocks, hipStream_t st)
{
    if (blocks == 1) product_few<TI, P, kStack, kGroupLog2, 1>(p, blocks, st);
    else if (blocks <= 16) product_few<TI, P, kStack, kGroupLog2, 2>(p, blocks, st);
    else product_few<TI, P, kStack, kGroupLog2, 4>(p, blocks, st);
}

template <class TI, int kGroupLog2, int MT, int NT, int WM, int WN, int WK, int kStages>
void product_tiles(const same::GroupProductArgs& p, const Laid& to, hipStream_t st)
{
    constexpr int P = sizeof(TI) == 4 ? 3 : 1, kTall = 16 * MT * WM, kWide = 16 * NT * WN;
    static_assert(WK <= 4 && kTall <= 128, "the workspace is for these");
    constexpr int kFit = kStages * sizeof(same::GroupStage<P, kGroupLog2, MT, NT, WM, WN, WK>) <= 163840 ? kStages : kStages - 1;
    const int blocks = (p.width + 127) / 128, filled = (blocks + WK - 1) / WK * WK;
    const int64_t tiles_a = (p.rows_a + kTall - 1) / kTall, tiles_b = ((p.rows_b + kWide - 1) / kWide + 7) / 8 * 8;
    const same::GroupRowsArgs rows = {p.a, p.rows_a, p.stride_a, p.width, blocks, filled, to.operands, to.sums, to.inverse};
    const unsigned sixteens = (unsigned)(tiles_a * MT * WM);
    bool whole = false;
    if constexpr (P == 3) {
        if ((whole = filled <= same::kWholeBlocks))
            hipLaunchKernelGGL((same::group_rows_kernel<TI, kGroupLog2, true>), dim3(sixteens), dim3((unsigned)(64 * filled)), 0, st, rows);
        else
            hipLaunchKernelGGL(same::group_row_powers_kernel, dim3(16 * sixteens), dim3(256), 0, st, rows);
    }
    if (!whole) hipLaunchKernelGGL((same::group_rows_kernel<TI, kGroupLog2, false>), dim3(sixteens, (unsigned)at_most((filled + 3) / 4, 65535)), dim3(256), 0, st, rows);
    const same::GroupTilesArgs tiles = {p, to.operands, to.sums, to.inverse, blocks, filled};
    hipLaunchKernelGGL((same::group_product_kernel<same::kHalfMatrix<TI>, P, kGroupLog2, MT, NT, WM, WN, WK, kFit>), dim3((unsigned)(tiles_a * tiles_b)), dim3(64 * WM * WN * WK), 0, st,
                       tiles);
}

template <class TI, int kGroupLog2>
void product_launch(same::GroupProductArgs& p, bool few, const Laid& to, hipStream_t st)
{
    const int blocks = (p.width + 127) / 128;
    if (few) {
        if constexpr (sizeof(TI) == 4) return p.rows_a <= 4 ? product_few_by_width<TI, 1, true, kGroupLog2>(p, blocks, st) : product_few_by_width<TI, 3, false, kGroupLog2>(p, blocks, st);
        else return product_few_by_width<TI, 1, false, kGroupLog2>(p, blocks, st);
    }
    // Tiles are as large as still gives every compute unit some, and where there are many those whose last round is the fuller one: by the
    // workgroups that run at once (LDS bounds them), and what a round takes to that of the next form.  us of the two launches, G128, by form:
    //   bf16                 64x256  64x128  64x64  32x128  32x64  16x128      binary32 (*)         64x256  32x128  32x64  16x64
    //   512 x 50,021 x 4096     250     268    446     409    643     716      512 x 50,021 x 4096     615     648   1251   1739
    //   2048 x 8192 x 4096      166     190    359     270    434     446      2048 x 8192 x 4096      389     467    959   1028
    //   64 x 50,021 x 1024       22      19     33      26     45      36      64 x 50,021 x 1024       32      35     57     76
    //   256 x 8000 x 1000        17      14     18      16     27      22      256 x 20,000 x 2000      93      80    128    176
    //   128 x 8192 x 8192        91      63     40      45     52      68      128 x 8192 x 8192       162      72     94    118
    //   32 x 50,021 x 4096       54      54     76      50     60      73      512 x 1000 x 4000        87      40     33     44
    //   32 x 4096 x 4096         43      30     21      21     16      19      40 x 10,000 x 2000       45      21     27     21
    //   1 x 20,000 x 8192        90      64     70      46     53      43      32 x 4096 x 4096         81      34     25     19
    // (*) without the search for the rows' powers of two, which adds the same to every form: about 1 us up to 1024 elements, beyond 2 to 3, a launch
    const auto tiles = [&](int64_t tall, int64_t wide) { return ((p.rows_a + tall - 1) / tall) * ((p.rows_b + wide - 1) / wide); };
    const auto rounds = [&](int64_t tall, int64_t wide, int64_t per_unit) { return (tiles(tall, wide) + per_unit * kComputeUnits - 1) / (per_unit * kComputeUnits); };
    if constexpr (sizeof(TI) == 4) {
        if (p.rows_a > 32 && 17 * rounds(64, 256, 1) <= 10 * rounds(32, 128, 2)) product_tiles<TI, kGroupLog2, 2, 4, 2, 4, 1, 2>(p, to, st);
        else if (p.rows_a > 16 && tiles(32, 64) > kComputeUnits)     product_tiles<TI, kGroupLog2, 2, 2, 1, 4, 1, 2>(p, to, st);
        else if (p.rows_a > 16 && tiles(32, 64) > kComputeUnits / 2) product_tiles<TI, kGroupLog2, 2, 2, 1, 2, 2, 2>(p, to, st);
        else                                                         product_tiles<TI, kGroupLog2, 1, 2, 1, 2, 4, 2>(p, to, st);
    } else {
        if (p.rows_a > 32 && 5 * rounds(64, 256, 2) <= 4 * rounds(64, 128, 3)) product_tiles<TI, kGroupLog2, 4, 4, 1, 4, 1, 2>(p, to, st);
        else if (p.rows_a > 32 && tiles(64, 64) > kComputeUnits)     product_tiles<TI, kGroupLog2, 4, 2, 1, 4, 1, 2>(p, to, st);
        else if (p.rows_a > 32 && tiles(64, 64) > kComputeUnits / 2) product_tiles<TI, kGroupLog2, 4, 2, 1, 2, 2, 3>(p, to, st);
        else if (p.rows_a > 16 && tiles(32, 64) > kComputeUnits)     product_tiles<TI, kGroupLog2, 2, 2, 1, 4, 1, 4>(p, to, st);
        else if (p.rows_a > 16)                                      product_tiles<TI, kGroupLog2, 2, 2, 1, 2, 4, 3>(p, to, st);
        else                                                         product_tiles<TI, kGroupLog2, 1, 2, 1, 4, 1, 4>(p, to, st);
    }
}

template <class TI>
void product_to(same::GroupProductArgs& p, int group_log2, bool few, const Laid& to, hipStream_t st)
{
    switch (group_log2) {
        case 5:  return product_launch<TI, 5>(p, few, to, st);
        case 6:  return product_launch<TI, 6>(p, few, to, st);
        default: return product_launch<TI, 7>(p, few, to, st);
    }
}

int check_product(const same_lda_rows* a, const same_lda_rows* b)
{
    int rc = check_rows("group_product", "a", a, kNumbers);
    if (!rc) rc = check_rows("group_product", "b", b, kGrouped);
    if (!rc && a->width != b->width) rc = fail_without_handle(SAME_LDA_EINVAL, "group_product: rows of %d and of %d elements", a->width, b->width);
    return rc;
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
    const int32_t chunks = (int32_t)same::micro_groups(x->width) * 16;
    const int64_t groups = at_most((x->rows * chunks + same::kRoundedAtOnce - 1) / same::kRoundedAtOnce, kComputeUnits * 64), step = groups * same::kRoundedAtOnce;
    const same::GroupQuantizeArgs a = {x->data, x->rows, x->stride, x->width, __builtin_ctz((unsigned)group_out->type), static_cast<uint32_t*>(group_out->data),
                                       reinterpret_cast<uint32_t*>(group_out->scales), chunks, 1.0f / (float)chunks, (int32_t)(step / chunks), (int32_t)(step % chunks)};
    const dim3 grid((unsigned)groups);
    switch (x->type) {
        case SAME_LDA_FLOAT:  hipLaunchKernelGGL(same::group_quantize_kernel<float>, grid, dim3(256), 0, st, a); break;
        case SAME_LDA_BFLOAT: hipLaunchKernelGGL(same::group_quantize_kernel<__bf16>, grid, dim3(256), 0, st, a); break;
        default:              hipLaunchKernelGGL(same::group_quantize_kernel<_Float16>, grid, dim3(256), 0, st, a); break;
    }
    return launched("group_quantize");
}

int same_lda_group_product_workspace(const same_lda_rows* a, const same_lda_rows* b, size_t* bytes)
{
    if (!bytes) return fail_without_handle(SAME_LDA_EINVAL, "group_product: bytes is null");
    const int rc = check_product(a, b);
    if (rc) return rc;
    *bytes = a->rows > 0 && b->rows > 0 ? rows_space(a, b).bytes : 0;
    return SAME_LDA_OK;
}

int same_lda_group_product(const same_lda_rows* a, const same_lda_rows* b, float scale, const same_lda_rows* out, void* workspace, size_t workspace_bytes,
                           void* hip_stream)
{
    int rc = check_product(a, b);
    if (rc) return rc;
    if (b->rows == 0) return SAME_LDA_OK;                                                  // no columns: out is not looked at
    if ((rc = check_rows("group_product", "out", out, kNumbers, INT32_MAX))) return rc;
    if (out->rows != a->rows || out->width != b->rows)
        return fail_without_handle(SAME_LDA_EINVAL, "group_product: %lld rows by %lld rows do not give %lld x %d", (long long)a->rows, (long long)b->rows,
                                   (long long)out->rows, out->width);
    if (!std::isfinite(scale)) return fail_without_handle(SAME_LDA_EINVAL, "group_product: the scale must be finite");
    if (a->rows == 0) return SAME_LDA_OK;
    const RowsSpace space = rows_space(a, b);
    if (space.bytes > 0 && (!workspace || workspace_bytes < space.bytes || (uintptr_t)workspace % 16))
        return fail_without_handle(SAME_LDA_EINVAL, "group_product: needs %zu bytes of workspace aligned to 16 (got %zu)", space.bytes, workspace ? workspace_bytes : (size_t)0);
    char* const w = static_cast<char*>(workspace);
    const Laid to = {reinterpret_cast<same::v4u32*>(w), reinterpret_cast<float*>(w + space.operands), reinterpret_cast<float*>(w + space.operands + space.sums)};
    const bool few = few_rows(a, b);
    const int64_t rows_each = rows_of_a(a);
    const int group_log2 = __builtin_ctz((unsigned)b->type);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    // slices of either operand: grids stay below 2^32 threads (the output's size bounds the tiles)
    for (int64_t i = 0; i < a->rows; i += rows_each)
        for (int64_t j = 0; j < b->rows; j += kRowsOfB) {
            same::GroupProductArgs p = {};
            p.rows_a = at_most(a->rows - i, rows_each);
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
                case SAME_LDA_FLOAT:  product_to<float>(p, group_log2, few, to, st); break;
                case SAME_LDA_BFLOAT: product_to<__bf16>(p, group_log2, few, to, st); break;
                default:              product_to<_Float16>(p, group_log2, few, to, st); break;
            }
        }
    return launched("group_product");
}

}  // extern "C"
