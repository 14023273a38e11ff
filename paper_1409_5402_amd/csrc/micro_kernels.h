// Rounding to microscaled four-bit floating point, and the product of two matrices in it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "element.h"
#include "micro_format.h"

namespace same {

// ---- Rounding.  Of a block's largest magnitude top the exponent e = floor(log2 top) - 2 puts top / 2^e into [4, 8): the
// largest size is 6, so what lies above 6 is rounded down to it.  Sizes are rounded to the nearest, ties to the even
// code: in units of .5 below 2, of 1 below 4, of 2 above.  A lane takes 8 elements, four lanes a block.
struct QuantizeArgs {
    const void* x;
    int64_t rows, stride;
    int32_t width;
    int32_t wide;            // chunks of 8 are aligned
    uint8_t* codes;
    uint8_t* scales;
};

__device__ __forceinline__ uint32_t micro_code(float x, float per)
{
    const float t = fabsf(x) * per;
    const float r = t < 2.0f ? rintf(2.0f * t) : t < 4.0f ? rintf(t) + 2.0f : fminf(rintf(0.5f * t) + 4.0f, 7.0f);
    return (uint32_t)r | (__float_as_uint(x) >> 31 << 3);
}

template <class TI>
__global__ __launch_bounds__(256) void micro_quantize_kernel(QuantizeArgs a)
{
    const int64_t pieces = micro_groups(a.width) * (kMicroGroup / 8);          // of 8 elements, per row
    const int64_t all = a.rows * pieces;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {   // whole groups of four lanes
        const int64_t row = at / pieces;
        const int first = (int)(at - row * pieces) * 8;
        const TI* const from = static_cast<const TI*>(a.x) + row * a.stride + first;
        float x[8];
        if (a.wide && first + 8 <= a.width) {
            load_chunk<TI, 8>(x, from);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = first + j < a.width ? to_float(from[j]) : 0.0f;
        }
        uint32_t top = 0u;                                                     // magnitudes order like their bits, NaN above infinity
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        uint32_t q = 0u, s = 255u;
        if (top < 0x7F800000u) {
            s = top >= 0x01000000u ? (top >> 23) - 2u : 0u;                    // 127 + e, at least 0
            const float per = __uint_as_float((254u - s) << 23);               // 2^-e: s <= 252
#pragma unroll
            for (int j = 0; j < 8; ++j) q |= micro_code(x[j], per) << (4 * j);
        }
        reinterpret_cast<uint32_t*>(a.codes)[at] = q;                          // rows of codes follow each other without a gap
        if ((at & 3) == 0) a.scales[at >> 2] = (uint8_t)s;
    }
}

// ---- Product: out[i][j] = scale * sum_k a[i][k] b[j][k], both in four bits, on the scaled matrix instructions, which
// take 32 elements and their scale byte from a lane and add in binary32.
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
constexpr int kFormatE2M1 = 4;

struct ProductArgs {
    const uint8_t *a, *a_scales, *b, *b_scales;
    int64_t rows_a, rows_b;
    int32_t groups;          // of 128 elements per row
    float scale;
    void* out;
    int64_t out_stride;
    int64_t tiles_a, tiles_b;
};

__device__ __forceinline__ v8i fragment(v4i x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

// Few rows of a (at most 16): the table is read once, straight from memory into the operands of 16x16x128 instructions: lane l
// gives block l / 16 of row l % 16 of a group of 128, so four lanes read the 64 bytes of a row's group.
template <class TO>
__global__ __launch_bounds__(256) void micro_product_few_kernel(ProductArgs p)
{
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int64_t pitch = (int64_t)p.groups * 64, spitch = (int64_t)p.groups * 4;
    const int64_t ra = r < p.rows_a ? r : p.rows_a - 1;                        // rows behind the last are computed from it and not written
    const uint8_t* const fa = p.a + ra * pitch + g * 16;
    const uint8_t* const sa = p.a_scales + ra * spitch + g;
    for (int64_t tile = (int64_t)blockIdx.x * 4 + wv; tile < p.tiles_b; tile += (int64_t)gridDim.x * 4) {
        const int64_t j = tile * 16 + r, rb = j < p.rows_b ? j : p.rows_b - 1;
        const uint8_t* const fb = p.b + rb * pitch + g * 16;
        const uint8_t* const sb = p.b_scales + rb * spitch + g;
        v4f acc = {};
        int k = 0;
        for (; k + 4 <= p.groups; k += 4) {
            v4i xa[4], xb[4];
            int ea[4], eb[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                xb[q] = *reinterpret_cast<const v4i*>(fb + (int64_t)(k + q) * 64);
                eb[q] = sb[(k + q) * 4];
                xa[q] = *reinterpret_cast<const v4i*>(fa + (int64_t)(k + q) * 64);
                ea[q] = sa[(k + q) * 4];
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(xa[q]), fragment(xb[q]), acc, kFormatE2M1, kFormatE2M1, 0, ea[q], 0, eb[q]);
        }
        for (; k < p.groups; ++k)
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(*reinterpret_cast<const v4i*>(fa + (int64_t)k * 64)),
                                                                   fragment(*reinterpret_cast<const v4i*>(fb + (int64_t)k * 64)), acc, kFormatE2M1, kFormatE2M1, 0,
                                                                   sa[k * 4], 0, sb[k * 4]);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t i = 4 * g + v;
            if (i < p.rows_a && j < p.rows_b) static_cast<TO*>(p.out)[i * p.out_stride + j] = (TO)(p.scale * acc[v]);
        }
    }
}

// Many rows: a workgroup of four waves (2 x 2) computes a tile of 64 F x 64 F sums, a wave a quarter of it as F x F sums of
// 32 x 32 (32x32x64 instructions: lane l gives block l / 32 of row l % 32).  The rows' bytes come through LDS in stages of 256
// elements, 128 bytes of codes and 8 of scales per row, straight from memory, one stage ahead of the one that is multiplied.
// A row's eight blocks of 16 bytes are stored in the order block ^ ((row / 2) % 8): eight lanes write a row, and any eight
// consecutive rows that are read at one block then lie in different banks.
constexpr int kStageGroups = 2;

template <int F>
struct ProductStage {
    v4i codes[2 * 64 * F][8];
    uint32_t scales[2 * 64 * F][2];
};

// The tile of workgroup b: workgroups go to the eight dies in turn, and a die takes a run of consecutive tiles, eight tile rows
// at a time and column by column, so that what runs on a die at once shares rows of both operands in its cache.
__device__ __forceinline__ void tile_of(int64_t b, const ProductArgs& p, int64_t& ta, int64_t& tb)
{
    const int64_t all = p.tiles_a * p.tiles_b, die = b & 7, each = all >> 3, more = all & 7;
    const int64_t t = die * each + (die < more ? die : more) + (b >> 3);
    const int64_t band = t / (8 * p.tiles_b), first = band * 8, in = p.tiles_a - first < 8 ? p.tiles_a - first : 8, at = t - first * p.tiles_b;
    ta = first + at % in;
    tb = at / in;
}

template <class TO, int F>
__global__ __launch_bounds__(256, F == 4 ? 1 : 2) void micro_product_kernel(ProductArgs p)
{
    constexpr int kRows = 64 * F;                                              // of either operand in a tile
    __shared__ ProductStage<F> stage0, stage1;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t pitch = (int64_t)p.groups * 64, spitch = (int64_t)p.groups * 4;
    const int stages = (p.groups + kStageGroups - 1) / kStageGroups;
    int64_t ta, tb;
    tile_of(blockIdx.x, p, ta, tb);
    const int64_t i0 = ta * kRows, j0 = tb * kRows;
    const int last_a = (int)(p.rows_a - i0 < kRows ? p.rows_a - i0 : kRows) - 1, last_b = (int)(p.rows_b - j0 < kRows ? p.rows_b - j0 : kRows) - 1;
    const uint8_t* const base_a = p.a + i0 * pitch;
    const uint8_t* const base_b = p.b + j0 * pitch;
    const uint8_t* const sbase_a = p.a_scales + i0 * spitch;
    const uint8_t* const sbase_b = p.b_scales + j0 * spitch;

    // a wave's instruction fills 8 rows of codes or 32 rows of scales; rows behind the last are filled from it
    const int crow = wv * 8 + (lane >> 3), cblock = (lane & 7) ^ ((crow >> 1) & 7);
    const int srow = wv * 32 + (lane >> 1);
    const auto load = [&](ProductStage<F>& to, int st) {
        const int group = st * kStageGroups;
        const int c = group + (cblock >> 2) < p.groups ? cblock : cblock & 3;   // the last stage may hold one group: any bytes for the other
        const int s = group + (lane & 1) < p.groups ? lane & 1 : 0;
#pragma unroll
        for (int i = 0; i < 2 * F; ++i) {
            const int row = i * 32 + crow;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base_a + (row < last_a ? row : last_a) * pitch + group * 64 + c * 16),
                                             (__attribute__((address_space(3))) void*)&to.codes[i * 32 + wv * 8][0], 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base_b + (row < last_b ? row : last_b) * pitch + group * 64 + c * 16),
                                             (__attribute__((address_space(3))) void*)&to.codes[kRows + i * 32 + wv * 8][0], 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < (F + 1) / 2; ++i) {
            if (F % 2 && wv * 32 + i * 128 >= kRows) break;
            const int row = i * 128 + srow;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(sbase_a + (row < last_a ? row : last_a) * spitch + group * 4 + s * 4),
                                             (__attribute__((address_space(3))) void*)&to.scales[i * 128 + wv * 32][0], 4, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(sbase_b + (row < last_b ? row : last_b) * spitch + group * 4 + s * 4),
                                             (__attribute__((address_space(3))) void*)&to.scales[kRows + i * 128 + wv * 32][0], 4, 0, 0);
        }
    };

    const int r = lane & 31, half = lane >> 5;
    const int ra = (wv >> 1) * 32 * F + r, rb = kRows + (wv & 1) * 32 * F + r;   // rows of the stage that this lane multiplies (and every 32nd on)
    const int turn = (r >> 1) & 7;
    v16f acc[F][F] = {};
    const auto multiply = [&](const ProductStage<F>& from, int steps) {
        uint32_t ea[F][2], eb[F][2];                                           // bytes 0 and 2: this lane's blocks of two steps
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                ea[f][w] = from.scales[ra + 32 * f][w] >> (8 * half);
                eb[f][w] = from.scales[rb + 32 * f][w] >> (8 * half);
            }
        const auto step = [&](auto which) {
            constexpr int s = decltype(which)::value;
            v4i xa[F], xb[F];
#pragma unroll
            for (int f = 0; f < F; ++f) {
                xa[f] = from.codes[ra + 32 * f][(2 * s + half) ^ turn];
                xb[f] = from.codes[rb + 32 * f][(2 * s + half) ^ turn];
            }
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int h = 0; h < F; ++h)
                    acc[f][h] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fragment(xa[f]), fragment(xb[h]), acc[f][h], kFormatE2M1, kFormatE2M1,
                                                                                (s & 1) * 2, (int)ea[f][s >> 1], (s & 1) * 2, (int)eb[h][s >> 1]);
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        if (steps > 2) {
            step(std::integral_constant<int, 2>());
            step(std::integral_constant<int, 3>());
        }
    };

    load(stage0, 0);
    for (int st = 0; st < stages; st += 2) {
        __builtin_amdgcn_s_waitcnt(0x0f70);                                    // vmcnt(0): this wave's part of the stage has come
        __syncthreads();
        if (st + 1 < stages) load(stage1, st + 1);
        multiply(stage0, p.groups - st * kStageGroups > 1 ? 4 : 2);
        if (st + 1 >= stages) break;
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
        if (st + 2 < stages) load(stage0, st + 2);
        multiply(stage1, p.groups - (st + 1) * kStageGroups > 1 ? 4 : 2);
    }

#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int h = 0; h < F; ++h)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int64_t i = i0 + (wv >> 1) * 32 * F + 32 * f + 8 * (v >> 2) + 4 * half + (v & 3), j = j0 + (wv & 1) * 32 * F + 32 * h + r;
                if (i < p.rows_a && j < p.rows_b) static_cast<TO*>(p.out)[i * p.out_stride + j] = (TO)(p.scale * acc[f][h][v]);
            }
}

}  // namespace same
