// Rounding to microscaled four-bit floating point, and the product of two matrices in it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

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

// ---- Product: out[i][j] = scale * sum_k a[i][k] b[j][k], both in four bits.  One 16x16x128 matrix instruction takes from
// lane l the 32 elements and the scale of block l / 16 of row l % 16 of a group of 128, and adds in binary32.
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
    int64_t tiles_b, tiles;  // tiles along the rows of b, all tiles
};

__device__ __forceinline__ v8i fragment(const uint8_t* p)
{
    const v4i x = *reinterpret_cast<const v4i*>(p);
    return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1);
}

template <class TO>
__global__ __launch_bounds__(256) void micro_product_kernel(ProductArgs p)
{
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int64_t pitch = (int64_t)p.groups * 64, spitch = (int64_t)p.groups * 4;
    for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const int64_t i0 = tile / p.tiles_b * 64 + wv * 16, j0 = tile % p.tiles_b * 64;
        const int64_t ra = i0 + r < p.rows_a ? i0 + r : p.rows_a - 1;          // rows behind the last are computed from it and not written
        const uint8_t* const fa = p.a + ra * pitch + g * 16;
        const uint8_t* const sa = p.a_scales + ra * spitch + g;
        const uint8_t* fb[4];
        const uint8_t* sb[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t rb = j0 + 16 * c + r < p.rows_b ? j0 + 16 * c + r : p.rows_b - 1;
            fb[c] = p.b + rb * pitch + g * 16;
            sb[c] = p.b_scales + rb * spitch + g;
        }
        v4f acc[4] = {};
        for (int k = 0; k < p.groups; ++k) {
            const v8i xa = fragment(fa + (int64_t)k * 64);
            const int ea = sa[k * 4];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                acc[c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(xa, fragment(fb[c] + (int64_t)k * 64), acc[c], kFormatE2M1, kFormatE2M1, 0, ea,
                                                                          0, sb[c][k * 4]);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t i = i0 + 4 * g + v, j = j0 + 16 * c + r;
                if (i < p.rows_a && j < p.rows_b) static_cast<TO*>(p.out)[i * p.out_stride + j] = (TO)(p.scale * acc[c][v]);
            }
    }
}

}  // namespace same
