// Microscaled four-bit floating point: a row is cut into blocks of 32 elements; an element is one of 0, .5, 1, 1.5, 2, 3, 4,
// 6 with a sign (two exponent bits, one fraction bit), two to a byte with the even element in the low half; a block has one
// byte s and stands for its elements times 2^(s - 127) (s = 255: NaN).  Rows are filled up with zero blocks to a multiple of
// 128 elements, what one matrix instruction takes, so a row of codes is a multiple of 64 bytes and one of scales of 4.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace same {

constexpr int kMicroBlock = 32;
constexpr int kMicroGroup = 128;

__host__ __device__ constexpr int64_t micro_groups(int64_t width) { return (width + kMicroGroup - 1) / kMicroGroup; }
__host__ __device__ constexpr int64_t micro_code_pitch(int64_t width) { return micro_groups(width) * (kMicroGroup / 2); }
__host__ __device__ constexpr int64_t micro_scale_pitch(int64_t width) { return micro_groups(width) * (kMicroGroup / kMicroBlock); }

// 2^(s - 127); s = 0 is a subnormal number
__device__ __forceinline__ float micro_power(uint32_t s)
{
    return __uint_as_float(s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23);
}

// elements [first, first + V) of a row; V = 8 and 2 start at multiples of V
template <int V>
__device__ __forceinline__ void load_micro(float (&x)[V], const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int first)
{
    static_assert(V == 8 || V == 2 || V == 1, "");
    typedef float v2f __attribute__((ext_vector_type(2)));
    const float power = micro_power(scales[first / kMicroBlock]);
    uint32_t q;
    if constexpr (V == 8) q = *reinterpret_cast<const uint32_t*>(codes + first / 2);
    else                  q = (uint32_t)codes[first / 2] >> (V == 1 ? 4 * (first & 1) : 0);
    v2f p[4];
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 0);              // two elements of a byte, times the scale: exact
    if constexpr (V == 8) {
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 1);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 2);
        p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, power, 3);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = p[j / 2][j % 2];
}

}  // namespace same
