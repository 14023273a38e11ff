// Grouped four-bit integers: an element is q s + b with q in 0 .. 15; the step s and the base b, two bfloat16 numbers, belong to a
// group of 32, 64 or 128 consecutive elements of a row.  Rows are filled up with codes 0 to a multiple of 128 elements: 64 bytes of
// codes, and 4 bytes (s, b) per group.  Of 128 elements the word 4 h + j of 32 bits has the eight elements from 32 j + 8 h on: a lane of
// a matrix instruction that takes 8 consecutive elements of 32 (16 x 16 x 32) loads 16 bytes for four instructions, each of
// which stays within a group, whatever its size.  In a word the element 2 t is the half byte t and 2 t + 1 the half byte 4 + t:
// a shift and a mask give two neighbours in the two halves of a register.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "micro_format.h"

namespace same {

__host__ __device__ constexpr int64_t group_scale_pitch(int64_t width, int group_log2) { return micro_groups(width) * (kMicroGroup >> group_log2) * 4; }

__device__ __forceinline__ float from_bfloat_bits(uint32_t b) { return __uint_as_float(b << 16); }

// Word of the chunk c of eight elements among the words of a row.
__host__ __device__ constexpr int group_word(int c) { return (c & ~15) | ((c & 3) << 2) | ((c >> 2) & 3); }

// The eight elements of a word: q s + b in binary32, rounded once (q s has at most twelve bits, but may be beyond binary32 where the sum is not).
__device__ __forceinline__ void grouped_numbers(float (&x)[8], uint32_t word, uint32_t sb)
{
    const float s = from_bfloat_bits(sb & 0xFFFFu), b = __uint_as_float(sb & 0xFFFF0000u);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf((float)((word >> (4 * (e >> 1) + 16 * (e & 1))) & 15u), s, b);
}

}  // namespace same
