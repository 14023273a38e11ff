// Rounding to grouped four-bit integers, and the product of rows of numbers with a matrix in them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "element.h"
#include "group_format.h"
#include "to_lds.h"

namespace same {

// ---- Rounding.  A lane takes 8 elements, 2^(group_log2 - 3) consecutive lanes a group.  The quotient (x - b) / s is taken as a product
// in binary32; where that leaves open on which side of a border between two codes it lies, x - b is compared with the border, exactly, and at
// the ends of the range the quotient is taken in binary64.  Bound by memory in binary32 (100,000 x 256: 20 to 23 us, 5 TB/s and more read and
// written), by its instructions on 16-bit rows, half as long (8192 x 8192 bf16: 73 us, 2.3 TB/s).
struct GroupQuantizeArgs {
    const void* x;
    int64_t rows, stride;
    int32_t width, group_log2;
    uint32_t* codes;
    uint32_t* scales;
    int32_t chunks;                  // of 8 elements of a filled row
    float inverse;                   // of chunks
    int32_t step_rows, step_chunks;  // what all workgroups take at once, kRoundedAtOnce each, in rows and chunks
};

constexpr int kRoundedAtOnce = 256;

// Without the quieting of signalling NaNs that the functions of the language ask for.
__device__ __forceinline__ float least3(float x, float y, float z)
{
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
}
__device__ __forceinline__ float most3(float x, float y, float z)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
}

// The least (or largest) of 4, 8 or 16 consecutive lanes, in all of them.
template <class F>
__device__ __forceinline__ float of_lanes(float x, int group_log2, F&& f)
{
    const auto with = [&](auto control) { x = f(x, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(control)::value, 0xF, 0xF, true))); };
    with(std::integral_constant<int, 0xB1>());                                 // lane ^ 1
    with(std::integral_constant<int, 0x4E>());                                 // lane ^ 2
    if (group_log2 > 5) with(std::integral_constant<int, 0x141>());            // 7 - lane of eight
    if (group_log2 > 6) with(std::integral_constant<int, 0x140>());            // 15 - lane of sixteen
    return x;
}

// the largest bfloat16 number that is not above x, which is finite; -0 becomes 0
__device__ __forceinline__ float bfloat_below(float x)
{
    const uint32_t bits = __float_as_uint(x);
    uint32_t cut = bits & 0xFFFF0000u;
    if ((bits >> 31) && cut != bits) cut += 0x00010000u;
    return fmaxf(__uint_as_float(cut), __uint_as_float(0xFF7F0000u)) + 0.0f;
}

template <class TI>
__device__ __forceinline__ void group_round(const GroupQuantizeArgs& a, Eight<TI>& raw, uint32_t row, int c, int lanes)
{
    const int count = a.width - 8 * c;
    float x[8], sum = 0.0f;
    if (count < 8) cut_eight(raw, 8 * c, a.width);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = to_float(raw.v[j]);
    if (count < 8)                                                             // behind the row's end: its elements' first, which changes nothing
#pragma unroll
        for (int j = 1; j < 8; ++j) x[j] = j < count ? x[j] : x[0];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += x[j];
    float least = least3(least3(x[0], x[1], x[2]), least3(x[3], x[4], x[5]), least3(x[6], x[7], x[7]));
    float most = most3(most3(x[0], x[1], x[2]), most3(x[3], x[4], x[5]), most3(x[6], x[7], x[7]));
    bool bad = !(fabsf(sum) < __builtin_inff());                               // an infinity, a NaN or a sum beyond binary32
    if (bad) {
        bad = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) bad |= (__float_as_uint(x[j]) & 0x7FFFFFFFu) >= 0x7F800000u;
    }
    most = count <= 0 ? -__builtin_inff() : bad ? __builtin_inff() : most;
    least = count <= 0 ? __builtin_inff() : bad ? -__builtin_inff() : least;
    most = of_lanes(most, a.group_log2, [](float p, float q) { return most3(p, q, q); });
    least = of_lanes(least, a.group_log2, [](float p, float q) { return least3(p, q, q); });
    bad = most == __builtin_inff();
    uint32_t word = 0u, sb = 0u;
    if (bad) {
        sb = 0x7FC07FC0u;
    } else if (least <= most) {                                            // else a group behind the row's end
        const float base = bfloat_below(least);
        // (most - base) / 15 by a product that is off by less than four units of its last place: enough unless it is as near to a
        // border between two bfloat16 numbers, or near the ends of the range
        const float range = most - base, near_step = range * 0.06666667f;
        uint32_t step_bits = (__float_as_uint(near_step) + 0x8000u) >> 16;
        const int border = (int)(__float_as_uint(near_step) & 0xFFFFu) - 0x8000;
        const bool ordinary = range >= 1e-30f && range <= 1e30f;
        if (!(ordinary && abs(border) > 4)) {
            step_bits = __float_as_uint((float)(__bf16)(float)(((double)most - (double)base) / 15.0)) >> 16;
            if (fabs((double)base + 15.0 * (double)from_bfloat_bits(step_bits)) > 3.4028234663852886e38) --step_bits;      // towards zero
        }
        const float step = from_bfloat_bits(step_bits);
        sb = __float_as_uint(base) | step_bits;
        if (step_bits) {
            const float inverse = __builtin_amdgcn_rcpf(step);                // to a unit of the last place
            float off = 1.0f;                                              // least distance to a border
            float near[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float t = (x[e] - base) * inverse;
                near[e] = rintf(t);
                off = fminf(off, 0.5f - fabsf(t - near[e]));
                near[e] = __builtin_amdgcn_fmed3f(near[e], 0.0f, 15.0f);
                // (elements behind the row's end repeat their chunk's first, whose code is cut off below)
            }
            if (!ordinary) {
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {                              // eight turns of the registers
                    const double exact = rint(((double)x[0] - (double)base) / (double)step);
                    const float first = (float)fmin(fmax(exact, 0.0), 15.0), x0 = x[0];
#pragma unroll
                    for (int j = 0; j < 7; ++j) { near[j] = near[j + 1]; x[j] = x[j + 1]; }
                    near[7] = first;
                    x[7] = x0;
                }
            } else if (!(off > 1.52587890625e-5f)) {                       // t is off by less than 2^-18: within 2^-16 of a border
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // x - base is d and a rest exactly; the borders next to near are numbers of binary32, which d keeps its side of or is
                    const float d = x[e] - base, back = d - x[e], rest = (x[e] - (d - back)) - (base + back);
                    const float up = (near[e] + 0.5f) * step, down = (near[e] - 0.5f) * step;
                    const int odd = (int)near[e] & 1;                          // no branches: bits
                    const int above = (d > up) | ((d == up) & ((rest > 0.0f) | ((rest == 0.0f) & odd)));
                    const int below = (d < down) | ((d == down) & ((rest < 0.0f) | ((rest == 0.0f) & odd)));
                    near[e] = __builtin_amdgcn_fmed3f(near[e] + (float)(above - below), 0.0f, 15.0f);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) word |= (uint32_t)near[e] << (4 * (e >> 1) + 16 * (e & 1));
            if (count < 8)
                for (int e = 0; e < 8; ++e)
                    if (e >= count) word &= ~(15u << (4 * (e >> 1) + 16 * (e & 1)));
        }
    }
    const int64_t first = (int64_t)row * a.chunks;                             // rows of codes follow each other without a gap
    a.codes[first + group_word(c)] = word;
    if ((c & (lanes - 1)) == 0) a.scales[(first + c) >> (a.group_log2 - 3)] = sb;
}

template <class TI>
__global__ __launch_bounds__(256) void group_quantize_kernel(GroupQuantizeArgs a)
{
    constexpr int kMany = kRoundedAtOnce / 256;
    const int lanes = 1 << (a.group_log2 - 3);
    const int64_t begin = (int64_t)blockIdx.x * kRoundedAtOnce;
    uint32_t row0 = (uint32_t)(begin / a.chunks);                              // of the workgroup; a lane's own by a short division
    int c0 = (int)(begin - (int64_t)row0 * a.chunks);
    const uint32_t rows = (uint32_t)a.rows;
    while (row0 < rows) {
        Eight<TI> raw[kMany];
        uint32_t row[kMany];
        int chunk[kMany];
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            const int at = c0 + q * 256 + (int)threadIdx.x;                    // below 2^17 + 512: the quotient is exact
            const int down = (int)(((float)at + 0.5f) * a.inverse);
            row[q] = row0 + (uint32_t)down;
            chunk[q] = at - down * a.chunks;
            raw[q] = eight_at(static_cast<const TI*>(a.x) + (int64_t)min(row[q], rows - 1u) * a.stride, 8 * chunk[q], a.width);
        }
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            if (row[q] >= rows) continue;                                      // whole blocks of 16 lanes
            group_round(a, raw[q], row[q], chunk[q], lanes);
        }
        row0 += (uint32_t)a.step_rows;
        c0 += a.step_chunks;
        if (c0 >= a.chunks) {
            c0 -= a.chunks;
            ++row0;
        }
    }
}

// ---- Product: out[i][j] = scale * sum_k a[i][k] (q_jk s_jg + b_jg), on the 16-bit matrix instructions.
//
// A code as the lower half of a byte is the eight-bit floating-point number q / 512 (four exponent bits, three fraction bits; below 8 it
// is subnormal), so the conversion of such bytes with a scale of 512 gives two codes as 16-bit numbers an instruction, exactly, and their products
// with 16-bit numbers are exact.  With D = sum a q and S = sum a over a group, both summed by matrix instructions in binary32 (S
// with a second operand of ones), the group adds s D + b S.  Rows in binary32 are cut into three bfloat16 numbers of eight bits
// each, whose sum they are, and take three instructions.
//
// bfloat16 ends at 2^-133, so what a number has below that is not in its pieces, and 15 S is beyond binary32 where S is not far from its end.  Rows in
// binary32 are therefore multiplied by a power of two before they are cut where their largest number is below 2^-64 (up to [2^-31, 2^-30): all bits are
// above 2^-133 then, and no sum is beyond binary32, of 2^20 products with 2^132 either) or not below 2^112 (down to [2^111, 2^112)), and the result
// by its inverse.  Other rows stay as they are: their sums would lose bits at one end for what they gain at the other.
typedef float v4f32 __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));
typedef _Float16 v8f16 __attribute__((ext_vector_type(8)));

struct GroupProductArgs {
    const void* a;
    int64_t rows_a, stride_a;
    int32_t width;
    int32_t type_out;                // as in same_lda_rows: 0 binary32, 1 bfloat16, 2 binary16
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t rows_b;
    int64_t pitch, scale_pitch;      // bytes of a row of codes and of scales
    float scale;
    void* out;
    int64_t out_stride;
    int32_t waves_per_row;           // of the kernel for few rows: waves that share the blocks of a row of b
};

__device__ __forceinline__ void store_number(const GroupProductArgs& p, int64_t i, int64_t j, float x)
{
    const int64_t at = i * p.out_stride + j;
    if (p.type_out == 0)      static_cast<float*>(p.out)[at] = x;
    else if (p.type_out == 1) static_cast<__bf16*>(p.out)[at] = (__bf16)x;
    else                      static_cast<_Float16*>(p.out)[at] = (_Float16)x;
}

struct Numbers {
    v4f32 lo, hi;
};

// Up to eight numbers of row i from column j on (none where count is not positive).
__device__ __forceinline__ void store_numbers(const GroupProductArgs& p, int64_t i, int64_t j, Numbers x, int count)
{
    const int64_t at = i * p.out_stride + j;
    if (count >= 8) {
        const float y[8] = {x.lo[0], x.lo[1], x.lo[2], x.lo[3], x.hi[0], x.hi[1], x.hi[2], x.hi[3]};
        if (p.type_out == 0)      store_eight(static_cast<float*>(p.out) + at, y, 8);
        else if (p.type_out == 1) store_eight(static_cast<__bf16*>(p.out) + at, y, 8);
        else                      store_eight(static_cast<_Float16*>(p.out) + at, y, 8);
    } else {
#pragma unroll 1
        for (int e = 0; e < count; ++e) {
            store_number(p, i, j + e, x.lo[0]);
            x.lo = {x.lo[1], x.lo[2], x.lo[3], x.hi[0]};
            x.hi = {x.hi[1], x.hi[2], x.hi[3], 0.0f};
        }
    }
}

// What the matrix instruction takes: bfloat16 for rows in bfloat16 and binary32, binary16 for rows in that.
template <class TI>
constexpr bool kHalfMatrix = __is_same(TI, _Float16);

// The eight codes of a word, element j and j + 4 in a register.
template <bool kHalf>
__device__ __forceinline__ v4u32 codes_up(uint32_t w)
{
    const uint32_t lo = w & 0x0F0F0F0Fu, hi = (w >> 4) & 0x0F0F0F0Fu;          // elements 0, 4, 1, 5 and 2, 6, 3, 7
    if constexpr (kHalf)
        return {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true))};
    else
        return {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true))};
}

template <bool kHalf>
__device__ __forceinline__ v4f32 mfma_16(v4u32 a, v4u32 b, v4f32 c)
{
    if constexpr (kHalf) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, a), __builtin_bit_cast(v8f16, b), c, 0, 0, 0);
    else                 return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf16, a), __builtin_bit_cast(v8bf16, b), c, 0, 0, 0);
}

// The largest magnitude of x, y and z, of which NaN has none.
__device__ __forceinline__ float largest3(float x, float y, float z)
{
    float r;
    asm("v_max3_f32 %0, |%1|, |%2|, |%3|" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
}

template <int N>
__device__ __forceinline__ float largest(float most, const float (&x)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 2) most = largest3(most, x[j], x[j + 1]);
    return most;
}

// The power of two, as its exponent, for a row whose largest magnitude is `most`: in -16 .. 118, 0 for zero, an infinity and NaN.
__device__ __forceinline__ int power_for(float most)
{
    const int e = __builtin_amdgcn_frexp_expf(most);                           // most is in [2^(e - 1), 2^e)
    return e < -63 ? -30 - e : e > 112 ? 112 - e : 0;
}

__device__ __forceinline__ float two_to(int power) { return __uint_as_float((uint32_t)(127 + power) << 23); }

// Eight numbers in binary32 as three operands of bfloat16 numbers that add up to them, element j and j + 4 in a register: the upper eight
// bits of what is left, which leaves the rest exactly.
__device__ __forceinline__ void three_pieces(v4u32 (&out)[3], const float (&from)[8])
{
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = from[j];
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = __float_as_uint(x[j]), hi = __float_as_uint(x[j + 4]);
            out[q][j] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
            x[j] -= __uint_as_float(lo & 0xFFFF0000u);
            x[j + 4] -= __uint_as_float(hi & 0xFFFF0000u);
        }
}

// Eight numbers as operands of the matrix instruction, in the codes' order: themselves, or three operands that add up to them.
template <class TI, int P>
__device__ __forceinline__ void pieces_of(v4u32 (&out)[P], const Eight<TI>& c)
{
    if constexpr (P == 1) {
        v4u32 x;
        __builtin_memcpy(&x, c.v, 16);
        out[0] = {__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[1], 0x05040100u),
                  __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
    } else {
        three_pieces(out, c.v);
    }
}

// An operand of ones: with it as the first, an instruction adds up the rows of the second, lane l the row l % 16.
template <bool kHalf>
__device__ __forceinline__ v4u32 all_ones()
{
    constexpr uint32_t one = kHalf ? 0x3C003C00u : 0x3F803F80u;
    return {one, one, one, one};
}

// Any number of rows, in two launches.  The first one lays the rows of a down as the lanes of the matrix instruction take them, cut into pieces
// and filled up with zeros: per 16 rows and block of 128 elements 4 P operands of 1 KB; and the sums S of their groups.  Rows in binary32 need
// their largest number first: those of up to kWholeBlocks blocks are taken whole by one workgroup, of longer ones another launch before it finds the
// powers of two (us without either, whole, with the launch: 64 x 50,021 x 1024 33.3, 34.4, -; 40 x 10,000 x 2000 22.5, 26.2, 24.9; 33 x 4096 x 4096 19.9,
// 28.5, 22.3).
constexpr int kWholeBlocks = 8;

struct GroupRowsArgs {
    const void* a;
    int64_t rows_a, stride_a;
    int32_t width;
    int32_t blocks, filled;          // of 128 elements in a row; with those that are zeros
    v4u32* operands;                 // [16 rows][filled][4][P][64]
    float* sums;                     // [16 rows][filled][groups of a block][16]
    float* inverse;                  // [16 rows][16]: of rows in binary32, the inverse of their power of two
};

// A workgroup per row, those that fill up the last 16 too.
__global__ __launch_bounds__(256) void group_row_powers_kernel(GroupRowsArgs a)
{
    __shared__ float of_wave[4];
    const int64_t i = (int64_t)blockIdx.x < a.rows_a ? blockIdx.x : a.rows_a - 1;
    const float* const row = static_cast<const float*>(a.a) + i * a.stride_a;
    float most = 0.0f;
    for (int at = (int)threadIdx.x * 8; at < a.width; at += 4 * 2048) {
        Eight<float> x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = eight_at(row, at + u * 2048, a.width);       // behind the row's end: its last eight again
#pragma unroll
        for (int u = 0; u < 4; ++u) most = largest(most, x[u].v);
    }
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x == 0) a.inverse[blockIdx.x] = two_to(-power_for(largest(0.0f, of_wave)));
}

// kWhole: the workgroup's waves have a block each of all that there are.
template <class TI, int kGroupLog2, bool kWhole>
__global__ __launch_bounds__(kWhole ? 64 * kWholeBlocks : 256) void group_rows_kernel(GroupRowsArgs a)
{
    constexpr bool kHalf = kHalfMatrix<TI>;
    constexpr int P = sizeof(TI) == 4 ? 3 : 1, kPer = 128 >> kGroupLog2, kSteps = 4 / kPer;             // groups of a block, instructions per group
    static_assert(!kWhole || P == 3, "only rows in binary32 need a whole row");
    __shared__ float of_wave[kWhole ? kWholeBlocks : 1][16];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, waves = blockDim.x >> 6, r = lane & 15, h = lane >> 4;
    const int64_t tile = blockIdx.x;
    const int64_t i = tile * 16 + r < a.rows_a ? tile * 16 + r : a.rows_a - 1;         // rows behind the last one: it again
    const TI* const row = static_cast<const TI*>(a.a) + i * a.stride_a;
    for (int k = blockIdx.y * waves + wv; k < a.filled; k += gridDim.y * waves) {
        Eight<TI> raw[4] = {};
        if (k < a.blocks)
#pragma unroll
            for (int t = 0; t < 4; ++t) raw[t] = eight_at(row, k * 128 + 32 * t + 8 * h, a.width);
#pragma unroll
        for (int t = 0; t < 4; ++t) cut_eight(raw[t], k * 128 + 32 * t + 8 * h, a.width);
        if constexpr (P == 3) {
            float factor;
            if constexpr (kWhole) {                                                    // as many waves as blocks: all of them get here, once
                float most = 0.0f;
#pragma unroll
                for (int t = 0; t < 4; ++t) most = largest(most, raw[t].v);
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                if (h == 0) of_wave[wv][r] = most;
                __syncthreads();
                for (int w = 0; w < waves; ++w) most = fmaxf(most, of_wave[w][r]);
                const int power = power_for(most);
                factor = two_to(power);
                if (threadIdx.x < 16) a.inverse[tile * 16 + r] = two_to(-power);
            } else {
                factor = __uint_as_float(0x7F000000u - __float_as_uint(a.inverse[tile * 16 + r]));       // 2^p from 2^-p: 254 less the exponent's bits
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[t].v[j] *= factor;
        }
        v4f32 total[kPer] = {};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            v4u32 c[P];
            pieces_of<TI, P>(c, raw[t]);
#pragma unroll
            for (int q = 0; q < P; ++q) {
                a.operands[((tile * a.filled + k) * (4 * P) + t * P + q) * 64 + lane] = c[q];
                total[t / kSteps] = mfma_16<kHalf>(all_ones<kHalf>(), c[q], total[t / kSteps]);
            }
        }
        if (h == 0)
#pragma unroll
            for (int g = 0; g < kPer; ++g) a.sums[((tile * a.filled + k) * kPer + g) * 16 + r] = total[g][0];
    }
}

// The second one: WM WN WK waves take 16 MT WM rows of a by 16 NT WN of b.  All operands come straight to LDS, kStages - 1 trips ahead, in
// pieces of 1 KB as the lanes take them (with codes fetched into registers by one wave and shared by way of LDS 512 x 50,021 x 1024 f16 took
// 108 us, so 106, before the change below).  WK waves share out the blocks of a row of b, and their sums are added in order at the end: more waves
// where rows of b are few.  S comes with the operands, for sum_g b_g S_g as matrix instructions before the loop waited for what it read: 106 us,
// now 82 to 84 on those numbers, random codes and steps, and 72 on positive ones with a few large in a row.
// Bound by what the matrix instructions and the unpacking of codes take on the same SIMD one after the other, and by the tiles' fetches from the
// caches (16 KB of rows and 16 KB of codes per 64 x 256 x 128): 512 x 50,021 x 4096 bf16 247 to 250 us, 840 to 850 TFLOP/s of the 1205 that a plain
// product of that type reaches; in binary32, three instructions each, 615 us.
struct GroupTilesArgs {
    GroupProductArgs p;
    const v4u32* operands;
    const float* sums;
    const float* inverse;
    int32_t blocks, filled;          // filled: a multiple of WK
};

template <int P, int kGroupLog2, int MT, int NT, int WM, int WN, int WK>
struct GroupStage {
    v4u32 rows[WK][WM][MT][4][P][64];
    v4u32 codes[WK][WN][NT][64];
    uint32_t scales[WK][WN][NT][16][128 >> kGroupLog2];
    static constexpr int kSums = WK * WM * MT * (128 >> kGroupLog2) * 16;
    float sums[kSums < 64 ? 64 : kSums];                                       // [WK][WM][MT][groups][16]
};

template <bool kHalf, int P, int kGroupLog2, int MT, int NT, int WM, int WN, int WK, int kStages>
__global__ __launch_bounds__(64 * WM * WN * WK, kStages * sizeof(GroupStage<P, kGroupLog2, MT, NT, WM, WN, WK>) * 3 <= 163840 && WM * WN * WK == 4 ? 3 : 2) void group_product_kernel(GroupTilesArgs a)
{
    constexpr int kPer = 128 >> kGroupLog2, kSteps = 4 / kPer;                         // groups of a block, instructions per group
    constexpr int kWaves = WM * WN * WK;
    using Stage = GroupStage<P, kGroupLog2, MT, NT, WM, WN, WK>;
    __shared__ union {
        Stage in[kStages];
        float out[WK > 1 ? WK - 1 : 1][WK > 1 ? MT * NT * 4 : 1][WK > 1 ? 64 * WM * WN : 1];
        float strip[WM * WN][16 * MT][16 * NT + 4];
    } lds;
    __shared__ v4f32 inverse[P == 3 ? 16 : 1];                                         // of up to 64 rows
    static_assert(P != 3 || 16 * MT * WM <= 64, "a piece of 64 rows");
    const GroupProductArgs& p = a.p;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, h = lane >> 4;
    const int wk = wv / (WM * WN), wm = wv / WN % WM, wn = wv % WN;
    // the tiles of the same rows of b on one of the eight dies, one after the other: they find the codes in its cache
    constexpr int kTall = 16 * MT * WM, kWide = 16 * NT * WN;
    const int64_t tiles_a = (p.rows_a + kTall - 1) / kTall, turn = blockIdx.x / 8, tile_b = turn / tiles_a * 8 + blockIdx.x % 8;
    const int64_t first_i = turn % tiles_a * kTall, first_j = tile_b * kWide;
    if (first_j >= p.rows_b) return;                                                   // the whole workgroup
    const int64_t i0 = first_i + wm * (16 * MT), j0 = first_j + wn * (16 * NT);
    const int trips = a.filled / WK;
    const int last = (int)(p.rows_b - first_j < kWide ? p.rows_b - first_j : kWide) - 1;     // rows behind the last are computed from it and not written

    // what a trip needs, in equal numbers for every wave (the last pieces are fetched twice where they do not go round)
    constexpr int kRows = WK * WM * MT * 4 * P, kCodes = WK * WN * NT, kWords = WK * WN * NT * 16 * kPer, kSums = Stage::kSums;
    constexpr int kRowsEach = (kRows + kWaves - 1) / kWaves, kCodesEach = (kCodes + kWaves - 1) / kWaves, kWordsEach = (kWords + 64 * kWaves - 1) / (64 * kWaves);
    constexpr int kSumsEach = (kSums + 64 * kWaves - 1) / (64 * kWaves), kEach = kRowsEach + kCodesEach + kWordsEach + kSumsEach;
    const uint8_t* const rows = reinterpret_cast<const uint8_t*>(a.operands + first_i / 16 * a.filled * (4 * P) * 64);
    const uint8_t* const codes = p.codes + first_j * p.pitch;
    const uint8_t* const words = p.scales + first_j * p.scale_pitch;
    const uint8_t* const sums = reinterpret_cast<const uint8_t*>(a.sums + first_i / 16 * a.filled * (kPer * 16));
    uint32_t code_at[kCodesEach], word_at[kWordsEach], sum_at[kSumsEach];              // of this lane, in the tile's rows
#pragma unroll
    for (int f = 0; f < kCodesEach; ++f) {
        const int e = min(f * kWaves + wv, kCodes - 1);
        code_at[f] = (uint32_t)min(e % (WN * NT) * 16 + r, last) * (uint32_t)p.pitch + 16 * h;
    }
#pragma unroll
    for (int f = 0; f < kWordsEach; ++f) {
        const int e = min((f * kWaves + wv) * 64, kWords - 64) + lane;
        word_at[f] = (uint32_t)min(e / kPer % kWide, last) * (uint32_t)p.scale_pitch + 4 * (e % kPer);
    }
#pragma unroll
    for (int f = 0; f < kSumsEach; ++f) {
        const int e = min(min((f * kWaves + wv) * 64, kSums < 64 ? 0 : kSums - 64) + lane, kSums - 1);
        sum_at[f] = (uint32_t)((e / (kPer * 16) % (WM * MT) * a.filled + e / (WM * MT * kPer * 16)) * (kPer * 16) + e % (kPer * 16)) * 4;
    }
    const auto fetch = [&](int trip) {
        Stage& to = lds.in[trip % kStages];
        const int t = trip < trips ? trip : trips - 1;                                 // behind the last one: it again, not used
#pragma unroll
        for (int f = 0; f < kRowsEach; ++f) {
            const int e = min(f * kWaves + wv, kRows - 1), k = e / (WM * MT * 4 * P), m = e / (4 * P) % (WM * MT), at = e % (4 * P);
            to_lds_16(uniform(rows + (int64_t)(m * a.filled + t * WK + k) * (4 * P * 1024) + at * 1024), lane * 16, &to.rows[0][0][0][0][0][0] + e * 64);
        }
#pragma unroll
        for (int f = 0; f < kCodesEach; ++f) {
            const int e = min(f * kWaves + wv, kCodes - 1), k = min(t * WK + e / (WN * NT), a.blocks - 1);      // blocks behind the row's end: its last, times zeros
            to_lds_16(uniform(codes + (int64_t)k * 64), code_at[f], &to.codes[0][0][0][0] + e * 64);
        }
#pragma unroll
        for (int f = 0; f < kWordsEach; ++f) {
            const int e = min((f * kWaves + wv) * 64, kWords - 64), k = min(t * WK + e / (kWide * kPer), a.blocks - 1);
            to_lds_4(uniform(words + (int64_t)k * (4 * kPer)), word_at[f], &to.scales[0][0][0][0][0] + e);
        }
#pragma unroll
        for (int f = 0; f < kSumsEach; ++f)
            to_lds_4(uniform(sums + (int64_t)t * (WK * kPer * 64)), sum_at[f], &to.sums[min((f * kWaves + wv) * 64, kSums < 64 ? 0 : kSums - 64)]);
    };
    static_assert(kWide * kPer % 64 == 0 && (kSums < 64 || kSums % 64 == 0), "a piece of scales is of one block, of sums a whole one");
    if constexpr (P == 3)
        if (wv == 0) to_lds_4(uniform(reinterpret_cast<const uint8_t*>(a.inverse + first_i)), 4 * min(lane, kTall - 1), inverse);
#pragma unroll
    for (int f = 0; f + 1 < kStages; ++f) fetch(f);

    v4f32 acc[MT][NT] = {};
#pragma unroll 1
    for (int trip = 0; trip < trips; ++trip) {
        arrived<(kStages - 2) * kEach>();
        fetch(trip + kStages - 1);                                                     // where the trip before this one read, which this barrier ended
        const Stage& in = lds.in[trip % kStages];
        v4u32 w[NT];
        uint32_t sb[NT][kPer];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            w[n] = in.codes[wk][wn][n][lane];
#pragma unroll
            for (int g = 0; g < kPer; ++g) sb[n][g] = in.scales[wk][wn][n][r][g];
        }
#pragma unroll
        for (int g = 0; g < kPer; ++g) {
            __builtin_amdgcn_sched_barrier(0);                                         // one group's operands in registers at a time: more of them spill
            v4u32 part[kSteps][MT][P];
            v4f32 total[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) total[m] = *reinterpret_cast<const v4f32*>(&in.sums[(((wk * WM + wm) * MT + m) * kPer + g) * 16 + 4 * h]);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < kSteps; ++t)
#pragma unroll
                    for (int q = 0; q < P; ++q) part[t][m][q] = in.rows[wk][wm][m][g * kSteps + t][q][lane];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                v4f32 d[MT] = {};
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const v4u32 b = codes_up<kHalf>(w[n][g * kSteps + t]);
#pragma unroll
                    for (int q = P - 1; q >= 0; --q)
#pragma unroll
                        for (int m = 0; m < MT; ++m) d[m] = mfma_16<kHalf>(part[t][m][q], b, d[m]);
                }
                const float step = from_bfloat_bits(sb[n][g] & 0xFFFFu), base = __uint_as_float(sb[n][g] & 0xFFFF0000u);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[m][n][q] = __builtin_fmaf(step, d[m][q], __builtin_fmaf(base, total[m][q], acc[m][n][q]));
            }
        }
    }
    arrived<0>();                                                                      // nothing is on its way to LDS any more
    if constexpr (WK > 1) {
        const int at = (wm * WN + wn) * 64 + lane;
        if (wk > 0)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int q = 0; q < 4; ++q) lds.out[wk - 1][(m * NT + n) * 4 + q][at] = acc[m][n][q];
        __syncthreads();
        if (wk == 0)
#pragma unroll
            for (int w = 0; w + 1 < WK; ++w)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[m][n][q] += lds.out[w][(m * NT + n) * 4 + q][at];
        __syncthreads();
        if (wk > 0) return;
    }
    // by way of LDS, so that a lane stores eight numbers of one row
    auto& strip = lds.strip[wm * WN + wn];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        v4f32 back = {1.0f, 1.0f, 1.0f, 1.0f};
        if constexpr (P == 3) back = inverse[(wm * MT + m) * 4 + h];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) strip[16 * m + 4 * h + q][16 * n + r] = p.scale * (P == 3 ? acc[m][n][q] * back[q] : acc[m][n][q]);
    }
    asm volatile("" ::: "memory");                                                     // a wave's accesses to LDS are done in their order
    const int col = lane % (2 * NT) * 8, count = p.rows_b - (j0 + col) < 8 ? (int)(p.rows_b - (j0 + col)) : 8;
    const int rows_here = p.rows_a - i0 < 16 * MT ? (int)(p.rows_a - i0) : 16 * MT;
#pragma unroll 1
    for (int row = lane / (2 * NT); row < rows_here; row += 32 / NT) {
        const v4f32 lo = *reinterpret_cast<const v4f32*>(&strip[row][col]), hi = *reinterpret_cast<const v4f32*>(&strip[row][col + 4]);
        store_numbers(p, i0 + row, j0 + col, {lo, hi}, count);
    }
}

// Few rows of a, up to 16 a workgroup.  A wave keeps its part of them, KB blocks of 128 elements, in registers and goes through the rows of b, 16 at
// a time, whose codes come straight from memory, those of the next turns while these are multiplied: every byte of b is read once (for every 16 rows of
// a where there are more), a once per workgroup.  Bound by memory where rows are long (1 x 50,021 x 4096 bf16: 30 us, 3.6 TB/s of codes and scales; 13 in binary32, G64: 41),
// by the launch and the one wait for a where they are short (1 x 100,000 x 256 f32, G64: 8.1 to 8.6 us).  Where a row of b has more than KB blocks, waves_per_row waves share it and add up their sums by way of LDS, in order.
// S depends on a alone; sum_g b_g S_g is a product of its own along the groups, eight in the first lanes of a bfloat16 instruction, S in three
// pieces.
// kStack: up to four rows in binary32, whose pieces take the matrix instruction's rows 4 q + i; else binary32 takes three instructions
// (P = 3), the last pieces of four blocks from LDS.
template <class TI, int P, bool kStack, int kGroupLog2, int KB>
__global__ __launch_bounds__(512, 2) void group_product_few_kernel(GroupProductArgs p)
{
    constexpr bool kHalf = kHalfMatrix<TI>;
    constexpr int kPer = 128 >> kGroupLog2, kSteps = 4 / kPer;             // groups of a block, instructions per group
    constexpr int kSets = (KB * kPer + 7) / 8;                                 // of eight groups
    constexpr bool kAside = P == 3 && KB == 4;
    constexpr int kKept = kAside ? 2 : P;
    __shared__ float part[2][8][16][17];                                       // [turn][wave][row of a][row of b]
    __shared__ v4u32 aside[kAside ? 8 : 1][kAside ? KB * 4 : 1][64];
    constexpr bool kPowers = sizeof(TI) == 4;                                  // each wave's part of a row by a power of two of its own
    float back[kPowers ? 4 : 1];                                               // the inverses for its sums
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, h = lane >> 4;
    const int kw = p.waves_per_row, streams = (int)(blockDim.x >> 6) / kw, stream = wv / kw, mine = wv - stream * kw;
    const int blocks = (p.width + 127) / 128, first = mine * KB;

    const int64_t first_i = (int64_t)blockIdx.y * 16;
    const int rows_here = p.rows_a - first_i < 16 ? (int)(p.rows_a - first_i) : 16;
    const int64_t tiles = (p.rows_b + 15) / 16, turns = (tiles + streams - 1) / streams;
    struct Codes {
        v4u32 w[KB];
        uint32_t sb[KB * kPer];
    };
    // of 16 rows of b; blocks behind the row's end are those of its last, times zeros; rows behind the last are that one, not written
    const auto load = [&](Codes& c, int64_t turn) {
        int64_t j = (turn * streams + stream) * 16 + r;
        j = j < p.rows_b ? j : p.rows_b - 1;
        const uint8_t* const codes = p.codes + j * p.pitch + 16 * h;
        const uint8_t* const scales = p.scales + j * p.scale_pitch;
#pragma unroll
        for (int k = 0; k < KB; ++k) {
            const int at = first + k < blocks ? first + k : blocks - 1;
            c.w[k] = *reinterpret_cast<const v4u32*>(codes + (int64_t)at * 64);
            struct alignas(4) Words { uint32_t v[kPer]; };
            const Words s = *reinterpret_cast<const Words*>(scales + (int64_t)at * (4 * kPer));
#pragma unroll
            for (int g = 0; g < kPer; ++g) c.sb[k * kPer + g] = s.v[g];
        }
    };
    // kRing turns are on their way or at work; what is asked for behind the last one is its last row again
    constexpr int kRing = kAside ? 2 : 4;
    Codes ring[kRing];
    // the wave's part of a: lane l has the elements 32 t + 8 h .. + 7 of row l % 16 of every block
    v4u32 x[KB][4][kKept], sums[kSets][3];
    {
        const int m = kStack ? r & 3 : r;
        const TI* const row = static_cast<const TI*>(p.a) + (first_i + (m < rows_here ? m : rows_here - 1)) * p.stride_a;
        Eight<TI> raw[KB][4];
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) raw[k][t] = eight_at(row, (first + k) * 128 + 32 * t + 8 * h, p.width);
        load(ring[0], blockIdx.x);                                             // behind the rows of a, which are waited for first
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) cut_eight(raw[k][t], (first + k) * 128 + 32 * t + 8 * h, p.width);
        if constexpr (kPowers) {
            float most = 0.0f;
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int t = 0; t < 4; ++t) most = largest(most, raw[k][t].v);
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const int power = power_for(most);
#pragma unroll
            for (int q = 0; q < 4; ++q) back[q] = two_to(-__shfl(power, 4 * h + q));
            if (__any(power != 0)) {
                const float factor = two_to(power);
#pragma unroll
                for (int k = 0; k < KB; ++k)
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int j = 0; j < 8; ++j) raw[k][t].v[j] *= factor;
            }
        }
        v4f32 total[kSets * 8];
#pragma unroll
        for (int g = 0; g < kSets * 8; ++g) total[g] = v4f32{};
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                v4u32 c[sizeof(TI) == 4 ? 3 : 1];
                pieces_of(c, raw[k][t]);
                if constexpr (kStack) {
                    const v4u32 zero = {};
                    c[0] = r < 4 ? c[0] : r < 8 ? c[1] : r < 12 ? c[2] : zero;
                }
                v4f32& sum = total[k * kPer + t / kSteps];
#pragma unroll
                for (int q = 0; q < P; ++q) sum = mfma_16<kHalf>(all_ones<kHalf>(), c[q], sum);
#pragma unroll
                for (int q = 0; q < kKept; ++q) x[k][t][q] = c[q];
                if constexpr (kAside) aside[wv][k * 4 + t][lane] = c[2];
            }
#pragma unroll
        for (int e = 0; e < kSets; ++e) {
            const v4f32* const of = total + 8 * e;
            const float y[8] = {of[0][0], of[2][0], of[4][0], of[6][0], of[1][0], of[3][0], of[5][0], of[7][0]};          // three_pieces pairs j with j + 4
            three_pieces(sums[e], y);
#pragma unroll
            for (int q = 0; q < 3; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) sums[e][q][j] = h == 0 ? sums[e][q][j] : 0u;
        }
    }

#pragma unroll
    for (int u = 1; u + 1 < kRing; ++u) load(ring[u], blockIdx.x + (int64_t)u * gridDim.x);

    int buffer = 0;
    const auto multiply = [&](const Codes& c, int64_t turn) {
        v4f32 acc = {};
#pragma unroll
        for (int e = 0; e < kSets; ++e) {
            v4u32 b;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int g = 8 * e + 2 * j;
                b[j] = g + 1 < KB * kPer ? __builtin_amdgcn_perm(c.sb[g + 1 < KB * kPer ? g + 1 : 0], c.sb[g < KB * kPer ? g : 0], 0x07060302u) : g < KB * kPer ? c.sb[g < KB * kPer ? g : 0] >> 16 : 0u;
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) acc = mfma_16<false>(sums[e][q], b, acc);
        }
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int g = 0; g < kPer; ++g) {
                v4f32 d = {};
#pragma unroll
                for (int t = g * kSteps; t < (g + 1) * kSteps; ++t) {
                    const v4u32 b = codes_up<kHalf>(c.w[k][t]);
                    if constexpr (kAside) d = mfma_16<kHalf>(aside[wv][k * 4 + t][lane], b, d);
#pragma unroll
                    for (int q = kKept - 1; q >= 0; --q) d = mfma_16<kHalf>(x[k][t][q], b, d);
                }
                const float step = from_bfloat_bits(c.sb[k * kPer + g] & 0xFFFFu);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[q] = __builtin_fmaf(step, d[q], acc[q]);
            }
        if constexpr (kPowers)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[q] *= back[q];
        const int64_t tile = turn * streams + stream;
        if (kw == 1) {                                                         // the same for the whole launch
            if constexpr (kStack)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    acc[q] += __shfl_xor(acc[q], 32);                          // (the fourth quarter is zero)
                    acc[q] += __shfl_xor(acc[q], 16);
                }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = 4 * h + q;
                if (i < rows_here && tile * 16 + r < p.rows_b) store_number(p, first_i + i, tile * 16 + r, p.scale * acc[q]);
            }
            return;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) part[buffer][wv][4 * h + q][r] = acc[q];
        __syncthreads();
        for (int e = (int)threadIdx.x - stream * kw * 64; e < 256; e += kw * 64) {
            const int i = e >> 4, j = e & 15;
            if (i < rows_here && tile * 16 + j < p.rows_b) {
                float all = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) {                                  // all on their way at once
                    const int of = stream * kw + (w < kw ? w : 0);
                    float y = part[buffer][of][i][j];
                    if constexpr (kStack) y += part[buffer][of][i + 4][j] + part[buffer][of][i + 8][j];
                    all += w < kw ? y : 0.0f;
                }
                store_number(p, first_i + i, tile * 16 + j, p.scale * all);
            }
        }
        buffer ^= 1;                                                           // the next turn's sums go elsewhere; the one after it is behind a barrier
    };
    for (int64_t turn = blockIdx.x;;) {
#pragma unroll
        for (int u = 0; u < kRing; ++u) {
            load(ring[(u + kRing - 1) % kRing], turn + (int64_t)(kRing - 1) * gridDim.x);
            multiply(ring[u], turn);
            turn += gridDim.x;
            if (turn >= turns) return;
        }
    }
}

}  // namespace same
