// Rounding to grouped four-bit integers, and the product of rows of numbers with a matrix in them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "element.h"
#include "group_format.h"

namespace same {

// ---- Rounding.  A lane takes 8 elements, 2^(group_log2 - 3) consecutive lanes a group.  The quotient (x - b) / s is taken in
// binary32; where that leaves open on which side of a border between two codes it lies (or leaves its range) it is taken in binary64.
struct GroupQuantizeArgs {
    const void* x;
    int64_t rows, stride;
    int32_t width, group_log2;
    uint32_t* codes;
    uint32_t* scales;
};

// the largest bfloat16 number that is not above x, which is finite; -0 becomes 0
__device__ __forceinline__ float bfloat_below(float x)
{
    const uint32_t bits = __float_as_uint(x);
    uint32_t cut = bits & 0xFFFF0000u;
    if ((bits >> 31) && cut != bits) cut += 0x00010000u;
    return fmaxf(__uint_as_float(cut), __uint_as_float(0xFF7F0000u)) + 0.0f;
}

template <class TI>
__global__ __launch_bounds__(256) void group_quantize_kernel(GroupQuantizeArgs a)
{
    const int64_t pieces = micro_groups(a.width) * (kMicroGroup / 8);          // of 8 elements, per row
    const int64_t all = a.rows * pieces;
    const int lanes = 1 << (a.group_log2 - 3);
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {   // whole blocks of 16 lanes
        const int64_t row = all >> 32 ? at / pieces : (int64_t)((uint32_t)at / (uint32_t)pieces);             // a division of 64 bits takes as long as the rest
        const int c = (int)(at - row * pieces), count = a.width - 8 * c;
        float x[8];
        load_eight<TI>(x, static_cast<const TI*>(a.x) + row * a.stride + (int64_t)c * 8, count);
        float least = __builtin_inff(), most = -__builtin_inff();
        int bad = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count) {
                bad |= (__float_as_uint(x[j]) & 0x7FFFFFFFu) >= 0x7F800000u;
                least = fminf(least, x[j]);
                most = fmaxf(most, x[j]);
            }
        for (int o = 1; o < lanes; o <<= 1) {
            least = fminf(least, __shfl_xor(least, o));
            most = fmaxf(most, __shfl_xor(most, o));
            bad |= __shfl_xor(bad, o);
        }
        uint32_t word = 0u, sb = 0u;
        if (bad) {
            sb = 0x7FC07FC0u;
        } else if (least <= most) {                                            // else a group behind the row's end
            const float base = bfloat_below(least);
            uint32_t step_bits = __float_as_uint((float)(__bf16)(float)(((double)most - (double)base) / 15.0)) >> 16;
            if ((double)base + 15.0 * (double)from_bfloat_bits(step_bits) > 3.4028234663852886e38) --step_bits;
            const float step = from_bfloat_bits(step_bits);
            sb = __float_as_uint(base) | step_bits;
            const float inverse = 1.0f / step;
            if (step_bits) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float t = (x[e] - base) * inverse, near = rintf(t);
                    float q = fminf(fmaxf(near, 0.0f), 15.0f);
                    // t is off by less than 2^-18; at a border or out of range: in binary64
                    if (!(fabsf(fabsf(t - near) - 0.5f) > 1.52587890625e-5f)) {
                        const double exact = rint(((double)x[e] - (double)base) / (double)step);
                        q = (float)fmin(fmax(exact, 0.0), 15.0);
                    }
                    if (e < count) word |= (uint32_t)q << (4 * (e >> 1) + 16 * (e & 1));
                }
            }
        }
        a.codes[(at - c) + group_word(c)] = word;                              // rows of codes follow each other without a gap
        if ((c & (lanes - 1)) == 0) a.scales[at >> (a.group_log2 - 3)] = sb;
    }
}

// ---- Product: out[i][j] = scale * sum_k a[i][k] (q_jk s_jg + b_jg), on the 16-bit matrix instructions.
//
// A code as the lower half of a byte is the eight-bit floating-point number q / 512 (four exponent bits, three fraction bits; below 8 it
// is subnormal), so the conversion of such bytes with a scale of 512 gives two codes as 16-bit numbers an instruction, exactly, and their products
// with 16-bit numbers are exact.  With D = sum a q and S = sum a over a group, both summed by matrix instructions in binary32 (S
// with a second operand of ones), the group adds s D + b S.  Rows in binary32 are cut into three bfloat16 numbers of eight bits
// each, whose sum they are, and take three instructions.
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

// Eight numbers of a row as operands of the matrix instruction, in the codes' order: themselves, or three operands that add up to them.
template <class TI, int P>
__device__ __forceinline__ void pieces_of(v4u32 (&out)[P], const TI* p, int count)
{
    if constexpr (P == 1) {
        Eight<TI> c;
        if (count >= 8) {
            c.load(p);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) c.v[j] = j < count ? p[j] : (TI)0.0f;
        }
        v4u32 x;
        __builtin_memcpy(&x, c.v, 16);
        out[0] = {__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[1], 0x05040100u),
                  __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
    } else {
        float x[8];
        load_eight<float>(x, p, count);
        three_pieces(out, x);
    }
}

// A wave takes 16 rows of a by 16 of b.
template <class TI, int kGroupLog2>
__global__ __launch_bounds__(256) void group_product_kernel(GroupProductArgs p)
{
    constexpr bool kHalf = kHalfMatrix<TI>;
    constexpr int P = sizeof(TI) == 4 ? 3 : 1, kSteps = 1 << (kGroupLog2 - 5), kPer = 128 >> kGroupLog2;   // instructions per group, groups of 128 elements
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, r = lane & 15, h = lane >> 4;
    const int64_t tiles_b = (p.rows_b + 15) / 16, tiles_a = (p.rows_a + 15) / 16, blocks = (p.width + 127) / 128;
    const v4u32 ones = kHalf ? v4u32{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u} : v4u32{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    for (int64_t tile = (int64_t)blockIdx.x * 4 + wv; tile < tiles_a * tiles_b; tile += (int64_t)gridDim.x * 4) {
        const int64_t i0 = tile / tiles_b * 16, j0 = tile % tiles_b * 16;
        const int64_t i = i0 + r < p.rows_a ? i0 + r : p.rows_a - 1, j = j0 + r < p.rows_b ? j0 + r : p.rows_b - 1;   // rows behind the last are computed from it and not written
        const TI* const x = static_cast<const TI*>(p.a) + i * p.stride_a;
        const uint8_t* const codes = p.codes + j * p.pitch + 16 * h;
        const uint32_t* const scales = reinterpret_cast<const uint32_t*>(p.scales + j * p.scale_pitch);
        v4f32 acc = {};
        for (int64_t k = 0; k < blocks; ++k) {
            const v4u32 w = *reinterpret_cast<const v4u32*>(codes + k * 64);
#pragma unroll
            for (int g = 0; g < kPer; ++g) {
                v4f32 d = {}, s = {};
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const int at = (int)k * 128 + 32 * (g * kSteps + t) + 8 * h;
                    v4u32 xs[P];
                    pieces_of<TI, P>(xs, x + at, p.width - at);
                    const v4u32 b = codes_up<kHalf>(w[g * kSteps + t]);
#pragma unroll
                    for (int q = 0; q < P; ++q) {
                        d = mfma_16<kHalf>(xs[q], b, d);
                        s = mfma_16<kHalf>(xs[q], ones, s);
                    }
                }
                const uint32_t sb = scales[k * kPer + g];
                const float step = from_bfloat_bits(sb & 0xFFFFu), base = __uint_as_float(sb & 0xFFFF0000u);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[q] = __builtin_fmaf(step, d[q], __builtin_fmaf(base, s[q], acc[q]));
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (i0 + 4 * h + q < p.rows_a && j0 + r < p.rows_b)
                store_number(p, i0 + 4 * h + q, j0 + r, p.scale * acc[q]);
    }
}

// Few rows of a, up to 16.  A wave keeps its part of them, KB blocks of 128 elements, in registers and goes through the rows of b, 16 at
// a time, whose codes come straight from memory, those of the next 16 while these are multiplied: every byte of b is read once, a once per
// workgroup.  Where a row of b has more than KB blocks, waves_per_row waves share it and add up their sums by way of LDS, in order.
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
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, h = lane >> 4;
    const int kw = p.waves_per_row, streams = (int)(blockDim.x >> 6) / kw, stream = wv / kw, mine = wv - stream * kw;
    const int blocks = (p.width + 127) / 128, first = mine * KB;

    // the wave's part of a: lane l has the elements 32 t + 8 h .. + 7 of row l % 16 of every block
    v4u32 x[KB][4][kKept], sums[kSets][3];
    {
        const int m = kStack ? r & 3 : r;
        const TI* const row = static_cast<const TI*>(p.a) + (m < p.rows_a ? m : p.rows_a - 1) * p.stride_a;
        float total[kSets * 8];
#pragma unroll
        for (int g = 0; g < kSets * 8; ++g) total[g] = 0.0f;
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int at = (first + k) * 128 + 32 * t + 8 * h;
                float y[8];
                load_eight<TI>(y, row + at, p.width - at);
                if constexpr (kStack) {
                    v4u32 c[3];
                    three_pieces(c, y);
                    const v4u32 zero = {};
                    x[k][t][0] = r < 4 ? c[0] : r < 8 ? c[1] : r < 12 ? c[2] : zero;
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = __uint_as_float(j < 4 ? x[k][t][0][j & 3] << 16 : x[k][t][0][j & 3] & 0xFFFF0000u);
                } else if constexpr (P == 3) {
                    v4u32 c[3];
                    three_pieces(c, y);
#pragma unroll
                    for (int q = 0; q < kKept; ++q) x[k][t][q] = c[q];
                    if constexpr (kAside) aside[wv][k * 4 + t][lane] = c[2];
                } else {
                    pieces_of<TI, 1>(x[k][t], row + at, p.width - at);
                }
                total[k * kPer + t / kSteps] += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
            }
#pragma unroll
        for (int g = 0; g < KB * kPer; ++g) {
            total[g] += __shfl_xor(total[g], 16);
            total[g] += __shfl_xor(total[g], 32);
        }
#pragma unroll
        for (int e = 0; e < kSets; ++e) {
            const float* const of = total + 8 * e;
            const float y[8] = {of[0], of[2], of[4], of[6], of[1], of[3], of[5], of[7]};          // three_pieces pairs j with j + 4
            three_pieces(sums[e], y);
#pragma unroll
            for (int q = 0; q < 3; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) sums[e][q][j] = h == 0 ? sums[e][q][j] : 0u;
        }
    }

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
                if (i < p.rows_a && tile * 16 + r < p.rows_b) store_number(p, i, tile * 16 + r, p.scale * acc[q]);
            }
            return;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) part[buffer][wv][4 * h + q][r] = acc[q];
        __syncthreads();
        for (int e = (int)threadIdx.x - stream * kw * 64; e < 256; e += kw * 64) {
            const int i = e >> 4, j = e & 15;
            if (i < p.rows_a && tile * 16 + j < p.rows_b) {
                float all = 0.0f;
                for (int w = stream * kw; w < (stream + 1) * kw; ++w) {
                    if constexpr (kStack) all += (part[buffer][w][i + 8][j] + part[buffer][w][i + 4][j]) + part[buffer][w][i][j];
                    else                  all += part[buffer][w][i][j];
                }
                store_number(p, i, tile * 16 + j, p.scale * all);
            }
        }
        buffer ^= 1;                                                           // the next turn's sums go elsewhere; the one after it is behind a barrier
    };
    Codes even, odd;
    int64_t turn = blockIdx.x;
    if (turn >= turns) return;
    load(even, turn);
    for (;;) {
        const int64_t next = turn + gridDim.x, after = next + gridDim.x;
        load(odd, next < turns ? next : turn);
        multiply(even, turn);
        if (next >= turns) break;
        load(even, after < turns ? after : next);
        multiply(odd, next);
        if (after >= turns) break;
        turn = after;
    }
}

}  // namespace same
