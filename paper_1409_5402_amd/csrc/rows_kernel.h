// Rows of a table for a list of tokens (or a matrix as it is) with dropout, and rows of tables in grouped four-bit integers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dropout.h"
#include "element.h"
#include "group_format.h"
#include "micro_format.h"
#include "tokens.h"

namespace same {

// out[i][j] = factor * table[token i][j] where (i, j) is kept, else zero: one rounding in binary32 and one to the output's type.
struct RowsArgs {
    const void* table;
    const uint8_t* scales;   // microscaled and grouped tables
    int64_t rows, stride;    // stride in elements (of codes: in bytes)
    int64_t scale_pitch;     // bytes, grouped tables
    int32_t group_log2;
    Tokens tokens;
    int64_t n;
    float factor;
    void* out;
    int64_t out_stride;
    int32_t width, chunks;   // chunks of 8 elements of a row, the last one may be cut
    float inverse;           // of chunks
    Drop drop;
};

struct MicroCode {};         // type of a table in microscaled four bits,
struct GroupCode {};         // in grouped four-bit integers

// Eight elements of a row of the table, as they come from memory.
template <class TI>
struct Piece {
    Eight<TI> c;
    __device__ __forceinline__ void load(const RowsArgs& a, int64_t t, int chunk) { c = eight_at(static_cast<const TI*>(a.table) + t * a.stride, chunk * 8, a.width); }
    __device__ __forceinline__ void numbers(float (&x)[8], const RowsArgs& a, int chunk)
    {
        cut_eight(c, chunk * 8, a.width);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = to_float(c.v[j]);
    }
};

template <>
struct Piece<MicroCode> {
    float x[8];
    __device__ __forceinline__ void load(const RowsArgs& a, int64_t t, int chunk)
    {
        load_micro<8>(x, static_cast<const uint8_t*>(a.table) + t * a.stride, a.scales + t * (a.stride / 16), chunk * 8);
    }
    __device__ __forceinline__ void numbers(float (&y)[8], const RowsArgs&, int)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j];
    }
};

template <>
struct Piece<GroupCode> {
    uint32_t word, sb;
    __device__ __forceinline__ void load(const RowsArgs& a, int64_t t, int chunk)
    {
        word = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.table) + t * a.stride)[group_word(chunk)];
        sb = reinterpret_cast<const uint32_t*>(a.scales + t * a.scale_pitch)[chunk >> (a.group_log2 - 3)];
    }
    __device__ __forceinline__ void numbers(float (&x)[8], const RowsArgs&, int) { grouped_numbers(x, word, sb); }
};

// Memory bound.  A thread takes kMany chunks: their tokens, their rows and, while these are on their way, what is kept of them.
template <class TI, class TO, bool kDrop>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a)
{
    constexpr int kMany = 2;
    DropKey key = {};
    if constexpr (kDrop) key = drop_key(a.drop);
    const int64_t all = a.n * a.chunks;
    for (int64_t base = (int64_t)blockIdx.x * (256 * kMany); base < all; base += (int64_t)gridDim.x * (256 * kMany)) {
        const int64_t row0 = base / a.chunks;                    // of the workgroup; a lane's own by a short division
        const int c0 = (int)(base - row0 * a.chunks);
        Piece<TI> piece[kMany] = {};
        int64_t row[kMany], t[kMany];
        int chunk[kMany];
        uint32_t kept[kMany];
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            const int off = c0 + q * 256 + (int)threadIdx.x;     // below 2^17 + 512: the quotient is exact
            const int down = (int)(((float)off + 0.5f) * a.inverse);
            row[q] = row0 + down;
            chunk[q] = off - down * a.chunks;
            t[q] = a.tokens.at(row[q] < a.n ? row[q] : a.n - 1);
        }
        if (a.rows > 0)
#pragma unroll
            for (int q = 0; q < kMany; ++q) piece[q].load(a, t[q] >= 0 && t[q] < a.rows ? t[q] : 0, chunk[q]);     // padding: the first row, not used
#pragma unroll
        for (int q = 0; q < kMany; ++q) kept[q] = kDrop ? kept_eight(key, (uint32_t)chunk[q], (uint32_t)row[q]) : 0xFFu;
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            if (row[q] >= a.n) continue;
            float x[8];
            piece[q].numbers(x, a, chunk[q]);
            const uint32_t used = t[q] >= 0 && t[q] < a.rows ? kept[q] : 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = used >> j & 1u ? x[j] * a.factor : 0.0f;
            store_eight<TO>(static_cast<TO*>(a.out) + row[q] * a.out_stride + (int64_t)chunk[q] * 8, x, a.width - chunk[q] * 8);
        }
    }
}

}  // namespace same
