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

template <class TI, class TO, bool kDrop>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a)
{
    constexpr int kMany = 2;                                     // chunks of a thread
    DropKey key = {};
    if constexpr (kDrop) key = drop_key(a.drop);
    const int64_t all = a.n * a.chunks;
    for (int64_t base = (int64_t)blockIdx.x * (256 * kMany); base < all; base += (int64_t)gridDim.x * (256 * kMany)) {
        const int64_t row0 = base / a.chunks;                    // of the workgroup; a lane's own by a short division
        const int c0 = (int)(base - row0 * a.chunks);
        float x[kMany][8];
        int64_t row[kMany];
        int chunk[kMany];
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            const int off = c0 + q * 256 + (int)threadIdx.x;     // below 2^17 + 512: the quotient is exact
            const int down = (int)(((float)off + 0.5f) * a.inverse);
            row[q] = row0 + down;
            chunk[q] = off - down * a.chunks;
            const bool in = base + q * 256 + threadIdx.x < all;
            const int64_t t = in ? a.tokens.at(row[q]) : -1;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[q][j] = 0.0f;
            if (t >= 0 && t < a.rows) {
                if constexpr (__is_same(TI, MicroCode))
                    load_micro<8>(x[q], static_cast<const uint8_t*>(a.table) + t * a.stride, a.scales + t * (a.stride / 16), chunk[q] * 8);
                else if constexpr (__is_same(TI, GroupCode))
                    load_grouped(x[q], static_cast<const uint8_t*>(a.table) + t * a.stride, a.scales + t * a.scale_pitch, chunk[q], a.group_log2);
                else
                    load_eight<TI>(x[q], static_cast<const TI*>(a.table) + t * a.stride + (int64_t)chunk[q] * 8, a.width - chunk[q] * 8);
            }
        }
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            if (base + q * 256 + threadIdx.x >= all) continue;
            uint32_t kept = 0xFFu;
            if constexpr (kDrop) kept = kept_eight(key, (uint32_t)chunk[q], (uint32_t)row[q]);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[q][j] = kept >> j & 1u ? x[q][j] * a.factor : 0.0f;
            store_eight<TO>(static_cast<TO*>(a.out) + row[q] * a.out_stride + (int64_t)chunk[q] * 8, x[q], a.width - chunk[q] * 8);
        }
    }
}

}  // namespace same
