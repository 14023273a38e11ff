// Rows of a table for a list of tokens (or a matrix as it is) with dropout, and rows of tables in grouped four-bit integers.
//
// A lane takes eight elements of a row, which a block of the generator decides and one vector load and store move (two of each in binary32),
// and two such pieces at once, both loads on their way before the generators' rounds.  Bound by memory: 65,536 x 1024 bf16 48 us, 5.6 TB/s
// read and written; 131,072 rows of 100,000 x 1024 bf16 93 us, 77 without dropout, a good half of whose rows come from the caches.  131,072 rows
// into bf16 out of groups of 64 take 69 us, 3.9 TB/s of stores where a fill reaches 6.8: a lane asks for 4 bytes of codes and 4 of a step and a base
// for 16 that it stores; with dropout 81, out of microscaled rows 82.
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
    int32_t step_rows, step_chunks;   // what all workgroups take at once, kChunksAtOnce each, in rows and chunks
    Drop drop;
};

struct MicroCode {};         // type of a table in microscaled four bits,
struct GroupCode {};         // in grouped four-bit integers

// Eight elements of a row of the table, as they come from memory.
template <class TI>
struct Piece {
    Eight<TI> c;
    __device__ __forceinline__ void load(const RowsArgs& a, int32_t t, int chunk) { c = eight_at(static_cast<const TI*>(a.table) + (int64_t)t * a.stride, chunk * 8, a.width); }
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
    __device__ __forceinline__ void load(const RowsArgs& a, int32_t t, int chunk)
    {
        load_micro<8>(x, static_cast<const uint8_t*>(a.table) + (int64_t)t * a.stride, a.scales + (int64_t)t * (a.stride / 16), chunk * 8);
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
    __device__ __forceinline__ void load(const RowsArgs& a, int32_t t, int chunk)
    {
        word = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(a.table) + (int64_t)t * a.stride)[group_word(chunk)];
        sb = reinterpret_cast<const uint32_t*>(a.scales + (int64_t)t * a.scale_pitch)[chunk >> (a.group_log2 - 3)];
    }
    __device__ __forceinline__ void numbers(float (&x)[8], const RowsArgs&, int) { grouped_numbers(x, word, sb); }
};

// A thread takes kMany chunks at a time: their tokens, their rows and, while these are on their way, what is kept of them.  Bound by memory
// without dropout, with it by the generator as well (some 70 instructions for eight elements).
constexpr int kMany = 2, kChunksAtOnce = 256 * kMany;

template <class TI, class TO, bool kDrop>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a)
{
    DropKey key = {};
    if constexpr (kDrop) key = drop_key(a.drop);
    const int64_t begin = (int64_t)blockIdx.x * kChunksAtOnce;
    uint32_t row0 = (uint32_t)(begin / a.chunks);                // of the workgroup; a lane's own by a short division
    int c0 = (int)(begin - (int64_t)row0 * a.chunks);
    const uint32_t n = (uint32_t)a.n, rows = (uint32_t)a.rows;   // below 2^31
    while (row0 < n) {
        Piece<TI> piece[kMany] = {};
        uint32_t row[kMany], kept[kMany][4];
        int32_t t[kMany];
        int chunk[kMany];
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            const int off = c0 + q * 256 + (int)threadIdx.x;     // below 2^17 + 512: the quotient is exact
            const int down = (int)(((float)off + 0.5f) * a.inverse);
            row[q] = row0 + (uint32_t)down;
            chunk[q] = off - down * a.chunks;
            t[q] = (int32_t)min(row[q], n - 1u);
        }
        if (a.tokens.ids) {                                      // all of them on their way at once
            if (a.tokens.wide) {
                int64_t id[kMany];
#pragma unroll
                for (int q = 0; q < kMany; ++q) id[q] = static_cast<const int64_t*>(a.tokens.ids)[t[q]];
#pragma unroll
                for (int q = 0; q < kMany; ++q) t[q] = id[q] >= 0 && id[q] < a.rows ? (int32_t)id[q] : -1;
            } else {
                int32_t id[kMany];
#pragma unroll
                for (int q = 0; q < kMany; ++q) id[q] = static_cast<const int32_t*>(a.tokens.ids)[t[q]];
#pragma unroll
                for (int q = 0; q < kMany; ++q) t[q] = (uint32_t)id[q] < rows ? id[q] : -1;
            }
        }
        if (rows > 0)
#pragma unroll
            for (int q = 0; q < kMany; ++q) piece[q].load(a, max(t[q], 0), chunk[q]);          // padding: the first row, not used
#pragma unroll
        for (int q = 0; q < kMany; ++q)
            if constexpr (kDrop) kept_halves(kept[q], key, (uint32_t)chunk[q], row[q]);
#pragma unroll
        for (int q = 0; q < kMany; ++q) {
            if (row[q] >= n) continue;
            float x[8];
            piece[q].numbers(x, a, chunk[q]);
            const uint32_t known = t[q] >= 0 ? ~0u : 0u;
            Eight<TO> out;
#pragma unroll
            for (int j = 0; j < 8; ++j) out.v[j] = (TO)(x[j] * a.factor);
            uint32_t w[sizeof(TO) * 2];
            __builtin_memcpy(w, out.v, sizeof w);
#pragma unroll
            for (int j = 0; j < (int)(sizeof(TO) * 2); ++j) {                  // two elements a word, or one
                uint32_t mask = known;
                if constexpr (kDrop) mask &= sizeof(TO) == 2 ? kept[q][j & 3] : (uint32_t)((int32_t)(j & 1 ? kept[q][j / 2] : kept[q][j / 2] << 16) >> 16);
                w[j] &= mask;
            }
            __builtin_memcpy(out.v, w, sizeof w);
            TO* const to = static_cast<TO*>(a.out) + (int64_t)row[q] * a.out_stride + chunk[q] * 8;
            const int count = a.width - chunk[q] * 8;
            if (count >= 8) {
                out.store(to);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < count) to[j] = out.v[j];
            }
        }
        row0 += (uint32_t)a.step_rows;
        c0 += a.step_chunks;
        if (c0 >= a.chunks) {
            c0 -= a.chunks;
            ++row0;
        }
    }
}

}  // namespace same
