// Tokens: ids of rows of a word table.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace same {

// Ids outside [0, rows) stand for no word (padding): a row of zeros, no gradient.
struct Tokens {
    const void* ids;      // [n] int32 or int64; null: token i is row i
    int32_t wide;         // ids are int64
    __device__ __forceinline__ int64_t at(int64_t i) const
    {
        if (!ids) return i;
        return wide ? static_cast<const int64_t*>(ids)[i] : (int64_t) static_cast<const int32_t*>(ids)[i];
    }
};

// A token on its way through the sort: its word and its place in the list, moved together (the scattered stores of a pass are what
// it waits for, and one of 8 bytes costs what one of 4 does).
struct alignas(8) Placed {
    int32_t word, pos;
};

}  // namespace same
