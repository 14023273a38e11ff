// Dropout from a counter-based generator: whether an element is kept follows from its place, so nothing is stored between a
// forward and a backward pass.
//
// Element (i, j) of a call's matrix has 32 random bits; it is kept where they are below round((1 - p) 2^32).  The bits of the
// columns 8 c .. 8 c + 7 come from two blocks of Philox4x32-10 under the call's seed at the counters (c, i, step, word) and
// (c, i, step, word | 2^27), word = 4 2^28 + the step's bits from 32 on (the sweeps' draws have the fields 0 to 3 there): column
// 8 c + e has half e % 2, the low one first, of word e / 2 of either block, those of the first on top.  The lower halves decide
// only where the upper ones equal the border's, once in 65,536 elements, so eight elements cost one block.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rng_binom.h"

namespace same {

struct Drop {
    uint32_t seed_lo, seed_hi;
    uint64_t step;
    const int64_t* step_at;      // device, added to step; or null
    uint32_t keep_hi, keep_lo;   // round((1 - p) 2^32) by halves: keep_hi in 0 .. 65536
};

// What a block's counter and key have in common for all elements.
struct DropKey {
    uint32_t k0, k1, c2, c3, keep_hi, keep_lo;
};

__device__ __forceinline__ DropKey drop_key(const Drop& d)
{
    const uint64_t step = d.step + (d.step_at ? (uint64_t)*d.step_at : 0ull);
    return {d.seed_lo, d.seed_hi, (uint32_t)step, 0x40000000u | ((uint32_t)(step >> 32) & 0x00FFFFFFu), d.keep_hi, d.keep_lo};
}

// Bit e: element 8 * chunk + e of row `row` is kept.
__device__ __forceinline__ uint32_t kept_eight(const DropKey& k, uint32_t chunk, uint32_t row)
{
    uint32_t x[4];
    philox4x32_10(chunk, row, k.c2, k.c3, k.k0, k.k1, x);
    uint32_t kept = 0u, least = ~0u;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        const uint32_t over = (e & 1 ? x[e / 2] >> 16 : x[e / 2] & 0xFFFFu) - k.keep_hi;      // negative: kept
        kept = __builtin_amdgcn_alignbit(kept, over, 31);                                     // kept << 1 | sign
        least = min(least, over);                                                             // 0: some element is on the border
    }
    if (least == 0u && k.keep_lo) {
        uint32_t y[4];
        philox4x32_10(chunk, row, k.c2, k.c3 | 0x08000000u, k.k0, k.k1, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t hi = e & 1 ? x[e / 2] >> 16 : x[e / 2] & 0xFFFFu, lo = e & 1 ? y[e / 2] >> 16 : y[e / 2] & 0xFFFFu;
            kept |= (hi == k.keep_hi && lo < k.keep_lo ? 1u : 0u) << e;
        }
    }
    return kept;
}

}  // namespace same
