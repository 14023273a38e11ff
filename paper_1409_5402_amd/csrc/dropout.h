// Dropout from a counter-based generator: whether an element is kept follows from its place, so nothing is stored between a
// forward and a backward pass.
//
// Element (i, j) of a call's matrix has 32 random bits; it is kept where they are below round((1 - p) 2^32).  The bits of the
// columns 8 c .. 8 c + 7 come from two blocks of Philox4x32-10 under the call's seed at the counters (c, i, step, word) and
// (c, i, step, word | 2^27), word = 4 2^28 + the step's bits from 32 on (the sweeps' draws have the fields 0 to 3 there): column
// 8 c + e has half e % 2, the low one first, of word e / 2 of either block, those of the first on top.  The lower halves decide
// only where the upper ones equal the border's, once in 65,536 elements, so eight elements cost one block (65,536 x 1024 bf16: 57 us with a
// comparison and a bit for each, 48 to 50 by halves of registers, which a copy takes too).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rng_binom.h"

namespace same {

struct Drop {
    uint32_t seed_lo, seed_hi;
    uint64_t step;
    const int64_t* step_at;      // device, added to step; or null
    uint32_t keep_hi, keep_lo;   // round((1 - p) 2^32) = 65536 keep_hi + keep_lo: keep_hi in 0 .. 65535, keep_lo in 0 .. 65536
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

typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));

// All ones in half e % 2 of word e / 2 where element 8 * chunk + e of row `row` is kept, else zeros.
__device__ __forceinline__ void kept_halves(uint32_t (&kept)[4], const DropKey& k, uint32_t chunk, uint32_t row)
{
    uint32_t x[4];
    philox4x32_10(chunk, row, k.c2, k.c3, k.k0, k.k1, x);
    const v2u16 border = {(uint16_t)k.keep_hi, (uint16_t)k.keep_hi}, one = {1, 1};
    v2u16 least = {0xFFFF, 0xFFFF};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const v2u16 half = __builtin_bit_cast(v2u16, x[w]);
        v2u16 over;                                                                           // 0 up to the border (the compiler takes the vectors apart)
        asm("v_pk_sub_u16 %0, %1, %2 clamp" : "=v"(over) : "v"(half), "v"(border));
        kept[w] = __builtin_bit_cast(uint32_t, (v2u16)(__builtin_elementwise_min(over, one) - one));
        least = __builtin_elementwise_min(least, (v2u16)(half ^ border));                     // 0: on it
    }
    const uint32_t on = __builtin_bit_cast(uint32_t, least);
    if ((on & 0xFFFFu) == 0u || (on >> 16) == 0u) {                                           // one chunk in 8192
        uint32_t y[4];
        philox4x32_10(chunk, row, k.c2, k.c3 | 0x08000000u, k.k0, k.k1, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int w = e / 2, up = 16 * (e % 2);
            if ((x[w] >> up & 0xFFFFu) == k.keep_hi && (y[w] >> up & 0xFFFFu) >= k.keep_lo) kept[w] &= ~(0xFFFFu << up);
        }
    }
}

// Bit e: element 8 * chunk + e of row `row` is kept.
__device__ __forceinline__ uint32_t kept_eight(const DropKey& k, uint32_t chunk, uint32_t row)
{
    uint32_t kept[4];
    kept_halves(kept, k, chunk, row);
    const uint32_t bits = (kept[0] & 0x00020001u) | (kept[1] & 0x00080004u) | (kept[2] & 0x00200010u) | (kept[3] & 0x00800040u);
    return (bits | bits >> 16) & 0xFFu;
}

// x where bit j of kept is set, else 0
__device__ __forceinline__ float if_kept(float x, uint32_t kept, int j)
{
    return __uint_as_float(__float_as_uint(x) & (uint32_t)((int32_t)(kept << (31 - j)) >> 31));
}

}  // namespace same
