// The order of tokens by word, for the gradient of a word table.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tokens.h"

namespace same {

// Stable radix sort of the words by digits of `bits` bits (at most kDigitBits), least significant first.  A workgroup owns a
// tile of 256 * R consecutive tokens.  Per pass: counts per (digit, tile); for every digit their exclusive sum over the tiles (up to
// kFewTiles tiles the placement adds them up for itself); placement, which adds up the digits before its own.
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr uint32_t kFewTiles = 64;                               // 50,000 tokens x 64: 52 us; beyond it does not pay, 100,000: 60 us by itself, 55 in a launch

__device__ __forceinline__ int32_t word_of(const Tokens& tokens, int64_t i, int64_t rows)
{
    const int64_t t = tokens.at(i);
    return t >= 0 && t < rows ? (int32_t)t : (int32_t)rows;
}

// from null: the first pass takes the words from the tokens
template <int R>
__global__ __launch_bounds__(256) void token_histogram(Tokens tokens, int64_t rows, const Placed* __restrict__ from, int64_t n, int shift, int bits,
                                                       uint32_t tiles, uint32_t* __restrict__ hist)   // tiles: a multiple of 4, the last ones may be empty
{
    __shared__ uint32_t h[kDigits];
    const uint32_t digits = 1u << bits;
    for (uint32_t d = threadIdx.x; d < digits; d += 256) h[d] = 0u;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * (256 * R);
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int64_t i = first + (int64_t)j * 256 + threadIdx.x;
        if (i < n) {
            const int32_t key = from ? from[i].word : word_of(tokens, i, rows);
            atomicAdd(&h[((uint32_t)key >> shift) & (digits - 1u)], 1u);
        }
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += 256) hist[(size_t)d * tiles + blockIdx.x] = h[d];
}

// Workgroup d: the counts of digit d in every tile become the number of its tokens in the tiles before, total[d] their number.
__global__ __launch_bounds__(256) void token_offsets(uint32_t* __restrict__ hist, uint32_t tiles, uint32_t* __restrict__ total)
{
    __shared__ uint32_t wave_total[4];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    uint32_t* const mine = hist + (size_t)blockIdx.x * tiles;
    uint32_t base = 0;
    for (uint32_t first = 0; first < tiles; first += 256) {
        const uint32_t at = first + threadIdx.x, x = at < tiles ? mine[at] : 0u;
        uint32_t incl = x;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 63) wave_total[wv] = incl;
        __syncthreads();
        uint32_t before = base;
        for (int i = 0; i < 4; ++i) { if (i < wv) before += wave_total[i]; base += wave_total[i]; }
        if (at < tiles) mine[at] = before + incl - x;
        __syncthreads();
    }
    if (threadIdx.x == 0) total[blockIdx.x] = base;
}

// A token's place: the tokens of lower digits, those of its digit in the tiles before, in the waves before its own, in the
// earlier rows of its wave and in the lower lanes of its row.
template <int R, bool kFew>
__global__ __launch_bounds__(256) void token_place(Tokens tokens, int64_t rows, const Placed* __restrict__ from, int64_t n, int shift, int bits, uint32_t tiles, const uint32_t* __restrict__ start,
                                                   const uint32_t* __restrict__ total, Placed* __restrict__ to)
{
    __shared__ uint32_t cnt[4][kDigits];
    __shared__ uint32_t wave_total[4];
    const uint32_t digits = 1u << bits;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (uint32_t d = lane; d < digits; d += 64) cnt[wv][d] = 0u;
    const uint32_t d0 = 2u * threadIdx.x;                          // a thread's two digits
    uint32_t t0 = 0u, t1 = 0u, p0 = 0u, p1 = 0u;                   // their tokens, and those of them in the tiles before
    if constexpr (kFew) {
        const auto sums = [&](uint32_t d, uint32_t& all, uint32_t& before) {
            const uint4* const row = reinterpret_cast<const uint4*>(start + (size_t)d * tiles);
#pragma unroll 4
            for (uint32_t q = 0; q < tiles / 4u; ++q) {
                const uint4 c = row[q];
                const uint32_t x[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                for (uint32_t j = 0; j < 4u; ++j) { all += x[j]; before += 4u * q + j < blockIdx.x ? x[j] : 0u; }
            }
        };
        if (d0 < digits) sums(d0, t0, p0);
        if (d0 + 1u < digits) sums(d0 + 1u, t1, p1);
    } else {
        if (d0 < digits) { t0 = total[d0]; p0 = start[(size_t)d0 * tiles + blockIdx.x]; }
        if (d0 + 1u < digits) { t1 = total[d0 + 1u]; p1 = start[(size_t)(d0 + 1u) * tiles + blockIdx.x]; }
    }
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * (256 * R) + (int64_t)wv * (R * 64) + lane;
    Placed x[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int64_t i = first + (int64_t)j * 64;
        const bool in = i < n;
        x[j] = !in ? Placed{0, 0} : from ? from[i] : Placed{word_of(tokens, i, rows), (int32_t)i};
        if (in) atomicAdd(&cnt[wv][((uint32_t)x[j].word >> shift) & (digits - 1u)], 1u);
    }
    uint32_t incl = t0 + t1;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o);
        if (lane >= o) incl += up;
    }
    if (lane == 63) wave_total[wv] = incl;
    __syncthreads();
    uint32_t below_digit = incl - t0 - t1;
    for (int i = 0; i < wv; ++i) below_digit += wave_total[i];
    p0 += below_digit;
    p1 += below_digit + t0;
    if (d0 < digits)
        for (int v = 0; v < 4; ++v) { const uint32_t c = cnt[v][d0]; cnt[v][d0] = p0; p0 += c; }
    if (d0 + 1u < digits)
        for (int v = 0; v < 4; ++v) { const uint32_t c = cnt[v][d0 + 1u]; cnt[v][d0 + 1u] = p1; p1 += c; }
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const bool in = first + (int64_t)j * 64 < n;
        const uint32_t dgt = ((uint32_t)x[j].word >> shift) & (digits - 1u);
        uint64_t peers = __ballot(in);                             // the lanes of this row that hold the same digit
        for (int bit = 0; bit < bits; ++bit) {
            const bool one = (dgt >> bit) & 1u;
            const uint64_t m = __ballot(one);
            peers &= one ? m : ~m;
        }
        if (in) {
            const uint32_t rank = (uint32_t)__popcll((unsigned long long)(peers & below));
            const uint32_t p = cnt[wv][dgt] + rank;                // every peer reads the place before the first one moves it on
            if (rank == 0u) cnt[wv][dgt] = p + (uint32_t)__popcll((unsigned long long)peers);
            if ((int64_t)p < n) to[p] = x[j];                      // always true; keeps a wrong count from becoming a wild store
        }
    }
}

// start[w] = first place of word w among the sorted tokens, rows + 1 entries (the last: the number of tokens of any word).  The
// token at place p writes the entries of the words after its predecessor's up to its own, the end those after the last: a few each
// where tokens are many, and the lanes of a wave share a long gap.
__global__ __launch_bounds__(256) void word_runs(const Placed* __restrict__ sorted, int64_t n, int64_t rows, int32_t* __restrict__ start)
{
    constexpr int64_t kOwn = 8;
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    int64_t lo = 0, hi = -1;                                       // first and last word to write
    if (p <= n) {
        lo = p > 0 ? (int64_t)sorted[p - 1].word + 1 : 0;
        hi = p < n ? sorted[p].word : rows;
    }
    for (int64_t w = lo; w <= hi && w < lo + kOwn; ++w) start[w] = (int32_t)p;
    uint64_t wide = __ballot(hi - lo >= kOwn);
    const int lane = threadIdx.x & 63;
    while (wide) {
        const int from = __builtin_ctzll(wide);
        wide &= wide - 1ull;
        const int64_t first = __shfl((long long)lo, from) + kOwn, last = __shfl((long long)hi, from), q = __shfl((long long)p, from);
        for (int64_t w = first + lane; w <= last; w += 64) start[w] = (int32_t)q;
    }
}

// The same where words are many for the tokens (16,385 in 140,000: 16 us by gaps): every word looks for its place.
__global__ __launch_bounds__(256) void word_runs_sparse(const Placed* __restrict__ sorted, int64_t n, int64_t rows, int32_t* __restrict__ start)
{
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w > rows) return;
    int64_t lo = 0, hi = n;
    while (lo < hi) { const int64_t mid = (lo + hi) >> 1; if (sorted[mid].word < (int32_t)w) lo = mid + 1; else hi = mid; }
    start[w] = (int32_t)lo;
}

}  // namespace same
