// Lookup of a word table's rows for a list of tokens, and the table's gradient by sorted tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "element.h"
#include "micro_format.h"

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

// ---- out[i] = scale * table[token i], one rounding in binary32 and one to the output's type.  A row is taken by a group of
// 2^lanes_log2 lanes, a chunk of V elements per lane and trip.  Memory bound: the table's rows once, the output once.
struct EmbedArgs {
    const void* table;
    const uint8_t* scales;   // microscaled tables
    int64_t rows, stride;    // stride in elements (microscaled: in bytes of codes)
    Tokens tokens;
    int64_t n;
    float scale;
    void* out;
    int64_t out_stride;
    int32_t chunks;          // chunks of a row
    int32_t lanes_log2;
};

template <class TI, class TO, int V>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t step = (int64_t)gridDim.x << (8 - a.lanes_log2);
    for (int64_t i = ((int64_t)blockIdx.x << (8 - a.lanes_log2)) + (threadIdx.x >> a.lanes_log2); i < a.n; i += step) {
        const int64_t t = a.tokens.at(i);
        const bool known = t >= 0 && t < a.rows;
        TO* const to = static_cast<TO*>(a.out) + i * a.out_stride;
        for (int c = lane; c < a.chunks; c += lanes) {
            float x[V];
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = 0.0f;
            if (known) {
                if constexpr (sizeof(TI) == 1) load_micro<V>(x, static_cast<const uint8_t*>(a.table) + t * a.stride, a.scales + t * (a.stride / 16), c * V);
                else                           load_chunk<TI, V>(x, static_cast<const TI*>(a.table) + t * a.stride + c * V);
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] *= a.scale;
            }
            store_chunk<TO, V>(to + c * V, x);
        }
    }
}

// ---- Gradient.  The tokens are sorted by word, stable, with the padding behind the last word; the positions of one word are
// then a run in ascending order, and its row of the gradient is one sum over the run in binary32, in an order that depends
// on the tokens alone (no atomics: two calls give the same bits).

// Stable radix sort of the words by digits of `bits` bits (at most kDigitBits), least significant first.  A workgroup owns a
// tile of consecutive tokens.  Per pass: counts per (digit, tile); their exclusive sum in that order; placement.
constexpr int kTileTokens = 4096;
constexpr int kTileRows = kTileTokens / 256;
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;

__device__ __forceinline__ int32_t word_of(const Tokens& tokens, int64_t i, int64_t rows)
{
    const int64_t t = tokens.at(i);
    return t >= 0 && t < rows ? (int32_t)t : (int32_t)rows;
}

// keys null: the first pass takes the words from the tokens
__global__ __launch_bounds__(256) void token_histogram(Tokens tokens, int64_t rows, const int32_t* __restrict__ keys, int64_t n, int shift, int bits,
                                                       uint32_t tiles, uint32_t* __restrict__ hist)
{
    __shared__ uint32_t h[kDigits];
    const uint32_t digits = 1u << bits;
    for (uint32_t d = threadIdx.x; d < digits; d += 256) h[d] = 0u;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTileTokens;
    for (int j = 0; j < kTileRows; ++j) {
        const int64_t i = first + (int64_t)j * 256 + threadIdx.x;
        if (i < n) {
            const int32_t key = keys ? keys[i] : word_of(tokens, i, rows);
            atomicAdd(&h[((uint32_t)key >> shift) & (digits - 1u)], 1u);
        }
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += 256) hist[(size_t)d * tiles + blockIdx.x] = h[d];
}

// exclusive sum in place, by one workgroup
__global__ __launch_bounds__(1024) void token_offsets(uint32_t* __restrict__ hist, int64_t cells)
{
    __shared__ uint32_t wave_total[16];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    uint32_t base = 0;
    for (int64_t first = 0; first < cells; first += 4096) {
        const int64_t at = first + threadIdx.x * 4;
        uint32_t x[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[j] = at + j < cells ? hist[at + j] : 0u; mine += x[j]; }
        uint32_t incl = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 63) wave_total[wv] = incl;
        __syncthreads();
        uint32_t before = base, all = base;
        for (int i = 0; i < 16; ++i) { if (i < wv) before += wave_total[i]; all += wave_total[i]; }
        uint32_t run = before + incl - mine;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (at + j < cells) hist[at + j] = run;
            run += x[j];
        }
        base = all;
        __syncthreads();
    }
}

// A token's place: the start of its (digit, tile) run, plus the tokens of the same digit in the waves before its own, in the
// earlier rows of its wave and in the lower lanes of its row.
__global__ __launch_bounds__(256) void token_place(Tokens tokens, int64_t rows, const int32_t* __restrict__ keys_in, const int32_t* __restrict__ pos_in,
                                                   int64_t n, int shift, int bits, uint32_t tiles, const uint32_t* __restrict__ start,
                                                   int32_t* __restrict__ keys_out, int32_t* __restrict__ pos_out)
{
    __shared__ uint32_t cnt[4][kDigits];
    const uint32_t digits = 1u << bits;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (uint32_t d = lane; d < digits; d += 64) cnt[wv][d] = 0u;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTileTokens + (int64_t)wv * (kTileRows * 64) + lane;
    int32_t key[kTileRows], pos[kTileRows];
#pragma unroll
    for (int j = 0; j < kTileRows; ++j) {
        const int64_t i = first + (int64_t)j * 64;
        const bool in = i < n;
        key[j] = in ? (keys_in ? keys_in[i] : word_of(tokens, i, rows)) : 0;
        pos[j] = in ? (pos_in ? pos_in[i] : (int32_t)i) : 0;
        if (in) atomicAdd(&cnt[wv][((uint32_t)key[j] >> shift) & (digits - 1u)], 1u);
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += 256) {
        uint32_t p = start[(size_t)d * tiles + blockIdx.x];
        for (int v = 0; v < 4; ++v) { const uint32_t c = cnt[v][d]; cnt[v][d] = p; p += c; }
    }
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
    for (int j = 0; j < kTileRows; ++j) {
        const bool in = first + (int64_t)j * 64 < n;
        const uint32_t dgt = ((uint32_t)key[j] >> shift) & (digits - 1u);
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
            if ((int64_t)p < n) {                                  // always true; keeps a wrong count from becoming a wild store
                keys_out[p] = key[j];
                pos_out[p] = pos[j];
            }
        }
    }
}

// start[w] = first place of word w among the sorted tokens, rows + 1 entries (the last: the number of tokens of any word)
__global__ __launch_bounds__(256) void word_runs(const int32_t* __restrict__ keys, int64_t n, int64_t rows, int32_t* __restrict__ start)
{
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w > rows) return;
    int64_t lo = 0, hi = n;
    while (lo < hi) { const int64_t mid = (lo + hi) >> 1; if (keys[mid] < (int32_t)w) lo = mid + 1; else hi = mid; }
    start[w] = (int32_t)lo;
}

// A run of more than kLongRun tokens is cut at the multiples of kLongRun: group j sums the places [j, j + 1) * kLongRun of long
// runs into two rows of partial sums (2j: the run that the range begins in, 2j + 1: a long run that starts behind the
// range's first place; such a run goes on behind the range's end, so there is one at most).  Short runs are summed by
// the group of their word.
constexpr int kLongRun = 256;

struct GradArgs {
    const void* grad;
    int64_t stride;
    const int32_t* pos;      // [n] sorted tokens: their places in the list
    const int32_t* keys;     // [n] and their words
    const int32_t* start;    // [rows + 1]
    int64_t rows;
    float scale;
    int32_t accumulate;
    void* out;
    int64_t out_stride;
    float* partial;          // [2 * ranges][width]
    int64_t ranges;
    int32_t width, chunks, lanes_log2;
};

template <class TI, int V>
__device__ __forceinline__ void sum_run(float (&acc)[V], const GradArgs& a, int64_t lo, int64_t hi, int c)
{
    const TI* const from = static_cast<const TI*>(a.grad) + c * V;
    int64_t p = lo;
    for (; p + 4 <= hi; p += 4) {
        float x[4][V];
#pragma unroll
        for (int q = 0; q < 4; ++q) load_chunk<TI, V>(x[q], from + (int64_t)a.pos[p + q] * a.stride);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += x[q][j];
    }
    for (; p < hi; ++p) {
        float x[V];
        load_chunk<TI, V>(x, from + (int64_t)a.pos[p] * a.stride);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += x[j];
    }
}

template <class TO, int V>
__device__ __forceinline__ void write_row(const GradArgs& a, int64_t w, int c, float (&acc)[V], bool any)
{
    TO* const to = static_cast<TO*>(a.out) + w * a.out_stride + c * V;
    if (a.accumulate) {
        if (!any) return;
        float old[V];
        load_chunk<TO, V>(old, to);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = old[j] + a.scale * acc[j];
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] *= a.scale;
    }
    store_chunk<TO, V>(to, acc);
}

template <class TI, class TO, int V>
__global__ __launch_bounds__(256) void embed_grad_kernel(GradArgs a)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int c = blockIdx.y * lanes + lane;
    const int64_t item0 = ((int64_t)blockIdx.x << (8 - a.lanes_log2)) + (threadIdx.x >> a.lanes_log2);
    if (c >= a.chunks) return;
    for (int64_t item = item0; item < a.ranges + a.rows; item += (int64_t)gridDim.x << (8 - a.lanes_log2)) {
        if (item < a.ranges) {
            const int64_t n = a.start[a.rows], lo = item * kLongRun;
            if (lo >= n) continue;
            const int64_t hi = lo + kLongRun < n ? lo + kLongRun : n;
            const int32_t w0 = a.keys[lo], w1 = a.keys[hi - 1];
            const int64_t s0 = a.start[w0], e0 = a.start[w0 + 1];
            if (e0 - s0 > kLongRun) {
                float acc[V] = {};
                sum_run<TI, V>(acc, a, lo, e0 < hi ? e0 : hi, c);
                store_chunk<float, V>(a.partial + (size_t)(2 * item) * a.width + c * V, acc);
            }
            const int64_t s1 = a.start[w1], e1 = a.start[w1 + 1];
            if (w1 != w0 && e1 - s1 > kLongRun) {
                float acc[V] = {};
                sum_run<TI, V>(acc, a, s1, hi, c);
                store_chunk<float, V>(a.partial + (size_t)(2 * item + 1) * a.width + c * V, acc);
            }
        } else {
            const int64_t w = item - a.ranges, lo = a.start[w], hi = a.start[w + 1];
            if (hi - lo > kLongRun) continue;
            float acc[V] = {};
            sum_run<TI, V>(acc, a, lo, hi, c);
            write_row<TO, V>(a, w, c, acc, hi > lo);
        }
    }
}

// The row of the long run that starts in range blockIdx.x, if there is one: its partial sums in order.
template <class TO, int V>
__global__ __launch_bounds__(256) void embed_grad_join_kernel(GradArgs a)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int c = blockIdx.y * lanes + lane;
    const int64_t item0 = ((int64_t)blockIdx.x << (8 - a.lanes_log2)) + (threadIdx.x >> a.lanes_log2);
    if (c >= a.chunks) return;
    const int64_t n = a.start[a.rows];
    for (int64_t item = item0; item * kLongRun < n; item += (int64_t)gridDim.x << (8 - a.lanes_log2)) {
        const int64_t first = item * kLongRun, behind = first + kLongRun < n ? first + kLongRun : n;
        int32_t w = a.keys[behind - 1];
        const int64_t s = a.start[w], e = a.start[w + 1];
        if (s < first || e - s <= kLongRun) continue;
        float acc[V];
        load_chunk<float, V>(acc, a.partial + (size_t)(s == first ? 2 * item : 2 * item + 1) * a.width + c * V);
        for (int64_t r = item + 1; r * kLongRun < e; ++r) {
            float x[V];
            load_chunk<float, V>(x, a.partial + (size_t)(2 * r) * a.width + c * V);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += x[j];
        }
        write_row<TO, V>(a, w, c, acc, true);
    }
}

}  // namespace same
