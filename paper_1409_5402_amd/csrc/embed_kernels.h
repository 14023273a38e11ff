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

// Two tokens and two chunks of their rows at once: with one load on its way per lane 262,144 rows of 1024 bf16 took 158 us, now 154 us.
template <class TI, class TO, int V>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a)
{
    constexpr int kTokens = 2, kChunks = 2;
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t step = (int64_t)gridDim.x << (8 - a.lanes_log2);
    for (int64_t i = ((int64_t)blockIdx.x << (8 - a.lanes_log2)) + (threadIdx.x >> a.lanes_log2); i < a.n; i += kTokens * step) {
        int64_t row[kTokens];
        bool known[kTokens];
#pragma unroll
        for (int q = 0; q < kTokens; ++q) {
            row[q] = i + q * step < a.n ? a.tokens.at(i + q * step) : -1;
            known[q] = row[q] >= 0 && row[q] < a.rows;
        }
        for (int c = lane; c < a.chunks; c += kChunks * lanes) {
            float x[kTokens][kChunks][V];
#pragma unroll
            for (int q = 0; q < kTokens; ++q)
#pragma unroll
                for (int h = 0; h < kChunks; ++h) {
                    const int at = c + h * lanes;
#pragma unroll
                    for (int j = 0; j < V; ++j) x[q][h][j] = 0.0f;
                    if (known[q] && at < a.chunks) {
                        if constexpr (sizeof(TI) == 1)
                            load_micro<V>(x[q][h], static_cast<const uint8_t*>(a.table) + row[q] * a.stride, a.scales + row[q] * (a.stride / 16), at * V);
                        else
                            load_chunk<TI, V>(x[q][h], static_cast<const TI*>(a.table) + row[q] * a.stride + (int64_t)at * V);
                    }
                }
#pragma unroll
            for (int q = 0; q < kTokens; ++q)
#pragma unroll
                for (int h = 0; h < kChunks; ++h) {
                    const int at = c + h * lanes;
                    if (i + q * step >= a.n || at >= a.chunks) continue;
#pragma unroll
                    for (int j = 0; j < V; ++j) x[q][h][j] *= a.scale;
                    store_chunk<TO, V>(static_cast<TO*>(a.out) + (i + q * step) * a.out_stride + (int64_t)at * V, x[q][h]);
                }
        }
    }
}

// ---- Gradient.  The tokens are sorted by word, stable, with the padding behind the last word; the positions of one word are
// then a run in ascending order, and its row of the gradient is one sum over the run in binary32.  The order of its additions
// depends on the tokens, and on whether they are taken in one launch (their number, the bytes of a row of grad, the table's size);
// not on how rows are cut into chunks and lanes, which addresses and strides decide, and no atomics: equal numbers, equal bits.

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

// A token on its way through the sort: its word and its place in the list, moved together (the scattered stores of a pass are what
// it waits for, and one of 8 bytes costs what one of 4 does).
struct alignas(8) Placed {
    int32_t word, pos;
};

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

// A run of more than kLongRun tokens is cut at the multiples of kLongRun: group j sums the places [j, j + 1) * kLongRun of long
// runs into two rows of partial sums (2j: the run that the range begins in, 2j + 1: a long run that starts behind the
// range's first place; such a run goes on behind the range's end, so there is one at most).  Short runs are summed by
// the group of their word.  A sum takes its rows eight at a time, a trip to memory each: with 64 tokens the longest
// chain is eight trips, with 256 the hottest words' chains were what a batch of 65,537 tokens waited for.
constexpr int kLongRun = 64;

struct GradArgs {
    const void* grad;
    int64_t stride;
    const Placed* sorted;    // [n]
    const int32_t* start;    // [rows + 1]
    int64_t rows;
    float scale;
    int32_t accumulate;
    void* out;
    int64_t out_stride;
    float* partial;          // [2 * ranges][width]
    int64_t ranges;
    int32_t width, chunks, lanes_log2;
    Tokens tokens;           // few tokens only: the list itself,
    int32_t n;               // its length
    int32_t words;           // the words of a workgroup, at most
    int32_t unit_log2;
};

// acc += the rows at places at(0) .. at(count - 1) of the list, count in [1, N]: all loads before the first addition (at(q) is a
// place to read from for q >= count too)
template <class TI, int V, int N, class At>
__device__ __forceinline__ void add_rows(float (&acc)[V], const TI* __restrict__ from, int64_t stride, int count, At at)
{
    float x[N][V];
#pragma unroll
    for (int q = 0; q < N; ++q) load_chunk<TI, V>(x[q], from + (int64_t)at(q) * stride);
#pragma unroll
    for (int q = 0; q < N; ++q)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = q < count ? acc[j] + x[q][j] : acc[j];
}

// By the 2^lanes_log2 lanes of a group, all of them active: a lane fetches one place of the run for all, or, where lanes are few,
// each fetches eight, those of the next rows while these are on their way (16,385 tokens into 140,000 x 16: 24 us with one place
// per lane and four lanes, now 15).
template <class TI, int V, bool kNarrow>
__device__ __forceinline__ void sum_run(float (&acc)[V], const GradArgs& a, int64_t lo, int64_t hi, int c)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const TI* const from = static_cast<const TI*>(a.grad) + (int64_t)c * V;
    if constexpr (kNarrow) {
        if (lo >= hi) return;
        int32_t place[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) place[q] = a.sorted[lo + q < hi ? lo + q : hi - 1].pos;
        for (int64_t p = lo; p < hi; p += 8) {
            int32_t here[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) here[q] = place[q];
            if (p + 8 < hi)
#pragma unroll
                for (int q = 0; q < 8; ++q) place[q] = a.sorted[p + 8 + q < hi ? p + 8 + q : hi - 1].pos;
            const auto at = [&](int i) { return here[i]; };
            const int left = hi - p < 8 ? (int)(hi - p) : 8;
            if (left > 2) add_rows<TI, V, 8>(acc, from, a.stride, left, at);
            else          add_rows<TI, V, 2>(acc, from, a.stride, left, at);
        }
        return;
    }
    for (int64_t base = lo; base < hi; base += lanes) {
        const int here = hi - base < lanes ? (int)(hi - base) : lanes;
        const int32_t mine = a.sorted[base + (lane < here ? lane : here - 1)].pos;
        for (int q = 0; q < here; q += 8) {
            const auto at = [&](int i) { return __shfl(mine, q + i < here ? q + i : here - 1, lanes); };
            const int left = here - q;
            if (left > 4)       add_rows<TI, V, 8>(acc, from, a.stride, left < 8 ? left : 8, at);
            else if (left > 2)  add_rows<TI, V, 4>(acc, from, a.stride, left, at);
            else if (left == 2) add_rows<TI, V, 2>(acc, from, a.stride, 2, at);
            else                add_rows<TI, V, 1>(acc, from, a.stride, 1, at);
        }
    }
}

template <class TO, int V>
__device__ __forceinline__ void write_row(const GradArgs& a, int64_t w, int c, float (&acc)[V], bool any)
{
    TO* const to = static_cast<TO*>(a.out) + w * a.out_stride + (int64_t)c * V;
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

// Memory bound where tokens are many: a million rows of 256 binary32 take 243 us, 4.6 TB/s of what has to be read and written;
// 65,537 rows of 1024 bf16 37 us, 5.3 TB/s.
template <class TI, class TO, int V, bool kNarrow>
__global__ __launch_bounds__(256) void embed_grad_kernel(GradArgs a)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int column = blockIdx.y * lanes + lane;
    const bool mine = column < a.chunks;
    const int c = mine ? column : a.chunks - 1;                     // lanes behind the row's end follow its last chunk and write nothing
    const int64_t item0 = ((int64_t)blockIdx.x << (8 - a.lanes_log2)) + (threadIdx.x >> a.lanes_log2);
    for (int64_t item = item0; item < a.ranges + a.rows; item += (int64_t)gridDim.x << (8 - a.lanes_log2)) {
        if (item < a.ranges) {
            const int64_t n = a.start[a.rows], lo = item * kLongRun;
            if (lo >= n) continue;
            const int64_t hi = lo + kLongRun < n ? lo + kLongRun : n;
            const int32_t w0 = a.sorted[lo].word, w1 = a.sorted[hi - 1].word;
            const int64_t s0 = a.start[w0], e0 = a.start[w0 + 1];
            if (e0 - s0 > kLongRun) {
                float acc[V] = {};
                sum_run<TI, V, kNarrow>(acc, a, lo, e0 < hi ? e0 : hi, c);
                if (mine) store_chunk<float, V>(a.partial + (size_t)(2 * item) * a.width + (int64_t)c * V, acc);
            }
            const int64_t s1 = a.start[w1], e1 = a.start[w1 + 1];
            if (w1 != w0 && e1 - s1 > kLongRun) {
                float acc[V] = {};
                sum_run<TI, V, kNarrow>(acc, a, s1, hi, c);
                if (mine) store_chunk<float, V>(a.partial + (size_t)(2 * item + 1) * a.width + (int64_t)c * V, acc);
            }
        } else {
            const int64_t w = item - a.ranges, lo = a.start[w], hi = a.start[w + 1];
            if (hi - lo > kLongRun) continue;
            float acc[V] = {};
            sum_run<TI, V, kNarrow>(acc, a, lo, hi, c);
            if (mine) write_row<TO, V>(a, w, c, acc, hi > lo);
        }
    }
}

// The rows of the long runs that start in the ranges of a workgroup, one range per group of lanes: the partial sums of a run in
// order.  A run of more than kLongJoin of them is left to the whole workgroup: kJoinParts of its groups sum consecutive parts, then the
// parts' sums are added in pairs, pairs of pairs and so on.  Groups are of few lanes (kJoinLanesLog2 at most): the hottest word's
// partial sums (2 MB of a million tokens of natural text at 256 elements) are then read by as many compute units as there are groups to
// a row.  The number of parts is that of the widest groups, so that narrower ones (rows of few chunks) give the same sums.
constexpr int kLongJoin = 32;
constexpr int kJoinLanesLog2 = 3;
constexpr int kJoinParts = 1024 >> kJoinLanesLog2;

// acc += rows first .. behind - 1 of the partial sums of a run: row 0 is `head`, row k is 2 (item + k)
template <int V>
__device__ __forceinline__ void add_partials(float (&acc)[V], const GradArgs& a, int64_t item, int64_t head, int64_t first, int64_t behind, int c)
{
    for (int64_t r = first; r < behind; r += 8) {
        const auto at = [&](int i) {
            const int64_t k = r + i < behind ? r + i : behind - 1;
            return (int32_t)(k == 0 ? head : 2 * (item + k));
        };
        add_rows<float, V, 8>(acc, a.partial + (int64_t)c * V, a.width, behind - r < 8 ? (int)(behind - r) : 8, at);
    }
}

template <class TO, int V>
__global__ __launch_bounds__(1024) void embed_grad_join_kernel(GradArgs a)
{
    __shared__ float part[512 * V];
    __shared__ int32_t later[1024 / kLongJoin + 2];                 // ranges that a long join starts in: at least kLongJoin apart
    __shared__ int32_t n_later;
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log2, groups = 1024 >> a.lanes_log2;
    const int64_t column = ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * lanes + lane;
    const int c = column < a.chunks ? (int)column : a.chunks - 1;
    const int64_t n = a.start[a.rows];
    if (threadIdx.x == 0) n_later = 0;
    __syncthreads();
    const int64_t item = (int64_t)blockIdx.x * groups + group, first = item * kLongRun;
    if (first < n) {
        const int64_t behind = first + kLongRun < n ? first + kLongRun : n;
        const int32_t w = a.sorted[behind - 1].word;
        const int64_t s = a.start[w], e = a.start[w + 1];
        if (s >= first && e - s > kLongRun) {
            const int64_t rows = (e - 1) / kLongRun - item + 1;
            if (rows <= kLongJoin) {
                float acc[V] = {};
                add_partials<V>(acc, a, item, s == first ? 2 * item : 2 * item + 1, 0, rows, c);
                if (column < a.chunks) write_row<TO, V>(a, w, c, acc, true);
            } else if (lane == 0) {
                later[atomicAdd(&n_later, 1)] = (int32_t)item;
            }
        }
    }
    __syncthreads();
    for (int q = 0; q < n_later; ++q) {
        const int64_t it = later[q], from = it * kLongRun;
        const int32_t w = a.sorted[from + kLongRun - 1].word;              // the run goes on behind its first range
        const int64_t s = a.start[w], e = a.start[w + 1];
        const int64_t rows = (e - 1) / kLongRun - it + 1, each = (rows + kJoinParts - 1) / kJoinParts;
        const int64_t lo = group * each, hi = lo + each < rows ? lo + each : rows;
        float acc[V] = {};
        if (group < kJoinParts) add_partials<V>(acc, a, it, s == from ? 2 * it : 2 * it + 1, lo, hi, c);
        for (int o = kJoinParts >> 1; o > 0; o >>= 1) {
            if (group >= o && group < 2 * o)
#pragma unroll
                for (int j = 0; j < V; ++j) part[j * 512 + threadIdx.x - (o << a.lanes_log2)] = acc[j];
            __syncthreads();
            if (group < o)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += part[j * 512 + threadIdx.x];
            __syncthreads();
        }
        if (group == 0 && column < a.chunks) write_row<TO, V>(a, w, c, acc, true);
    }
}

// Few tokens: one launch.  A workgroup owns up to `words` words, reads the whole list, keeps the places of its words' tokens in order
// and sorts them by word in LDS.  A word's row is then summed by a group of lanes, or, of a run of more than kLongRun tokens, by all
// groups: the run is cut into 256 pieces, of 16 tokens at least, every kColumns-th piece is added up in order, then these sums in
// pairs, pairs of pairs and so on.  A group takes a piece at a time and kColumns is the least number of groups that a workgroup has, so
// the additions are the same for every number of groups, and a term passes 64 + 16 + 4 of them at most.  (One part per group was
// 73 us for 16,384 tokens of one word x 64 f32, this is 78; batches of natural text take the same time within 5 %.)
// The words go to the workgroups in turn, 2^unit_log2 at a time (128 bytes of the table): with consecutive words the
// workgroup of the most frequent ones had most of the tokens (8192 tokens, 30,000 x 1024 bf16: 103 us, in turn 37).
constexpr int kFewTokens = 16384;                                   // 1024 for each of the kRows of the kernel that takes the most
constexpr int kFewWords = 256;                                      // most words of a workgroup
constexpr int kColumns = 16;

// (two workgroups per compute unit where 64 registers are enough, which is where V < 8)
template <class TI, class TO, int V, int kRows>
__global__ __launch_bounds__(1024, V < 8 && kRows == 8 ? 8 : 4) void embed_grad_few_kernel(GradArgs a)
{
    constexpr int kTokens = 1024 * kRows;
    __shared__ union {
        uint32_t list[kTokens];                                     // number of the word in the upper half, place in the lower
        float part[1024 * V];
    } lds;
    __shared__ uint16_t sorted[kTokens];                         // places, by word
    __shared__ uint32_t cnt[16][kFewWords];                         // per wave and word: tokens, then the next position among the sorted
    __shared__ uint32_t first[kFewWords + 1];
    __shared__ uint32_t found[kRows * 16 + 1];                      // per 64 tokens of the list: those of the workgroup's words, then how many come before
    __shared__ uint16_t long_words[kTokens / kLongRun];
    __shared__ int32_t n_long;
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_log2, groups = 1024 >> a.lanes_log2;
    const int wv = threadIdx.x >> 6, wlane = threadIdx.x & 63;
    const uint64_t below = (1ull << wlane) - 1ull;
    // its word k is word ((k >> unit_log2) * workgroups + workgroup << unit_log2) + k % 2^unit_log2 of the table
    const auto word_at = [&](int k) { return ((((int64_t)(k >> a.unit_log2) * gridDim.x + blockIdx.x) << a.unit_log2) + (k & ((1 << a.unit_log2) - 1))); };
    uint32_t t[kRows];                                              // numbers k, or ~0 for others' words
    uint64_t in[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
        const int64_t w = j * 1024 + (int)threadIdx.x < a.n ? a.tokens.at(j * 1024 + threadIdx.x) : -1;
        const uint32_t unit = (uint32_t)(w >> a.unit_log2), turn = unit / gridDim.x;
        t[j] = w >= 0 && w < a.rows && unit - turn * gridDim.x == blockIdx.x ? (turn << a.unit_log2) + ((uint32_t)w & ((1u << a.unit_log2) - 1u)) : ~0u;
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
        in[j] = __ballot(t[j] != ~0u);
        if (wlane == 0) found[j * 16 + wv] = (uint32_t)__popcll((unsigned long long)in[j]);
    }
    if (threadIdx.x == 0) n_long = 0;
    for (int w = wlane; w < a.words; w += 64) cnt[wv][w] = 0u;
    __syncthreads();
    if (wv == 0) {                                                  // exclusive sum of kRows * 16 counts, kRows / 4 a lane
        uint32_t x[kRows / 4], incl = 0u;
#pragma unroll
        for (int j = 0; j < kRows / 4; ++j) { x[j] = found[wlane * (kRows / 4) + j]; incl += x[j]; }
        const uint32_t mine = incl;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t up = __shfl_up(incl, o);
            if (wlane >= o) incl += up;
        }
        uint32_t run = incl - mine;
#pragma unroll
        for (int j = 0; j < kRows / 4; ++j) { found[wlane * (kRows / 4) + j] = run; run += x[j]; }
        if (wlane == 63) found[kRows * 16] = run;
    }
    __syncthreads();
    const uint32_t count = found[kRows * 16];
    if (count > 0) {                                                // the same for the whole workgroup
#pragma unroll
        for (int j = 0; j < kRows; ++j)
            if ((in[j] >> wlane) & 1ull)
                lds.list[found[j * 16 + wv] + (uint32_t)__popcll((unsigned long long)(in[j] & below))] = t[j] << 16 | (uint32_t)(j * 1024 + threadIdx.x);
        __syncthreads();
        // stable sort: a wave takes a sixteenth of the list, rounded up to rows of 64
        const uint32_t each = ((count + 15u) / 16u + 63u) & ~63u, lo = wv * each, hi = lo + each < count ? lo + each : count;
        for (uint32_t p = lo + wlane; p < hi; p += 64) atomicAdd(&cnt[wv][lds.list[p] >> 16], 1u);
        __syncthreads();
        for (int w = threadIdx.x; w < a.words; w += 1024) {
            uint32_t all = 0u;
            for (int v = 0; v < 16; ++v) { const uint32_t c = cnt[v][w]; cnt[v][w] = all; all += c; }
            first[w] = all;
        }
        __syncthreads();
        if (wv == 0) {                                              // exclusive sum of the words' counts, kFewWords / 64 a lane
            constexpr int kEach = kFewWords / 64;
            uint32_t x[kEach], incl = 0u;
#pragma unroll
            for (int j = 0; j < kEach; ++j) { x[j] = wlane * kEach + j < a.words ? first[wlane * kEach + j] : 0u; incl += x[j]; }
            const uint32_t mine = incl;
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t up = __shfl_up(incl, o);
                if (wlane >= o) incl += up;
            }
            uint32_t run = incl - mine;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if (wlane * kEach + j <= a.words) first[wlane * kEach + j] = run;
                run += x[j];
            }
            if (wlane == 63 && a.words == kFewWords) first[kFewWords] = run;
        }
        __syncthreads();
        for (uint32_t row = lo; row < lo + each; row += 64) {       // whole rows: the ballots need every lane
            const uint32_t p = row + wlane;
            const bool have = p < hi;
            const uint32_t entry = have ? lds.list[p] : 0u, word = entry >> 16;
            uint64_t peers = __ballot(have);
#pragma unroll
            for (int bit = 0; bit < 8; ++bit) {
                const bool one = (word >> bit) & 1u;
                const uint64_t m = __ballot(one);
                peers &= one ? m : ~m;
            }
            if (have) {
                const uint32_t rank = (uint32_t)__popcll((unsigned long long)(peers & below)), at = cnt[wv][word] + rank;
                if (rank == 0u) cnt[wv][word] = at + (uint32_t)__popcll((unsigned long long)peers);
                sorted[first[word] + at] = (uint16_t)entry;
            }
        }
        __syncthreads();
    }

    const int column = blockIdx.y * lanes + lane;
    const bool mine = column < a.chunks;
    const int c = mine ? column : a.chunks - 1;
    const TI* const from = static_cast<const TI*>(a.grad) + (int64_t)c * V;
    // acc += the rows at the sorted positions p .. p_behind - 1
    const auto sum = [&](float (&acc)[V], uint32_t p, uint32_t p_behind) {
        for (; p < p_behind; p += 8) {
            const auto at = [&](int i) { return (int32_t)sorted[p + i < p_behind ? p + i : p_behind - 1]; };
            const int left = (int)(p_behind - p);
            if (left > 4)       add_rows<TI, V, 8>(acc, from, a.stride, left < 8 ? left : 8, at);
            else if (left > 1)  add_rows<TI, V, 4>(acc, from, a.stride, left, at);
            else                add_rows<TI, V, 1>(acc, from, a.stride, 1, at);
        }
    };
    for (int word = group; word < a.words && word_at(word) < a.rows; word += groups) {
        const uint32_t p = count ? first[word] : 0u, p_behind = count ? first[word + 1] : 0u;
        if (p_behind - p > kLongRun) {
            if (lane == 0) long_words[atomicAdd(&n_long, 1)] = (uint16_t)word;
            continue;
        }
        float acc[V] = {};
        sum(acc, p, p_behind);
        if (mine) write_row<TO, V>(a, word_at(word), c, acc, p_behind > p);
    }
    __syncthreads();
    for (int q = 0; q < n_long; ++q) {                              // in any order: each is a sum of its own
        const int word = long_words[q];
        const uint32_t p0 = first[word], behind = first[word + 1], each = max(8u * ((behind - p0 + 2047u) / 2048u), 16u);   // 8 at a time
        const uint32_t pieces = (behind - p0 + each - 1u) / each;
        float acc[V] = {};                                          // of the first kColumns groups: a column each
        for (uint32_t k0 = 0; k0 < pieces; k0 += groups) {
            const uint32_t p = p0 + (k0 + (uint32_t)group) * each;
            float piece[V] = {};
            sum(piece, p, p + each < behind ? p + each : behind);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += piece[j];
            if (groups > kColumns) {
                if (group >= kColumns)
#pragma unroll
                    for (int j = 0; j < V; ++j) lds.part[j * 1024 + threadIdx.x] = piece[j];
                __syncthreads();
                if (group < kColumns)
                    for (int o = kColumns; o < groups && k0 + (uint32_t)o < pieces; o += kColumns)
#pragma unroll
                        for (int j = 0; j < V; ++j) acc[j] += lds.part[j * 1024 + threadIdx.x + (o << a.lanes_log2)];
                __syncthreads();
            }
        }
        for (int o = kColumns >> 1; o > 0; o >>= 1) {
            if (group >= o && group < 2 * o)
#pragma unroll
                for (int j = 0; j < V; ++j) lds.part[j * 1024 + threadIdx.x] = acc[j];
            __syncthreads();
            if (group < o)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += lds.part[j * 1024 + threadIdx.x + (o << a.lanes_log2)];
            __syncthreads();
        }
        if (group == 0 && mine) write_row<TO, V>(a, word_at(word), c, acc, true);
    }
}

}  // namespace same
