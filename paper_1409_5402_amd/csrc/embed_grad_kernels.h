// The gradient of a word table's lookup by sorted tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "dropout.h"
#include "element.h"
#include "tokens.h"

namespace same {

// ---- Gradient.  The tokens are sorted by word, stable, with the padding behind the last word; the positions of one word are
// then a run in ascending order, and its row of the gradient is one sum over the run in binary32.  The order of its additions
// depends on the tokens, and on whether they are taken in one launch (their number, the bytes of a row of grad, the table's size);
// not on how rows are cut into chunks and lanes, which addresses and strides decide, and no atomics: equal numbers, equal bits.

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
    Drop drop;               // of the lookup, where it had one
};

// Which elements of a row of grad count: all, or those that the lookup's dropout kept.  Chunks of V elements, 8 a multiple of V: the 8 / V
// lanes that hold eight columns share out the rows of a trip, so that a generator's block is made once (131,072 x 333 bf16: each lane for
// itself 193 us, now 128; without dropout 95).
// kApart: the blocks one after another and not side by side, for which registers are too few in some kernels (us apart and not: few tokens,
// V = 8, 4096 x 1024 f32 into bf16 56, 88; V = 4, 8000 x 50 27.2, 26.4; sorted tokens, V = 8, 131,072 x 1024 bf16 145, 140; V = 1, 131,072 x 333
// bf16 128, 137).
struct KeepAll {
    static constexpr bool kDrop = false;
    __device__ __forceinline__ KeepAll(const GradArgs&, int) {}
};

template <int V, bool kApart>
struct KeepSome {
    static constexpr bool kDrop = true;
    static constexpr int kShare = 8 / V;
    DropKey key;
    uint32_t eight;          // columns 8 * eight .. + 7 hold the chunk, from bit `shift` on
    int sub;                 // which of the lanes that share them
    bool shared;             // there are as many
    __device__ __forceinline__ KeepSome(const GradArgs& a, int column)
        : key(drop_key(a.drop)), eight((uint32_t)(column / kShare)), sub(column % kShare), shared(1 << a.lanes_log2 >= kShare) {}

    // kept[q]: of the elements of row at(q), q < count, bit j for the chunk's j-th; place(q) is at(q) for a q that differs between lanes
    template <int N, class At, class Place>
    __device__ __forceinline__ void rows(uint32_t (&kept)[N], int count, At at, Place place) const
    {
        if (kShare == 1 || N == 1 || !shared) {
            if constexpr (kApart) {
                uint64_t all = 0u;                                     // a byte per row
#pragma unroll 1
                for (int q = 0; q < count; ++q) all |= (uint64_t)((kept_eight(key, eight, (uint32_t)place(q)) >> (sub * V)) & 255u) << (8 * q);
#pragma unroll
                for (int q = 0; q < N; ++q) kept[q] = (uint32_t)(all >> (8 * q));
            } else {
#pragma unroll
                for (int q = 0; q < N; ++q)
                    if (q < count) kept[q] = kept_eight(key, eight, (uint32_t)at(q)) >> (sub * V);
            }
            return;
        }
        uint32_t lo = 0u, hi = 0u;                                     // a byte per row
#pragma unroll(kApart ? 1 : 8)
        for (int i = 0; i < (N + kShare - 1) / kShare; ++i) {
            const int q = sub + kShare * i;
            const int32_t row = place(q < count ? q : count - 1);
            if (q < count) {
                const uint32_t bits = kept_eight(key, eight, (uint32_t)row) << (8 * (q & 3));
                if (q < 4) lo |= bits; else hi |= bits;
            }
        }
        lo |= (uint32_t)__builtin_amdgcn_mov_dpp((int)lo, 0xB1, 0xF, 0xF, true);                           // lane ^ 1
        if (N > 4) hi |= (uint32_t)__builtin_amdgcn_mov_dpp((int)hi, 0xB1, 0xF, 0xF, true);
        if (kShare > 2) {
            lo |= (uint32_t)__builtin_amdgcn_mov_dpp((int)lo, 0x4E, 0xF, 0xF, true);                       // lane ^ 2
            if (N > 4) hi |= (uint32_t)__builtin_amdgcn_mov_dpp((int)hi, 0x4E, 0xF, 0xF, true);
        }
        if (kShare > 4) {
            lo |= (uint32_t)__builtin_amdgcn_mov_dpp((int)lo, 0x141, 0xF, 0xF, true);                      // 7 - lane of eight: the other four
            if (N > 4) hi |= (uint32_t)__builtin_amdgcn_mov_dpp((int)hi, 0x141, 0xF, 0xF, true);
        }
#pragma unroll
        for (int q = 0; q < N; ++q) kept[q] = (q < 4 ? lo >> (8 * (q & 3)) : hi >> (8 * (q & 3))) >> (sub * V);
    }
};

template <int V, bool kDrop, bool kApart>
using Keep = typename std::conditional<kDrop, KeepSome<V, kApart>, KeepAll>::type;

// acc += the rows at places at(0) .. at(count - 1) of the list, count in [1, N]: all loads before the first addition (at(q) is a
// place to read from for q >= count too)
template <class TI, int V, int N, class At, class Place, class K>
__device__ __forceinline__ void add_rows(float (&acc)[V], const TI* __restrict__ from, int64_t stride, int count, At at, Place place, const K& keep)
{
    float x[N][V];
#pragma unroll
    for (int q = 0; q < N; ++q) load_chunk<TI, V>(x[q], from + (int64_t)at(q) * stride);
    if constexpr (K::kDrop) {
        uint32_t kept[N] = {};
        keep.template rows<N>(kept, count, at, place);
#pragma unroll
        for (int q = 0; q < N; ++q)
#pragma unroll
            for (int j = 0; j < V; ++j) x[q][j] = if_kept(x[q][j], kept[q], j);
    }
#pragma unroll
    for (int q = 0; q < N; ++q)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = q < count ? acc[j] + x[q][j] : acc[j];
}

// By the 2^lanes_log2 lanes of a group, all of them active: a lane fetches one place of the run for all, or, where lanes are few,
// each fetches eight, those of the next rows while these are on their way (16,385 tokens into 140,000 x 16: 24 us with one place
// per lane and four lanes, now 15).
template <class TI, int V, bool kNarrow, class K>
__device__ __forceinline__ void sum_run(float (&acc)[V], const GradArgs& a, int64_t lo, int64_t hi, int c, const K& keep)
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
            const auto place = [&](int i) { return a.sorted[p + i].pos; };
            const int left = hi - p < 8 ? (int)(hi - p) : 8;
            if (left > 2) add_rows<TI, V, 8>(acc, from, a.stride, left, at, place, keep);
            else          add_rows<TI, V, 2>(acc, from, a.stride, left, at, place, keep);
        }
        return;
    }
    for (int64_t base = lo; base < hi; base += lanes) {
        const int here = hi - base < lanes ? (int)(hi - base) : lanes;
        const int32_t mine = a.sorted[base + (lane < here ? lane : here - 1)].pos;
        for (int q = 0; q < here; q += 8) {
            const auto at = [&](int i) { return __shfl(mine, q + i < here ? q + i : here - 1, lanes); };
            const auto& place = at;
            const int left = here - q;
            if (left > 4)       add_rows<TI, V, 8>(acc, from, a.stride, left < 8 ? left : 8, at, place, keep);
            else if (left > 2)  add_rows<TI, V, 4>(acc, from, a.stride, left, at, place, keep);
            else if (left == 2) add_rows<TI, V, 2>(acc, from, a.stride, 2, at, place, keep);
            else                add_rows<TI, V, 1>(acc, from, a.stride, 1, at, place, keep);
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
template <class TI, class TO, int V, bool kNarrow, bool kDrop>
__global__ __launch_bounds__(256) void embed_grad_kernel(GradArgs a)
{
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int column = blockIdx.y * lanes + lane;
    const bool mine = column < a.chunks;
    const int c = mine ? column : a.chunks - 1;                     // lanes behind the row's end follow its last chunk and write nothing
    const Keep<V, kDrop, (V < 8)> keep(a, column);
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
                sum_run<TI, V, kNarrow>(acc, a, lo, e0 < hi ? e0 : hi, c, keep);
                if (mine) store_chunk<float, V>(a.partial + (size_t)(2 * item) * a.width + (int64_t)c * V, acc);
            }
            const int64_t s1 = a.start[w1], e1 = a.start[w1 + 1];
            if (w1 != w0 && e1 - s1 > kLongRun) {
                float acc[V] = {};
                sum_run<TI, V, kNarrow>(acc, a, s1, hi, c, keep);
                if (mine) store_chunk<float, V>(a.partial + (size_t)(2 * item + 1) * a.width + (int64_t)c * V, acc);
            }
        } else {
            const int64_t w = item - a.ranges, lo = a.start[w], hi = a.start[w + 1];
            if (hi - lo > kLongRun) continue;
            float acc[V] = {};
            sum_run<TI, V, kNarrow>(acc, a, lo, hi, c, keep);
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
        add_rows<float, V, 8>(acc, a.partial + (int64_t)c * V, a.width, behind - r < 8 ? (int)(behind - r) : 8, at, at, KeepAll(a, c));
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

// (two workgroups per compute unit where 64 registers are enough, which is where V < 8; with dropout they are not: 4000 x 128 f32 into 20,000
// words 55 us, with one 22)
template <class TI, class TO, int V, int kRows, bool kDrop>
__global__ __launch_bounds__(1024, V < 8 && kRows == 8 && !kDrop ? 8 : 4) void embed_grad_few_kernel(GradArgs a)
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
    const Keep<V, kDrop, V == 8> keep(a, column);
    // acc += the rows at the sorted positions p .. p_behind - 1
    const auto sum = [&](float (&acc)[V], uint32_t p, uint32_t p_behind) {
        for (; p < p_behind; p += 8) {
            const auto at = [&](int i) { return (int32_t)sorted[p + i < p_behind ? p + i : p_behind - 1]; };
            const auto& place = at;
            const int left = (int)(p_behind - p);
            if (left > 4)       add_rows<TI, V, 8>(acc, from, a.stride, left < 8 ? left : 8, at, place, keep);
            else if (left > 1)  add_rows<TI, V, 4>(acc, from, a.stride, left, at, place, keep);
            else                add_rows<TI, V, 1>(acc, from, a.stride, 1, at, place, keep);
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
