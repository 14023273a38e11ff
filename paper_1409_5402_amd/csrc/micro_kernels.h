// Rounding to microscaled four-bit floating point, and the product of two matrices in it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "element.h"
#include "micro_format.h"

namespace same {

// ---- Rounding.  Of a block's largest magnitude top the exponent e = floor(log2 top) - 2 puts top / 2^e into [4, 8): the
// largest size is 6, so what lies above 6 is rounded down to it.  Sizes are rounded to the nearest, ties to the even
// code: in units of .5 below 2, of 1 below 4, of 2 above.  A lane takes 8 elements, four lanes a block.
struct QuantizeArgs {
    const void* x;
    int64_t rows, stride;
    int32_t width;
    int32_t wide;            // chunks of 8 are aligned
    uint8_t* codes;
    uint8_t* scales;
};

// Codes of the 8 elements from `first` of a row of `width` on, and their block's scale; by four consecutive lanes together.
template <class TI>
__device__ __forceinline__ uint32_t micro_piece(const TI* __restrict__ row, int first, int width, bool wide, uint32_t& scale)
{
    float x[8];
    if (wide && first + 8 <= width) {
        load_chunk<TI, 8>(x, row + first);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = first + j < width ? to_float(row[first + j]) : 0.0f;
    }
    uint32_t top = 0u;                                                         // magnitudes order like their bits, NaN above infinity
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    uint32_t q = 0u;
    scale = 255u;
    if (top < 0x7F800000u) {
        scale = top >= 0x01000000u ? (top >> 23) - 2u : 0u;                    // 127 + e, at least 0
        const float power = micro_power(scale);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[0], x[1], power, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[2], x[3], power, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[4], x[5], power, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[6], x[7], power, 3);
    }
    return q;
}

// Memory bound: 8192 x 8192 bf16 take 40 us, 4.3 TB/s; the conversion is two elements per instruction.
template <class TI>
__global__ __launch_bounds__(256) void micro_quantize_kernel(QuantizeArgs a)
{
    const int64_t pieces = micro_groups(a.width) * (kMicroGroup / 8);          // of 8 elements, per row
    const int64_t all = a.rows * pieces;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {   // whole groups of four lanes
        const int64_t row = all >> 32 ? at / pieces : (int64_t)((uint32_t)at / (uint32_t)pieces);             // a division of 64 bits takes as long as the rest
        uint32_t s;
        const uint32_t q = micro_piece(static_cast<const TI*>(a.x) + row * a.stride, (int)(at - row * pieces) * 8, a.width, a.wide, s);
        reinterpret_cast<uint32_t*>(a.codes)[at] = q;                          // rows of codes follow each other without a gap
        if ((at & 3) == 0) a.scales[at >> 2] = (uint8_t)s;
    }
}

// ---- Product: out[i][j] = scale * sum_k a[i][k] b[j][k], both in four bits, on the scaled matrix instructions, which
// take 32 elements and their scale byte from a lane and add in binary32.
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
constexpr int kFormatE2M1 = 4;

struct ProductArgs {
    const uint8_t *a, *a_scales, *b, *b_scales;
    int64_t rows_a, rows_b;
    int32_t groups;          // of 128 elements per row
    float scale;
    void* out;
    int64_t out_stride;
    int64_t tiles_a, tiles_b;
    int32_t wide;            // 16 bytes of a row of out are aligned
    int64_t stride_a;        // where a is a matrix of numbers: its stride and width,
    int32_t width;
    int32_t wide_a;          // and whether chunks of 8 are aligned
};

__device__ __forceinline__ v8i fragment(v4i x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

// Few rows of a (at most 16 * MF): the table is read once, straight from memory into the operands of 16x16x128 instructions: lane l
// gives block l / 16 of row l % 16 of a group of 128, so four lanes read the 64 bytes of a row's group.  A wave takes 16 * RF
// rows of the table; with KW = 4 the four waves of a workgroup take a quarter of the groups each and their sums are added in
// order, so that long rows are in flight from more waves.
template <int N>
struct alignas(4) ScaleWords {
    uint32_t v[N];
};

// 13 x 50,021 x 4096 takes 26 us, 4.2 TB/s; 1 x 100,000 x 256 5.4 us, a launch and the way to memory.
// With TI a type of numbers the rows of a are such numbers, few enough (kRoundMost of them) for every workgroup to round them for itself:
// one launch in place of two (the most, as calls: 16 x 40,000 x 1024 9.0 us, rounded before 14.6; 2 x 20,000 x 8192 19.2, 19.8; with the
// 53,248 of 13 x 50,021 x 4096 it would be 44, 34).
constexpr int kRoundMost = 16384, kRoundRows = 64;

template <class TO, int MF, int RF, int KW, class TI>
__global__ __launch_bounds__(256) void micro_product_few_kernel(ProductArgs p)
{
    constexpr int kUnroll = MF * RF >= 8 ? 2 : 4;                              // groups in flight
    constexpr bool kRound = !std::is_void<TI>::value;
    __shared__ v4f others[KW > 1 ? KW - 1 : 1][MF][RF][64];
    __shared__ alignas(16) uint32_t rounded[kRound ? (kRoundMost + 16 * MF * kMicroGroup) / 8 : 1];
    __shared__ alignas(16) uint8_t rounded_scales[kRound ? (kRoundMost + 16 * MF * kMicroGroup) / 32 : 4];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int64_t pitch = (int64_t)p.groups * 64, spitch = (int64_t)p.groups * 4;
    const uint8_t *a = p.a, *a_scales = p.a_scales;
    if constexpr (kRound) {
        const int pieces = p.groups * 16, all = (int)p.rows_a * pieces;        // whole groups of four lanes
        for (int at = threadIdx.x; at < all; at += 256) {
            const int row = at / pieces;
            uint32_t s;
            const uint32_t q = micro_piece(reinterpret_cast<const TI*>(p.a) + row * p.stride_a, (at - row * pieces) * 8, p.width, p.wide_a, s);
            rounded[at] = q;
            if ((at & 3) == 0) rounded_scales[at >> 2] = (uint8_t)s;
        }
        __syncthreads();
        a = reinterpret_cast<const uint8_t*>(rounded);
        a_scales = rounded_scales;
    }
    const uint8_t* fa[MF];
    const uint8_t* sa[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int64_t i = 16 * f + r < p.rows_a ? 16 * f + r : p.rows_a - 1;   // rows behind the last are computed from it and not written
        fa[f] = a + i * pitch + g * 16;
        sa[f] = a_scales + i * spitch;
    }
    const int each = (p.groups + KW - 1) / KW, part = KW > 1 ? wv : 0;
    const int k0 = part * each, k1 = k0 + each < p.groups ? k0 + each : p.groups;
    for (int64_t tile = (int64_t)blockIdx.x * (4 / KW) + (KW > 1 ? 0 : wv); tile < p.tiles_b; tile += (int64_t)gridDim.x * (4 / KW)) {
        const uint8_t* fb[RF];
        const uint8_t* sb[RF];
#pragma unroll
        for (int f = 0; f < RF; ++f) {
            const int64_t j = (tile * RF + f) * 16 + r, row = j < p.rows_b ? j : p.rows_b - 1;
            fb[f] = p.b + row * pitch + g * 16;
            sb[f] = p.b_scales + row * spitch;
        }
        v4f acc[MF][RF] = {};
        const auto groups = [&](int k, auto many) {
            constexpr int N = decltype(many)::value;
            v4i xa[N][MF], xb[N][RF];
            ScaleWords<N> ea[MF], eb[RF];
#pragma unroll
            for (int f = 0; f < RF; ++f) {
                eb[f] = *reinterpret_cast<const ScaleWords<N>*>(sb[f] + (int64_t)k * 4);
#pragma unroll
                for (int q = 0; q < N; ++q) xb[q][f] = *reinterpret_cast<const v4i*>(fb[f] + (int64_t)(k + q) * 64);
            }
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                ea[f] = *reinterpret_cast<const ScaleWords<N>*>(sa[f] + (int64_t)k * 4);
#pragma unroll
                for (int q = 0; q < N; ++q) xa[q][f] = *reinterpret_cast<const v4i*>(fa[f] + (int64_t)(k + q) * 64);
            }
#pragma unroll
            for (int q = 0; q < N; ++q)
#pragma unroll
                for (int f = 0; f < MF; ++f)
#pragma unroll
                    for (int h = 0; h < RF; ++h)
                        acc[f][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fragment(xa[q][f]), fragment(xb[q][h]), acc[f][h], kFormatE2M1, kFormatE2M1,
                                                                                     0, (int)(ea[f].v[q] >> (8 * g)), 0, (int)(eb[h].v[q] >> (8 * g)));
        };
        int k = k0;
        for (; k + kUnroll <= k1; k += kUnroll) groups(k, std::integral_constant<int, kUnroll>());
        for (; k < k1; ++k) groups(k, std::integral_constant<int, 1>());
        if constexpr (KW > 1) {
            __syncthreads();                                                   // the sums of the tile before have been read
            if (wv > 0)
#pragma unroll
                for (int f = 0; f < MF; ++f)
#pragma unroll
                    for (int h = 0; h < RF; ++h) others[wv - 1][f][h][lane] = acc[f][h];
            __syncthreads();
            if (wv > 0) continue;
#pragma unroll
            for (int q = 0; q < KW - 1; ++q)
#pragma unroll
                for (int f = 0; f < MF; ++f)
#pragma unroll
                    for (int h = 0; h < RF; ++h) acc[f][h] += others[q][f][h][lane];
        }
#pragma unroll
        for (int f = 0; f < MF; ++f)
#pragma unroll
            for (int h = 0; h < RF; ++h)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int64_t i = 16 * f + 4 * g + v, j = (tile * RF + h) * 16 + r;
                    if (i < p.rows_a && j < p.rows_b) static_cast<TO*>(p.out)[i * p.out_stride + j] = (TO)(p.scale * acc[f][h][v]);
                }
    }
}

// Many rows: a workgroup of WM x WN waves computes a tile of (32 FM WM) x (32 FN WN) sums, a wave FM x FN sums of 32 x 32 of it
// (32x32x64 instructions: lane l gives block l / 32 of row l % 32).  The rows' bytes come through LDS straight from memory.
// Codes come in stages of two groups of 128 elements, 128 bytes of a row, one stage ahead of the one that is multiplied.  A row's
// eight blocks of 16 bytes are stored in the order block ^ ((row / 2) % 8): eight lanes write a row, and any eight
// consecutive rows that are read at one block then lie in different banks.  A row's scales are fetched for kScaleGroups
// groups at once: what a compute unit's loads cost is the lines that they touch, and with 8 bytes per row and stage the
// scales touched as many as the codes (65 x 50,021 x 4096: 36.6 us, with kScaleGroups = 4 33.5 us).
// 8192 x 8192 x 8192 to bf16 takes 275 to 282 us, 4.0 PFLOP/s (tiles of 256 x 256 by eight waves): its loads alone take 231 us and its
// products alone 211 (6.4 PFLOP/s is what the instructions reach by themselves on random numbers, 9.2 on zeros).  2048 x 100,000
// x 256 to binary32 takes 166 us, 5.0 TB/s; a kernel that only stores the same tiles takes 127.
constexpr int kStageGroups = 2;

template <int R, int kStages, int kScaleGroups>
struct ProductSpace {
    v4i codes[kStages][R][8];
    uint32_t scales[kScaleGroups > kStageGroups ? 2 : kStages][R][kScaleGroups];
    uint32_t ahead[kStages > 1 ? 512 : 1];                                     // what is fetched for the cache alone
};

// The tile of workgroup b: workgroups go to the eight dies in turn, and a die takes a run of consecutive tiles, eight tile rows
// at a time and column by column, so that what runs on a die at once shares rows of both operands in its cache.
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t tiles_a, uint32_t tiles_b, uint32_t& ta, uint32_t& tb)
{
    const uint32_t all = tiles_a * tiles_b, die = b & 7u, each = all >> 3, more = all & 7u;
    const uint32_t t = die * each + (die < more ? die : more) + (b >> 3);
    const uint32_t first = t / (8u * tiles_b) * 8u, in = tiles_a - first < 8u ? tiles_a - first : 8u, at = t - first * tiles_b;
    tb = at / in;
    ta = first + at - tb * in;
}

// 16 or 4 bytes per lane from base + offset straight to consecutive places of LDS from `to` on.  Written as assembly because the
// compiler takes the builtin for a store that any later read from LDS may depend on, and waits for it there: here the only
// readers are behind arrived().  No vector register is written.  The copy of the base is for two waits that the compiler does not
// look for inside: a base that the vector unit has just written, and the state between writing m0 and using it.
__device__ __forceinline__ void to_lds_16(const uint8_t* base, uint32_t offset, const void* to)
{
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)to;
    uint64_t copy;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(copy) : "s"(at), "v"(offset), "s"(base) : "m0");
}
__device__ __forceinline__ void to_lds_4(const uint8_t* base, uint32_t offset, const void* to)
{
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)to;
    uint64_t copy;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0" : "=&s"(copy) : "s"(at), "v"(offset), "s"(base) : "m0");
}
// f(0), f(1), ... f(N - 1), the argument a constant
template <class F, int... I>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f)
{
    (f(std::integral_constant<int, I>()), ...);
}

// All of this wave's loads but the last N have come (they end in their order), then all waves'.
template <int N>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    __syncthreads();
}

// A wave's sums go out by way of LDS, 32 rows of its part of the tile at a time, so that a lane stores 16 bytes of one row.
template <int FM, int FN, int WM, int WN>
constexpr int kStripPitch = 32 * FN + 8;                                       // floats: the two halves of a wave write to different banks

template <class TO, int FM, int FN, int WM, int WN, int kStages, int kScaleGroups>
__global__ __launch_bounds__(64 * WM * WN, FM * FN * WM * WN > 16 ? WM * WN / 4 : kStages == 1 ? 4 : 2) void micro_product_kernel(ProductArgs p)
{
    constexpr int kW = WM * WN, kA = 32 * FM * WM, kB = 32 * FN * WN;          // waves, rows of a and of b
    constexpr int kPitch = kStripPitch<FM, FN, WM, WN>;
    union Space {
        ProductSpace<kA + kB, kStages, kScaleGroups> in;
        float strip[kW][32 * kPitch];
    };
    __shared__ Space space;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t pitch = (int64_t)p.groups * 64, spitch = (int64_t)p.groups * 4;
    uint32_t ta, tb;
    tile_of(blockIdx.x, (uint32_t)p.tiles_a, (uint32_t)p.tiles_b, ta, tb);
    const int64_t i0 = (int64_t)ta * kA, j0 = (int64_t)tb * kB;
    const int last_a = (int)(p.rows_a - i0 < kA ? p.rows_a - i0 : kA) - 1, last_b = (int)(p.rows_b - j0 < kB ? p.rows_b - j0 : kB) - 1;
    const int stages = (p.groups + kStageGroups - 1) / kStageGroups;
    const bool odd = p.groups % kStageGroups;

    // Codes: an instruction of a wave fills 8 rows.  Rows behind the last are filled from it.
    constexpr int kCodeA = kA / (8 * kW), kCodes = (kA + kB) / (8 * kW);
    static_assert(kA % (8 * kW) == 0 && kB % (8 * kW) == 0, "every wave fetches the same number of pieces of either operand");
    const int crow = wv * 8 + (lane >> 3), cblock = (lane & 7) ^ ((crow >> 1) & 7);
    uint32_t from[kCodes];
#pragma unroll
    for (int i = 0; i < kCodeA; ++i) from[i] = (uint32_t)min(i * 8 * kW + crow, last_a) * (uint32_t)pitch + cblock * 16;
#pragma unroll
    for (int i = kCodeA; i < kCodes; ++i) from[i] = (uint32_t)min((i - kCodeA) * 8 * kW + crow, last_b) * (uint32_t)pitch + cblock * 16;
    const uint8_t* const codes_a = p.a + i0 * pitch;
    const uint8_t* const codes_b = p.b + j0 * pitch;
    const auto load = [&](int st, auto which) {                                // instruction `which` of stage st
        constexpr int i = decltype(which)::value;
        auto& to = space.in.codes[st & (kStages - 1)];
        if constexpr (i < kCodeA) to_lds_16(codes_a + (int64_t)st * 128, from[i], &to[i * 8 * kW + wv * 8][0]);
        else                      to_lds_16(codes_b + (int64_t)st * 128, from[i], &to[kA + (i - kCodeA) * 8 * kW + wv * 8][0]);
    };
    // Before the last stage is loaded: where it holds one group, the lanes of the other fetch the first one's bytes again.
    const auto last_stage_next = [&] {
        if (!odd) return;
#pragma unroll
        for (int i = 0; i < kCodes; ++i) from[i] -= cblock >= 4 ? 64 : 0;
    };

    // Scales: pieces of kPiece groups of a row, a lane each; where the row ends inside a piece it is the row's last kPiece groups.
    constexpr int kPiece = kScaleGroups > kStageGroups ? 4 : 1, kPieces = kScaleGroups / kPiece, kRowsAtOnce = 64 / kPieces;
    static_assert((kA + kB) % (kRowsAtOnce * kW) == 0 && kA % kRowsAtOnce == 0, "");
    const uint8_t* const scales_a = p.a_scales + i0 * spitch;
    const uint8_t* const scales_b = p.b_scales + j0 * spitch;
    const auto first_of_piece = [&](int g) { return min(g / kPiece * kPiece, p.groups - kPiece); };   // of the piece that holds group g
    const auto load_scales = [&](int c) {                                      // groups c * kScaleGroups and on
        auto& to = space.in.scales[c & (sizeof(space.in.scales) / sizeof(space.in.scales[0]) - 1)];
        const int first = first_of_piece(c * kScaleGroups + (lane % kPieces) * kPiece);
#pragma unroll
        for (int i = 0; i < (kA + kB) / (kRowsAtOnce * kW); ++i) {
            const int row0 = (i * kW + wv) * kRowsAtOnce, row = row0 + lane / kPieces;   // of a, then of b: the same for a whole wave
            const uint32_t at = (uint32_t)(row0 < kA ? min(row, last_a) : min(row - kA, last_b)) * (uint32_t)spitch + (uint32_t)first * 4;
            if constexpr (kPiece == 4) to_lds_16(row0 < kA ? scales_a : scales_b, at, &to[row0][0]);
            else                       to_lds_4(row0 < kA ? scales_a : scales_b, at, &to[row0][0]);
        }
    };

    // A line of memory that no workgroup of the die has read yet takes as long as a stage's products, and all that share it wait.
    // Every workgroup therefore touches some lines of a stage kAhead stages before it loads it: of a's rows the part that is its own
    // among the kShareA tiles of a tile row that run on a die at once, of b's likewise.
    constexpr int kAhead = 2, kShareA = 4, kShareB = 8, kTouchA = kA / (kShareA * kW), kTouchB = kB / (kShareB * kW);
    static_assert(kTouchA + kTouchB <= 64, "");
    const bool touch_a = lane < kTouchA;
    const int touch_row = touch_a ? (int)(tb % kShareA) * (kTouchA * kW) + wv * kTouchA + lane : (int)(ta % kShareB) * (kTouchB * kW) + wv * kTouchB + (lane - kTouchA) % kTouchB;
    const uint8_t* const touch_from = touch_a ? codes_a + min(touch_row, last_a) * pitch : codes_b + min(touch_row, last_b) * pitch;
    const auto touch = [&](int st) {
        const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)&space.in.ahead[wv * 64];
        if (lane < kTouchA + kTouchB)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(at), "v"(touch_from + (int64_t)min(st, stages - 1) * 128) : "m0");
    };

    const int r = lane & 31, half = lane >> 5;
    const int wi = wv / WN * 32 * FM, wj = wv % WN * 32 * FN;                  // the wave's part of the tile
    const int turn = (r >> 1) & 7;
    v16f acc[FM][FN] = {};
    constexpr int kSteps = 4, kReads = FM + FN, kRow = FM * FN;
    uint32_t ea[FM][2], eb[FN][2];                                             // bytes 0 and 2: this lane's blocks of two steps
    uint32_t words[kReads][2];                                                 // the next stage's as they are read
    v4i xa[2][FM], xb[2][FN];                                                  // blocks of this step and the next
    const auto fetch = [&](int st, int s, int q) {                             // read q of step s of a stage: first all that its first row of products needs
        const auto& at = space.in.codes[st & (kStages - 1)];
        if (q < FN) xb[s & 1][q] = at[kA + wj + 32 * q + r][(2 * s + half) ^ turn];
        else        xa[s & 1][q - FN] = at[wi + 32 * (q - FN) + r][(2 * s + half) ^ turn];
    };
    const auto fetch_scales = [&](int st, int q) {
        const int g = st * kStageGroups, h = min(g + 1, p.groups - 1), c = g / kScaleGroups;
        const auto& at = space.in.scales[c & (sizeof(space.in.scales) / sizeof(space.in.scales[0]) - 1)];
        const int row = q < FN ? kA + wj + 32 * q + r : wi + 32 * (q - FN) + r;
        words[q][0] = at[row][g / kPiece * kPiece - c * kScaleGroups + g - first_of_piece(g)];
        words[q][1] = at[row][h / kPiece * kPiece - c * kScaleGroups + h - first_of_piece(h)];
    };
    const auto exponents = [&](uint32_t keep) {                                // a second group that is not there counts 2^-254 times: nothing
#pragma unroll
        for (int q = 0; q < kReads; ++q) {
            uint32_t(&e)[2] = q < FN ? eb[q] : ea[q - FN];
            e[0] = words[q][0] >> (8 * half);
            e[1] = words[q][1] >> (8 * half) & keep;
        }
    };
    const uint32_t keep_last = odd ? 0u : ~0u;
    // Multiplies a stage in four steps of 64 elements, a product of 32 x 32 x 64 per slot; in the slots' shadows the blocks of the
    // next step are read from LDS and with kMore the next stage is loaded.  In the middle of the last step the next stage has to have
    // arrived: its first blocks are read before the last products are done, and every wave has read what the stage after it
    // will overwrite.  A slot's product lasts 32 cycles, what stands beside it should not last longer.
    const auto multiply = [&](int st, auto more) {
        constexpr bool kMore = decltype(more)::value;
        if constexpr (kMore) {
            if (st + 2 == stages) last_stage_next();
            const int g = (st + 1) * kStageGroups;                             // scales that no stage before the next needs
            if constexpr (kScaleGroups > kStageGroups) {
                if (st * kStageGroups % kScaleGroups == 0 && st * kStageGroups + kScaleGroups < p.groups) load_scales(st * kStageGroups / kScaleGroups + 1);
            } else {
                load_scales(g / kScaleGroups);
            }
        }
        each_of(std::make_integer_sequence<int, kSteps * kRow>(), [&](auto slot) {
            constexpr int m = decltype(slot)::value, s = m / kRow, at = m % kRow, f = at / FN, h = at % FN;
            if constexpr (s + 1 < kSteps) {
                constexpr int q0 = at * kReads / kRow, q1 = (at + 1) * kReads / kRow;
                each_of(std::make_integer_sequence<int, q1 - q0>(), [&](auto q) { fetch(st, s + 1, q0 + decltype(q)::value); });
            }
            if constexpr (kMore && m < 2 * kRow) {
                constexpr int l0 = m * kCodes / (2 * kRow), l1 = (m + 1) * kCodes / (2 * kRow);
                each_of(std::make_integer_sequence<int, l1 - l0>(), [&](auto q) { load(st + 1, std::integral_constant<int, l0 + decltype(q)::value>()); });
            }
            if constexpr (kMore && m == 2 * kRow) touch(st + 1 + kAhead);
            if constexpr (kMore && s + 1 == kSteps) {
                constexpr int kFrom = kRow / 2;
                if constexpr (at == kFrom) arrived<1>();
                if constexpr (at >= kFrom) {
                    constexpr int q0 = (at - kFrom) * kReads / (kRow - kFrom), q1 = (at + 1 - kFrom) * kReads / (kRow - kFrom);
                    each_of(std::make_integer_sequence<int, q1 - q0>(), [&](auto q) {
                        fetch(st + 1, 0, q0 + decltype(q)::value);
                        fetch_scales(st + 1, q0 + decltype(q)::value);
                    });
                }
            }
            acc[f][h] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fragment(xa[s & 1][f]), fragment(xb[s & 1][h]), acc[f][h], kFormatE2M1, kFormatE2M1,
                                                                        (s & 1) * 2, (int)ea[f][s >> 1], (s & 1) * 2, (int)eb[h][s >> 1]);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (kMore) exponents(st + 2 < stages ? ~0u : keep_last);
    };
    if (stages == 1) last_stage_next();
    each_of(std::make_integer_sequence<int, kCodes>(), [&](auto i) { load(0, i); });
    load_scales(0);
    if constexpr (kStages > 1) {
#pragma unroll
        for (int st = 1; st <= kAhead; ++st) touch(st);
        arrived<kAhead>();
    } else {
        arrived<0>();
    }
#pragma unroll
    for (int q = 0; q < kReads; ++q) fetch(0, 0, q);
#pragma unroll
    for (int q = 0; q < kReads; ++q) fetch_scales(0, q);
    exponents(stages > 1 ? ~0u : keep_last);
    if constexpr (kStages > 1)
        for (int st = 0; st + 1 < stages; ++st) multiply(st, std::true_type());
    multiply(stages - 1, std::false_type());

    arrived<0>();                                                              // nothing is on its way to LDS, and no wave reads blocks from it any more
    float* const strip = space.strip[wv];
    constexpr int V = 16 / sizeof(TO), kAcross = 32 * FN / V;                  // elements of a store, stores of a row
    TO* const out = static_cast<TO*>(p.out) + (i0 + wi) * p.out_stride + j0 + wj;
    const int64_t behind_i = p.rows_a - i0 - wi, behind_j = p.rows_b - j0 - wj;
#pragma unroll
    for (int f = 0; f < FM; ++f) {
#pragma unroll
        for (int h = 0; h < FN; ++h)
#pragma unroll
            for (int v = 0; v < 16; ++v) strip[(8 * (v >> 2) + 4 * half + (v & 3)) * kPitch + 32 * h + r] = p.scale * acc[f][h][v];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (p.wide && behind_i >= 32 * FM && behind_j >= 32 * FN) {
#pragma unroll
            for (int q = 0; q < 32 * kAcross / 64; ++q) {
                const int at = q * 64 + lane, row = at / kAcross, column = at % kAcross * V;
                float x[V];
                load_chunk<float, V>(x, strip + row * kPitch + column);
                store_chunk<TO, V>(out + (32 * f + row) * p.out_stride + column, x);
            }
        } else {
            for (int at = lane; at < 32 * 32 * FN; at += 64) {
                const int row = at / (32 * FN), column = at % (32 * FN);
                if (32 * f + row < behind_i && column < behind_j) out[(32 * f + row) * p.out_stride + column] = (TO)strip[row * kPitch + column];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

}  // namespace same
