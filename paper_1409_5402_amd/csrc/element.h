// Element types of the word-table operators and chunks of consecutive elements that one lane moves at a time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace same {

// A number in binary32 from any of the three types (exact), and rounded to it (once, to nearest, ties to even:
// the conversions are single instructions on gfx950).
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__bf16 x) { return (float)x; }
__device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }

// V consecutive elements, moved by the widest accesses that their alignment allows (up to 16 bytes).
template <class T, int V>
struct alignas(V * sizeof(T) < 16 ? V * sizeof(T) : 16) Chunk {
    T v[V];
};

template <class T, int V>
__device__ __forceinline__ void load_chunk(float (&x)[V], const T* __restrict__ p)
{
    const Chunk<T, V> c = *reinterpret_cast<const Chunk<T, V>*>(p);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = to_float(c.v[j]);
}

template <class T, int V>
__device__ __forceinline__ void store_chunk(T* __restrict__ p, const float (&x)[V])
{
    Chunk<T, V> c;
#pragma unroll
    for (int j = 0; j < V; ++j) c.v[j] = (T)x[j];
    *reinterpret_cast<Chunk<T, V>*>(p) = c;
}

// Eight elements at the alignment of one: whole vectors all the same, global memory is read and written at any address.
typedef uint32_t v4u32 __attribute__((ext_vector_type(4)));
typedef v4u32 v4u32_anywhere __attribute__((aligned(2)));

template <class T>
struct Eight {
    T v[8];
    static constexpr int kVectors = sizeof(T) / 2;
    __device__ __forceinline__ void load(const T* p)
    {
        v4u32 x[kVectors];
#pragma unroll
        for (int q = 0; q < kVectors; ++q) x[q] = reinterpret_cast<const v4u32_anywhere*>(p)[q];
        __builtin_memcpy(v, x, sizeof v);
    }
    __device__ __forceinline__ void store(T* p) const
    {
        v4u32 x[kVectors];
        __builtin_memcpy(x, v, sizeof v);
#pragma unroll
        for (int q = 0; q < kVectors; ++q) reinterpret_cast<v4u32_anywhere*>(p)[q] = x[q];
    }
};

// Elements at .. at + 7 of a row, zeros behind its end, in two steps: a whole load, of the row's last eight elements where the chunk crosses
// its end, and moving those into place.  Many loads are then on their way together.
template <class T>
__device__ __forceinline__ Eight<T> eight_at(const T* row, int at, int width)
{
    Eight<T> c;
    if (width >= 8) {
        c.load(row + (at < width - 8 ? at : width - 8));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const T x = row[at + j < width ? at + j : width - 1];
            c.v[j] = at + j < width ? x : (T)0.0f;
        }
    }
    return c;
}

template <class T>
__device__ __forceinline__ void cut_eight(Eight<T>& c, int at, int width)
{
    const int over = at + 8 - width;
    if (over <= 0 || width < 8) return;
#pragma unroll
    for (int by = 1; by <= 4; by *= 2)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const T other = j + by < 8 ? c.v[j + by < 8 ? j + by : 7] : (T)0.0f;
            c.v[j] = over & by ? other : c.v[j];
        }
#pragma unroll
    for (int j = 0; j < 8; ++j) c.v[j] = over >= 8 ? (T)0.0f : c.v[j];
}

template <class T>
__device__ __forceinline__ void load_eight(float (&x)[8], const T* row, int at, int width)
{
    Eight<T> c = eight_at(row, at, width);
    cut_eight(c, at, width);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = to_float(c.v[j]);
}

template <class T>
__device__ __forceinline__ void store_eight(T* p, const float (&x)[8], int count)
{
    Eight<T> c;
#pragma unroll
    for (int j = 0; j < 8; ++j) c.v[j] = (T)x[j];
    if (count >= 8) {
        c.store(p);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count) p[j] = c.v[j];
    }
}

}  // namespace same
