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

}  // namespace same
