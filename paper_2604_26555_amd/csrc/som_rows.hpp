// Rows of the local models' element types: sixteen bytes at a time, in float32 registers in between.
#pragma once

#include "som_internal.hpp"

namespace som {

// Sixteen bytes at the alignment of an element.  Global memory serves such accesses at any address of this target, so rows of
// any length and stride take the same path.
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(2)));

template <class T>
struct Piece {
    static constexpr int N = 16 / sizeof(T);          // elements
    union {
        words4 w;
        T e[N];
    };
    __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const words4*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<words4*>(p) = w; }
};

// The pieces of a row of D elements, D >= Piece::N: the last one ends at the row's end and so overlaps the one before where
// N does not divide D (both hold the same values there).
template <class T>
__device__ __forceinline__ int64_t piece_at(int c, int D)
{
    constexpr int N = Piece<T>::N;
    const int at = c * N;
    return at + N <= D ? at : D - N;
}

} // namespace som
