// Rows of the local models' element types: sixteen bytes at a time, in float32 registers in between.
#pragma once

#include "som_internal.hpp"

namespace som {

// N elements, sixteen bytes unless said otherwise, at the alignment of an element.  Global memory serves such accesses at any address of
// this target, so rows of any length and stride take the same path.
template <class T, int COUNT = 16 / sizeof(T)>
struct Piece {
    static constexpr int N = COUNT;
    T e[N];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(e, p, sizeof(e)); }
    __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, e, sizeof(e)); }
};

// The pieces of a row of D elements, D >= Piece::N: the last one ends at the row's end and so overlaps the one before where
// N does not divide D (both hold the same values there).
template <class T, int N = Piece<T>::N>
__device__ __forceinline__ int64_t piece_at(int c, int D)
{
    const int at = c * N;
    return at + N <= D ? at : D - N;
}

// A wavefront's writes to LDS before, its reads behind (the same wavefront's LDS accesses take effect in order).
__device__ __forceinline__ void wave_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// Lanes that share a row of `pieces` pieces: a power of two, at most `most`.
inline int row_lanes(int64_t pieces, int most)
{
    int l = 1;
    while (l < most && l < pieces) l *= 2;
    return l;
}

} // namespace som
