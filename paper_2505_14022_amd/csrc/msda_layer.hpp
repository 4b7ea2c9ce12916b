// What the layer operators share: element types, 16-byte pieces of rows, the host's view of a launch.
#pragma once

#include "msda_device.hpp"

namespace msda {
namespace {

typedef __bf16 bf16_t;

// A piece of VEC consecutive elements in memory.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Piece {
    T v[VEC];
};

template <typename T, int VEC>
__device__ __forceinline__ void load_piece(float (&f)[VEC], const T* p) {
    const Piece<T, VEC> x = *reinterpret_cast<const Piece<T, VEC>*>(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = (float)x.v[i];
}

// Elements are rounded to nearest-even. For waves that store whole cache lines: a streaming store that leaves lines in
// part goes to memory in parts.
template <typename T, int VEC>
__device__ __forceinline__ void store_piece(T* p, const float (&f)[VEC]) {
    Piece<T, VEC> x;
#pragma unroll
    for (int i = 0; i < VEC; ++i) x.v[i] = (T)f[i];
    if constexpr (sizeof(x) == 16) stream_store(reinterpret_cast<uint4*>(p), __builtin_bit_cast(uint4, x));
    else *reinterpret_cast<Piece<T, VEC>*>(p) = x;
}

}  // namespace
}  // namespace msda
