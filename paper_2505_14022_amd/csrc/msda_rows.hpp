// What the kernels that own rows of channels share (layer norm, root-mean-square norm, rows in 8 bits): sums over a
// row's lanes, columns of weights, and how many lanes a row gets.
#pragma once

#include <type_traits>

#include "msda_layer.hpp"

namespace msda {
namespace {

// Sums of NX values over the G lanes of a row; every lane of the row gets them. With G = NT the row is
// the workgroup's: `red` holds the waves' sums, and all threads take part.
template <int NT, int G, int NX>
__device__ __forceinline__ void row_sums(float (&x)[NX], float* red) {
#pragma unroll
    for (int k = 0; k < NX; ++k) x[k] = group_sum<(G < 64 ? G : 64)>(x[k]);
    if constexpr (G > 64) {
        constexpr int W = NT / 64;
        __syncthreads();  // the last sums have been read
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < NX; ++k) red[k * W + (threadIdx.x >> 6)] = x[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NX; ++k) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) t += red[k * W + w];
            x[k] = t;
        }
    }
}

// The lane's columns of weight or bias (`none` without one), in 16-byte pieces if `pieces`.
template <int VEC, int G, int NV>
__device__ __forceinline__ void load_columns(float (&w)[NV][VEC], const float* from, float none, int g, int C, bool pieces) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * G + g) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[j][i] = none;
        if (!from || c >= C) continue;
        if (VEC % 4 == 0 && pieces) {
#pragma unroll
            for (int i = 0; i + 3 < VEC; i += 4) {
                const float4 x = *reinterpret_cast<const float4*>(from + c + i);
                w[j][i] = x.x;
                w[j][i + 1] = x.y;
                w[j][i + 2] = x.z;
                w[j][i + 3] = x.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[j][i] = from[c + i];
        }
    }
}

// Lanes per row and the row's pieces per lane: a lane keeps at most 16 elements, since the backward holds
// five values of each. Called with a functor taking (threads, lanes, pieces) as integral constants.
template <int N>
using Int = std::integral_constant<int, N>;

template <int VEC, typename F>
hipError_t by_row(int C, F f) {
    const int n = (C + VEC - 1) / VEC;
    if (n <= 8) return f(Int<256>(), Int<8>(), Int<1>());
    if (n <= 16) return f(Int<256>(), Int<16>(), Int<1>());
    if (n <= 32) return f(Int<256>(), Int<32>(), Int<1>());
    if (n <= 64) return f(Int<256>(), Int<64>(), Int<1>());
    if (n <= 128) return f(Int<256>(), Int<64>(), Int<2>());
    if (n <= 256) return f(Int<256>(), Int<256>(), Int<1>());
    if (n <= 512) return f(Int<256>(), Int<256>(), Int<2>());
    if (n <= 1024) return f(Int<1024>(), Int<1024>(), Int<1>());
    if constexpr (VEC < 16) {
        if (n <= 2048) return f(Int<1024>(), Int<1024>(), Int<2>());
    }
    if constexpr (VEC <= 4) {
        if (n <= 4096) return f(Int<1024>(), Int<1024>(), Int<4>());
    }
    if constexpr (VEC == 1) return f(Int<1024>(), Int<1024>(), Int<16>());
    return hipErrorInvalidValue;
}

// Rows of a workgroup of the backward (as by_row, for the host).
inline int rows_per_block(int64_t C, int vec) {
    const int64_t n = (C + vec - 1) / vec;
    return n <= 8 ? 32 : n <= 16 ? 16 : n <= 32 ? 8 : n <= 128 ? 4 : 1;
}

}  // namespace
}  // namespace msda
