// What the kernels that make 8-bit codes share: the largest magnitude of values that have a scale in common, its scale, and
// codes from values.
#pragma once

#include "msda_layer.hpp"

namespace msda {
namespace {

// The larger of `most` and the magnitudes of a and b; a NaN stays.
__device__ __forceinline__ float larger(float most, float a, float b) {
    return __builtin_elementwise_maximum(most, __builtin_elementwise_maximum(__builtin_fabsf(a), __builtin_fabsf(b)));
}
// Magnitudes as integers, which are ordered as they are, infinities and NaN last.
__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// The scale of values whose largest magnitude has these bits: 0 below 2^-100, NaN if it is not finite.
constexpr uint32_t kNotFinite = 0x7f800000u, kLeast = 0x0d800000u;  // bits of infinity, and of 2^-100
__device__ __forceinline__ float scale_of(uint32_t bits) {
    if (bits >= kNotFinite) return __builtin_nanf("");
    return bits < kLeast ? 0.f : __builtin_bit_cast(float, bits) * (1.f / 127.f);
}

// VEC values in steps of 1 / inverse, to the nearest code, even ones between two. At most 127 (1 + 2^-22) of them make the
// largest value, so no code is beyond 127. 1.5 * 2^23 added to a number of this size leaves it, rounded so, in the
// sum's low bits, of which the lowest byte is the code. With inverse 0 (and finite values) all are 0.
template <int VEC>
__device__ __forceinline__ Piece<int8_t, VEC> codes_of(const float (&t)[VEC], float inverse) {
#pragma clang fp contract(off)  // the product is rounded, and then the sum
    constexpr float kWhole = 12582912.f;
    Piece<int8_t, VEC> x;
    uint32_t b[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float scaled = t[i] * inverse;
        b[i] = __builtin_bit_cast(uint32_t, scaled + kWhole);
    }
    if constexpr (VEC % 4 == 0) {
        uint32_t w[VEC / 4];
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) {
            const uint32_t lo = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u);
            const uint32_t hi = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u);
            w[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
        }
        __builtin_memcpy(&x, w, VEC);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x.v[i] = (int8_t)b[i];
    }
    return x;
}

}  // namespace
}  // namespace msda
