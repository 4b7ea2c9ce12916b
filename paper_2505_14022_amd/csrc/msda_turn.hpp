// What the kernels that turn channel pairs by positions share: sines and cosines of turns, and quotients of small numbers.
#pragma once

#include "msda_layer.hpp"

namespace msda {
namespace {

// cos and sin of `turns` whole turns: k / 4 + f with |f| <= 1/8; for |x| <= pi / 4 the first terms left
// out, x^11 / 11! and x^12 / 12!, are below 2e-9.
__device__ __forceinline__ void cos_sin(double turns, float& c, float& s) {
    turns -= rint(turns);
    const double k = rint(4.0 * turns);
    const float x = (float)((turns - 0.25 * k) * 6.283185307179586);
    const float x2 = x * x;
    float sx = 2.7557319e-6f;                      // 1 / 9!
    sx = __builtin_fmaf(sx, x2, -1.9841270e-4f);   // 1 / 7!
    sx = __builtin_fmaf(sx, x2, 8.3333333e-3f);    // 1 / 5!
    sx = __builtin_fmaf(sx, x2, -1.6666667e-1f);   // 1 / 3!
    sx = __builtin_fmaf(sx * x2, x, x);
    float cx = -2.7557319e-7f;                     // 1 / 10!
    cx = __builtin_fmaf(cx, x2, 2.4801587e-5f);    // 1 / 8!
    cx = __builtin_fmaf(cx, x2, -1.3888889e-3f);   // 1 / 6!
    cx = __builtin_fmaf(cx, x2, 4.1666667e-2f);    // 1 / 4!
    cx = __builtin_fmaf(cx, x2, -0.5f);
    cx = __builtin_fmaf(cx, x2, 1.f);
    const int q = (int)k & 3;
    const float a = q & 1 ? sx : cx, b = q & 1 ? cx : sx;
    c = q == 1 || q == 2 ? -a : a;
    s = q >= 2 ? -b : b;
}

// n / d for n < 2^16 and d <= 2^16, with m = ceil(2^32 / d): m d - 2^32 < d, so the quotient is over by less
// than n / 2^32 < 1 / d.
struct Div16 {
    uint32_t m;
    int d;
};
__device__ __forceinline__ int div16(int n, Div16 v) {
    return v.d == 1 ? n : (int)(((uint64_t)(uint32_t)n * v.m) >> 32);
}
inline Div16 make_div16(int d) { return {(uint32_t)((((uint64_t)1 << 32) + d - 1) / d), d}; }

}  // namespace
}  // namespace msda
