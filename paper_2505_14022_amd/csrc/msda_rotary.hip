// Rotary positions of several axes: pair i of a token is turned by angle_i = sum over axes of pos * freq.
// Bound by memory: each element is read and written once. The angles are the same for every head, so a
// workgroup forms the cosines and sines of its tokens once, in LDS, and then streams its tokens' channels
// past them. An angle is reduced in fp64, in turns (pos * freq / 2 pi), so that a position of 10^7 keeps
// its angle to fp32 accuracy; what is left, at most an eighth of a turn, goes through the Taylor series of
// sine and cosine in fp32.
#include "msda_layer.h"
#include "msda_layer.hpp"

namespace msda {
namespace {

constexpr int kPairs = 2048;  // pairs of a workgroup's tokens: 16 KB of cosines and sines

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
Div16 make_div16(int d) { return {(uint32_t)((((uint64_t)1 << 32) + d - 1) / d), d}; }

// VEC pairs per item (two 16-byte pieces), or one. An item of a head beyond the pairs copies VEC channels.
template <typename T, int VEC>
struct Item {
    int64_t from, to;  // of its head's first channel
    int c0, c1, pair;  // first channels of its pieces (c1 < 0: one piece, copied), and its first pair in LDS
    Piece<T, VEC> u, v;
};

template <typename T, int VEC>
__device__ __forceinline__ void take_item(const RotaryParams& p, Item<T, VEC>& it, const T* x, int i, Div16 per_token, Div16 items) {
    const int t = div16(i, per_token), j = i - t * per_token.d;
    const int m = div16(j, items), k = j - m * items.d;
    const int r = k * VEC;
    it.from = t * p.xs[1] + m * p.xs[2];
    it.to = t * p.os[1] + m * p.os[2];
    it.pair = t * p.R + r;
    if (r >= p.R) {
        it.c0 = p.R + r;  // 2R + the channels of the copying items before
        it.c1 = -1;
    } else {
        it.c0 = p.interleaved ? 2 * r : r;
        it.c1 = p.interleaved ? 2 * r + VEC : p.R + r;
        it.v = *reinterpret_cast<const Piece<T, VEC>*>(x + it.from + it.c1);
    }
    it.u = *reinterpret_cast<const Piece<T, VEC>*>(x + it.from + it.c0);
}

template <typename T, int VEC>
__device__ __forceinline__ void turn_item(const RotaryParams& p, const Item<T, VEC>& it, T* out, const float* s_cos, const float* s_sin) {
    float u[VEC], v[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        u[j] = (float)it.u.v[j];
        v[j] = (float)it.v.v[j];
    }
    // plain stores: a wave writes every other 16 or 32 bytes, and the rest of the lines with its next store (streaming
    // stores took 83 us in place of 65 for 8 x 40000 tokens of 8 x 32 channels in bf16)
    auto put = [](T* to, const float (&f)[VEC]) { *reinterpret_cast<Piece<T, VEC>*>(to) = to_piece<T>(f); };
    T* to = out + it.to;
    if (it.c1 < 0) {
        put(to + it.c0, u);
        return;
    }
    const float* cs = s_cos + it.pair;
    const float* sn = s_sin + it.pair;
    if (VEC > 1 && p.interleaved) {
        // u and v are the item's first VEC / 2 pairs and its others
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
            const float a = u[2 * j], b = u[2 * j + 1];
            u[2 * j] = a * cs[j] - b * sn[j];
            u[2 * j + 1] = a * sn[j] + b * cs[j];
            const float d = v[2 * j], e = v[2 * j + 1];
            v[2 * j] = d * cs[VEC / 2 + j] - e * sn[VEC / 2 + j];
            v[2 * j + 1] = d * sn[VEC / 2 + j] + e * cs[VEC / 2 + j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float a = u[j], b = v[j];
            u[j] = a * cs[j] - b * sn[j];
            v[j] = a * sn[j] + b * cs[j];
        }
    }
    put(to + it.c0, u);
    put(to + it.c1, v);
}

// A thread's first item is on its way while the workgroup forms the cosines and sines.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p, int tokens, Div16 per_token, Div16 items) {
    __shared__ float s_cos[kPairs], s_sin[kPairs];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int n = blockIdx.y;
    const int nt = (int)(p.T - t0 < tokens ? p.T - t0 : tokens);
    const T* x = static_cast<const T*>(p.x) + n * p.xs[0] + t0 * p.xs[1];
    T* out = static_cast<T*>(p.out) + n * p.os[0] + t0 * p.os[1];
    const int count = nt * per_token.d;  // at most 2^16
    Item<T, VEC> first;
    if ((int)threadIdx.x < count) take_item(p, first, x, threadIdx.x, per_token, items);
    const float* pos = p.pos + n * p.pos_item + t0 * p.A;
    for (int i = threadIdx.x; i < nt * p.R; i += 256) {
        const int t = i / p.R, r = i - t * p.R;
        double turns = 0.0;
        for (int a = 0; a < p.A; ++a) turns += (double)pos[t * p.A + a] * (double)p.freqs[a * p.R + r];
        float c, s;
        cos_sin(turns * 0.15915494309189535, c, s);
        s_cos[i] = c;
        s_sin[i] = p.sign * s;
    }
    __syncthreads();
    if ((int)threadIdx.x < count) turn_item(p, first, out, s_cos, s_sin);
    for (int i = threadIdx.x + 256; i < count; i += 256) {
        Item<T, VEC> it;
        take_item(p, it, x, i, per_token, items);
        turn_item(p, it, out, s_cos, s_sin);
    }
}

template <typename T, int VEC>
hipError_t launch_typed(const RotaryParams& p, hipStream_t stream) {
    const int items = p.R / VEC + (p.D - 2 * p.R) / VEC;
    // tokens per workgroup: about two items a thread, as many pairs as LDS holds, and enough workgroups
    int tokens = 512 / (items * p.M);
    if (p.R > 0 && tokens > kPairs / p.R) tokens = kPairs / p.R;
    if (tokens < 1) tokens = 1;
    while (tokens > 1 && (p.T + tokens - 1) / tokens * p.N < 1024) tokens = (tokens + 1) / 2;
    const int64_t gx = (p.T + tokens - 1) / tokens;
    if (gx > 0x7fffffff) return hipErrorInvalidValue;
    const int most = 65535;  // batch items of a launch
    for (int n0 = 0; n0 < p.N; n0 += most) {
        RotaryParams c = p;
        c.N = p.N - n0 < most ? p.N - n0 : most;
        c.x = static_cast<const T*>(p.x) + n0 * p.xs[0];
        c.out = static_cast<T*>(p.out) + n0 * p.os[0];
        c.pos = p.pos + n0 * p.pos_item;
        hipLaunchKernelGGL((rotary_kernel<T, VEC>), dim3((unsigned)gx, c.N), dim3(256), 0, stream, c, tokens,
                           make_div16(items * p.M), make_div16(items));
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t stream) {
    if (dtype == MSDA_F32) return p.vec ? launch_typed<float, 4>(p, stream) : launch_typed<float, 1>(p, stream);
    if (dtype == MSDA_F16) return p.vec ? launch_typed<_Float16, 8>(p, stream) : launch_typed<_Float16, 1>(p, stream);
    return p.vec ? launch_typed<bf16_t, 8>(p, stream) : launch_typed<bf16_t, 1>(p, stream);
}

}  // namespace msda
