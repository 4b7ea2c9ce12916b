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

// The cosines and sines of the workgroup's tokens, into LDS.
__device__ __forceinline__ void form_angles(const RotaryParams& p, const float* pos, int nt, float* s_cos, float* s_sin) {
    for (int i = threadIdx.x; i < nt * p.R; i += 256) {
        const int t = i / p.R, r = i - t * p.R;
        double turns = 0.0;
        for (int a = 0; a < p.A; ++a) turns += (double)pos[t * p.A + a] * (double)p.freqs[a * p.R + r];
        float c, s;
        cos_sin(turns * 0.15915494309189535, c, s);
        s_cos[i] = c;
        s_sin[i] = p.sign * s;
    }
}

// Heads of whole 16-byte pieces: a thread writes one piece at a time, so that a wave's stores are whole cache lines.
// With the pairs in halves it reads its piece's partner too, which a neighbour's read brings into the cache. (Both
// pieces of a pair in one thread: its stores are every other 32 bytes of a head of 32 channels, and both passes over
// 8 x 40000 x 8 x 32 in bf16 take 165 us, 170 to 176 with more loads ahead, in place of 134.)
// In place, a piece is read by two threads before either writes: each turn takes whole heads, and the barrier is between.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void rotary_pieces_kernel(RotaryParams p, int tokens, Div16 per_token, Div16 per_head) {
    __shared__ float s_cos[kPairs], s_sin[kPairs];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int n = blockIdx.y, nt = (int)(p.T - t0 < tokens ? p.T - t0 : tokens);
    const T* x = static_cast<const T*>(p.x) + n * p.xs[0] + t0 * p.xs[1];
    T* out = static_cast<T*>(p.out) + n * p.os[0] + t0 * p.os[1];
    const int count = nt * per_token.d;              // at most 2^16
    const int width = 256 / per_head.d * per_head.d; // pieces of whole heads that 256 threads take
    const int half = p.R / VEC, turned = 2 * half;   // pieces of a head from a pair's one channel to the other, and all turned
    for (int base = 0; base < count; base += width) {
        const int i = base + threadIdx.x;
        const bool mine = (int)threadIdx.x < width && i < count;
        const int t = div16(i, per_token), j = i - t * per_token.d, m = div16(j, per_head), k = j - m * per_head.d;
        const bool beside = p.interleaved, lower = k < half;
        const int pair = t * p.R + (beside ? k * (VEC / 2) : (lower ? k : k - half) * VEC);
        Piece<T, VEC> u, v;
        if (mine) {
            const T* from = x + t * p.xs[1] + m * p.xs[2] + k * VEC;
            u = *reinterpret_cast<const Piece<T, VEC>*>(from);
            if (!beside && k < turned) v = *reinterpret_cast<const Piece<T, VEC>*>(from + (lower ? half : -half) * VEC);
        }
        // the first pieces are on their way meanwhile
        if (base == 0) form_angles(p, p.pos + n * p.pos_item + t0 * p.A, nt, s_cos, s_sin);
        __syncthreads();
        if (!mine) continue;
        float y[VEC];
        if (k >= turned) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = (float)u.v[e];
        } else if (beside) {
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) {
                const float a = (float)u.v[2 * e], b = (float)u.v[2 * e + 1], c = s_cos[pair + e], s = s_sin[pair + e];
                y[2 * e] = a * c - b * s;
                y[2 * e + 1] = a * s + b * c;
            }
        } else {
            const float sign = lower ? -1.f : 1.f;  // a c - b s, and b c + a s
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                y[e] = (float)u.v[e] * s_cos[pair + e] + sign * ((float)v.v[e] * s_sin[pair + e]);
        }
        store_piece(out + t * p.os[1] + m * p.os[2] + k * VEC, y);
    }
}

// Other heads: a thread turns one pair at a time, or copies one channel.
template <typename T>
__global__ __launch_bounds__(256) void rotary_pairs_kernel(RotaryParams p, int tokens, Div16 per_token, Div16 per_head) {
    __shared__ float s_cos[kPairs], s_sin[kPairs];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int n = blockIdx.y, nt = (int)(p.T - t0 < tokens ? p.T - t0 : tokens);
    form_angles(p, p.pos + n * p.pos_item + t0 * p.A, nt, s_cos, s_sin);
    __syncthreads();
    const T* x = static_cast<const T*>(p.x) + n * p.xs[0] + t0 * p.xs[1];
    T* out = static_cast<T*>(p.out) + n * p.os[0] + t0 * p.os[1];
    for (int i = threadIdx.x; i < nt * per_token.d; i += 256) {  // at most 2^16
        const int t = div16(i, per_token), j = i - t * per_token.d, m = div16(j, per_head), k = j - m * per_head.d;
        const T* from = x + t * p.xs[1] + m * p.xs[2];
        T* to = out + t * p.os[1] + m * p.os[2];
        if (k >= p.R) {
            to[p.R + k] = from[p.R + k];
            continue;
        }
        const int c0 = p.interleaved ? 2 * k : k, c1 = p.interleaved ? 2 * k + 1 : p.R + k;
        const float a = (float)from[c0], b = (float)from[c1], c = s_cos[t * p.R + k], s = s_sin[t * p.R + k];
        to[c0] = (T)(a * c - b * s);
        to[c1] = (T)(a * s + b * c);
    }
}

// What a head is to the threads: pieces of `vec` channels, or pairs and copied channels.
int items_of_head(const RotaryParams& p, int vec) { return vec > 1 ? p.D / vec : p.D - p.R; }

// Tokens per workgroup: about four items a thread, as many pairs as LDS holds, and enough workgroups.
int tokens_of_workgroup(const RotaryParams& p, int items) {
    int tokens = 1024 / (items * p.M);
    if (p.R > 0 && tokens > kPairs / p.R) tokens = kPairs / p.R;
    if (tokens < 1) tokens = 1;
    while (tokens > 1 && (p.T + tokens - 1) / tokens * p.N < 1024) tokens = (tokens + 1) / 2;
    return tokens;
}

template <typename T, int VEC>
hipError_t launch_typed(const RotaryParams& p, hipStream_t stream) {
    const int items = items_of_head(p, VEC), tokens = tokens_of_workgroup(p, items);
    const int64_t gx = (p.T + tokens - 1) / tokens;
    const int most = 65535;  // batch items of a launch
    for (int n0 = 0; n0 < p.N; n0 += most) {
        RotaryParams c = p;
        c.N = p.N - n0 < most ? p.N - n0 : most;
        c.x = static_cast<const T*>(p.x) + n0 * p.xs[0];
        c.out = static_cast<T*>(p.out) + n0 * p.os[0];
        c.pos = p.pos + n0 * p.pos_item;
        const dim3 grid((unsigned)gx, c.N);
        const Div16 per_token = make_div16(items * p.M), per_head = make_div16(items);
        if constexpr (VEC > 1)
            hipLaunchKernelGGL((rotary_pieces_kernel<T, VEC>), grid, dim3(256), 0, stream, c, tokens, per_token, per_head);
        else hipLaunchKernelGGL((rotary_pairs_kernel<T>), grid, dim3(256), 0, stream, c, tokens, per_token, per_head);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t rotary_workgroups(const RotaryParams& p, int dtype) {
    const int tokens = tokens_of_workgroup(p, items_of_head(p, p.vec ? 16 / dtype_size(dtype) : 1));
    return (p.T + tokens - 1) / tokens;
}

hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t stream) {
    if (dtype == MSDA_F32) return p.vec ? launch_typed<float, 4>(p, stream) : launch_typed<float, 1>(p, stream);
    if (dtype == MSDA_F16) return p.vec ? launch_typed<_Float16, 8>(p, stream) : launch_typed<_Float16, 1>(p, stream);
    return p.vec ? launch_typed<bf16_t, 8>(p, stream) : launch_typed<bf16_t, 1>(p, stream);
}

}  // namespace msda
