// New keys and values into a paged cache of 8 bits, the keys turned by their positions on the way.
//   u' = max(u where tokens stood in the page, most * (1 / 127)),  old codes rne(code * (u / u')),  new ones rne(x * (1 / u'))
// Bound by memory (2 or 4 bytes read and 1 written for each channel), or by latency for single tokens. A workgroup has one page of
// one sequence, and each of its waves in turn one head's keys or values of that page: nothing is shared between heads
// but the positions' cosines and sines, which the workgroup forms once, in LDS. The largest value has to be known before the
// first code can be written, so a wave reads its tokens twice, the second time from a cache.
#include "msda_cache.hpp"
#include "msda_turn.hpp"

namespace msda {
namespace {

constexpr int kUnits = 4;  // heads (of keys or of values) of a workgroup, one to a wave
constexpr uint32_t kNotFinite = 0x7f800000u, kLeast = 0x0d800000u;  // bits of infinity, and of 2^-100

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)x, m, 64);
        x = o > x ? o : x;
    }
    return x;
}

// Channels c .. c + VEC - 1 of a head, turned by the token's cosines and sines.
template <typename T, int VEC>
__device__ __forceinline__ void load_turned(float (&y)[VEC], const T* head, int c, int R, bool interleaved, const float* cs,
                                            const float* sn) {
    load_piece(y, head + c);
    if (c >= 2 * R) return;
    if (interleaved) {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const float a = y[e], b = y[e + 1], co = cs[(c + e) / 2], si = sn[(c + e) / 2];
                y[e] = a * co - b * si;
                y[e + 1] = a * si + b * co;
            }
        } else {
            const float b = (float)head[c ^ 1], co = cs[c / 2], si = sn[c / 2];
            y[0] = c & 1 ? b * si + y[0] * co : y[0] * co - b * si;
        }
    } else {
        const bool lower = c < R;
        const int pair = lower ? c : c - R;
        float o[VEC];
        load_piece(o, head + (lower ? c + R : c - R));
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[e] = lower ? y[e] * cs[pair + e] - o[e] * sn[pair + e] : o[e] * sn[pair + e] + y[e] * cs[pair + e];
    }
}

template <typename T, int VEC>
__global__ __launch_bounds__(64 * kUnits) void append_kernel(AppendParams p, Div16 per_token) {
    extern __shared__ float turns[];
    const Cache& c = p.c;
    const int lane = threadIdx.x & 63, wave = wave_index();
    const Place at = c.start ? find_place(c, blockIdx.x, c.page, 2, lane) : Place{(int)blockIdx.x, 0};
    if (at.n < 0) return;
    const Tokens t(c, at.n);
    // the page's column in the table, and its new tokens: slots s0 .. s1 - 1
    const int column = (max(t.first, 0) >> c.page_shift) + at.block;
    const int64_t base = (int64_t)column << c.page_shift;
    const int s0 = (int)max((int64_t)t.first - base, (int64_t)0), s1 = (int)min((int64_t)t.length - base, (int64_t)c.page);
    if (s0 >= s1) return;
    const int page = page_at(c, at.n, column);
    if (page < 0) return;
    const int nt = s1 - s0;
    const int64_t token0 = t.start + (base + s0 - t.first);  // the call's token in slot s0

    const int unit = blockIdx.y * kUnits + wave, units = 2 * c.Mkv;  // keys' heads, then values'
    const float *cs = turns, *sn = turns + nt * p.R;
    if (blockIdx.y * kUnits < (unsigned)c.Mkv && p.R > 0) {
        for (int i = threadIdx.x; i < nt * p.R; i += 64 * kUnits) {
            const int k = i / p.R, r = i - k * p.R;
            double turn = 0.0;
            if (p.pos)
                for (int a = 0; a < p.A; ++a) turn += (double)p.pos[(token0 + k) * p.A + a] * (double)p.freqs[a * p.R + r];
            else turn = (double)(base + s0 + k) * (double)p.freqs[r];
            float co, si;
            cos_sin(turn * 0.15915494309189535, co, si);
            turns[i] = co;
            turns[nt * p.R + i] = si;
        }
        __syncthreads();
    }
    if (unit >= units) return;
    const bool keys = unit < c.Mkv;
    const int head = keys ? unit : unit - c.Mkv, R = keys ? p.R : 0;
    const int64_t* stride = keys ? p.ks : p.vs;
    const T* from = static_cast<const T*>(keys ? p.k : p.v) + token0 * stride[0] + head * stride[1];
    const int64_t slab = (int64_t)page * c.Mkv + head;
    int8_t* codes = (keys ? c.k : c.v) + slab * c.page * c.D;
    float* scale = (keys ? c.k_scale : c.v_scale) + slab;
    const float old = s0 > 0 ? *scale : 0.f;

    const int count = nt * per_token.d;  // pieces
    uint32_t most = 0;
#pragma unroll 4
    for (int i = lane; i < count; i += 64) {
        const int k = div16(i, per_token), ch = (i - k * per_token.d) * VEC;
        float y[VEC];
        load_turned<T, VEC>(y, from + k * stride[0], ch, R, p.interleaved, cs + k * p.R, sn + k * p.R);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, y[e]) & 0x7fffffffu;
            most = bits > most ? bits : most;
        }
    }
    most = wave_max(most);
    float u = most < kLeast ? 0.f : __builtin_bit_cast(float, most) * (1.f / 127.f);
    u = old > u ? old : u;
    const bool odd = most >= kNotFinite || !(fabsf(old) < __builtin_huge_valf());
    const float inverse = u > 0.f && !odd ? 1.f / u : 0.f;
    if (old > 0.f && u > old && !odd) {
        const float ratio = old / u;
        for (int i = lane * 16; i < s0 * c.D; i += 64 * 16) {
            auto x = *reinterpret_cast<const Piece<int8_t, 16>*>(codes + i);
#pragma unroll
            for (int e = 0; e < 16; ++e) x.v[e] = (int8_t)(int)rintf((float)x.v[e] * ratio);
            *reinterpret_cast<Piece<int8_t, 16>*>(codes + i) = x;
        }
    }
#pragma unroll 4
    for (int i = lane; i < count; i += 64) {
        const int k = div16(i, per_token), ch = (i - k * per_token.d) * VEC;
        float y[VEC];
        load_turned<T, VEC>(y, from + k * stride[0], ch, R, p.interleaved, cs + k * p.R, sn + k * p.R);
        Piece<int8_t, VEC> x;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x.v[e] = odd ? 0 : (int8_t)(int)fminf(fmaxf(rintf(y[e] * inverse), -127.f), 127.f);
        *reinterpret_cast<Piece<int8_t, VEC>*>(codes + (s0 + k) * c.D + ch) = x;
    }
    if (lane == 0) *scale = odd ? __builtin_nanf("") : u;
}

template <typename T, int VEC>
hipError_t launch_typed(const AppendParams& p, hipStream_t stream) {
    // cosines and sines of a page's tokens, of which a call with one token each has one
    const int tokens = p.c.start ? (p.c.page < p.c.T ? p.c.page : p.c.T) : 1;
    const size_t lds = (size_t)tokens * p.R * 2 * sizeof(float);
    const auto kernel = append_kernel<T, VEC>;
    if (lds > 65536) {
        hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)place_count(p.c, p.c.page, 2), (unsigned)((2 * p.c.Mkv + kUnits - 1) / kUnits));
    hipLaunchKernelGGL(kernel, grid, dim3(64 * kUnits), lds, stream, p, make_div16(p.c.D / VEC));
    return hipGetLastError();
}

}  // namespace

int64_t append_workgroups(const AppendParams& p) { return place_count(p.c, p.c.page, 2) * ((2 * p.c.Mkv + kUnits - 1) / kUnits); }

hipError_t launch_append(const AppendParams& p, int dtype, hipStream_t stream) {
    if (dtype == MSDA_F32) return p.vec ? launch_typed<float, 4>(p, stream) : launch_typed<float, 1>(p, stream);
    if (dtype == MSDA_F16) return p.vec ? launch_typed<_Float16, 8>(p, stream) : launch_typed<_Float16, 1>(p, stream);
    return p.vec ? launch_typed<bf16_t, 8>(p, stream) : launch_typed<bf16_t, 1>(p, stream);
}

}  // namespace msda
