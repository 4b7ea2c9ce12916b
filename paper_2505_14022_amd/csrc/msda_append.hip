// New keys and values into a paged cache of 8 bits, the keys turned by their positions on the way.
//   u' = max(u where tokens stood in the page, most * (1 / 127)),  old codes rne(code * (u / u')) if u' > u,  new ones rne(x * (1 / u'))
// Bound by memory (2 or 4 bytes read and 1 written for each channel), or by latency for single tokens. A workgroup has one page of
// one sequence, and each of its waves one head's keys or values of that page: nothing is shared between heads
// but the positions' cosines and sines, which the workgroup forms once, in LDS. A lane takes two 16-byte pieces at a time, a
// pair's two where the channels of a pair lie in halves. The largest value has to be known before the first code can be
// written: what a lane has loaded first stays in its registers (4 times two pieces, half a page of 64 tokens of 128 channels in 16
// bits), and the rest is read again, from a cache. (Chunks of up to 2048 tokens of 16 sequences, 8 heads of 128 channels in
// fp16: 54 us, 2.9 TB/s, the waves waiting for memory in 60 % of their time; with 8 times two pieces, of which the registers leave room
// for fewer waves, 72; with none 96.)
#include "msda_cache.hpp"
#include "msda_codes.hpp"
#include "msda_turn.hpp"

namespace msda {
namespace {

constexpr int kUnits = 4;  // heads (of keys or of values) of a workgroup, one to a wave

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)x, m, 64);
        x = o > x ? o : x;
    }
    return x;
}

constexpr int kHeld = 4;  // items that a lane keeps

// Two pieces of VEC channels of a head, from channels c0 and c1 on: a pair's two, or neighbours.
struct Item {
    int token, c0, c1;
    bool turned;
};
template <int VEC>
__device__ __forceinline__ Item item_of(int i, Div16 per_token, int R, bool interleaved) {
    const int k = div16(i, per_token), j = i - k * per_token.d;
    const int turned = R / VEC;  // items that are turned, of a head
    if (!interleaved && j < turned) return {k, j * VEC, R + j * VEC, true};
    return {k, 2 * j * VEC, (2 * j + 1) * VEC, j < turned};
}
template <int VEC>
__device__ __forceinline__ void turn(float (&y0)[VEC], float (&y1)[VEC], const Item& x, bool interleaved, const float* cs,
                                     const float* sn) {
    if (!x.turned) return;
    auto pair = [](float& a, float& b, float c, float s) {
        const float u = a * c - b * s;
        b = a * s + b * c;
        a = u;
    };
    if constexpr (VEC > 1) {
        if (interleaved) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                pair(y0[e], y0[e + 1], cs[(x.c0 + e) / 2], sn[(x.c0 + e) / 2]);
                pair(y1[e], y1[e + 1], cs[(x.c1 + e) / 2], sn[(x.c1 + e) / 2]);
            }
            return;
        }
    }
    const int first = interleaved ? x.c0 / 2 : x.c0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) pair(y0[e], y1[e], cs[first + e], sn[first + e]);
}

template <typename T, int VEC>
__global__ __launch_bounds__(64 * kUnits, 4) void append_kernel(AppendParams p, Div16 per_token, Div16 pairs) {
    extern __shared__ float turns[];
    const Cache& c = p.c;
    const int lane = threadIdx.x & 63, wave = wave_index();
    const Place t = find_place(c, blockIdx.x, c.page, 2, lane);
    if (t.n < 0) return;
    // the page's column in the table, and its new tokens: slots s0 .. s1 - 1
    const int column = (max(t.first, 0) >> c.page_shift) + t.block;
    const int64_t base = (int64_t)column << c.page_shift;
    const int s0 = (int)max((int64_t)t.first - base, (int64_t)0), s1 = (int)min((int64_t)t.length - base, (int64_t)c.page);
    if (s0 >= s1) return;
    const int page = page_at(c, t.n, column);
    if (page < 0) return;
    const int nt = s1 - s0;
    const int64_t token0 = t.start + (base + s0 - t.first);  // the call's token in slot s0

    const int unit = blockIdx.y * kUnits + wave, units = 2 * c.Mkv;  // keys' heads, then values'
    const float *cs = turns, *sn = turns + nt * p.R;
    const bool turns_any = blockIdx.y * kUnits < (unsigned)c.Mkv && p.R > 0;
    // The cosines and sines of the page's new tokens; all of the workgroup's waves take part.
    auto form_turns = [&]() {
        if (!turns_any) return;
        for (int i = threadIdx.x; i < nt * p.R; i += 64 * kUnits) {
            const int k = div16(i, pairs), r = i - k * p.R;
            double by = 0.0;
            if (p.pos)
                for (int a = 0; a < p.A; ++a) by += (double)p.pos[(token0 + k) * p.A + a] * (double)p.freqs[a * p.R + r];
            else by = (double)(base + s0 + k) * (double)p.freqs[r];
            float co, si;
            cos_sin(by * 0.15915494309189535, co, si);
            turns[i] = co;
            turns[nt * p.R + i] = si;
        }
        __syncthreads();
    };
    if (unit >= units) {
        form_turns();
        return;
    }
    const bool keys = unit < c.Mkv;
    const int head = keys ? unit : unit - c.Mkv, R = keys ? p.R : 0;
    const int64_t* stride = keys ? p.ks : p.vs;
    const T* from = static_cast<const T*>(keys ? p.k : p.v) + token0 * stride[0] + head * stride[1];
    const int64_t slab = (int64_t)page * c.Mkv + head;
    int8_t* codes = (keys ? c.k : c.v) + slab * c.page * c.D;
    float* scale = (keys ? c.k_scale : c.v_scale) + slab;
    const float old = s0 > 0 ? *scale : 0.f;

    const int count = nt * per_token.d;  // items
    float top = 0.f;
    Piece<T, VEC> held[kHeld][2];
    auto load = [&](int i, Piece<T, VEC> (&x)[2]) {
        const Item it = item_of<VEC>(i, per_token, R, p.interleaved);
        const T* row = from + it.token * stride[0];
        x[0] = *reinterpret_cast<const Piece<T, VEC>*>(row + it.c0);
        x[1] = *reinterpret_cast<const Piece<T, VEC>*>(row + it.c1);
    };
    auto values = [&](const Item& it, const Piece<T, VEC> (&x)[2], float (&y0)[VEC], float (&y1)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            y0[e] = (float)x[0].v[e];
            y1[e] = (float)x[1].v[e];
        }
        turn<VEC>(y0, y1, it, p.interleaved, cs + it.token * p.R, sn + it.token * p.R);
    };
    auto look = [&](int i, const Piece<T, VEC> (&x)[2]) {
        float y0[VEC], y1[VEC];
        values(item_of<VEC>(i, per_token, R, p.interleaved), x, y0, y1);
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = larger(top, y0[e], y1[e]);
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
        if (lane + 64 * h < count) load(lane + 64 * h, held[h]);
    form_turns();
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
        if (lane + 64 * h < count) look(lane + 64 * h, held[h]);
    for (int i = lane + 64 * kHeld; i < count; i += 64) {
        Piece<T, VEC> x[2];
        load(i, x);
        look(i, x);
    }
    float u = scale_of(wave_max(magnitude_bits(top)));
    const bool odd = u != u || !(old >= 0.f && old < __builtin_huge_valf());
    u = old > u ? old : u;
    const float inverse = u > 0.f && !odd ? 1.f / u : 0.f;
    if (u > old && !odd) {
        const float ratio = old / u;  // of a page of scale 0, whatever its codes are, it makes zeros
        for (int i = lane * 16; i < s0 * c.D; i += 64 * 16) {
            auto x = *reinterpret_cast<const Piece<int8_t, 16>*>(codes + i);
#pragma unroll
            for (int e = 0; e < 16; ++e) x.v[e] = (int8_t)(int)rintf((float)x.v[e] * ratio);
            *reinterpret_cast<Piece<int8_t, 16>*>(codes + i) = x;
        }
    }
    auto write = [&](int i, const Piece<T, VEC> (&x)[2]) {
        const Item it = item_of<VEC>(i, per_token, R, p.interleaved);
        float y0[VEC], y1[VEC];
        values(it, x, y0, y1);
        Piece<int8_t, VEC> z0 = {}, z1 = {};
        if (!odd) {
            z0 = codes_of<VEC>(y0, inverse);
            z1 = codes_of<VEC>(y1, inverse);
        }
        int8_t* row = codes + (s0 + it.token) * c.D;
        *reinterpret_cast<Piece<int8_t, VEC>*>(row + it.c0) = z0;
        *reinterpret_cast<Piece<int8_t, VEC>*>(row + it.c1) = z1;
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
        if (lane + 64 * h < count) write(lane + 64 * h, held[h]);
    for (int i = lane + 64 * kHeld; i < count; i += 64) {
        Piece<T, VEC> x[2];
        load(i, x);
        write(i, x);
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
    hipLaunchKernelGGL(kernel, grid, dim3(64 * kUnits), lds, stream, p, make_div16(p.c.D / (2 * VEC)),
                       make_div16(p.R > 0 ? p.R : 1));
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
