// Root-mean-square norm with a residual addition, its backward pass, and rows in 8 bits.
//   s = x + residual;  rstd = (mean(s^2) + eps)^(-1/2);  out = s * rstd * weight
//   codes: t = s * weight (or x), u = max|t| / 127, code = rne(t / u), the row's scale u * rstd (or u)
//   grad_x = rstd * (g - xh * mean(g * xh)) + grad_sum,  xh = s * rstd,  g = grad_out * weight
// Bound by memory, as layer norm is, and built like it: a row stays in the registers of the lanes that own it. A row's
// rstd divides its values and their largest alike, so the codes do not depend on it: they need the largest |t| and the
// sum of squares, which are found in one reduction, and the codes come from fp32 operations that do not depend on the
// order of any sum. A NaN stays the largest, and is told with
// the infinities by the largest's bits.
// Measured: 9973 rows x 2568 in fp16 with a residual, its sum and 8-bit results 33 to 36 us, 5.0 to 5.4 TB/s (a large copy
// 5.1); 39894 x 1024 in bf16 with a residual 40 to 47 forward, 53 backward and 5 for the sums; 16 x 4096 5.0.
#include "msda_codes.hpp"
#include "msda_rows.hpp"
#include "msda_serve.h"

namespace msda {
namespace {

// The largest of G lanes' values and the sum of others, as row_sums.
template <int NT, int G>
__device__ __forceinline__ void row_sum_and_max(float& sum, uint32_t& most, float* red, uint32_t* red_most) {
    constexpr int L = G < 64 ? G : 64;
    sum = group_sum<L>(sum);
#pragma unroll
    for (int m = 1; m < L; m *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)most, m, 64);
        most = o > most ? o : most;
    }
    if constexpr (G > 64) {
        constexpr int W = NT / 64;
        __syncthreads();  // the last ones have been read
        if ((threadIdx.x & 63) == 0) {
            red[threadIdx.x >> 6] = sum;
            red_most[threadIdx.x >> 6] = most;
        }
        __syncthreads();
        sum = 0.f;
        most = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            sum += red[w];
            most = red_most[w] > most ? red_most[w] : most;
        }
    }
}

template <typename T, int VEC, int NT, int G, int NV, RmsResult RESULT>
__global__ __launch_bounds__(NT) void rms_fwd_kernel(RmsParams p) {
    __shared__ float red[NT / 64];
    __shared__ uint32_t red_most[NT / 64];
    const int g = threadIdx.x % G;
    const int C = p.C;
    const float inv_c = 1.f / (float)C;
    float w[NV][VEC];
    if constexpr (RESULT != kCodes) load_columns<VEC, G, NV>(w, p.weight, 1.f, g, C, p.columns);
    const T* x = static_cast<const T*>(p.x);
    const T* r = static_cast<const T*>(p.residual);
    const int64_t step = (int64_t)gridDim.x * (NT / G);
    int64_t row = (int64_t)blockIdx.x * (NT / G) + threadIdx.x / G;
    // the next row's pieces are on their way while a row is reduced
    Piece<T, VEC> nx[NV], nr[NV];
    auto fetch = [&](int64_t of) {
        if (of >= p.rows) return;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + g) * VEC;
            if (c < C) {
                nx[j] = *reinterpret_cast<const Piece<T, VEC>*>(x + of * C + c);
                if (RESULT != kCodes && r) nr[j] = *reinterpret_cast<const Piece<T, VEC>*>(r + of * C + c);
            }
        }
    };
    fetch(row);
    for (; row < p.rows; row += step) {
        const int64_t at = row * C;
        float s[NV][VEC];
        float sum = 0.f, top = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + g) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[j][i] = (float)nx[j].v[i] + (RESULT != kCodes && r ? (float)nr[j].v[i] : 0.f);
            if (c < C) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    if constexpr (RESULT != kCodes) sum += s[j][i] * s[j][i];
                }
                if constexpr (RESULT != kNormed) {
                    auto t = [&](int i) { return RESULT == kCodes ? s[j][i] : s[j][i] * w[j][i]; };
#pragma unroll
                    for (int i = 0; i < VEC; i += 2) top = larger(top, t(i), i + 1 < VEC ? t(i + 1) : 0.f);
                }
            }
        }
        fetch(row + step);
        uint32_t most = magnitude_bits(top);
        if constexpr (RESULT == kNormed) {
            float one[1] = {sum};
            row_sums<NT, G>(one, red);
            sum = one[0];
        } else {
            row_sum_and_max<NT, G>(sum, most, red, red_most);
        }
        const float rstd = RESULT == kCodes ? 1.f : 1.f / sqrtf(sum * inv_c + p.eps);
        if constexpr (RESULT == kNormed) {
            if (g == 0 && p.rstd) p.rstd[row] = rstd;
        }
        float inverse = 0.f;
        if constexpr (RESULT != kNormed) {
            const float u = scale_of(most);
            if (u > 0.f) inverse = 1.f / u;
            if (g == 0) p.scale[row] = u * rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + g) * VEC;
            if (c < C) {
                if (RESULT != kCodes && p.sum) store_piece(static_cast<T*>(p.sum) + at + c, s[j]);
                if constexpr (RESULT == kNormed) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) s[j][i] = s[j][i] * rstd * w[j][i];
                    store_piece(static_cast<T*>(p.out) + at + c, s[j]);
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        if constexpr (RESULT == kNormedCodes) s[j][i] *= w[j][i];
                        if (most >= kNotFinite) s[j][i] = 0.f;
                    }
                    *reinterpret_cast<Piece<int8_t, VEC>*>(p.codes + at + c) = codes_of<VEC>(s[j], inverse);
                }
            }
        }
    }
}

template <typename T, int VEC, int NT, int G, int NV>
__global__ __launch_bounds__(NT) void rms_bwd_kernel(RmsParams p) {
    constexpr int kRows = NT / G;
    __shared__ float red[NT / 64];
    __shared__ float cols[kRows > 1 ? NT * NV * VEC : 1];
    const int g = threadIdx.x % G;
    const int C = p.C;
    const float inv_c = 1.f / (float)C;
    float w[NV][VEC], gw[NV][VEC];
    load_columns<VEC, G, NV>(w, p.weight, 1.f, g, C, p.columns);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) gw[j][i] = 0.f;
    const T* x = static_cast<const T*>(p.x);
    const T* r = static_cast<const T*>(p.residual);
    const T* go = static_cast<const T*>(p.grad_out);
    const T* gs = static_cast<const T*>(p.grad_sum);
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G; row < p.rows;
         row += (int64_t)gridDim.x * kRows) {
        const int64_t at = row * C;
        const float rstd = p.rstd[row];
        float xh[NV][VEC], gv[NV][VEC];
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + g) * VEC;
            if (c < C) {
                load_piece(xh[j], x + at + c);
                load_piece(gv[j], go + at + c);
                if (r) {
                    float y[VEC];
                    load_piece(y, r + at + c);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) xh[j][i] += y[i];
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    xh[j][i] *= rstd;
                    gw[j][i] += gv[j][i] * xh[j][i];
                    gv[j][i] *= w[j][i];
                    s[0] += gv[j][i] * xh[j][i];
                }
            }
        }
        row_sums<NT, G>(s, red);
        const float m1 = s[0] * inv_c;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + g) * VEC;
            if (c < C) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) gv[j][i] = rstd * (gv[j][i] - xh[j][i] * m1);
                if (gs) {
                    float y[VEC];
                    load_piece(y, gs + at + c);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) gv[j][i] += y[i];
                }
                store_piece(static_cast<T*>(p.grad_x) + at + c, gv[j]);
            }
        }
    }
    if (!p.partial) return;
    float* part = p.partial + (int64_t)blockIdx.x * C;
    if constexpr (kRows > 1) {
        // the workgroup's rows: one after the other's columns in LDS, then added up column by column
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) cols[(threadIdx.x / G) * (G * NV * VEC) + (j * G + g) * VEC + i] = gw[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < C; c += NT) {
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < kRows; ++k) t += cols[k * (G * NV * VEC) + c];
            part[c] = t;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * G + g) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (c + i < C) part[c + i] = gw[j][i];
        }
    }
}

template <RmsResult RESULT, typename T, int VEC>
hipError_t launch_forward_of(const RmsParams& p, hipStream_t stream) {
    return by_row<VEC>(p.C, [&](auto nt, auto g, auto nv) {
        constexpr int NT = decltype(nt)::value, G = decltype(g)::value, NV = decltype(nv)::value;
        const int64_t need = (p.rows + NT / G - 1) / (NT / G);
        const int64_t most = 2048 * 256 / NT;  // every CU full: lanes keep the weight over several rows
        hipLaunchKernelGGL((rms_fwd_kernel<T, VEC, NT, G, NV, RESULT>), dim3((unsigned)(need < most ? need : most)),
                           dim3(NT), 0, stream, p);
        return hipGetLastError();
    });
}

template <RmsResult RESULT, typename T>
hipError_t launch_forward_typed(const RmsParams& p, hipStream_t stream) {
    return p.vec ? launch_forward_of<RESULT, T, 16 / sizeof(T)>(p, stream) : launch_forward_of<RESULT, T, 1>(p, stream);
}

template <RmsResult RESULT>
hipError_t launch_forward(const RmsParams& p, int dtype, hipStream_t stream) {
    if (dtype == MSDA_F32) return launch_forward_typed<RESULT, float>(p, stream);
    if (dtype == MSDA_F16) return launch_forward_typed<RESULT, _Float16>(p, stream);
    return launch_forward_typed<RESULT, bf16_t>(p, stream);
}

template <typename T, int VEC>
hipError_t launch_backward_of(const RmsParams& p, hipStream_t stream) {
    return by_row<VEC>(p.C, [&](auto nt, auto g, auto nv) {
        constexpr int NT = decltype(nt)::value, G = decltype(g)::value, NV = decltype(nv)::value;
        hipLaunchKernelGGL((rms_bwd_kernel<T, VEC, NT, G, NV>), dim3(p.blocks), dim3(NT), 0, stream, p);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t launch_backward_typed(const RmsParams& p, hipStream_t stream) {
    return p.vec ? launch_backward_of<T, 16 / sizeof(T)>(p, stream) : launch_backward_of<T, 1>(p, stream);
}

}  // namespace

hipError_t launch_rms_forward(const RmsParams& p, RmsResult result, int dtype, hipStream_t stream) {
    if (result == kNormed) return launch_forward<kNormed>(p, dtype, stream);
    if (result == kNormedCodes) return launch_forward<kNormedCodes>(p, dtype, stream);
    return launch_forward<kCodes>(p, dtype, stream);
}

hipError_t launch_rms_backward(const RmsParams& p, int dtype, hipStream_t stream) {
    if (p.rows == 0) return p.grad_weight ? launch_column_zeros(p.grad_weight, nullptr, p.C, stream) : hipSuccess;
    hipError_t e = dtype == MSDA_F32   ? launch_backward_typed<float>(p, stream)
                   : dtype == MSDA_F16 ? launch_backward_typed<_Float16>(p, stream)
                                       : launch_backward_typed<bf16_t>(p, stream);
    if (e != hipSuccess || !p.partial) return e;
    return launch_column_sums(p.partial, p.grad_weight, nullptr, p.C, p.blocks, stream);
}

}  // namespace msda
