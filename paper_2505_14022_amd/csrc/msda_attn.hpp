// Dense attention: what the forward and the two backward kernels share.
//
// A wave owns 32 rows (queries) or 32 keys, one per lane of each half wave, and walks over tiles of the
// other axis that its workgroup stages in LDS. All products are 32 x 32 matrix instructions with fp32 sums,
// arranged so that the owner is the column: the scores of the owner's column lie in the lane's own registers
// (16 of each 32, the other half wave holds the rest), softmax statistics are lane values, and a column of
// probabilities is already the operand of the next product: its registers hold rows
//   8 (r / 4) + 4 h + r % 4        (h: half wave, r: register)
// and a sum over rows may take them in any order as long as the other operand's rows are read in the same
// order. So nothing is exchanged between lanes but one maximum per tile.
#pragma once

#include <type_traits>

#include "msda_layer.h"
#include "msda_layer.hpp"

namespace msda {
namespace {

typedef float acc_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// tanh(x) = 1 - 2 / (e^2x + 1), off by an fp32 rounding of 1; with fp32 operands, where that shows in
// the result, |x| < 1/4 goes through the series x - x^3/3 + 2x^5/15 - 17x^7/315 (next term: 8e-8 of x).
template <bool SERIES>
__device__ __forceinline__ float tanh_of(float x) {
    const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(exp2_of(2.f * kLog2e * x) + 1.f);
    if constexpr (!SERIES) return t;
    const float x2 = x * x;
    float s = __builtin_fmaf(x2, -17.f / 315.f, 2.f / 15.f);
    s = __builtin_fmaf(s, x2, -1.f / 3.f);
    s = __builtin_fmaf(s * x2, x, x);
    return fabsf(x) < 0.25f ? s : t;
}

// The value of both half waves' lanes l and l ^ 32: x of the lower half in lo, of the upper in hi.
__device__ __forceinline__ void both_halves(float x, float& lo, float& hi) {
    const int u = __builtin_bit_cast(int, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const int a = r[0], b = r[1];
    lo = __builtin_bit_cast(float, a);
    hi = __builtin_bit_cast(float, b);
}
__device__ __forceinline__ float halves_sum(float x) {
    float a, b;
    both_halves(x, a, b);
    return a + b;
}
__device__ __forceinline__ float halves_max(float x) {
    float a, b;
    both_halves(x, a, b);
    return fmaxf(a, b);
}

// Matrix operands of an element type. A fragment is 16 bytes per lane: K / 2 elements of the lane's
// row or column; half wave h holds the upper or lower half of every K summed positions.
template <typename T>
struct Op;

template <typename T, typename V>
struct Op16 {
    using Frag = V;
    static constexpr int K = 16;
    static constexpr int kTile = 64;  // keys or rows staged at a time
    // Rows row0 + {4h .. 4h+3, 8+4h .. 8+4h+3} at channel c0 + lane % 32: ds_read_tr16 turns 4 rows x 16
    // channels, read as 8 bytes per lane, into 4 rows of one channel per lane (in each 16 lanes).
    static __device__ __forceinline__ Frag column(const T* tile, int stride, int row0, int c0, int lane) {
        const T* at = tile + (row0 + 4 * (lane >> 5) + ((lane & 15) >> 2)) * stride + c0 + (lane & 16) + (lane & 3) * 4;
        using P = __attribute__((address_space(3))) short4_t;
        const short4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P*)at);
        const short4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P*)(at + 8 * stride));
        typedef short short8_t __attribute__((ext_vector_type(8)));
        const short8_t x = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(Frag, x);
    }
    static __device__ __forceinline__ Frag pack(const float* x) {
        Frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (T)x[i];
        return f;
    }
};
template <>
struct Op<_Float16> : Op16<_Float16, _Float16 __attribute__((ext_vector_type(8)))> {
    static __device__ __forceinline__ acc_t mma(Frag a, Frag b, acc_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Op<bf16_t> : Op16<bf16_t, bf16_t __attribute__((ext_vector_type(8)))> {
    static __device__ __forceinline__ acc_t mma(Frag a, Frag b, acc_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Op<float> {
    using Frag = float __attribute__((ext_vector_type(4)));
    static constexpr int K = 8;
    static constexpr int kTile = 32;
    static __device__ __forceinline__ Frag column(const float* tile, int stride, int row0, int c0, int lane) {
        const float* at = tile + (row0 + 4 * (lane >> 5)) * stride + c0 + (lane & 31);
        Frag f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = at[i * stride];
        return f;
    }
    static __device__ __forceinline__ Frag pack(const float* x) {
        Frag f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = x[i];
        return f;
    }
    static __device__ __forceinline__ acc_t mma(Frag a, Frag b, acc_t c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// A fragment of a row in LDS (or global memory, 16-byte aligned): positions c * K ..., half h.
template <typename T>
__device__ __forceinline__ typename Op<T>::Frag row_frag(const T* row, int c, int lane) {
    return *reinterpret_cast<const typename Op<T>::Frag*>(row + c * Op<T>::K + (lane >> 5) * (Op<T>::K / 2));
}

// 16 bytes of a row in global memory from channel d on; channels from D on are zero.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T* row, int d, int D, bool vec) {
    constexpr int n = 16 / sizeof(T);
    uint4 x = make_uint4(0, 0, 0, 0);
    if (vec) {
        if (d < D) x = *reinterpret_cast<const uint4*>(row + d);
    } else {
        Piece<T, n> y;
#pragma unroll
        for (int i = 0; i < n; ++i) y.v[i] = d + i < D ? row[d + i] : (T)0.f;
        x = __builtin_bit_cast(uint4, y);
    }
    return x;
}

// Whether 16 bytes hold an infinity or NaN.
template <typename T>
__device__ __forceinline__ bool not_finite(uint4 x) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
    constexpr uint32_t e = std::is_same_v<T, float> ? 0x7f800000u : std::is_same_v<T, bf16_t> ? 0x7f80u : 0x7c00u;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bad |= (u[i] & e) == e;
        if constexpr (sizeof(T) == 2) bad |= (u[i] & (e << 16)) == (e << 16);
    }
    return bad;
}

// Geometry of a tile in LDS: rows padded by 16 bytes, which spreads a column of 16-byte reads over the banks.
template <typename T, int DP>
struct TileOf {
    static constexpr int kRows = Op<T>::kTile;
    static constexpr int kPer = 16 / sizeof(T);          // elements of a 16-byte chunk
    static constexpr int kChunks = DP / kPer;            // chunks of a row
    static constexpr int kStride = DP + kPer;
    static constexpr int kElems = kRows * kStride;
};

// acc (channels x owners) += sum over the 32 rows of a tile of weight * row, where a weight of zero takes
// nothing from the row, whatever it holds: for tiles with infinities or NaN of which some pairs are masked.
// `w` holds the owner's weights in the register order above.
template <typename T, int DP>
__device__ __forceinline__ void add_rows(acc_t (&acc)[DP / 32], const acc_t& w, const T* tile, int stride, int lane) {
    const int h = lane >> 5;
#pragma unroll 1
    for (int r = 0; r < 16; ++r) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) x = i == r ? w[i] : x;
        float half[2];
        both_halves(x, half[0], half[1]);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const T* row = tile + (8 * (r >> 2) + 4 * hh + (r & 3)) * stride + 4 * h;
#pragma unroll
            for (int t = 0; t < DP / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float y = (float)row[t * 32 + 8 * (i >> 2) + (i & 3)];
                    acc[t][i] += half[hh] == 0.f ? 0.f : half[hh] * y;
                }
        }
    }
}

// acc += tile^T (32 rows from tile on) times the owner's weights.
template <typename T, int DP>
__device__ __forceinline__ void add_product(acc_t (&acc)[DP / 32], const acc_t& w, const T* tile, int stride, int lane) {
    using O = Op<T>;
#pragma unroll
    for (int c = 0; c < 32 / O::K; ++c) {
        float x[O::K / 2];
#pragma unroll
        for (int i = 0; i < O::K / 2; ++i) x[i] = w[c * (O::K / 2) + i];
        const typename O::Frag b = O::pack(x);
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) acc[t] = O::mma(O::column(tile, stride, c * O::K, t * 32, lane), b, acc[t]);
    }
}

// 32 rows of a tile times the owner's fragments.
template <typename T, int DP>
__device__ __forceinline__ acc_t row_product(const T* tile, int stride, const typename Op<T>::Frag* own, int lane) {
    acc_t s = {};
#pragma unroll
    for (int c = 0; c < DP / Op<T>::K; ++c) s = Op<T>::mma(row_frag(tile + (lane & 31) * stride, c, lane), own[c], s);
    return s;
}

// ---------------------------------------------------------------- masks

// The documents of a tile: the smallest and largest that are not padding, and whether none is padding.
// Which tiles a workgroup visits, and which of those need their pairs tested, follows from these.
struct Range {
    int lo, hi, whole;
};
__device__ __forceinline__ Range range_of(const int4 x) { return {x.x, x.y, x.z}; }
__device__ __forceinline__ bool meet(Range a, Range b, bool common) {
    return a.hi >= 0 && b.hi >= 0 && (common || (a.lo <= b.hi && b.lo <= a.hi));
}

// Range of the documents of tokens first .. last, by one wave.
__device__ __forceinline__ Range wave_range(const int* doc, int first, int last, int lane) {
    int lo = 0x7fffffff, hi = -1, whole = 1;
    for (int i = first + lane; i <= last; i += 64) {
        const int d = doc[i];
        if (d >= 0) {
            lo = min(lo, d);
            hi = max(hi, d);
        } else {
            whole = 0;
        }
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        lo = min(lo, __shfl_xor(lo, m, 64));
        hi = max(hi, __shfl_xor(hi, m, 64));
        whole &= __shfl_xor(whole, m, 64);
    }
    return {__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi),
            __builtin_amdgcn_readfirstlane(whole)};
}

// Walks over the tiles of [at, end) that `test` accepts, 64 at a time: one lane tests one tile. The result
// is the same in every wave of a workgroup, whose test does not depend on the wave.
struct TileWalk {
    int at, end;
    uint64_t left = 0;
    template <typename F>
    __device__ __forceinline__ int next(int lane, F test) {
        while (left == 0) {
            if (at >= end) return -1;
            const int t = at + lane;
            left = __ballot(t < end && test(t));
            at += 64;
        }
        const int b = __builtin_ctzll(left);
        left &= left - 1;
        return __builtin_amdgcn_readfirstlane(at - 64 + b);
    }
};

// Work of workgroup b: consecutive items go to one XCD (workgroup b runs on XCD b % 8), so that the rows of
// a slab read its keys through one L2.
__device__ __forceinline__ int xcd_item(int b, int grid) { return (b & 7) * (grid >> 3) + (b >> 3); }
int xcd_grid(int64_t items) { return (int)((items + 7) / 8 * 8); }

// Stores four consecutive channels of a result row.
template <typename T>
__device__ __forceinline__ void store_four(T* row, int d, int D, const float (&x)[4]) {
    if (D % 4 == 0) {
        if (d < D) {
            Piece<T, 4> y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y.v[i] = (T)x[i];
            *reinterpret_cast<Piece<T, 4>*>(row + d) = y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d + i < D) row[d + i] = (T)x[i];
    }
}

// Calls f with the kernels' element type, and with the channels they hold.
template <typename F>
hipError_t by_channels(int D, F f) {
    if (D <= 32) return f(std::integral_constant<int, 32>());
    if (D <= 64) return f(std::integral_constant<int, 64>());
    return f(std::integral_constant<int, 128>());
}

}  // namespace
}  // namespace msda
