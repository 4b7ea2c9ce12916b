// Matrix product of 8-bit integers with a scale for each row of both:
//   out[t, o] = (sum_k a[t, k] b[o, k]) (a_scale[t] b_scale[o]) + bias[o]
// Sums are 32-bit integers from the matrix instructions, exact up to 131071 products of two codes. The rows of b (a
// layer's weights) are the instructions' rows and the tokens their columns, so that a lane holds consecutive channels of
// one token and stores them together.
// Few tokens: bound by reading b once. A workgroup owns 16 channels and its waves share the sum: each reads rows of b
// straight into its registers, and the waves' sums are added in LDS. Many tokens: bound by the matrix unit. Tiles of both go to LDS past the
// registers while the previous ones are multiplied; 16-byte pieces of a row of 128 are permuted by the row's number, so that
// reads of one column of pieces spread over the banks.
// Measured: 8 tokens x 4096 by 6144 channels 9.1 us, 2.8 TB/s (bf16 results); 8192 x 4096 by 12288 380 to 410 us, 2.0 to 2.2 POP/s (the
// library's int8 product, 32-bit results, 433; its best, 8192 cubed, 2.4 POP/s); 1019 x 1360 by 2050 in fp32 14. Sums stored from where
// the matrix instructions leave them, 8 bytes a lane, took 584 for the second, and the builtin for loads to LDS, after which the
// compiler waits for all of them before any read, 404. Rows of 4097 codes, which start at any byte: 8 tokens by 6144 channels 26 us,
// 4096 by 4096 95 (4096 codes 73), 8000 x 2001 by 8000 187 (1.4 POP/s).
#include "msda_layer.hpp"
#include "msda_serve.h"

namespace msda {
namespace {

typedef int int4_t __attribute__((ext_vector_type(4)));
typedef int int16_t_ __attribute__((ext_vector_type(16)));

// Pieces k .. k + 15 of a row, zeros from K on.
template <bool PIECES>
__device__ __forceinline__ int4_t load_codes(const int8_t* row, int k, int K) {
    int4_t x = {0, 0, 0, 0};
    if (PIECES) {
        if (k < K) x = *reinterpret_cast<const int4_t*>(row + k);
    } else if (K >= 16) {
        // the row's last 16 codes, those before k shifted out, where fewer than 16 are left: no lane takes a way of its own
        const int from = min(k, K - 16), skip = k - from;
        unsigned __int128 codes;
        __builtin_memcpy(&codes, row + from, 16);
        if (skip < 16) x = __builtin_bit_cast(int4_t, codes >> (8 * skip));
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k + i < K) x[i / 4] |= (int)(uint8_t)row[k + i] << (8 * (i % 4));
    }
    return x;
}

// Four consecutive channels of a token, from their sums.
template <typename T>
__device__ __forceinline__ void store_sums(const ProductParams& p, int64_t t, int o, const int (&sum)[4], float a_scale) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int c = o + e < p.O ? o + e : p.O - 1;
        y[e] = __builtin_fmaf((float)sum[e], a_scale * p.b_scale[c], p.bias ? p.bias[c] : 0.f);
    }
    T* to = static_cast<T*>(p.out) + t * p.O + o;
    if (p.wide && o + 4 <= p.O) {
        Piece<T, 4> x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[e] = (T)y[e];
        *reinterpret_cast<Piece<T, 4>*>(to) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (o + e < p.O) to[e] = (T)y[e];
    }
}

constexpr int kRowWaves = 8, kRowSteps = 4;  // waves of a workgroup, and 64-byte steps of a wave that are loaded together

template <typename T, int NT, bool PIECES>
__global__ __launch_bounds__(64 * kRowWaves) void product_rows_kernel(ProductParams p, int across) {
    __shared__ int4_t part[kRowWaves][NT][64];
    const int lane = threadIdx.x & 63, wave = wave_index(), r = lane & 15, g = lane >> 4;
    const int t0 = (blockIdx.x / across) * 16 * NT, o0 = (blockIdx.x % across) * 16;
    const int8_t* b = p.b + (int64_t)min(o0 + r, p.O - 1) * p.K;
    const int8_t* a[NT];
    int4_t acc[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        a[n] = p.a + (int64_t)min(t0 + n * 16 + r, p.T - 1) * p.K;
        acc[n] = int4_t{0, 0, 0, 0};
    }
    for (int k0 = wave * kRowSteps * 64; k0 < p.K; k0 += kRowWaves * kRowSteps * 64) {
        int4_t x[kRowSteps], y[NT][kRowSteps];
#pragma unroll
        for (int s = 0; s < kRowSteps; ++s) {
            x[s] = load_codes<PIECES>(b, k0 + s * 64 + g * 16, p.K);
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n][s] = load_codes<PIECES>(a[n], k0 + s * 64 + g * 16, p.K);
        }
#pragma unroll
        for (int s = 0; s < kRowSteps; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[s], y[n][s], acc[n], 0, 0, 0);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) part[wave][n][lane] = acc[n];
    __syncthreads();
    if (wave >= NT) return;
    int4_t sum = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) sum += part[w][wave][lane];
    const int t = t0 + wave * 16 + r, o = o0 + 4 * g;
    if (t >= p.T || o >= p.O) return;
    const int four[4] = {sum[0], sum[1], sum[2], sum[3]};
    store_sums<T>(p, t, o, four, p.a_scale[t]);
}

// ---------------------------------------------------------------- tiles

__device__ const int4_t kZeroPiece[1] = {{0, 0, 0, 0}};

constexpr int kBand = 8;  // tiles of tokens that are worked on together

// 16 bytes from every lane's address to LDS, lane after lane from `to` on (the same in all lanes). By the instruction's name, and
// not by its builtin, after which the compiler has every read of LDS wait for all of these loads: the kernel waits for
// those that it needs with wait_loads.
__device__ __forceinline__ void load_to_lds(const void* from, void* to) {
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)to;
    uint32_t keep;  // m0 is the compiler's; what is written to it needs one instruction's time before such a load
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(keep)
                 : "s"(__builtin_amdgcn_readfirstlane(at)), "v"(from)
                 : "memory");
}

// Waits until at most N of the wave's loads are under way.
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
}

// Tiles of BM tokens and BN channels, WM x WN waves, 128 bytes of every row at a time, of which NS are in LDS. Rows that are
// not whole pieces (PIECES false) go through registers, since loads to LDS want their addresses aligned.
template <typename T, int BM, int BN, int WM, int WN, int NS, bool PIECES>
__global__ __launch_bounds__(64 * WM * WN) void product_tiles_kernel(ProductParams p, int across) {
    constexpr int kWaves = WM * WN, kTM = BM / WM / 32, kTN = BN / WN / 32;  // 32 x 32 blocks of a wave
    constexpr int kRows = BM + BN, kLoads = kRows / 8 / kWaves;              // 8 rows a load of a wave
    __shared__ __attribute__((aligned(16))) int8_t tile[NS][kRows * 128];
    __shared__ float a_scale[BM];
    const int lane = threadIdx.x & 63, wave = wave_index(), wm = wave / WN, wn = wave % WN;
    // An XCD takes consecutive tiles (workgroup b runs on XCD b % 8), down a band of kBand and then across, so that those
    // that it has at work read few rows of either operand.
    const int item = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3), down = (p.T + BM - 1) / BM;
    const int band = item / (kBand * across), in = item - band * (kBand * across), high = min(kBand, down - band * kBand);
    if (high <= 0 || in >= high * across) return;  // past the last band's tiles: the grid is a multiple of 8
    const int t0 = (band * kBand + in % high) * BM, o0 = in / high * BN;
    const int8_t* from[kLoads];
    int piece[kLoads];  // of the row, which the lane's place in LDS holds
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int row = (wave * kLoads + i) * 8 + (lane >> 3);
        piece[i] = (lane & 7) ^ (row >> 1 & 7);
        from[i] = row < BM ? p.a + (int64_t)min(t0 + row, p.T - 1) * p.K : p.b + (int64_t)min(o0 + row - BM, p.O - 1) * p.K;
        from[i] += piece[i] * 16;
    }
    auto load = [&](int k0, int s) {
        auto put = [&](int i, const void* src) {
            load_to_lds(src, tile[s] + (wave * kLoads + i) * 1024);
        };
        if (k0 + 128 <= p.K) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) put(i, from[i] + k0);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) put(i, k0 + piece[i] * 16 < p.K ? (const void*)(from[i] + k0) : (const void*)kZeroPiece);
        }
    };
    int16_t_ acc[kTN][kTM];
#pragma unroll
    for (int n = 0; n < kTN; ++n)
#pragma unroll
        for (int m = 0; m < kTM; ++m) acc[n][m] = int16_t_{};
    const int lr = lane & 31, lh = lane >> 5;
    auto fragment = [&](int s, int row, int step) {
        return *reinterpret_cast<const int4_t*>(tile[s] + row * 128 + (((step * 2 + lh) ^ (row >> 1 & 7)) << 4));
    };
    for (int i = threadIdx.x; i < BM; i += 64 * kWaves) a_scale[i] = p.a_scale[min(t0 + i, p.T - 1)];
    auto multiply = [&](int s) {
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            int4_t x[kTN], y[kTM];
#pragma unroll
            for (int n = 0; n < kTN; ++n) x[n] = fragment(s, BM + (wn * kTN + n) * 32 + lr, step);
#pragma unroll
            for (int m = 0; m < kTM; ++m) y[m] = fragment(s, (wm * kTM + m) * 32 + lr, step);
#pragma unroll
            for (int n = 0; n < kTN; ++n)
#pragma unroll
                for (int m = 0; m < kTM; ++m) acc[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[n], y[m], acc[n][m], 0, 0, 0);
        }
    };
    if constexpr (PIECES) {
        static_assert(NS == 2 || NS == 3, "at most one buffer is on its way while another is read");
#pragma unroll
        for (int i = 0; i < NS - 1; ++i)
            if (i * 128 < p.K) load(i * 128, i);
        int s = 0, last = NS - 1;
        for (int k0 = 0; k0 < p.K; k0 += 128) {
            // the wave's pieces of this buffer are in LDS, those of the next ones may be on their way
            if (NS > 2 && k0 + 128 < p.K) wait_loads<(NS > 2 ? 1 : 0) * kLoads>();
            else wait_loads<0>();
            __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();        // everybody's are, and the buffer before it has been read
            asm volatile("" ::: "memory");
            if (k0 + (NS - 1) * 128 < p.K) load(k0 + (NS - 1) * 128, last);
            multiply(s);
            last = s;
            s = s + 1 == NS ? 0 : s + 1;
        }
    } else {
        static_assert(NS == 2, "a buffer that is read, and one that is written");
        int4_t held[kLoads];
        auto take = [&](int k0) {
            if (k0 + 128 <= p.K) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) __builtin_memcpy(&held[i], from[i] + k0, 16);
            } else {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) held[i] = load_codes<false>(from[i] - piece[i] * 16, k0 + piece[i] * 16, p.K);
            }
        };
        auto leave = [&](int s) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) *reinterpret_cast<int4_t*>(tile[s] + (wave * kLoads + i) * 1024 + lane * 16) = held[i];
        };
        take(0);
        leave(0);
        int s = 0;
        for (int k0 = 0; k0 < p.K; k0 += 128, s ^= 1) {
            __syncthreads();  // this buffer is written, and the other one has been read
            if (k0 + 128 < p.K) take(k0 + 128);
            multiply(s);
            if (k0 + 128 < p.K) leave(s ^ 1);
        }
    }
    // Sums change lanes through LDS, so that a lane has kPer consecutive channels (the same ones all along: their scales
    // stay in registers) and a wave stores whole pieces of rows.
    constexpr int kPer = 16 / sizeof(T), kAcross = 32 * kTN / kPer, kDown = 64 / kAcross, kWide = 32 * kTN + 4;
    static_assert(kWaves * 32 * kWide * 4 <= sizeof(tile), "the waves' sums fit into the tiles");
    __syncthreads();  // the tiles have been read
    int* mine = reinterpret_cast<int*>(&tile[0][0]) + wave * 32 * kWide;
    const int o = o0 + wn * 32 * kTN + lane % kAcross * kPer;
    float b_scale[kPer], bias[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int c = min(o + e, p.O - 1);
        b_scale[e] = p.b_scale[c];
        bias[e] = p.bias ? p.bias[c] : 0.f;
    }
#pragma unroll
    for (int m = 0; m < kTM; ++m) {
#pragma unroll
        for (int n = 0; n < kTN; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<int4_t*>(mine + lr * kWide + n * 32 + 8 * q + 4 * lh) =
                    int4_t{acc[n][m][4 * q], acc[n][m][4 * q + 1], acc[n][m][4 * q + 2], acc[n][m][4 * q + 3]};
        wave_lds_sync();
#pragma unroll
        for (int i = 0; i < 32 / kDown; ++i) {
            const int row = i * kDown + lane / kAcross, t = t0 + (wm * kTM + m) * 32 + row;
            const int* from = mine + row * kWide + lane % kAcross * kPer;
            const float by = a_scale[(wm * kTM + m) * 32 + row];
            Piece<T, kPer> y;
#pragma unroll
            for (int e = 0; e < kPer; e += 4) {
                const int4_t x = *reinterpret_cast<const int4_t*>(from + e);
#pragma unroll
                for (int k = 0; k < 4; ++k) y.v[e + k] = (T)__builtin_fmaf((float)x[k], by * b_scale[e + k], bias[e + k]);
            }
            T* to = static_cast<T*>(p.out) + (int64_t)t * p.O + o;
            if (t < p.T && o < p.O) {
                if (p.wide) {
                    stream_store(reinterpret_cast<uint4*>(to), __builtin_bit_cast(uint4, y));
                } else {
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (o + e < p.O) to[e] = y.v[e];
                }
            }
        }
        wave_lds_sync();
    }
}

template <typename T, int NT>
void launch_rows(const ProductParams& p, int64_t workgroups, hipStream_t stream) {
    const dim3 grid((unsigned)workgroups), block(64 * kRowWaves);
    const int across = (p.O + 15) / 16;
    if (p.pieces) hipLaunchKernelGGL((product_rows_kernel<T, NT, true>), grid, block, 0, stream, p, across);
    else hipLaunchKernelGGL((product_rows_kernel<T, NT, false>), grid, block, 0, stream, p, across);
}

template <typename T, int BM, int BN, int WM, int WN, int NS>
void launch_tiles(const ProductParams& p, int64_t workgroups, hipStream_t stream) {
    const dim3 grid((unsigned)((workgroups + 7) / 8 * 8)), block(64 * WM * WN);
    const int across = (p.O + BN - 1) / BN;
    if (p.pieces) hipLaunchKernelGGL((product_tiles_kernel<T, BM, BN, WM, WN, NS, true>), grid, block, 0, stream, p, across);
    else hipLaunchKernelGGL((product_tiles_kernel<T, BM, BN, WM, WN, 2, false>), grid, block, 0, stream, p, across);
}

template <typename T>
hipError_t launch_typed(const ProductParams& p, hipStream_t stream) {
    const ProductPlan plan = product_plan(p);
    if (plan.channels == 16) {
        if (plan.tokens == 16) launch_rows<T, 1>(p, plan.workgroups, stream);
        else if (plan.tokens == 32) launch_rows<T, 2>(p, plan.workgroups, stream);
        else launch_rows<T, 4>(p, plan.workgroups, stream);
    } else if (plan.tokens == 256) {
        launch_tiles<T, 256, 256, 2, 4, 2>(p, plan.workgroups, stream);
    } else if (plan.tokens == 128) {
        launch_tiles<T, 128, 128, 2, 2, 2>(p, plan.workgroups, stream);
    } else {
        launch_tiles<T, 64, 64, 2, 2, 3>(p, plan.workgroups, stream);
    }
    return hipGetLastError();
}

}  // namespace

ProductPlan product_plan(const ProductParams& p) {
    ProductPlan a;
    auto tiles = [&](int tokens, int channels) {
        return ((int64_t)p.T + tokens - 1) / tokens * (((int64_t)p.O + channels - 1) / channels);
    };
    auto take = [&](int tokens, int channels, int waves) {
        a.tokens = tokens;
        a.channels = channels;
        a.waves = waves;
        a.workgroups = tiles(tokens, channels);
    };
    // Few tokens and tiles: 64 x 4096 by 4096 12.9 us against 13.6, by 1024 of 8192 20 against 24, but each 64 tokens read b again.
    // The larger tile as soon as every CU has one: 1024 x 4096 by 4096 with tiles of 64, 128 and 256 35, 27.5 and 56 us, 512
    // tokens 20, 25 and 55; 4096 tokens 111, 83 and 70, 2048 62, 42 and 58.
    if (p.T <= 64) {
        take(p.T <= 16 ? 16 : p.T <= 32 ? 32 : 64, 16, kRowWaves);
    } else if (tiles(256, 256) >= 256) {
        take(256, 256, 8);
    } else if (tiles(128, 128) >= 256) {
        take(128, 128, 4);
    } else {
        take(64, 64, 4);
    }
    return a;
}

hipError_t launch_product(const ProductParams& p, int dtype, hipStream_t stream) {
    if (dtype == MSDA_F32) return launch_typed<float>(p, stream);
    if (dtype == MSDA_F16) return launch_typed<_Float16>(p, stream);
    return launch_typed<bf16_t>(p, stream);
}

}  // namespace msda
