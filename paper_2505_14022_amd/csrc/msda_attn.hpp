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

// The power of two by which probabilities (at most 1) are scaled as an operand: fp16 would round those below 6e-5, which
// a row over many thousand keys is full of, to fewer bits. A probability is over 1 by what its score and maximum are rounded to:
// 2^5 are left to fp16's largest number for scores of 10^7, whose rounding in fp32 is 1.
template <typename T>
constexpr int kProbShift = std::is_same_v<T, _Float16> ? 11 : 0;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// tanh(x) = 1 - 2 / (e^2x + 1), off by an fp32 rounding or two of 1. Where that shows in the result (SERIES: with fp32 operands, or
// a large cap, which it is multiplied by), |x| < 1/4 goes through the series x - x^3/3 + 2x^5/15 - 17x^7/315 + 62x^9/2835 (next
// term: 8.5e-9 of x). Of s * a, with a2 = 2 log2(e) a.
template <bool SERIES>
__device__ __forceinline__ float tanh_of(float s, float a, float a2) {
    const float t = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(exp2_of(s * a2) + 1.f), 1.f);
    if constexpr (!SERIES) return t;
    const float x = s * a, x2 = x * x;
    float y = __builtin_fmaf(x2, 62.f / 2835.f, -17.f / 315.f);
    y = __builtin_fmaf(y, x2, 2.f / 15.f);
    y = __builtin_fmaf(y, x2, -1.f / 3.f);
    y = __builtin_fmaf(y * x2, x, x);
    return fabsf(x) < 0.25f ? y : t;
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

// Whether 16 bytes hold an infinity or NaN: an exponent of all ones carries into the sign's place when one is
// added to it, and no other does.
template <typename T>
__device__ __forceinline__ bool not_finite(uint4 x) {
    constexpr uint32_t e = std::is_same_v<T, float> ? 0x7f800000u : std::is_same_v<T, bf16_t> ? 0x7f807f80u : 0x7c007c00u;
    constexpr uint32_t one = std::is_same_v<T, float> ? 0x00800000u : std::is_same_v<T, bf16_t> ? 0x00800080u : 0x04000400u;
    constexpr uint32_t sign = std::is_same_v<T, float> ? 0x80000000u : 0x80008000u;
    return (((x.x & e) + one) | ((x.y & e) + one) | ((x.z & e) + one) | ((x.w & e) + one)) & sign;
}

// Geometry of the tiles that a workgroup of NW waves stages in LDS. Rows are padded by 16 bytes, which spreads
// a column of 16-byte reads over the banks. A lone wave (few owners) takes half tiles: what it has in flight
// stays in its registers.
// The backward kernels take wide tiles of 16-bit rows of 32 channels, whose staging would be a third of the work (kv 205 us
// -> 193, q 147 -> 141 for DETR-encoder self-attention); the forward would lose a wave per SIMD to their LDS (130 -> 156).
constexpr int kWideTile = 128;
template <typename T, int DP, int NW, bool WIDE>
struct TileOf {
    static constexpr int kRows = NW == 1 ? 32 : WIDE && DP == 32 && sizeof(T) == 2 ? kWideTile : Op<T>::kTile;
    static constexpr int kBlocks = kRows / 32 < 2 ? 1 : 2;  // blocks of 32 that are worked on together
    static constexpr int kPer = 16 / sizeof(T);          // elements of a 16-byte chunk
    static constexpr int kChunks = DP / kPer;            // chunks of a row
    static constexpr int kStride = DP + kPer;
    static constexpr int kElems = kRows * kStride;
    static constexpr int kLoads = kRows * kChunks / (64 * NW);  // chunks per thread
    static constexpr int kStep = 64 * NW / kChunks;             // rows between two chunks of a thread
    // row of the thread's a-th chunk, and the first channel of all of them
    static __device__ __forceinline__ int row(int a) { return (int)threadIdx.x / kChunks + a * kStep; }
    static __device__ __forceinline__ int channel() { return (int)threadIdx.x % kChunks * kPer; }
    static __device__ __forceinline__ void put(T* tile, int a, uint4 x) {
        *reinterpret_cast<uint4*>(tile + row(a) * kStride + channel()) = x;
    }
};

// 16 bytes at a byte offset below 2^31 from a base that is the same in all lanes.
__device__ __forceinline__ uint4 load_at(const void* base, int offset) {
    return *reinterpret_cast<const uint4*>(static_cast<const char*>(base) + (uint32_t)offset);
}

// Channels d .. of a row in global memory, zero from D on. Rows are whole 16-byte chunks.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T* row, int d, int D) {
    return d < D ? *reinterpret_cast<const uint4*>(row + d) : make_uint4(0, 0, 0, 0);
}

// What a masked pair holds must reach nothing, but in a matrix product zero times an infinity or a NaN is a NaN. In
// calls with masks the tiles that are summed over are therefore staged with zeros in place of such values, and
// what they make of an owner's channel that does see them is noted in LDS, two bits per channel: 1 infinity, 2 minus
// infinity, both NaN; it is added to the result as it is written. (A rare path that holds no sums, so it costs
// the others no registers.)
template <int DP>
struct Odd {
    static constexpr int kWords = DP / 16;  // per owner
    uint32_t* mine;                         // the lane's owner's
    bool any = false;

    __device__ __forceinline__ void start(uint32_t* words, int owner, int lane, bool masks) {
        mine = words + owner * kWords;
        if (masks)
            for (int i = lane >> 5; i < kWords; i += 2) mine[i] = 0;
    }
    // `w`: the owner's weights of 32 rows in the register order above; row_at(r): row r's D channels in memory (asked
    // for rows of nonzero weight only). Half wave h notes every other word.
    template <typename T, typename F>
    __device__ __forceinline__ void note(const acc_t& w, int D, int lane, F row_at) {
        any = true;
#pragma unroll 1
        for (int r = 0; r < 16; ++r) {
            float x = 0.f, half[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) x = i == r ? w[i] : x;
            both_halves(x, half[0], half[1]);
#pragma unroll 1
            for (int hh = 0; hh < 2; ++hh) {
                const float y = hh ? half[1] : half[0];
                if (y == 0.f) continue;
                const T* row = row_at(8 * (r >> 2) + 4 * hh + (r & 3));
#pragma unroll 1
                for (int k = lane >> 5; k < kWords; k += 2) {
                    uint32_t bits = mine[k];
#pragma unroll 1
                    for (int c = 0; c < 16 && k * 16 + c < D; ++c) {
                        const float v = (float)row[k * 16 + c];
                        const uint32_t code = fabsf(v) < kInf ? 0u : v != v ? 3u : (v > 0.f) == (y > 0.f) ? 1u : 2u;
                        bits |= code << (2 * c);
                    }
                    mine[k] = bits;
                }
            }
        }
    }
    // Adds what was noted to channels d .. d + 3 of the owner's result.
    __device__ __forceinline__ void apply(float (&x)[4], int d) const {
        if (!any) return;
        wave_lds_sync();  // each half wave has noted every other word
        const uint32_t codes = mine[d >> 4] >> (2 * (d & 15));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t code = codes >> (2 * e) & 3u;
            x[e] += code == 0u ? 0.f : code == 1u ? kInf : code == 2u ? -kInf : __builtin_nanf("");
        }
    }
};

// A chunk without its infinities and NaN.
template <typename T>
__device__ __forceinline__ uint4 finite_only(uint4 x) {
    auto y = __builtin_bit_cast(Piece<T, 16 / sizeof(T)>, x);
#pragma unroll
    for (int i = 0; i < (int)(16 / sizeof(T)); ++i) y.v[i] = fabsf((float)y.v[i]) < kInf ? y.v[i] : (T)0.f;
    return __builtin_bit_cast(uint4, y);
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

// s + 32 rows of a tile times the owner's fragments, of D channels.
template <typename T, int DP>
__device__ __forceinline__ acc_t row_product(const T* tile, int stride, const typename Op<T>::Frag* own, int lane, int D,
                                             acc_t s) {
#pragma unroll
    for (int c = 0; c < DP / Op<T>::K; ++c) {
        if (sizeof(T) == 2 || c * Op<T>::K < D)  // in fp32 a chunk beyond D is 256 cycles of products of zeros
            s = Op<T>::mma(row_frag(tile + (lane & 31) * stride, c, lane), own[c], s);
    }
    return s;
}

// ---------------------------------------------------------------- masks

// The documents of a tile: the smallest and largest that are not padding, and whether none is padding.
// Which tiles a workgroup visits, and which of those need their pairs tested, follows from these.
struct Range {
    int lo, hi, whole;
};
__device__ __forceinline__ bool meet(Range a, Range b, bool common) {
    return (a.hi >= 0) & (b.hi >= 0) & (common | ((a.lo <= b.hi) & (b.lo <= a.hi)));
}

// Walks over the tiles of [at, end) that `test` accepts, 64 at a time: one lane tests one tile and keeps its
// documents, so that going on to the next tile reads no memory. The result is the same in every wave of a
// workgroup, whose test does not depend on the wave.
struct TileWalk {
    int at = 0, end = 0;
    uint64_t left = 0;
    Range held = {0, 0, 1};
    // Whether there is a tile left to visit.
    template <typename F>
    __device__ __forceinline__ bool more(int lane, const int4* ranges, F test) {
        while (left == 0) {
            if (at >= end) return false;
            const int t = at + lane;
            if (ranges && t < end) {
                const int4 x = ranges[t];
                held = {x.x, x.y, x.z};
            }
            left = __ballot(t < end && test(t, held));
            at += 64;
        }
        return true;
    }
    // Drops the tiles found so far that `test` does not accept any more.
    template <typename F>
    __device__ __forceinline__ void test_again(int lane, F test) {
        left &= __ballot(test(at - 64 + lane, held));
    }
    // The next tile or -1; its documents into `of` (with `ranges`).
    template <typename F>
    __device__ __forceinline__ int next(int lane, const int4* ranges, Range& of, F test) {
        if (!more(lane, ranges, test)) return -1;
        const int b = __builtin_ctzll(left);
        left &= left - 1;
        if (ranges)
            of = {__builtin_amdgcn_readlane(held.lo, b), __builtin_amdgcn_readlane(held.hi, b),
                  __builtin_amdgcn_readlane(held.whole, b)};
        return __builtin_amdgcn_readfirstlane(at - 64 + b);
    }
};

// Work of workgroup b: consecutive items go to one XCD (workgroup b runs on XCD b % 8), so that the rows of
// a slab read its keys through one L2.
__device__ __forceinline__ int xcd_item(int b, int grid) { return (b & 7) * (grid >> 3) + (b >> 3); }
[[maybe_unused]] int xcd_grid(int64_t items) { return (int)((items + 7) / 8 * 8); }

// What a workgroup works on: a block of owners and a run of the other axis' tiles.
struct Work {
    int slab, block, split, n, kv, common, off;
    bool any;
    Range docs;  // of the block's owners
    TileWalk walk;
    // last_first: blocks from the last to the first, so that causal rows with the most keys go first
    __device__ __forceinline__ Work(const AttnParams& p, bool last_first) {
        const int item = xcd_item(blockIdx.x, gridDim.x), per_slab = p.blocks * p.splits;
        any = item < p.N * p.Mkv * per_slab;
        slab = item / per_slab;
        const int rest = item - slab * per_slab;
        block = rest / p.splits;
        split = rest - block * p.splits;
        if (last_first) block = p.blocks - 1 - block;
        n = slab / p.Mkv;
        kv = slab - n * p.Mkv;
        off = p.Lk - p.Lq;
        common = any && p.prefix ? min(max(p.prefix[n], 0), p.Lk) : 0;
        docs = {0, 0, 1};
        if (any && p.own_ranges) {
            const int4 x = p.own_ranges[(int64_t)n * p.blocks + block];
            docs = {x.x, x.y, x.z};
        }
        walk.at = split * p.chunk;
        walk.end = min(walk.at + p.chunk, p.tiles);
    }
    __device__ __forceinline__ const int4* tile_ranges(const AttnParams& p) const {
        return p.tile_ranges ? p.tile_ranges + (int64_t)n * p.tiles : nullptr;
    }
    // With splits, notes whether this one has any tile to visit: the rest of it is not written otherwise.
    __device__ __forceinline__ bool note_split(const AttnParams& p, bool visits_any) const {
        if (p.splits == 1) return true;
        if (threadIdx.x == 0) p.filled[((int64_t)slab * p.blocks + block) * p.splits + split] = visits_any;
        return visits_any;
    }
};

// Whether any of a block of rows, up to query i_last and of documents `rows`, sees any of the keys from j_first on, of
// documents `keys`.
__device__ __forceinline__ bool sees(const AttnParams& p, const Work& w, int i_last, Range rows, int j_first, Range keys) {
    const bool first = j_first < w.common, in_order = !p.causal | (j_first <= i_last + w.off) | first;
    return in_order & (!p.q_doc | meet(rows, keys, first));
}

// The row that a lane owns, and what it sees: keys up to `last` of document `doc`, or below `common`.
struct Row32 {
    int row, i, head, doc, last;
    int64_t at;    // its place in [N, Lq, M]
    int64_t stat;  // its place in [N, M, Lq]
    float slope;
    float2 pos;
    int last0, doc0;  // of the wave's first row
    bool one_doc, no_pad;

    template <int NW>
    static __device__ __forceinline__ Row32 of(const AttnParams& p, const Work& w, int wave, int lane, bool biased) {
        Row32 x;
        const int first = w.block * 32 * NW;
        x.row = first + wave * 32 + (lane & 31);
        const int row = min(x.row, p.R - 1);
        x.i = row / p.G;
        x.head = w.kv * p.G + row - x.i * p.G;
        x.at = ((int64_t)w.n * p.Lq + x.i) * p.M + x.head;
        x.stat = ((int64_t)w.n * p.M + x.head) * p.Lq + x.i;
        x.doc = p.q_doc ? p.q_doc[(int64_t)w.n * p.Lq + x.i] : 0;
        x.last = x.doc < 0 ? -1 : p.causal ? max(x.i + w.off, w.common - 1) : p.Lk - 1;
        x.slope = 0.f;
        x.pos = make_float2(0.f, 0.f);
        if (biased && p.slopes) {
            x.slope = p.slopes[x.head] * kLog2e;
            x.pos = reinterpret_cast<const float2*>(p.q_pos)[(int64_t)w.n * p.Lq + x.i];
        }
        x.doc0 = __builtin_amdgcn_readfirstlane(x.doc);
        x.one_doc = __all((x.doc == x.doc0) & (x.doc >= 0));
        x.no_pad = __all(x.doc >= 0);
        x.last0 = p.causal ? __builtin_amdgcn_readfirstlane(x.last) : p.Lk - 1;  // rows go up with their lanes
        return x;
    }
};

// The keys of a staged tile as the rows' masks need them: the document, kCommon for one that all documents
// see, or -1 for one that nobody sees, whichever negative document a caller gave it.
constexpr int kCommon = -2;

// Keys and values staged tile by tile, for kernels that own rows: two buffers in LDS, and the next tile in
// registers while the waves work on the current one. All loads of a tile are issued together; what must not
// count (keys past the last, padding) is dropped when the tile is put into LDS.
// SUMMED: what the kernel sums over: the values (forward), the keys (grad_q) or nothing (delta).
// BUFFERS 1: for a lone wave, which has read a tile before it writes the next, so that twice as many waves fit, and
// for kernels that wait before they write.
enum Summed { kValues, kKeys, kNothing };
template <typename T, int DP, int NW, bool BIASED, Summed SUMMED, int BUFFERS = NW == 1 ? 1 : 2>
struct KeyTiles {
    using Tile = TileOf<T, DP, NW, SUMMED != kValues>;
    static constexpr int kBuffers = BUFFERS;
    struct Shared {
        T k[kBuffers][Tile::kElems], v[kBuffers][Tile::kElems];
        int doc[kBuffers][Tile::kRows];
        float2 pos[kBuffers][BIASED ? Tile::kRows : 1];
        int odd[kBuffers][NW];  // per wave: some of what it staged was not finite
    };
    Shared& sh;
    const AttnParams& p;
    Work& w;
    const T *k, *v;
    const int* docs;
    int t, lane, i_last, k_off, v_off;  // byte offsets of the thread's first chunk from a tile's first key
    bool masks, clean;          // clean: all of the tile's keys count
    Range kr;
    uint4 kx[Tile::kLoads], vx[Tile::kLoads];
    int doc_x[Tile::kLoads];
    float2 pos_x[Tile::kLoads];

    __device__ __forceinline__ KeyTiles(Shared& s, const AttnParams& q, Work& work, int l) : sh(s), p(q), w(work), lane(l) {
        k = static_cast<const T*>(p.k) + w.n * p.ks[0] + w.kv * p.ks[2];
        v = static_cast<const T*>(p.v) + w.n * p.vs[0] + w.kv * p.vs[2];
        docs = p.k_doc ? p.k_doc + (int64_t)w.n * p.Lk : nullptr;
        i_last = (min((w.block + 1) * 32 * NW, p.R) - 1) / p.G;
        masks = p.q_doc || p.causal;
        kr = {0, 0, 1};
        k_off = (Tile::row(0) * (int)p.ks[1] + Tile::channel()) * (int)sizeof(T);
        v_off = (Tile::row(0) * (int)p.vs[1] + Tile::channel()) * (int)sizeof(T);
#pragma unroll
        for (int a = 0; a < Tile::kLoads; ++a) {
            kx[a] = vx[a] = make_uint4(0, 0, 0, 0);  // what lanes of channels from D on put into LDS
            doc_x[a] = 0;
            pos_x[a] = make_float2(0.f, 0.f);
        }
    }
    // Whether the workgroup's rows see any of its run of tiles.
    __device__ __forceinline__ bool any() {
        return w.walk.more(lane, w.tile_ranges(p), [&](int u, Range of) { return sees(p, w, i_last, w.docs, u * Tile::kRows, of); });
    }
    // Leaves the tiles that rows of documents `docs` do not see. (The tile that has been fetched stays.)
    __device__ __forceinline__ void only(Range docs) {
        w.docs = docs;
        w.walk.test_again(lane, [&](int u, Range of) { return sees(p, w, i_last, w.docs, u * Tile::kRows, of); });
    }
    // Finds the next tile that the workgroup's rows see, and loads it.
    __device__ __forceinline__ void fetch() {
        t = w.walk.next(lane, w.tile_ranges(p), kr,
                        [&](int u, Range of) { return sees(p, w, i_last, w.docs, u * Tile::kRows, of); });
        if (t < 0) return;
        const int j0 = t * Tile::kRows;
        const bool full = j0 + Tile::kRows <= p.Lk;
        clean = full && kr.whole;
        const T* kt = k + j0 * p.ks[1];
        const T* vt = v + j0 * p.vs[1];
        if (full) {
            if (Tile::channel() < p.D) {
#pragma unroll
                for (int a = 0; a < Tile::kLoads; ++a) {
                    kx[a] = load_at(kt + a * Tile::kStep * p.ks[1], k_off);
                    vx[a] = load_at(vt + a * Tile::kStep * p.vs[1], v_off);
                }
            }
        } else {
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a)
                if (j0 + Tile::row(a) < p.Lk && Tile::channel() < p.D) {
                    kx[a] = load_at(kt + a * Tile::kStep * p.ks[1], k_off);
                    vx[a] = load_at(vt + a * Tile::kStep * p.vs[1], v_off);
                }
        }
        if (!clean || masks) {
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a) {
                const int j = j0 + Tile::row(a);
                doc_x[a] = 0;
                if (docs) doc_x[a] = docs[min(j, p.Lk - 1)];
            }
        }
        if (BIASED && p.slopes) {
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a)
                if (Tile::channel() == 0)
                    pos_x[a] = reinterpret_cast<const float2*>(p.k_pos)[(int64_t)w.n * p.Lk + min(j0 + Tile::row(a), p.Lk - 1)];
        }
    }
    // Puts the tile into buffer b.
    __device__ __forceinline__ void stage(int b) {
        if (!clean) {
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a) {
                if (t * Tile::kRows + Tile::row(a) >= p.Lk) doc_x[a] = -1;
                if (doc_x[a] < 0) kx[a] = vx[a] = make_uint4(0, 0, 0, 0);
            }
        }
        if (masks && SUMMED != kNothing) {
            bool odd = false;
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a) odd |= not_finite<T>(SUMMED == kValues ? vx[a] : kx[a]);
            const bool some = __any(odd);
            if (some) {
#pragma unroll
                for (int a = 0; a < Tile::kLoads; ++a) {
                    uint4& x = SUMMED == kValues ? vx[a] : kx[a];
                    if (SUMMED == kKeys) {  // such a key is nobody's: see attn_grad_q_kernel
                        const uint64_t row = __ballot(not_finite<T>(x)) >> (lane / Tile::kChunks * Tile::kChunks);
                        if (row & (((uint64_t)1 << Tile::kChunks) - 1)) doc_x[a] = -1;
                    }
                    x = finite_only<T>(x);
                }
            }
            if (lane == 0) sh.odd[b][threadIdx.x >> 6] = some;
        }
#pragma unroll
        for (int a = 0; a < Tile::kLoads; ++a) {
            Tile::put(sh.k[b], a, kx[a]);
            Tile::put(sh.v[b], a, vx[a]);
        }
        if (Tile::channel() == 0) {
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a) {
                const int j = t * Tile::kRows + Tile::row(a);
                if (!clean || masks) sh.doc[b][Tile::row(a)] = doc_x[a] < 0 ? -1 : j < w.common ? kCommon : doc_x[a];
                if (BIASED) sh.pos[b][Tile::row(a)] = pos_x[a];
            }
        }
    }
    // Whether something that was staged in buffer b was not finite.
    __device__ __forceinline__ bool any_odd(int b) const {
        int some = 0;
        if (masks) {
#pragma unroll
            for (int i = 0; i < NW; ++i) some |= sh.odd[b][i];
        }
        return some;
    }
    // Notes what the weights of the block of 32 values from key j0 on meet that was not finite in buffer b.
    __device__ __forceinline__ void note_odd(Odd<DP>& odd, const acc_t& weight, int b, int j0) const {
        if (any_odd(b)) odd.template note<T>(weight, p.D, lane, [&](int r) { return v + (j0 + r) * p.vs[1]; });
    }
    // Whether all rows of the wave see all keys of the tile just loaded.
    __device__ __forceinline__ bool whole(const Row32& own) const {
        const int j1 = t * Tile::kRows + Tile::kRows - 1;
        bool x = j1 <= own.last0 && j1 < p.Lk;
        if (p.q_doc)
            x = x && kr.whole && ((own.one_doc && kr.lo == own.doc0 && kr.hi == own.doc0) || (own.no_pad && j1 < w.common));
        return x;
    }
};

// What is done to the scores, each with kernels of its own: nothing, capping, a bias (and capping, if asked for), or capping far
// out (and a bias, if asked for). With 16-bit operands, whose probabilities are rounded to 2^-11 or less, the short form of
// tanh serves caps up to kShortCap, where a score is 2^-14 off; the last kernels take tanh's series. (Both forms in one kernel:
// 666 us for 649 in the step of 2 x 4096 packed causal rows x 16 heads x 128, 143 for 137 for a token over 16411 keys; the series in
// all biased kernels: 309 for 280 in a capped step of 2 x 2000 rows x 8 heads x 64.)
enum Extras { kPlain, kCap, kBias, kFarCap };
constexpr float kShortCap = 256.f;
template <typename T>
Extras extras_of(const AttnParams& p) {
    if (sizeof(T) == 2 && p.softcap > kShortCap) return kFarCap;
    return p.slopes ? kBias : p.softcap > 0.f ? kCap : kPlain;
}

// The row of the register r of a 32 x 32 block.
__device__ __forceinline__ int block_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// Raw scores of a block made scores in units of log 2, but for a factor, which is returned and left to the
// exponent: the scale, or the cap, of which `s` holds the tanh then. `ds` (if given) is multiplied by the cap's
// derivative 1 - tanh^2.
template <typename T, int EXTRAS>
__device__ __forceinline__ float cap_scores(const AttnParams& p, acc_t& s, acc_t* ds) {
    if (EXTRAS >= kBias && !(p.softcap > 0.f)) return p.scale * kLog2e;
    const float a = p.scale / p.softcap, a2 = 2.f * kLog2e * a;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = tanh_of<std::is_same_v<T, float> || EXTRAS == kFarCap>(s[r], a, a2);
        if (ds) (*ds)[r] *= __builtin_fmaf(-s[r], s[r], 1.f);
    }
    return p.softcap * kLog2e;
}

// Replaces the values of pairs that are not seen in a block of one lane's row and the 32 keys from jt on in the tile. `last`: the
// row's last key, counted from the tile's first; `codes`: the tile's keys. Four at a time, or the compiler holds the
// comparisons of all in scalar registers and spills them.
template <int N>
__device__ __forceinline__ void hide(acc_t (&x)[N], float with, int jt, int h, int last, int doc, const int* codes) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int4 c4 = *reinterpret_cast<const int4*>(codes + jt + 8 * g + 4 * h);
        const int code[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool seen = ((code[e] == doc) | (code[e] == kCommon)) & (jt + 8 * g + 4 * h + e <= last);
#pragma unroll
            for (int n = 0; n < N; ++n) x[n][4 * g + e] = seen ? x[n][4 * g + e] : with;
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

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
