// Attention over a paged cache of 8-bit keys and values with a scale for each page and head.
//   z = cap(scale k_scale q . k_code),  lse = log sum exp z,  out = sum exp(z - lse) v_scale v_code
// For single tokens it is bound by reading the cache once, for chunks of a prompt by the vector work around its products. One
// pass over the keys with a running maximum and sum, everything in registers: a wave has 16 rows (queries of the heads that
// share a key head), 32 or 48, as columns of 16 x 16 x 32 instructions, and takes 32 keys at a time.
//   scores: keys are the instruction's rows. A lane (column n, quarter g) reads consecutive bytes of key n of 16, in an order
//     of channels that the queries follow, and gets the scores of keys 4 g .. 4 g + 3 of both halves of the 32;
//   values: a sum over keys may take them in any order, so the lane's eight probabilities are its operand as they are, and it
//     reads DP / 16 bytes of each of its eight keys, which are the rows n DP / 16 .. of the other operand.
// So nothing is exchanged between lanes but a maximum, and the cache goes from memory to registers. A code c becomes
// fp16 without a conversion: byte c ^ 0x80 below the exponent of 1024 is 1152 + c, less 1152 is c.
// A page's key scale is a factor of its scores. Its value scale goes into the exponent, so that it costs nothing for each key: an
// operand is a probability in units of the row's largest so far, times its value scale in units of the pages' largest. That
// keeps its digits where value scales are within 2^8 of each other. Where they are not ("apart"), a row would lose what it has to a
// scale that it does not see, or sees with a small probability: the largest product of the two that the row has seen is the
// unit then, and the sum of the probabilities has exponents of its own. A workgroup that meets such scales begins anew in that way.
// Roundings: queries are scaled by a power of two to their row's largest and held in fp16 (in fp32 as the sum of two), exact for
// fp16 and for all of bf16 within 2^28 of the largest; probabilities are rounded to fp16 for the product (in fp32 the sum of
// two), times 2^14, so that those of long rows keep their bits; their sum is taken before that. Statistics and sums are fp32.
// Measured: one token each of 32 sequences of 11 to 16 thousand keys, 32 heads of 128 channels on 8, bf16: 165 us and 5 to
// join the runs, 5.3 TB/s (a large copy reaches 5.1); two chunks of up to 2048 tokens over up to 10240, the same heads:
// 646 us, 696 TFLOP/s (a large product 1366), two waves per SIMD at 245 registers, of which the vector unit works in 73 % of the cycles and
// the matrix unit in 27 %. (Before it looked for scales that are apart it took 634, with 32 rows a wave 692, with 16 1164. A
// kernel whose waves share fp16 tiles in LDS, so that a code is turned once for 128 rows, took 705: its barriers and reads of LDS
// cost what it saved.)
#include "msda_attn.hpp"
#include "msda_cache.hpp"

namespace msda {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kCacheWaves = 4;
constexpr float kShift = 14.f;  // probabilities times 2^14 as an operand

// Bytes A and B (0 .. 3) of the words x and y of codes, as two fp16 numbers.
template <int A, int B>
__device__ __forceinline__ uint32_t two_codes(uint32_t x, uint32_t y) {
    // selector: 0 .. 3 bytes of y (second operand), 4 .. 7 of x, 12 zero
    const uint32_t u = __builtin_amdgcn_perm(x, y, 0x0c000c00u | (4 + A) | (uint32_t)B << 16) ^ 0x64806480u;
    const half2v h = __builtin_bit_cast(half2v, u) - half2v{(_Float16)1152.f, (_Float16)1152.f};
    return __builtin_bit_cast(uint32_t, h);
}

// The bytes of two words, the same way: c ^ 0x80 for four at once, and the exponent's byte from a constant.
__device__ __forceinline__ half8 eight_codes(uint32_t lo, uint32_t hi) {
    const half2v off = {(_Float16)1152.f, (_Float16)1152.f};
    auto two = [&](uint32_t x, uint32_t selector) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, __builtin_amdgcn_perm(x, 0x64646464u, selector)) - off);
    };
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    const uint4 w = make_uint4(two(lo, 0x00050004u), two(lo, 0x00070006u), two(hi, 0x00050004u), two(hi, 0x00070006u));
    return __builtin_bit_cast(half8, w);
}

// The largest of the four lanes of a column.
__device__ __forceinline__ float column_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, 64));
    return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float column_sum(float x) {
    x += __shfl_xor(x, 16, 64);
    return x + __shfl_xor(x, 32, 64);
}

// A workgroup's block of rows and run of tokens.
struct CacheWork {
    int n, item, kv, head0, heads, split;  // item: of (block, key head, heads), in the order of the partial results
    int token0, tokens;  // the block's first token of the call, and how many
    int place0;          // its place in the sequence
    int end;             // tokens of the sequence that exist
    // Work item `at`: runs of a block's rows are neighbours, then the blocks of a key head, the last first: with an order
    // they have the most keys.
    __device__ __forceinline__ bool find(const CacheAttnParams& p, int at, int lane) {
        split = at % p.splits;
        const int rest = at / p.splits;
        return find_block(p, p.blocks - 1 - rest % p.blocks, rest / p.blocks, lane);
    }
    // Block `block` of tokens, part `part` of the heads.
    __device__ __forceinline__ bool find_block(const CacheAttnParams& p, int block, int part, int lane) {
        const int per_block = p.c.Mkv * p.groups;
        if (part >= per_block) return false;
        item = block * per_block + part;
        kv = part / p.groups;
        head0 = (part - kv * p.groups) * p.group;
        heads = min(p.group, p.G - head0);
        head0 += kv * p.G;
        const Place t = find_place(p.c, block, p.tokens, 1, lane);
        if (t.n < 0) return false;
        n = t.n;
        const int skip = t.block * p.tokens;
        tokens = min(p.tokens, t.count - skip);
        if (tokens <= 0) return false;
        token0 = t.start + skip;
        place0 = t.first + skip;
        end = (int)min((int64_t)t.length, (int64_t)p.c.width << p.c.page_shift);
        return true;
    }
    // Keys that token i of the block sees.
    __device__ __forceinline__ int limit(const CacheAttnParams& p, int i) const {
        return p.causal ? min(max(place0 + i + 1, 0), end) : end;
    }
    // Runs in which the block's rows see any key.
    __device__ __forceinline__ int runs(const CacheAttnParams& p) const {
        const int most = limit(p, tokens - 1);
        return most <= 0 ? 0 : min((most - 1) / p.run + 1, p.splits);
    }
};

__device__ __forceinline__ float lane_value(float x, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// The pages of 64 columns of the sequence's table, one to a lane.
template <bool APART>
struct Pages {
    int first;                  // column of lane 0
    int page;                   // -1: no tokens
    float k_scale, bias;        // bias: log2 of the value scale in units of unit(), and kShift
    // Without APART, the same in all lanes: the largest value scale so far, and of the first 64 pages; whether any is not within 1 / 64
    // and 4 of the latter, so that they may be more than 2^8 from each other.
    float most = 0.f, first_most = 0.f;
    bool apart = false;
    __device__ __forceinline__ float unit() const { return !APART && most > 0.f ? most : 1.f; }
    // Loads columns `column` ..; returns the factor from the old unit to the new one.
    __device__ __forceinline__ float load(const CacheAttnParams& p, const CacheWork& w, int column, int end, int lane) {
        first = column;
        page = -1;
        k_scale = 0.f;
        float v_scale = 0.f;
        if (((int64_t)(column + lane) << p.c.page_shift) < end) page = page_at(p.c, w.n, column + lane);
        if (page >= 0) {
            const int64_t at = (int64_t)page * p.c.Mkv + w.kv;
            k_scale = p.c.k_scale[at];
            v_scale = p.c.v_scale[at];
        }
        // the scores of a page that makes NaN are NaN, which a row that does not see it replaces
        const bool odd = !(k_scale >= 0.f && k_scale < kInf && v_scale >= 0.f && v_scale < kInf);
        if (odd) k_scale = __builtin_nanf("");
        if (odd || v_scale < 1.17549435e-38f) v_scale = 0.f;  // logarithms are those of normal numbers
        float turn = 1.f;
        if constexpr (!APART) {
            const float before = most;
            most = lane_value(fmaxf(group_max<64>(v_scale), most), 0);
            if (before > 0.f) turn = before / most;
            else first_most = most;
            const bool near = v_scale > 0.f && v_scale * 64.f >= first_most && v_scale <= 4.f * first_most;
            if (__any(page >= 0 && !near)) apart = true;
        }
        bias = (page >= 0 ? __builtin_amdgcn_logf(v_scale) - __builtin_amdgcn_logf(unit()) : 0.f) + kShift;
        return turn;
    }
};

// lse of a row's maximum (in units of log 2) and sum.
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2; }

// Where the maxima and sums of partial results lie: behind their channels.
template <int DP>
__device__ __forceinline__ float2* stats_of(const CacheAttnParams& p, int rows) {
    return reinterpret_cast<float2*>(p.part + (int64_t)p.blocks * p.c.Mkv * p.groups * rows * p.splits * DP);
}

// Four channels of a row, joined from partial results.
struct Joined {
    float m = -kInf, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void take(float2 ml, float4 y) {
        const float top = fmaxf(m, ml.x), base = top == -kInf ? 0.f : top;
        const float u = exp2_of(m - base), v = exp2_of(ml.x - base);
        m = top;
        l = l * u + ml.y * v;
        x[0] = x[0] * u + y.x * v;
        x[1] = x[1] * u + y.y * v;
        x[2] = x[2] * u + y.z * v;
        x[3] = x[3] * u + y.w * v;
    }
    // at: the row's place in [T, M]
    template <typename T>
    __device__ __forceinline__ void store(const CacheAttnParams& p, int64_t at, int d) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] *= inv;
        store_four(static_cast<T*>(p.out) + at * p.c.D, d, p.c.D, x);
        if (p.lse && d == 0) p.lse[at] = lse_of(m, l);
    }
};

// The queries of rows row0 + 16 j + col of the block, 8 channels from d_of(s) on for each step, as fp16 operands (in fp32
// the sum of q and low); how many keys a row sees (and the least and the most of the wave's rows); and the factor that
// makes a raw score one in units of log 2, or with CAP in natural ones. meanwhile() is called while the queries are on their
// way.
template <typename T, int NQ, int STEPS, int CAP, int NL, typename F, typename W>
__device__ __forceinline__ void load_queries(const CacheAttnParams& p, const CacheWork& w, int row0, int col, F d_of,
                                             half8 (&q)[NQ][STEPS], half8 (&low)[NL][STEPS], int (&limit)[NQ], float (&unit)[NQ],
                                             int& lowest, int& highest, W meanwhile) {
    lowest = 0x7fffffff;
    highest = 0;
    Piece<T, 8> x[NQ][STEPS];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        const int row = row0 + j * 16 + col, i = row / p.group, h = row - i * p.group;
        const bool mine = i < w.tokens && h < w.heads;
        limit[j] = mine ? w.limit(p, i) : 0;
        highest = max(highest, limit[j]);
        if (mine) lowest = min(lowest, limit[j]);
        const T* from = static_cast<const T*>(p.q) + (int64_t)(w.token0 + (mine ? i : 0)) * p.qs[0] + (int64_t)(w.head0 + (mine ? h : 0)) * p.qs[1];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int d = d_of(s);
            const bool in = mine && d < p.c.D;
            constexpr int kPer = 16 / sizeof(T);
            x[j][s] = {};
            if (p.vec) {
#pragma unroll
                for (int e = 0; e < 8; e += kPer) {
                    Piece<T, kPer> y = {};
                    if (in) y = *reinterpret_cast<const Piece<T, kPer>*>(from + d + e);
#pragma unroll
                    for (int k = 0; k < kPer; ++k) x[j][s].v[e + k] = y.v[k];
                }
            } else if (in) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[j][s].v[e] = from[d + e];
            }
        }
    }
    meanwhile();
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf((float)x[j][s].v[e]));
        top = column_max(top);
        int shift = top > 0.f && top < kInf ? 14 - ((int)(__builtin_bit_cast(uint32_t, top) >> 23) - 127) : 0;
        shift = min(shift, 126);
        const float up = __builtin_bit_cast(float, (uint32_t)(shift + 127) << 23);
        unit[j] = fminf(p.scale * (CAP > 0 ? 1.f : kLog2e) * __builtin_bit_cast(float, (uint32_t)(127 - shift) << 23), 3.4e38f);
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = (float)x[j][s].v[e] * up;
                q[j][s][e] = (_Float16)y;
                if constexpr (std::is_same_v<T, float>) low[j][s][e] = (_Float16)(y - (float)q[j][s][e]);
            }
    }
#pragma unroll
    for (int k = 1; k < 16; k *= 2) {
        lowest = min(lowest, __shfl_xor(lowest, k, 64));
        highest = max(highest, __shfl_xor(highest, k, 64));
    }
    lowest = __builtin_amdgcn_readfirstlane(lowest);
    highest = __builtin_amdgcn_readfirstlane(highest);
}

// What a group of four keys gets from its page; less: 2^-bias.
struct GroupScales {
    float k_scale, bias, less;
    bool there;
};
// Raw scores of a lane's row with NG groups of four keys, key + 16 t .. key + 16 t + 3, made scores but for the factors `by`. whole: the
// row sees all of them; otherwise those below `limit`, of groups that have a page. Returns the largest score, and with APART the
// largest exponent of an operand. CAP: capped by tanh, in its short form for 16-bit results and caps up to kShortCap (a score is
// 2^-14 off then), else its series.
template <int CAP, bool APART, int NG>
__device__ __forceinline__ float2 finish_scores(const CacheAttnParams& p, float4v (&s)[NG], float (&by)[NG], float unit,
                                                const GroupScales (&of)[NG], bool whole, int key, int limit) {
    float top = -kInf, weighed = -kInf;
#pragma unroll
    for (int t = 0; t < NG; ++t) {
        by[t] = unit * of[t].k_scale;
        if constexpr (CAP > 0) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                s[t][r] = p.cap_unit * tanh_of<(CAP == 2)>(s[t][r] * by[t], p.cap_inverse, p.cap_exponent);
            by[t] = 1.f;
        }
        if (!whole) {
            const int stop = of[t].there ? limit : 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) s[t][r] = key + 16 * t + r < stop ? s[t][r] * by[t] : -kInf;
            by[t] = 1.f;
        }
        const float most = fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])) * by[t];
        top = fmaxf(top, most);
        if constexpr (APART) weighed = fmaxf(weighed, most + of[t].bias);
    }
    return make_float2(top, weighed);
}
// The running maximum after a lane's `top`, and the factor of what was summed before.
__device__ __forceinline__ float raise(float& m, float top) {
    const float now = fmaxf(m, column_max(top));
    const float fade = exp2_of(m - (now == -kInf ? 0.f : now));
    m = now;
    return fade;
}
// Scores made operands (probabilities times 2^kShift and the value scale, see above) in fp16, with TWO the sum of prob and low; the
// probabilities are added to l in units of 2^m, m being the row's largest score so far. Operands' exponents are relative to m too, or
// with APART to `ref`, the largest exponent of an operand so far less kShift.
template <bool TWO, bool APART, int NG>
__device__ __forceinline__ void weigh(const float4v (&s)[NG], const float (&by)[NG], const GroupScales (&of)[NG], float m, float ref,
                                      float& l, half8 (&prob)[NG / 2], half8* low) {
    const float base = m == -kInf ? 0.f : m, from = !APART ? base : ref == -kInf ? 0.f : ref;
#pragma unroll
    for (int t = 0; t < NG; ++t) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float x = exp2_of(__builtin_fmaf(s[t][r], by[t], of[t].bias - from));
            sum += APART ? exp2_of(__builtin_fmaf(s[t][r], by[t], -base)) : x;
            prob[t / 2][4 * (t % 2) + r] = (_Float16)x;
            if constexpr (TWO) low[t / 2][4 * (t % 2) + r] = (_Float16)(x - (float)prob[t / 2][4 * (t % 2) + r]);
        }
        l += APART ? sum : sum * of[t].less;
    }
}

// Rows row0 .. row0 + 16 NQ - 1 of a workgroup's kRows, and its run of keys. Returns false, with nothing stored, if APART has to be
// set for them.
template <typename T, int DP, int NQ, int CAP, bool APART, int kRows>
__device__ __forceinline__ bool attend(const CacheAttnParams& p, int thread, int row0, float* joined, float2* stats, int* failed) {
    constexpr bool kTwo = std::is_same_v<T, float>;
    constexpr int kSteps = DP / 32, kBytes = DP / 16, kWords = (kBytes + 3) / 4;
    constexpr int kStride = DP + 4;  // of a row in LDS
    const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), col = lane & 15, g = lane >> 4;
    CacheWork w;
    if (!w.find(p, xcd_item(blockIdx.x, gridDim.x), lane)) return true;
    if (w.split >= max(w.runs(p), 1)) return true;
    const Cache& c = p.c;

    int limit[NQ], lowest, highest;
    float unit[NQ];
    half8 q[NQ][kSteps], q_low[kTwo ? NQ : 1][kSteps];
    const int run0 = w.split * p.run, first_key = run0 + 32 * wave, most = w.limit(p, w.tokens - 1);
    Pages<APART> pages;
    load_queries<T, NQ, kSteps, CAP>(p, w, row0, col,
                                     [&](int s) { return DP == 32 ? g * 8 : (s / 2) * 64 + g * 16 + (s % 2) * 8; }, q, q_low, limit,
                                     unit, lowest, highest, [&]() { pages.load(p, w, first_key >> c.page_shift, most, lane); });

    float4v o[NQ][kBytes];
    float m[NQ], l[NQ], ref[NQ];  // ref: see weigh
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        m[j] = ref[j] = -kInf;
        l[j] = 0.f;
#pragma unroll
        for (int u = 0; u < kBytes; ++u) o[j][u] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    // byte offsets of the lane within 16 keys; channels from D on are read as others: they meet zeros, or rows of no result
    uint32_t k_at[DP == 32 ? 1 : DP / 64];
#pragma unroll
    for (int u = 0; u < (DP == 32 ? 1 : DP / 64); ++u) {
        const int d = DP == 32 ? g * 8 : u * 64 + g * 16;
        k_at[u] = col * c.D + (d < c.D ? d : 0);
    }
    const uint32_t v_at = 4 * g * c.D + (col * kBytes < c.D ? col * kBytes : 0);

    const int run1 = pages.apart ? 0 : (int)min((int64_t)highest, (int64_t)run0 + p.run);
    for (int key0 = first_key; key0 < run1; key0 += 32 * kCacheWaves) {
        const int columns[2] = {key0 >> c.page_shift, (key0 + 16) >> c.page_shift};
        if (columns[1] >= pages.first + 64) {
            const float turn = pages.load(p, w, columns[0], most, lane);
            if (pages.apart) break;
            if constexpr (!APART) {
#pragma unroll
                for (int j = 0; j < NQ; ++j)
#pragma unroll
                    for (int u = 0; u < kBytes; ++u) o[j][u] *= turn;
            }
        }
        uint4 kx[2][DP == 32 ? 1 : DP / 64];
        uint32_t vx[8][kWords];
        GroupScales of[2];
        bool whole = key0 + 32 <= lowest;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int at = columns[t] - pages.first, slot = (key0 + 16 * t) & (c.page - 1);
            const int page = __builtin_amdgcn_readlane(pages.page, at);
            whole = whole && page >= 0;
            const float bias = lane_value(pages.bias, at);
            of[t] = {lane_value(pages.k_scale, at), bias, exp2_of(-bias), page >= 0};
            const int64_t base = (((int64_t)max(page, 0) * c.Mkv + w.kv) << c.page_shift) * c.D + (int64_t)slot * c.D;
#pragma unroll
            for (int u = 0; u < (DP == 32 ? 1 : DP / 64); ++u) {
                if constexpr (DP == 32) {
                    const uint2 y = *reinterpret_cast<const uint2*>(c.k + base + k_at[u]);
                    kx[t][u] = make_uint4(y.x, y.y, 0, 0);
                } else {
                    kx[t][u] = *reinterpret_cast<const uint4*>(c.k + base + k_at[u]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int8_t* from = c.v + base + (int64_t)i * c.D + v_at;
                if constexpr (kBytes == 8) {
                    const uint2 y = *reinterpret_cast<const uint2*>(from);
                    vx[4 * t + i][0] = y.x;
                    vx[4 * t + i][1] = y.y;
                } else if constexpr (kBytes == 4) {
                    vx[4 * t + i][0] = *reinterpret_cast<const uint32_t*>(from);
                } else {
                    vx[4 * t + i][0] = *reinterpret_cast<const uint16_t*>(from);
                }
            }
        }
        float4v s[NQ][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int j = 0; j < NQ; ++j) s[j][t] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const uint4 x = kx[t][k / 2];
                const half8 f = k % 2 ? eight_codes(x.z, x.w) : eight_codes(x.x, x.y);
#pragma unroll
                for (int j = 0; j < NQ; ++j) {
                    s[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, q[j][k], s[j][t], 0, 0, 0);
                    if constexpr (kTwo) s[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, q_low[j][k], s[j][t], 0, 0, 0);
                }
            }
        }
        half8 prob[NQ][1], prob_low[kTwo ? NQ : 1][1];
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
            float by[2];
            const float2 top = finish_scores<CAP, APART>(p, s[j], by, unit[j], of, whole, key0 + 4 * g, limit[j]);
            if (__any(top.x > m[j])) {
                const float fade = raise(m[j], top.x);
                l[j] *= fade;
                if constexpr (!APART) {
#pragma unroll
                    for (int u = 0; u < kBytes; ++u) o[j][u] *= fade;
                }
            }
            if constexpr (APART) {
                if (__any(top.y - kShift > ref[j])) {
                    const float fade = raise(ref[j], top.y - kShift);
#pragma unroll
                    for (int u = 0; u < kBytes; ++u) o[j][u] *= fade;
                }
            }
            weigh<kTwo, APART>(s[j], by, of, m[j], ref[j], l[j], prob[j], prob_low[kTwo ? j : 0]);
        }
#pragma unroll
        for (int u = 0; u < kBytes; ++u) {
            uint32_t f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = vx[2 * i][u / 4], b = vx[2 * i + 1][u / 4];
                f[i] = u % 4 == 0 ? two_codes<0, 0>(a, b) : u % 4 == 1 ? two_codes<1, 1>(a, b) : u % 4 == 2 ? two_codes<2, 2>(a, b) : two_codes<3, 3>(a, b);
            }
            const half8 v = __builtin_bit_cast(half8, make_uint4(f[0], f[1], f[2], f[3]));
#pragma unroll
            for (int j = 0; j < NQ; ++j) {
                o[j][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, prob[j][0], o[j][u], 0, 0, 0);
                if constexpr (kTwo) o[j][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, prob_low[j][0], o[j][u], 0, 0, 0);
            }
        }
    }

#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        l[j] = column_sum(l[j]);
        const float by = !APART ? pages.unit() : m[j] == -kInf ? 0.f : exp2_of(ref[j] - m[j]);
#pragma unroll
        for (int u = 0; u < kBytes; ++u) o[j][u] = o[j][u] * exp2_of(-kShift) * by;
    }
#pragma unroll
    for (int j = 0; j < NQ; ++j) {  // 16 rows at a time
        if (j > 0) __syncthreads();  // the last ones have been read
        float* mine = joined + (wave * 16 + col) * kStride;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int u = 0; u < kBytes; u += 2)
                *reinterpret_cast<float2*>(mine + (4 * g + r) * kBytes + u) = make_float2(o[j][u][r], o[j][u + 1][r]);
        if (g == 0) stats[wave * 16 + col] = make_float2(m[j], l[j]);
        if (!APART && j == 0 && lane == 0) failed[wave] = pages.apart;
        __syncthreads();
        if (!APART && j == 0) {
            int any = 0;
#pragma unroll
            for (int v = 0; v < kCacheWaves; ++v) any |= failed[v];
            if (any) return false;
        }
        for (int k = thread; k < 16 * (DP / 4); k += 64 * kCacheWaves) {
            const int in = k / (DP / 4), d = k % (DP / 4) * 4, row = row0 + j * 16 + in, i = row / p.group, h = row - i * p.group;
            if (i >= w.tokens || h >= w.heads) continue;
            Joined x;
#pragma unroll
            for (int v = 0; v < kCacheWaves; ++v)
                x.take(stats[v * 16 + in], *reinterpret_cast<const float4*>(joined + (v * 16 + in) * kStride + d));
            if (p.splits > 1) {
                const int64_t at = ((int64_t)w.item * kRows + row) * p.splits + w.split;
                *reinterpret_cast<float4*>(p.part + at * DP + d) = make_float4(x.x[0], x.x[1], x.x[2], x.x[3]);
                if (d == 0) stats_of<DP>(p, kRows)[at] = make_float2(x.m, x.l);
            } else {
                x.template store<T>(p, (int64_t)(w.token0 + i) * p.M + w.head0 + h, d);
            }
        }
    }
    return true;
}

// Waves per SIMD that the registers of the kernel for 16, 32 and 48 rows leave room for, so that the part for scales that are apart
// takes no more. (128 channels in 16 bits, 32 rows: three keep some of the queries in memory, and a chunk of 2048 tokens over 10240 takes
// 692 us for 748; in fp32 they would keep most of their sums there, 1051 us for 413.)
template <typename T>
constexpr int row_waves(int DP, int NQ) {
    constexpr int of32[3][2] = {{6, 4}, {5, 3}, {3, 2}}, of16[3][3] = {{7, 5, 4}, {5, 4, 3}, {4, 3, 2}};
    const int width = DP == 32 ? 0 : DP == 64 ? 1 : 2;
    return sizeof(T) == 4 ? of32[width][NQ - 1] : of16[width][NQ - 1];
}

// A workgroup's waves share 16 NQ rows and take the 32 keys in turn; their results are joined in LDS. Value scales that are apart
// are found on the way, and the rows begun anew: sixteen at a time, and from the arguments and the thread's number as if they were
// others, so that nothing that this needs takes registers from the first part. (With the choice made for each step of one loop, two chunks took 700 us for 640;
// with one loop after the other, and all rows in both, 645 to 700, and a chunk of 1024 tokens 273 to 318 for 246.)
template <typename T, int DP, int NQ, int CAP>
__global__ __launch_bounds__(64 * kCacheWaves, row_waves<T>(DP, NQ)) void cache_attn_kernel(CacheAttnParams p) {
    __shared__ __attribute__((aligned(16))) float joined[kCacheWaves * 16 * (DP + 4)];
    __shared__ float2 stats[kCacheWaves * 16];
    __shared__ int failed[kCacheWaves];
    if (attend<T, DP, NQ, CAP, false, 16 * NQ>(p, threadIdx.x, 0, joined, stats, failed)) return;
    for (int row0 = 0; row0 < 16 * NQ; row0 += 16) {
        __syncthreads();  // what is in LDS has been read
        auto* arguments = (const __attribute__((address_space(4))) CacheAttnParams*)__builtin_amdgcn_kernarg_segment_ptr();
        int thread = threadIdx.x;
        asm volatile("" : "+s"(arguments), "+v"(thread) : : "memory");
        attend<T, DP, 1, CAP, true, 16 * NQ>(*(const CacheAttnParams*)arguments, thread, row0, joined, stats, failed);
    }
}

// Joins the runs of a block's rows: DP / 4 lanes to a row, a workgroup for each block.
template <typename T, int DP>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnParams p, int rows) {
    const int lane = threadIdx.x & 63, per_block = p.c.Mkv * p.groups;
    CacheWork w;
    if (!w.find_block(p, blockIdx.x / per_block, blockIdx.x % per_block, lane)) return;
    const int runs = max(w.runs(p), 1);
    for (int k = threadIdx.x; k < w.tokens * p.group * (DP / 4); k += 256) {
        const int row = k / (DP / 4), d = k % (DP / 4) * 4, i = row / p.group, h = row - i * p.group;
        if (h >= w.heads) continue;
        const int64_t at = ((int64_t)w.item * rows + row) * p.splits;
        Joined x;
#pragma unroll 4
        for (int s = 0; s < runs; ++s)
            x.take(stats_of<DP>(p, rows)[at + s], *reinterpret_cast<const float4*>(p.part + (at + s) * DP + d));
        x.template store<T>(p, (int64_t)(w.token0 + i) * p.M + w.head0 + h, d);
    }
}

template <typename T, int DP, int CAP>
hipError_t launch_rows(const CacheAttnParams& p, const CacheAttnPlan& plan, hipStream_t stream) {
    const dim3 grid((unsigned)plan.workgroups), block(64 * kCacheWaves);
    if (plan.rows == 16) hipLaunchKernelGGL((cache_attn_kernel<T, DP, 1, CAP>), grid, block, 0, stream, p);
    else if (plan.rows == 32) hipLaunchKernelGGL((cache_attn_kernel<T, DP, 2, CAP>), grid, block, 0, stream, p);
    else if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((cache_attn_kernel<T, DP, 3, CAP>), grid, block, 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL((cache_join_kernel<T, DP>), dim3((unsigned)((int64_t)p.blocks * p.c.Mkv * p.groups)), dim3(256), 0, stream, p,
                       plan.rows);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const CacheAttnParams& p, const CacheAttnPlan& plan, hipStream_t stream) {
    return by_channels(p.c.D, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        if (p.softcap == 0.f) return launch_rows<T, DP, 0>(p, plan, stream);
        if constexpr (sizeof(T) == 2) {
            if (p.softcap <= kShortCap) return launch_rows<T, DP, 1>(p, plan, stream);
        }
        return launch_rows<T, DP, 2>(p, plan, stream);
    });
}

}  // namespace

// Rows of a workgroup by what a sequence has on average, and runs so that the card is full.
CacheAttnPlan cache_attn_plan(const CacheAttnParams& p, int dtype) {
    CacheAttnPlan a;
    const Cache& c = p.c;
    const int64_t mean = c.start && c.N > 0 ? (c.T + c.N - 1) / c.N : 1, G = p.G;
    auto blocks_of = [&](int rows) {
        a.rows = rows;
        a.group = (int)(G < rows ? G : rows);
        a.groups = (int)((G + a.group - 1) / a.group);
        a.tokens = a.rows / a.group;
        a.blocks = place_count(c, a.tokens, 1);
        return a.blocks * c.Mkv * a.groups;
    };
    // More rows of a wave share the codes' way to fp16, but make fewer workgroups. bf16, 32 heads of 128 channels on 8 key heads,
    // with 16, 32 and 48 rows: 8 sequences of 8000 keys with 4 new tokens 42, 47 and 67 us, with 16 63, 55 and 74; one of 8192
    // with 1024 253, 187 and 190; two of 10240 with 2048 1164, 692 and 633. 64 channels, 16 sequences of 4000 with 512 of 8
    // heads: 134, 112 and 113. In fp32 (products of two fp16 parts) 48 rows do not fit into the registers: two of 8192 with 2048,
    // 16 heads of 128 on 4, 517, 413 and 749.
    int64_t items = mean * G <= 16 ? blocks_of(16) : blocks_of(32);
    if (dtype != MSDA_F32 && mean * G >= 1024) {
        items = blocks_of(48);
        if (items < 1024) items = blocks_of(32);
    }
    const int64_t longest = (int64_t)c.width * c.page, least = 256;  // tokens of a run
    int64_t splits = items > 0 ? 1024 / items : 1;
    if (splits > longest / least) splits = longest / least;
    // the partial results have to fit into half a GB
    const int64_t row_bytes = (attn_channels(c.D) + 2) * 4, most = ((int64_t)512 << 20) / (items * a.rows * row_bytes + 1);
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    int64_t run = (longest + splits - 1) / splits;
    run = (run + 32 * kCacheWaves - 1) / (32 * kCacheWaves) * (32 * kCacheWaves);
    a.run = (int)(run < 1 ? 32 * kCacheWaves : run);
    a.splits = (int)((longest + a.run - 1) / a.run);
    if (a.splits < 1) a.splits = 1;
    a.workgroups = (items * a.splits + 7) / 8 * 8;  // see xcd_item
    a.bytes = a.splits > 1 ? (size_t)(items * a.rows * a.splits) * row_bytes : 0;
    return a;
}

hipError_t launch_cache_attn(const CacheAttnParams& p, const CacheAttnPlan& plan, int dtype, hipStream_t stream) {
    if (dtype == MSDA_F32) return launch_typed<float>(p, plan, stream);
    if (dtype == MSDA_F16) return launch_typed<_Float16>(p, plan, stream);
    return launch_typed<bf16_t>(p, plan, stream);
}

}  // namespace msda
