// Dense attention, backward.
//   P = exp(z - lse);  dP_ij = grad_out_i . v_j;  delta_i = sum_d grad_out_i out_i
//   dS = scale P (dP - delta) (1 - tanh^2);  grad_q_i = sum_j dS_ij k_j;  grad_k_j = sum_i dS_ij q_i;  grad_v_j = sum_i P_ij grad_out_i
// The probabilities are formed again from lse. Two kernels, each owning what it sums, so no atomics and
// results that do not depend on scheduling: attn_grad_q_kernel owns rows and walks over the keys (three products),
// attn_grad_kv_kernel owns keys and walks over all the rows that share them (four products). The scores are thus
// formed twice: seven products in place of the five of a kernel that scatters grad_q, whose
// atomics would move rows x channels x key blocks fp32 values instead.
// Where the owners are few the other axis is split over workgroups, and a last kernel adds the splits.
#include "msda_attn.hpp"

namespace msda {
namespace {

// Powers of two by which probabilities are scaled for the product with grad_out: fp16 would round those below 6e-5 (any
// row over 16 thousand keys) to fewer bits.
template <typename T>
constexpr float kProbShift = std::is_same_v<T, _Float16> ? 8.f : 0.f;

// A capped score in units of log 2, and the cap's derivative 1 - tanh^2.
template <typename T>
__device__ __forceinline__ float capped_score(float s, float cap_in, float cap, float& slack) {
    const float t = tanh_of<std::is_same_v<T, float>>(s * cap_in);
    slack = 1.f - t * t;
    return cap * t;
}

template <typename T, int DP, int NW>
__global__ __launch_bounds__(64 * NW) void attn_grad_q_kernel(AttnParams p) {
    using O = Op<T>;
    using Tile = TileOf<T, DP>;
    constexpr int kTile = Tile::kRows, kBlocks = kTile / 32, NT = 64 * NW;
    constexpr int kLoads = kTile * Tile::kChunks / NT;
    __shared__ __attribute__((aligned(16))) T s_k[2][Tile::kElems], s_v[2][Tile::kElems];
    __shared__ __attribute__((aligned(16))) int s_doc[2][kTile];
    __shared__ __attribute__((aligned(16))) float2 s_pos[2][kTile];
    __shared__ int s_bad[2][NW];

    const int item = xcd_item(blockIdx.x, gridDim.x);
    const int per_slab = p.blocks * p.splits;
    if (item >= p.N * p.Mkv * per_slab) return;
    const int slab = item / per_slab, rest = item - slab * per_slab;
    const int split = rest % p.splits;
    const int block = p.blocks - 1 - rest / p.splits;
    const int n = slab / p.Mkv, kv = slab - n * p.Mkv;
    const int lane = threadIdx.x & 63, wave = wave_index(), h = lane >> 5;
    const int off = p.Lk - p.Lq;
    const int common = p.prefix ? min(max(p.prefix[n], 0), p.Lk) : 0;

    const int row = block * 32 * NW + wave * 32 + (lane & 31);
    const int rowc = min(row, p.R - 1);
    const int i = rowc / p.G, head = kv * p.G + rowc - i * p.G;
    const int64_t at_row = (((int64_t)n * p.Lq + i) * p.M + head) * p.D;
    const int64_t at_stat = ((int64_t)n * p.M + head) * p.Lq + i;
    const int doc = p.q_doc ? p.q_doc[(int64_t)n * p.Lq + i] : 0;
    typename O::Frag q[DP / O::K], go[DP / O::K];
    float delta = 0.f;
    {
        const T* qr = static_cast<const T*>(p.q) + n * p.qs[0] + (int64_t)i * p.qs[1] + (int64_t)head * p.qs[2];
        const T* gr = static_cast<const T*>(p.grad_out) + at_row;
        const T* orow = static_cast<const T*>(p.o) + at_row;
#pragma unroll
        for (int c = 0; c < DP / O::K; ++c) {
            const int d = c * O::K + h * (O::K / 2);
            q[c] = __builtin_bit_cast(typename O::Frag, load_chunk(qr, d, p.D, p.q_vec));
            const uint4 g = load_chunk(gr, d, p.D, p.out_vec);
            go[c] = __builtin_bit_cast(typename O::Frag, g);
            const auto o = __builtin_bit_cast(typename O::Frag, load_chunk(orow, d, p.D, p.out_vec));
#pragma unroll
            for (int e = 0; e < O::K / 2; ++e) delta += (float)go[c][e] * (float)o[e];
        }
        delta = halves_sum(delta);
        if (split == 0 && h == 0 && row < p.R) p.delta[at_stat] = delta;
    }
    int last = p.causal ? max(i + off, common - 1) : p.Lk - 1;
    if (doc < 0) last = -1;
    const float lse = p.lse[at_stat] == -kInf ? kInf : p.lse[at_stat] * kLog2e;  // a row that saw nothing: p = 0
    const float slope = p.slopes ? p.slopes[head] * kLog2e : 0.f;
    const float2 pos = p.slopes ? reinterpret_cast<const float2*>(p.q_pos)[(int64_t)n * p.Lq + i] : make_float2(0.f, 0.f);

    const int i_last = (min((block + 1) * 32 * NW, p.R) - 1) / p.G;
    Range rows = {0, 0, 1};
    if (p.q_doc) rows = wave_range(p.q_doc + (int64_t)n * p.Lq, block * 32 * NW / p.G, i_last, lane);
    const int doc0 = __builtin_amdgcn_readfirstlane(doc);
    const bool one_doc = __all(doc == doc0 && doc >= 0), no_pad = __all(doc >= 0);
    const int last0 = p.causal ? __builtin_amdgcn_readfirstlane(last) : p.Lk - 1;
    const int4* k_ranges = p.k_ranges + (int64_t)n * p.k_tiles;
    auto visit = [&](int t) {
        const bool first = t * kTile < common;
        if (p.causal && t * kTile > i_last + off && !first) return false;
        return !p.q_doc || meet(rows, range_of(k_ranges[t]), first);
    };

    const T* k = static_cast<const T*>(p.k) + n * p.ks[0] + kv * p.ks[2];
    const T* v = static_cast<const T*>(p.v) + n * p.vs[0] + kv * p.vs[2];
    const bool masks = p.q_doc || p.causal;
    uint4 kx[kLoads], vx[kLoads];
    int doc_x = 0;
    float2 pos_x = make_float2(0.f, 0.f);
    auto fetch = [&](int t) {
        const int j0 = t * kTile;
#pragma unroll
        for (int a = 0; a < kLoads; ++a) {
            const int id = threadIdx.x + a * NT, r = id / Tile::kChunks, d = (id % Tile::kChunks) * Tile::kPer;
            kx[a] = vx[a] = make_uint4(0, 0, 0, 0);
            if (j0 + r < p.Lk && (!p.k_doc || p.k_doc[(int64_t)n * p.Lk + j0 + r] >= 0)) {
                kx[a] = load_chunk(k + (int64_t)(j0 + r) * p.ks[1], d, p.D, p.k_vec);
                vx[a] = load_chunk(v + (int64_t)(j0 + r) * p.vs[1], d, p.D, p.v_vec);
            }
        }
        if (threadIdx.x < kTile) {
            const int j = j0 + threadIdx.x;
            doc_x = j >= p.Lk ? -1 : p.k_doc ? p.k_doc[(int64_t)n * p.Lk + j] : 0;
            if (p.slopes && j < p.Lk) pos_x = reinterpret_cast<const float2*>(p.k_pos)[(int64_t)n * p.Lk + j];
        }
    };
    auto stage = [&](int b) {
        bool bad = false;
#pragma unroll
        for (int a = 0; a < kLoads; ++a) {
            const int id = threadIdx.x + a * NT, r = id / Tile::kChunks, d = (id % Tile::kChunks) * Tile::kPer;
            *reinterpret_cast<uint4*>(&s_k[b][r * Tile::kStride + d]) = kx[a];
            *reinterpret_cast<uint4*>(&s_v[b][r * Tile::kStride + d]) = vx[a];
            if (masks) bad |= not_finite<T>(kx[a]);
        }
        if (threadIdx.x < kTile) {
            s_doc[b][threadIdx.x] = doc_x;
            if (p.slopes) s_pos[b][threadIdx.x] = pos_x;
        }
        if (masks) {
            const int any = __any(bad);
            if (lane == 0) s_bad[b][wave] = any;
        }
    };

    acc_t gq[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) gq[t] = acc_t{};
    TileWalk walk;
    walk.at = (int)((int64_t)p.k_tiles * split / p.splits);
    walk.end = (int)((int64_t)p.k_tiles * (split + 1) / p.splits);
    int t = walk.next(lane, visit);
    if (t >= 0) fetch(t);
    for (int b = 0; t >= 0; b ^= 1) {
        stage(b);
        __syncthreads();
        const int here = t;
        t = walk.next(lane, visit);
        if (t >= 0) fetch(t);
        const int j0 = here * kTile, j1 = j0 + kTile - 1;
        bool whole = j1 <= last0 && j1 < p.Lk;
        if (p.q_doc) {
            const Range kr = range_of(k_ranges[here]);
            whole = whole && kr.whole && ((one_doc && kr.lo == doc0 && kr.hi == doc0) || (no_pad && j1 < common));
        }
        bool apart = false;
        if (masks && !whole) {
#pragma unroll
            for (int w = 0; w < NW; ++w) apart |= s_bad[b][w] != 0;
        }
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            const T* kt = &s_k[b][kb * 32 * Tile::kStride];
            acc_t s = row_product<T, DP>(kt, Tile::kStride, q, lane);
            acc_t ds = row_product<T, DP>(&s_v[b][kb * 32 * Tile::kStride], Tile::kStride, go, lane);
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] -= delta;
            float unit = p.scale * kLog2e;
            if (p.softcap > 0.f) {
                const float a = p.scale / p.softcap, cap = p.softcap * kLog2e;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float slack;
                    s[r] = capped_score<T>(s[r], a, cap, slack);
                    ds[r] *= slack;
                }
                unit = 1.f;
            }
            if (p.slopes) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float2 kp = s_pos[b][kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3)];
                    const float dx = pos.x - kp.x, dy = pos.y - kp.y;
                    s[r] = s[r] * unit - slope * __builtin_amdgcn_sqrtf(dx * dx + dy * dy);
                }
                unit = 1.f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] *= exp2_of(__builtin_fmaf(s[r], unit, -lse));
            if (!whole) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int jt = kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3), kd = s_doc[b][jt];
                    const bool seen = j0 + jt <= last && kd >= 0 && (!p.q_doc || kd == doc || j0 + jt < common);
                    ds[r] = seen ? ds[r] : 0.f;
                }
            }
            if (apart) add_rows<T, DP>(gq, ds, kt, Tile::kStride, lane);
            else add_product<T, DP>(gq, ds, kt, Tile::kStride, lane);
        }
    }
    if (row >= p.R) return;
    if (p.splits > 1) {
        float* part = p.part + (((int64_t)slab * p.R + row) * p.splits + split) * DP;
#pragma unroll
        for (int u = 0; u < DP / 32; ++u)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(part + u * 32 + 8 * g + 4 * h) =
                    make_float4(gq[u][4 * g], gq[u][4 * g + 1], gq[u][4 * g + 2], gq[u][4 * g + 3]);
        return;
    }
    T* out = static_cast<T*>(p.grad_q) + at_row;
#pragma unroll
    for (int u = 0; u < DP / 32; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = gq[u][4 * g + e] * p.scale;
            store_four(out, u * 32 + 8 * g + 4 * h, p.D, x);
        }
}

template <typename T, int DP, int NW>
__global__ __launch_bounds__(64 * NW) void attn_grad_kv_kernel(AttnParams p) {
    using O = Op<T>;
    using Tile = TileOf<T, DP>;
    constexpr int kTile = Tile::kRows, kBlocks = kTile / 32, NT = 64 * NW;
    constexpr int kLoads = kTile * Tile::kChunks / NT;
    __shared__ __attribute__((aligned(16))) T s_q[2][Tile::kElems], s_g[2][Tile::kElems];
    __shared__ __attribute__((aligned(16))) float s_lse[2][kTile], s_delta[2][kTile], s_slope[2][kTile];
    __shared__ __attribute__((aligned(16))) int s_doc[2][kTile], s_last[2][kTile];
    __shared__ __attribute__((aligned(16))) float2 s_pos[2][kTile];
    __shared__ int s_bad[2][NW];

    const int item = xcd_item(blockIdx.x, gridDim.x);
    const int per_slab = p.blocks * p.splits;
    if (item >= p.N * p.Mkv * per_slab) return;
    const int slab = item / per_slab, rest = item - slab * per_slab;
    const int split = rest % p.splits, block = rest / p.splits;  // the first keys have the most rows
    const int n = slab / p.Mkv, kv = slab - n * p.Mkv;
    const int lane = threadIdx.x & 63, wave = wave_index(), h = lane >> 5;
    const int off = p.Lk - p.Lq;
    const int common = p.prefix ? min(max(p.prefix[n], 0), p.Lk) : 0;

    // the lane's key, in registers with its value
    const int key = block * 32 * NW + wave * 32 + (lane & 31);
    const int j = min(key, p.Lk - 1);
    const int doc = p.k_doc ? p.k_doc[(int64_t)n * p.Lk + j] : 0;
    const bool pad = key >= p.Lk || doc < 0;  // what padding holds must reach nothing
    typename O::Frag k[DP / O::K], v[DP / O::K];
    {
        const T* kr = static_cast<const T*>(p.k) + n * p.ks[0] + (int64_t)j * p.ks[1] + kv * p.ks[2];
        const T* vr = static_cast<const T*>(p.v) + n * p.vs[0] + (int64_t)j * p.vs[1] + kv * p.vs[2];
#pragma unroll
        for (int c = 0; c < DP / O::K; ++c) {
            const int d = c * O::K + h * (O::K / 2);
            uint4 x = make_uint4(0, 0, 0, 0), y = x;
            if (!pad) {
                x = load_chunk(kr, d, p.D, p.k_vec);
                y = load_chunk(vr, d, p.D, p.v_vec);
            }
            k[c] = __builtin_bit_cast(typename O::Frag, x);
            v[c] = __builtin_bit_cast(typename O::Frag, y);
        }
    }
    const float2 pos = p.slopes ? reinterpret_cast<const float2*>(p.k_pos)[(int64_t)n * p.Lk + j] : make_float2(0.f, 0.f);
    const bool is_common = key < common;

    // what the workgroup's keys are seen by at most, and the wave's at least
    const int j_first = block * 32 * NW, j_end = min(j_first + 32 * NW, p.Lk);
    Range keys = {0, 0, 1};
    if (p.k_doc) keys = wave_range(p.k_doc + (int64_t)n * p.Lk, j_first, j_end - 1, lane);
    const int doc0 = __builtin_amdgcn_readfirstlane(doc);
    const bool one_doc = __all(doc == doc0 && doc >= 0), no_pad = __all(!pad);
    const int wave_last = block * 32 * NW + wave * 32 + 31;
    const int4* row_ranges = p.row_ranges + (int64_t)n * p.row_tiles;
    auto visit = [&](int t) {
        if (p.causal && j_first > (min((t + 1) * kTile, p.R) - 1) / p.G + off && j_first >= common) return false;
        return !p.q_doc || meet(keys, range_of(row_ranges[t]), j_first < common);
    };

    const bool masks = p.q_doc || p.causal;
    uint4 qx[kLoads], gx[kLoads];
    float lse_x = 0.f, delta_x = 0.f, slope_x = 0.f;
    int doc_x = -1, last_x = -1;
    float2 pos_x = make_float2(0.f, 0.f);
    auto fetch = [&](int t) {
        const int r0 = t * kTile;
#pragma unroll
        for (int a = 0; a < kLoads; ++a) {
            const int id = threadIdx.x + a * NT, r = id / Tile::kChunks, d = (id % Tile::kChunks) * Tile::kPer;
            qx[a] = gx[a] = make_uint4(0, 0, 0, 0);
            if (r0 + r < p.R) {
                const int i = (r0 + r) / p.G, head = kv * p.G + r0 + r - i * p.G;
                if (!p.q_doc || p.q_doc[(int64_t)n * p.Lq + i] >= 0) {
                    const T* qr = static_cast<const T*>(p.q) + n * p.qs[0] + (int64_t)i * p.qs[1] + (int64_t)head * p.qs[2];
                    qx[a] = load_chunk(qr, d, p.D, p.q_vec);
                    gx[a] = load_chunk(static_cast<const T*>(p.grad_out) + (((int64_t)n * p.Lq + i) * p.M + head) * p.D, d,
                                       p.D, p.out_vec);
                }
            }
        }
        if (threadIdx.x < kTile) {
            const int r = r0 + threadIdx.x;
            lse_x = kInf;
            delta_x = 0.f;
            last_x = doc_x = -1;
            if (r < p.R) {
                const int i = r / p.G, head = kv * p.G + r - i * p.G;
                const int64_t at = ((int64_t)n * p.M + head) * p.Lq + i;
                const float x = p.lse[at];
                if (x != -kInf) lse_x = x * kLog2e;
                delta_x = p.delta[at];
                doc_x = p.q_doc ? p.q_doc[(int64_t)n * p.Lq + i] : 0;
                last_x = doc_x < 0 ? -1 : p.causal ? max(i + off, common - 1) : p.Lk - 1;
                if (p.slopes) {
                    slope_x = p.slopes[head] * kLog2e;
                    pos_x = reinterpret_cast<const float2*>(p.q_pos)[(int64_t)n * p.Lq + i];
                }
            }
        }
    };
    auto stage = [&](int b) {
        bool bad = false;
#pragma unroll
        for (int a = 0; a < kLoads; ++a) {
            const int id = threadIdx.x + a * NT, r = id / Tile::kChunks, d = (id % Tile::kChunks) * Tile::kPer;
            *reinterpret_cast<uint4*>(&s_q[b][r * Tile::kStride + d]) = qx[a];
            *reinterpret_cast<uint4*>(&s_g[b][r * Tile::kStride + d]) = gx[a];
            if (masks) bad |= not_finite<T>(qx[a]) || not_finite<T>(gx[a]);
        }
        if (threadIdx.x < kTile) {
            s_lse[b][threadIdx.x] = lse_x;
            s_delta[b][threadIdx.x] = delta_x;
            s_doc[b][threadIdx.x] = doc_x;
            s_last[b][threadIdx.x] = last_x;
            if (p.slopes) {
                s_slope[b][threadIdx.x] = slope_x;
                s_pos[b][threadIdx.x] = pos_x;
            }
        }
        if (masks) {
            const int any = __any(bad);
            if (lane == 0) s_bad[b][wave] = any;
        }
    };

    acc_t gk[DP / 32], gv[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) gk[t] = gv[t] = acc_t{};
    TileWalk walk;
    walk.at = (int)((int64_t)p.row_tiles * split / p.splits);
    walk.end = (int)((int64_t)p.row_tiles * (split + 1) / p.splits);
    int t = walk.next(lane, visit);
    if (t >= 0) fetch(t);
    for (int b = 0; t >= 0; b ^= 1) {
        stage(b);
        __syncthreads();
        const int here = t;
        t = walk.next(lane, visit);
        if (t >= 0) fetch(t);
        // rows past the last have grad_out = 0 and p = 0, keys past the last are not written
        bool whole = !p.causal || wave_last <= here * kTile / p.G + off || wave_last < common;
        if (p.q_doc) {
            const Range rr = range_of(row_ranges[here]);
            whole = whole && rr.whole && ((one_doc && rr.lo == doc0 && rr.hi == doc0) || (no_pad && wave_last < common));
        }
        bool apart = false;
        if (masks && !whole) {
#pragma unroll
            for (int w = 0; w < NW; ++w) apart |= s_bad[b][w] != 0;
        }
#pragma unroll
        for (int rb = 0; rb < kBlocks; ++rb) {
            const T* qt = &s_q[b][rb * 32 * Tile::kStride];
            const T* gt = &s_g[b][rb * 32 * Tile::kStride];
            acc_t s = row_product<T, DP>(qt, Tile::kStride, k, lane);
            acc_t ds = row_product<T, DP>(gt, Tile::kStride, v, lane);
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] -= s_delta[b][rb * 32 + 8 * (r >> 2) + 4 * h + (r & 3)];
            float unit = p.scale * kLog2e;
            if (p.softcap > 0.f) {
                const float a = p.scale / p.softcap, cap = p.softcap * kLog2e;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float slack;
                    s[r] = capped_score<T>(s[r], a, cap, slack);
                    ds[r] *= slack;
                }
                unit = 1.f;
            }
            if (p.slopes) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = rb * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
                    const float2 qp = s_pos[b][at];
                    const float dx = qp.x - pos.x, dy = qp.y - pos.y;
                    s[r] = s[r] * unit - s_slope[b][at] * __builtin_amdgcn_sqrtf(dx * dx + dy * dy);
                }
                unit = 1.f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = exp2_of(__builtin_fmaf(s[r], unit, kProbShift<T> - s_lse[b][rb * 32 + 8 * (r >> 2) + 4 * h + (r & 3)]));
                ds[r] *= s[r];
                if constexpr (kProbShift<T> != 0.f) ds[r] *= 1.f / (1 << (int)kProbShift<T>);
            }
            if (!whole) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = rb * 32 + 8 * (r >> 2) + 4 * h + (r & 3), qd = s_doc[b][at];
                    const bool seen = key <= s_last[b][at] && !pad && (!p.q_doc || qd == doc || is_common);
                    s[r] = seen ? s[r] : 0.f;
                    ds[r] = seen ? ds[r] : 0.f;
                }
            }
            if (apart) {
                add_rows<T, DP>(gv, s, gt, Tile::kStride, lane);
                add_rows<T, DP>(gk, ds, qt, Tile::kStride, lane);
            } else {
                add_product<T, DP>(gv, s, gt, Tile::kStride, lane);
                add_product<T, DP>(gk, ds, qt, Tile::kStride, lane);
            }
        }
    }
    if (key >= p.Lk) return;
    const float v_unit = exp2_of(-kProbShift<T>);
    if (p.splits > 1) {
        float* part = p.part + (((int64_t)slab * p.Lk + key) * p.splits + split) * 2 * DP;
#pragma unroll
        for (int u = 0; u < DP / 32; ++u)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int d = u * 32 + 8 * g + 4 * h;
                *reinterpret_cast<float4*>(part + d) =
                    make_float4(gk[u][4 * g], gk[u][4 * g + 1], gk[u][4 * g + 2], gk[u][4 * g + 3]);
                *reinterpret_cast<float4*>(part + DP + d) =
                    make_float4(gv[u][4 * g] * v_unit, gv[u][4 * g + 1] * v_unit, gv[u][4 * g + 2] * v_unit,
                                gv[u][4 * g + 3] * v_unit);
            }
        return;
    }
    const int64_t at = (((int64_t)n * p.Lk + key) * p.Mkv + kv) * p.D;
#pragma unroll
    for (int u = 0; u < DP / 32; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = u * 32 + 8 * g + 4 * h;
            float x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = gk[u][4 * g + e] * p.scale;
                y[e] = gv[u][4 * g + e] * v_unit;
            }
            store_four(static_cast<T*>(p.grad_k) + at, d, p.D, x);
            store_four(static_cast<T*>(p.grad_v) + at, d, p.D, y);
        }
}

// Adds the splits of a row of grad_q (KV false), or of a key of grad_k and grad_v: DP / 4 lanes per row and result.
template <typename T, int DP, bool KV>
__global__ __launch_bounds__(256) void attn_sum_kernel(AttnParams p) {
    constexpr int kLanes = (KV ? 2 : 1) * DP / 4;
    const int64_t per_slab = KV ? p.Lk : p.R;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
    if (at >= (int64_t)p.N * p.Mkv * per_slab) return;
    const int e0 = (threadIdx.x % kLanes) * 4;
    const float* part = p.part + at * p.splits * (kLanes * 4) + e0;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
        const float4 y = *reinterpret_cast<const float4*>(part + (int64_t)s * (kLanes * 4));
        x[0] += y.x;
        x[1] += y.y;
        x[2] += y.z;
        x[3] += y.w;
    }
    const int64_t slab = at / per_slab, n = slab / p.Mkv;
    const int own = (int)(at - slab * per_slab), kv = (int)(slab - n * p.Mkv);
    const bool values = KV && e0 >= DP;
    if (!values) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] *= p.scale;
    }
    T* out;
    if constexpr (KV) {
        out = static_cast<T*>(values ? p.grad_v : p.grad_k) + ((n * p.Lk + own) * p.Mkv + kv) * p.D;
    } else {
        const int i = own / p.G;
        out = static_cast<T*>(p.grad_q) + ((n * p.Lq + i) * p.M + kv * p.G + own - i * p.G) * p.D;
    }
    store_four(out, e0 % DP, p.D, x);
}

template <typename T, bool KV>
hipError_t launch_typed(const AttnParams& p, int waves, hipStream_t stream) {
    return by_channels(p.D, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        const dim3 grid((unsigned)xcd_grid((int64_t)p.N * p.Mkv * p.blocks * p.splits));
        if constexpr (KV) {
            if (waves == 4) hipLaunchKernelGGL((attn_grad_kv_kernel<T, DP, 4>), grid, dim3(256), 0, stream, p);
            else hipLaunchKernelGGL((attn_grad_kv_kernel<T, DP, 1>), grid, dim3(64), 0, stream, p);
        } else {
            if (waves == 4) hipLaunchKernelGGL((attn_grad_q_kernel<T, DP, 4>), grid, dim3(256), 0, stream, p);
            else hipLaunchKernelGGL((attn_grad_q_kernel<T, DP, 1>), grid, dim3(64), 0, stream, p);
        }
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.splits == 1) return e;
        const int64_t lanes = (int64_t)p.N * p.Mkv * (KV ? (int64_t)p.Lk * 2 : p.R) * (DP / 4);
        hipLaunchKernelGGL((attn_sum_kernel<T, DP, KV>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, stream, p);
        return hipGetLastError();
    });
}

template <bool KV>
hipError_t launch_grad(const AttnParams& p, int dtype, int waves, hipStream_t stream) {
    if (dtype == MSDA_F32) return launch_typed<float, KV>(p, waves, stream);
    if (dtype == MSDA_F16) return launch_typed<_Float16, KV>(p, waves, stream);
    return launch_typed<bf16_t, KV>(p, waves, stream);
}

}  // namespace

hipError_t launch_attn_grad_q(const AttnParams& p, int dtype, int waves, hipStream_t stream) {
    return launch_grad<false>(p, dtype, waves, stream);
}

hipError_t launch_attn_grad_kv(const AttnParams& p, int dtype, int waves, hipStream_t stream) {
    return launch_grad<true>(p, dtype, waves, stream);
}

}  // namespace msda
