// Dense attention, forward.
//   z_ij = cap(scale q_i . k_j) - slope |q_pos_i - k_pos_j|,  lse_i = log sum_j exp z_ij,  out_i = sum_j exp(z_ij - lse_i) v_j
// One pass over the keys with a running maximum and sum (kept in units of log 2 and in fp32): a workgroup
// owns 32 rows per wave, stages one tile of keys and values after the other in LDS (the next tile's loads
// run while a tile is worked on), and skips the tiles of which its rows see nothing. Probabilities
// are rounded to the operands' type for the product with the values, unnormalized (at most 1), while their sum
// is taken before the rounding: the result's error is then the rounding's, averaged over the keys.
// With few rows the keys are split over workgroups, whose partial results a second kernel joins.
#include "msda_attn.hpp"

namespace msda {
namespace {

template <typename T, int DP, int NW>
__global__ __launch_bounds__(64 * NW) void attn_fwd_kernel(AttnParams p) {
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
    const int block = p.blocks - 1 - rest / p.splits;  // causal rows with the most keys go first
    const int n = slab / p.Mkv, kv = slab - n * p.Mkv;
    const int lane = threadIdx.x & 63, wave = wave_index(), h = lane >> 5;
    const int off = p.Lk - p.Lq;
    const int common = p.prefix ? min(max(p.prefix[n], 0), p.Lk) : 0;

    // the lane's row, its query in registers, and the keys that it sees: up to `last`, of document `doc`
    const int row = block * 32 * NW + wave * 32 + (lane & 31);
    const int rowc = min(row, p.R - 1);
    const int i = rowc / p.G, head = kv * p.G + rowc - i * p.G;
    typename O::Frag q[DP / O::K];
    {
        const T* qr = static_cast<const T*>(p.q) + n * p.qs[0] + (int64_t)i * p.qs[1] + (int64_t)head * p.qs[2];
#pragma unroll
        for (int c = 0; c < DP / O::K; ++c)
            q[c] = __builtin_bit_cast(typename O::Frag, load_chunk(qr, c * O::K + h * (O::K / 2), p.D, p.q_vec));
    }
    const int doc = p.q_doc ? p.q_doc[(int64_t)n * p.Lq + i] : 0;
    int last = p.causal ? max(i + off, common - 1) : p.Lk - 1;
    if (doc < 0) last = -1;
    const float slope = p.slopes ? p.slopes[head] * kLog2e : 0.f;
    const float2 pos = p.slopes ? reinterpret_cast<const float2*>(p.q_pos)[(int64_t)n * p.Lq + i] : make_float2(0.f, 0.f);

    // what all of the workgroup's rows see at most, and all of the wave's rows at least
    const int i_last = (min((block + 1) * 32 * NW, p.R) - 1) / p.G;
    Range rows = {0, 0, 1};
    if (p.q_doc) rows = wave_range(p.q_doc + (int64_t)n * p.Lq, block * 32 * NW / p.G, i_last, lane);
    const int doc0 = __builtin_amdgcn_readfirstlane(doc);
    const bool one_doc = __all(doc == doc0 && doc >= 0), no_pad = __all(doc >= 0);
    const int last0 = p.causal ? __builtin_amdgcn_readfirstlane(last) : p.Lk - 1;  // rows go up with their lanes
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
            // padding is not read: what it holds must reach nothing
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
            if (masks) bad |= not_finite<T>(vx[a]);
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

    acc_t o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[t] = acc_t{};
    float m = -kInf, l = 0.f;
    TileWalk walk;
    walk.at = (int)((int64_t)p.k_tiles * split / p.splits);
    walk.end = (int)((int64_t)p.k_tiles * (split + 1) / p.splits);
    int t = walk.next(lane, visit);
    if (t >= 0) fetch(t);
    for (int b = 0; t >= 0; b ^= 1) {
        stage(b);
        __syncthreads();  // buffer b is written; the tile before it, in the other buffer, has been read by every wave
        const int here = t;
        t = walk.next(lane, visit);
        if (t >= 0) fetch(t);

        acc_t s[kBlocks];
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb)
            s[kb] = row_product<T, DP>(&s_k[b][kb * 32 * Tile::kStride], Tile::kStride, q, lane);
        // scores in units of log 2 once multiplied by `unit`; without cap and bias that product is left to the exponent
        float unit = p.scale * kLog2e;
        if (p.softcap > 0.f) {
            const float a = p.scale / p.softcap, cap = p.softcap * kLog2e;
#pragma unroll
            for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kb][r] = cap * tanh_of<std::is_same_v<T, float>>(s[kb][r] * a);
            unit = 1.f;
        }
        if (p.slopes) {
#pragma unroll
            for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float2 kp = s_pos[b][kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3)];
                    const float dx = pos.x - kp.x, dy = pos.y - kp.y;
                    s[kb][r] = s[kb][r] * unit - slope * __builtin_amdgcn_sqrtf(dx * dx + dy * dy);
                }
            unit = 1.f;
        }
        const int j0 = here * kTile, j1 = j0 + kTile - 1;
        bool whole = j1 <= last0 && j1 < p.Lk;
        if (p.q_doc) {
            const Range kr = range_of(k_ranges[here]);
            whole = whole && kr.whole && ((one_doc && kr.lo == doc0 && kr.hi == doc0) || (no_pad && j1 < common));
        }
        if (!whole) {
#pragma unroll
            for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int jt = kb * 32 + 8 * (r >> 2) + 4 * h + (r & 3), kd = s_doc[b][jt];
                    const bool seen = j0 + jt <= last && kd >= 0 && (!p.q_doc || kd == doc || j0 + jt < common);
                    s[kb][r] = seen ? s[kb][r] : -kInf;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
        top = halves_max(top) * unit;
        if (__any(top > m)) {
            const float m_new = fmaxf(m, top);
            const float fade = exp2_of(m - (m_new == -kInf ? 0.f : m_new));
            m = m_new;
            l *= fade;
#pragma unroll
            for (int u = 0; u < DP / 32; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[u][r] *= fade;
        }
        const float base = m == -kInf ? 0.f : m;  // a row that has seen nothing yet
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = exp2_of(__builtin_fmaf(s[kb][r], unit, -base));
                l += s[kb][r];
            }
        bool apart = false;
        if (masks && !whole) {
#pragma unroll
            for (int w = 0; w < NW; ++w) apart |= s_bad[b][w] != 0;
        }
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            const T* tile = &s_v[b][kb * 32 * Tile::kStride];
            if (apart) add_rows<T, DP>(o, s[kb], tile, Tile::kStride, lane);
            else add_product<T, DP>(o, s[kb], tile, Tile::kStride, lane);
        }
    }
    l = halves_sum(l);
    if (row >= p.R) return;
    if (p.splits > 1) {
        const int64_t at = ((int64_t)slab * p.R + row) * p.splits + split;
        float* part = p.part + at * DP;
#pragma unroll
        for (int u = 0; u < DP / 32; ++u)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(part + u * 32 + 8 * g + 4 * h) =
                    make_float4(o[u][4 * g], o[u][4 * g + 1], o[u][4 * g + 2], o[u][4 * g + 3]);
        if (h == 0) {
            float2* stats = reinterpret_cast<float2*>(p.part + (int64_t)p.N * p.Mkv * p.R * p.splits * DP);
            stats[at] = make_float2(m, l);
        }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = static_cast<T*>(p.out) + (((int64_t)n * p.Lq + i) * p.M + head) * p.D;
#pragma unroll
    for (int u = 0; u < DP / 32; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = o[u][4 * g + e] * inv;
            store_four(out, u * 32 + 8 * g + 4 * h, p.D, x);
        }
    if (p.lse && h == 0)
        p.lse[((int64_t)n * p.M + head) * p.Lq + i] = l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Joins the splits of a row: DP / 4 lanes per row, four channels each.
template <typename T, int DP>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnParams p) {
    constexpr int kLanes = DP / 4;
    const int64_t rows = (int64_t)p.N * p.Mkv * p.R;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
    if (at >= rows) return;
    const int d = (threadIdx.x % kLanes) * 4;
    const float2* stats = reinterpret_cast<const float2*>(p.part + rows * p.splits * DP) + at * p.splits;
    const float* part = p.part + at * p.splits * DP + d;
    float top = -kInf;
    for (int s = 0; s < p.splits; ++s) top = fmaxf(top, stats[s].x);
    const float base = top == -kInf ? 0.f : top;
    float x[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
        const float2 ml = stats[s];
        const float w = exp2_of(ml.x - base);
        const float4 y = *reinterpret_cast<const float4*>(part + (int64_t)s * DP);
        l += w * ml.y;
        x[0] += w * y.x;
        x[1] += w * y.y;
        x[2] += w * y.z;
        x[3] += w * y.w;
    }
    const int64_t slab = at / p.R;
    const int row = (int)(at - slab * p.R), i = row / p.G;
    const int64_t n = slab / p.Mkv;
    const int head = (int)(slab - n * p.Mkv) * p.G + row - i * p.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= inv;
    store_four(static_cast<T*>(p.out) + ((n * p.Lq + i) * p.M + head) * p.D, d, p.D, x);
    if (p.lse && d == 0)
        p.lse[(n * p.M + head) * p.Lq + i] = l == 0.f ? -kInf : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

// Documents of each tile of keys, or of each tile of rows (the queries that its rows belong to).
__global__ __launch_bounds__(256) void attn_ranges_kernel(AttnParams p, int tile, int with_rows) {
    const int lane = threadIdx.x & 63;
    const int per = p.k_tiles + (with_rows ? p.row_tiles : 0);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave_index();
    if (item >= (int64_t)p.N * per) return;
    const int64_t n = item / per;
    int t = (int)(item - n * per);
    const bool keys = t < p.k_tiles;
    if (!keys) t -= p.k_tiles;
    const int first = keys ? t * tile : t * tile / p.G;
    const int last = keys ? min((t + 1) * tile, p.Lk) - 1 : (min((t + 1) * tile, p.R) - 1) / p.G;
    const Range r = wave_range(keys ? p.k_doc + n * p.Lk : p.q_doc + n * p.Lq, first, last, lane);
    int4* into = keys ? p.k_ranges + n * p.k_tiles : p.row_ranges + n * p.row_tiles;
    if (lane == 0) into[t] = make_int4(r.lo, r.hi, r.whole, 0);
}

template <typename T>
hipError_t launch_typed(const AttnParams& p, int waves, hipStream_t stream) {
    return by_channels(p.D, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        const dim3 grid((unsigned)xcd_grid((int64_t)p.N * p.Mkv * p.blocks * p.splits));
        if (waves == 4) hipLaunchKernelGGL((attn_fwd_kernel<T, DP, 4>), grid, dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((attn_fwd_kernel<T, DP, 1>), grid, dim3(64), 0, stream, p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.splits == 1) return e;
        const int64_t rows = (int64_t)p.N * p.Mkv * p.R;
        hipLaunchKernelGGL((attn_join_kernel<T, DP>), dim3((unsigned)((rows * (DP / 4) + 255) / 256)), dim3(256), 0,
                           stream, p);
        return hipGetLastError();
    });
}

}  // namespace

int attn_tile(int dtype) { return dtype == MSDA_F32 ? Op<float>::kTile : Op<_Float16>::kTile; }
int attn_channels(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

AttnPlan attn_plan(const AttnParams& p, int dtype, bool own_keys) {
    const int64_t own = own_keys ? p.Lk : p.R;
    const int64_t tiles = own_keys ? p.row_tiles : p.k_tiles;
    AttnPlan a;
    a.waves = own <= 32 ? 1 : 4;
    a.blocks = (int)((own + 32 * a.waves - 1) / (32 * a.waves));
    // enough waves for two on each of the 1024 SIMDs, of at least four tiles each
    const int64_t waves = (int64_t)p.N * p.Mkv * a.blocks * a.waves;
    int64_t splits = (2048 + waves - 1) / waves;
    if (splits > tiles / 4) splits = tiles / 4;
    a.splits = (int)(splits < 1 ? 1 : splits > 256 ? 256 : splits);
    (void)dtype;
    return a;
}

hipError_t launch_attn_ranges(const AttnParams& p, int dtype, bool rows, hipStream_t stream) {
    const int64_t items = (int64_t)p.N * (p.k_tiles + (rows ? p.row_tiles : 0));
    hipLaunchKernelGGL(attn_ranges_kernel, dim3((unsigned)((items + 3) / 4)), dim3(256), 0, stream, p, attn_tile(dtype),
                       rows ? 1 : 0);
    return hipGetLastError();
}

hipError_t launch_attn_forward(const AttnParams& p, int dtype, int waves, hipStream_t stream) {
    if (dtype == MSDA_F32) return launch_typed<float>(p, waves, stream);
    if (dtype == MSDA_F16) return launch_typed<_Float16>(p, waves, stream);
    return launch_typed<bf16_t>(p, waves, stream);
}

}  // namespace msda
