// Dense attention, backward.
//   P = exp(z - lse);  dP_ij = grad_out_i . v_j;  delta_i = sum_d grad_out_i out_i
//   dS = scale P (dP - delta) (1 - tanh^2);  grad_q_i = sum_j dS_ij k_j;  grad_k_j = sum_i dS_ij q_i;  grad_v_j = sum_i P_ij grad_out_i
// The probabilities are formed again from lse. Two kernels, each owning what it sums, so no atomics and
// results that do not depend on scheduling: attn_grad_q_kernel owns rows and walks over the keys (three products),
// attn_grad_kv_kernel owns keys and walks over all the rows that share them (four products). The scores are thus
// formed twice: seven products in place of the five of a kernel that scatters grad_q, whose
// atomics would move rows x channels x key blocks fp32 values instead.
// Where the owners are few the other axis is split over workgroups, and a last kernel adds the splits.
// Measured, with the products of the pairs that are seen, grad_q and grad_kv: bf16, 2 x 4947 rows x 8 heads x 32, padded:
// 121 and 179 us, 437 and 394 TFLOP/s, bound by the vector work of a pair as the forward; 2 x 4096 packed causal rows x
// 16 heads x 128 on 4 key heads, capped: 145 and 307 us, 300 and 188 TFLOP/s (the second has room for one wave per SIMD:
// k, v and two sums of 128 channels); fp32, 3 x 1023 rows over 2999 x 5 x 48: 181 and 272 us, 53 and 47 TFLOP/s, the matrix unit
// busy in 60 % of the cycles in which a CU has waves, which are 70 % of the kernels' (1080 workgroups for 512 places).
// Where 16-bit rows may have few keys, a third kernel forms delta before them.
#include "msda_attn.hpp"

namespace msda {
namespace {

// The power of two that an owner's score gradients carry as an operand in fp16, which holds 2^-14 .. 2^16 with all its bits:
// P (dP - delta) is about grad_out / keys, so rows of 16 thousand keys and a grad_out of 1e-3 would be rounded to 3 % of
// grad_q, and large ones would overflow. It is set by the largest so far, like a softmax's running maximum: that is kept
// within 2^10 .. 2^15, and the sums follow where it has to come down. What is lost is then at most 2^-35 of the largest. bf16
// has the exponents of fp32 and needs none. The maximum made fp16 steps 2 to 5 % longer.
template <typename T, int DP>
struct Carried {
    static constexpr bool kAny = std::is_same_v<T, _Float16>;
    float up = 0.f, unit = 1.f;  // its exponent, and itself
    float limit = 0.f;           // of the operands that the power of two holds for; 0 before the first
    // `w`: gradients of 32 scores of the lane's owner, which go into `sum`.
    __device__ __forceinline__ void keep(acc_t& w, acc_t (&sum)[DP / 32]) {
        if constexpr (!kAny) return;
        float top = fabsf(w[0]);
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, fabsf(w[r]));
        if (!__any(top > limit)) return;
        top = halves_max(top);
        if (!(top > limit && top < kInf)) return;
        // at most 2^60: a dP of fp16 values is below 2^39, and what is below 2^-84 reaches no fp16 result
        const int by = min(11 - __builtin_amdgcn_frexp_expf(top), 60 - (int)up);
        up += (float)by;
        unit = __builtin_ldexpf(1.f, (int)up);
        limit = 0x1p15f;
#pragma unroll
        for (int r = 0; r < 16; ++r) w[r] = __builtin_ldexpf(w[r], by);
#pragma unroll
        for (int u = 0; u < DP / 32; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[u][r] = __builtin_ldexpf(sum[u][r], by);
    }
    __device__ __forceinline__ float taken_out(float x) const { return kAny ? __builtin_ldexpf(x, -(int)up) : x; }
};

// Waves per SIMD that the kernels' registers have to leave room for.
constexpr int grad_q_waves(int DP, size_t element) { return DP == 32 ? 3 : DP == 128 && element == 4 ? 1 : 2; }
constexpr int grad_kv_waves(int DP) { return DP == 32 ? 3 : DP == 64 ? 2 : 1; }

// In calls with masks, a key that holds an infinity or a NaN is taken as hidden: its products with zeros (of pairs that
// are) must not reach grad_q, and nothing else is lost. A row that sees it has a score of minus infinity, or of plus or minus
// the cap, with which it passes no gradient; or one of plus infinity or NaN, and then its lse is NaN and so is its gradient.
template <typename T, int DP, int NW, int EXTRAS>
__global__ __launch_bounds__(64 * NW, grad_q_waves(DP, sizeof(T))) void attn_grad_q_kernel(AttnParams p) {
    using O = Op<T>;
    using Keys = KeyTiles<T, DP, NW, EXTRAS >= kBias, kKeys>;
    using Tile = typename Keys::Tile;
    __shared__ __attribute__((aligned(16))) typename Keys::Shared sh;
    Work w(p, true);
    if (!w.any) return;
    const int lane = threadIdx.x & 63, wave = wave_index(), h = lane >> 5;
    Keys keys(sh, p, w, lane);
    const bool any = w.note_split(p, keys.any());
    if (!any && w.split > 0) return;  // the first split writes delta
    const Row32 own = Row32::of<NW>(p, w, wave, lane, EXTRAS >= kBias);
    typename O::Frag q[DP / O::K], go[DP / O::K];
    float delta = 0.f;
    {
        const T* qr = static_cast<const T*>(p.q) + w.n * p.qs[0] + own.i * p.qs[1] + own.head * p.qs[2];
        const T* gr = static_cast<const T*>(p.grad_out) + own.at * p.row_width;
        const T* orow = static_cast<const T*>(p.o) + own.at * p.row_width;
#pragma unroll
        for (int c = 0; c < DP / O::K; ++c) {
            const int d = c * O::K + h * (O::K / 2);
            q[c] = __builtin_bit_cast(typename O::Frag, load_chunk(qr, d, p.D));
            go[c] = __builtin_bit_cast(typename O::Frag, load_chunk(gr, d, p.D));
            if (p.delta_known) continue;
            const auto o = __builtin_bit_cast(typename O::Frag, load_chunk(orow, d, p.D));
#pragma unroll
            for (int e = 0; e < O::K / 2; ++e) delta += (float)go[c][e] * (float)o[e];
        }
        if (p.delta_known) {
            delta = p.delta[own.stat];
        } else {
            delta = halves_sum(delta);
            if (w.split == 0 && h == 0 && own.row < p.R) p.delta[own.stat] = delta;
        }
        if (!any) return;
    }
    const float lse = p.lse[own.stat] == -kInf ? kInf : p.lse[own.stat] * kLog2e;  // a row that saw nothing: p = 0
    acc_t minus_delta, gq[DP / 32];
#pragma unroll
    for (int r = 0; r < 16; ++r) minus_delta[r] = -delta;  // where the sums of dP begin
#pragma unroll
    for (int u = 0; u < DP / 32; ++u) gq[u] = acc_t{};
    Carried<T, DP> carried;
    auto body = [&](int b, int j0, int sub, bool partial) {  // the tile's keys from sub on
#pragma unroll
        for (int kb = 0; kb < Tile::kBlocks; ++kb) {
            const T* kt = sh.k[b] + (sub + kb * 32) * Tile::kStride;
            acc_t s = row_product<T, DP>(kt, Tile::kStride, q, lane, p.D, acc_t{});
            acc_t ds = row_product<T, DP>(sh.v[b] + (sub + kb * 32) * Tile::kStride, Tile::kStride, go, lane, p.D, minus_delta);
            float unit = p.scale * kLog2e;
            if constexpr (EXTRAS >= kCap) unit = cap_scores<T, EXTRAS>(p, s, &ds);
            if constexpr (EXTRAS >= kBias) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float2 kp = sh.pos[b][sub + kb * 32 + block_row(r, h)];
                    const float dx = own.pos.x - kp.x, dy = own.pos.y - kp.y;
                    s[r] = s[r] * unit - own.slope * __builtin_amdgcn_sqrtf(dx * dx + dy * dy);
                }
                unit = 1.f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] *= exp2_of(__builtin_fmaf(s[r], unit, carried.up - lse));
            if (partial) {
                acc_t x[1] = {ds};
                hide(x, 0.f, sub + kb * 32, h, own.last - j0, own.doc, sh.doc[b]);
                ds = x[0];
            }
            carried.keep(ds, gq);
            add_product<T, DP>(gq, ds, kt, Tile::kStride, lane);
        }
    };
    keys.fetch();
    for (int b = 0; keys.t >= 0; b ^= 1) {
        keys.stage(b);
        const bool whole = keys.whole(own);
        const int j0 = keys.t * Tile::kRows;
        __syncthreads();  // buffer b is written, and every wave has read the other one, which is next
        const bool partial = !whole || keys.any_odd(b);
        keys.fetch();
#pragma unroll 1
        for (int sub = 0; sub < Tile::kRows; sub += 32 * Tile::kBlocks) body(b, j0, sub, partial);
    }
    if (own.row >= p.R) return;
    float* part = p.part + (((int64_t)w.slab * p.R + own.row) * p.splits + w.split) * DP;
    T* out = static_cast<T*>(p.grad_q) + own.at * p.D;
#pragma unroll
    for (int u = 0; u < DP / 32; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = u * 32 + 8 * g + 4 * h;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = lse == lse ? carried.taken_out(gq[u][4 * g + e]) * p.scale : lse;
            if (p.splits > 1) *reinterpret_cast<float4*>(part + d) = make_float4(x[0], x[1], x[2], x[3]);
            else store_four(out, d, p.D, x);
        }
}

// Where a row has few keys, dP - delta is small beside dP, and the rounding of out to 16 bits, which delta holds, is
// the largest part of the gradients' error: of two keys, grad_q and grad_k were 4 times as far off as by their own
// roundings. As a row's probabilities add up to one, sum_j P (dP - delta) is what delta lacks. This kernel writes delta, and
// mends that of the rows that see at most kFewKeys keys: a row of n keys gains 1 part in n of its error, so there is nothing
// to be had of longer ones. A workgroup walks over the tiles that its rows see, wherever they are, and leaves those that only
// rows with more keys see: long rows cost it a tile or two, or none where the tables of documents say that they are. A
// row is mended once all of its keys have been visited: one that is left out may have a value that outweighs its probability.
// 6 us in the first shape above and 35 in the second, whose out and grad_out take 12 at a copy's rate (two waves per SIMD wait
// for them, and a few workgroups for their tiles); grad_q reads delta in place of out then.
template <typename T, int DP, int NW, int EXTRAS>
__global__ __launch_bounds__(64 * NW, grad_q_waves(DP, sizeof(T))) void attn_delta_kernel(AttnParams p) {
    using O = Op<T>;
    using Keys = KeyTiles<T, DP, NW, EXTRAS >= kBias, kNothing, 1>;
    using Tile = typename Keys::Tile;
    __shared__ __attribute__((aligned(16))) typename Keys::Shared sh;
    __shared__ int2 s_open[NW];
    Work w(p, true);
    if (!w.any) return;
    const int lane = threadIdx.x & 63, wave = wave_index(), h = lane >> 5;
    Keys keys(sh, p, w, lane);
    const Row32 own = Row32::of<NW>(p, w, wave, lane, EXTRAS >= kBias);
    typename O::Frag q[DP / O::K], go[DP / O::K];
    const T* gr = static_cast<const T*>(p.grad_out) + own.at * p.row_width;
    const T* orow = static_cast<const T*>(p.o) + own.at * p.row_width;
    float delta = 0.f;
#pragma unroll
    for (int c = 0; c < DP / O::K; ++c) {
        const int d = c * O::K + h * (O::K / 2);
        go[c] = __builtin_bit_cast(typename O::Frag, load_chunk(gr, d, p.D));
        const auto o = __builtin_bit_cast(typename O::Frag, load_chunk(orow, d, p.D));
#pragma unroll
        for (int e = 0; e < O::K / 2; ++e) delta += (float)go[c][e] * (float)o[e];
    }
    delta = halves_sum(delta);
    const float lse = p.lse[own.stat] == -kInf ? kInf : p.lse[own.stat] * kLog2e;
    acc_t minus_delta;
#pragma unroll
    for (int r = 0; r < 16; ++r) minus_delta[r] = -delta;
    float lack = 0.f, met = 0.f;  // met: keys seen so far, of this half wave's
    // rows that may turn out to have few keys; without documents a row's place says how many it sees
    bool open = own.row < p.R && own.last >= 0 && (p.q_doc || own.last < kFewKeys);
    if (p.tile_ranges) {  // not if the tiles that are of its document, or common, from end to end are enough
        const int4* ranges = w.tile_ranges(p);
        int enough = kFewKeys;
        for (int t0 = 0; t0 < p.tiles && __any(open); t0 += 64) {
            const int t = t0 + lane;
            int4 x = make_int4(0, -1, 0, 0);
            if (t < p.tiles && (t + 1) * Tile::kRows <= p.Lk) x = ranges[t];
            uint64_t all = __ballot(x.z && ((x.x == x.y && w.docs.lo <= x.x && x.x <= w.docs.hi) || (t + 1) * Tile::kRows <= w.common));
            for (; all && __any(open); all &= all - 1) {
                const int b = __builtin_ctzll(all), end = (t0 + b + 1) * Tile::kRows;
                const bool seen = end - 1 <= own.last && (end <= w.common || __builtin_amdgcn_readlane(x.x, b) == own.doc);
                enough -= seen ? Tile::kRows : 0;
                open = open && enough >= 0;
            }
        }
    }
    // Whether a row of the workgroup is open; the walk goes on with what such rows see.
    auto any_open = [&]() {
        int lo = open ? own.doc : 0x7fffffff, hi = open ? own.doc : -1;
#pragma unroll
        for (int m = 16; m; m >>= 1) {  // both half waves hold the same rows
            lo = min(lo, __shfl_xor(lo, m, 64));
            hi = max(hi, __shfl_xor(hi, m, 64));
        }
        if (lane == 0) s_open[wave] = make_int2(lo, hi);
        __syncthreads();  // and every wave has read the tile
        for (int i = 0; i < NW; ++i) {
            lo = min(lo, s_open[i].x);
            hi = max(hi, s_open[i].y);
        }
        keys.only({__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi), 1});
        return w.docs.hi >= 0;
    };
    auto body = [&](int j0, int sub, bool partial) {  // the tile's keys from sub on
#pragma unroll
        for (int kb = 0; kb < Tile::kBlocks; ++kb) {
            acc_t s = row_product<T, DP>(sh.k[0] + (sub + kb * 32) * Tile::kStride, Tile::kStride, q, lane, p.D, acc_t{});
            const acc_t e = row_product<T, DP>(sh.v[0] + (sub + kb * 32) * Tile::kStride, Tile::kStride, go, lane, p.D, minus_delta);
            float unit = p.scale * kLog2e;
            if constexpr (EXTRAS >= kCap) unit = cap_scores<T, EXTRAS>(p, s, nullptr);
            if constexpr (EXTRAS >= kBias) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float2 kp = sh.pos[0][sub + kb * 32 + block_row(r, h)];
                    const float dx = own.pos.x - kp.x, dy = own.pos.y - kp.y;
                    s[r] = s[r] * unit - own.slope * __builtin_amdgcn_sqrtf(dx * dx + dy * dy);
                }
                unit = 1.f;
            }
            acc_t x[2];  // the probabilities, and a one for each
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[0][r] = exp2_of(__builtin_fmaf(s[r], unit, -lse));
                x[1][r] = 1.f;
            }
            if (partial) hide(x, 0.f, sub + kb * 32, h, own.last - j0, own.doc, sh.doc[0]);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (x[0][r] > 0.f) lack += x[0][r] * e[r];  // padding's dP may be anything
                met += x[1][r];
            }
        }
    };
    if (any_open()) {
        const T* qr = static_cast<const T*>(p.q) + w.n * p.qs[0] + own.i * p.qs[1] + own.head * p.qs[2];
#pragma unroll
        for (int c = 0; c < DP / O::K; ++c)
            q[c] = __builtin_bit_cast(typename O::Frag, load_chunk(qr, c * O::K + h * (O::K / 2), p.D));
        keys.fetch();
        while (keys.t >= 0) {
            keys.stage(0);
            const bool whole = keys.whole(own);
            const int j0 = keys.t * Tile::kRows;
            __syncthreads();  // the tile is written
            keys.fetch();
            if (whole && Tile::kRows > kFewKeys) {
                open = false;
            } else if (__any(open)) {
#pragma unroll 1
                for (int sub = 0; sub < Tile::kRows; sub += 32 * Tile::kBlocks) body(j0, sub, !whole);
                open = open && halves_sum(met) <= kFewKeys;
            }
            if (!any_open()) break;
        }
    }
    lack = halves_sum(lack);
    if (h == 0 && own.row < p.R) p.delta[own.stat] = open && fabsf(lack) < kInf ? delta + lack : delta;
}

template <typename T, int DP, int NW, int EXTRAS>
__global__ __launch_bounds__(64 * NW, grad_kv_waves(DP)) void attn_grad_kv_kernel(AttnParams p) {
    using O = Op<T>;
    using Tile = TileOf<T, DP, NW, true>;
    __shared__ __attribute__((aligned(16))) T s_q[2][Tile::kElems], s_g[2][Tile::kElems];
    __shared__ __attribute__((aligned(16))) float s_lse[2][Tile::kRows], s_delta[2][Tile::kRows];
    __shared__ __attribute__((aligned(16))) int s_doc[2][Tile::kRows], s_last[2][Tile::kRows];
    __shared__ __attribute__((aligned(16))) float s_slope[2][EXTRAS >= kBias ? Tile::kRows : 1];
    __shared__ __attribute__((aligned(16))) float2 s_pos[2][EXTRAS >= kBias ? Tile::kRows : 1];
    __shared__ int s_odd[2][NW];
    __shared__ uint32_t odd_words[2][32 * NW * Odd<DP>::kWords];
    Work w(p, false);  // the first keys have the most rows
    if (!w.any) return;
    const int lane = threadIdx.x & 63, wave = wave_index(), h = lane >> 5;
    const int j_first = w.block * 32 * NW;
    auto visits = [&](int u, Range of) {
        return sees(p, w, (min((u + 1) * Tile::kRows, p.R) - 1) / p.G, of, j_first, w.docs);
    };
    if (!w.note_split(p, w.walk.more(lane, w.tile_ranges(p), visits))) return;

    // the lane's key, in registers with its value
    const int key = j_first + wave * 32 + (lane & 31);
    const int j = min(key, p.Lk - 1);
    const int doc = p.k_doc ? p.k_doc[(int64_t)w.n * p.Lk + j] : 0;
    const bool pad = key >= p.Lk || doc < 0;  // what padding holds must reach nothing
    typename O::Frag k[DP / O::K], v[DP / O::K];
    {
        const T* kr = static_cast<const T*>(p.k) + w.n * p.ks[0] + j * p.ks[1] + w.kv * p.ks[2];
        const T* vr = static_cast<const T*>(p.v) + w.n * p.vs[0] + j * p.vs[1] + w.kv * p.vs[2];
#pragma unroll
        for (int c = 0; c < DP / O::K; ++c) {
            const int d = pad ? p.D : c * O::K + h * (O::K / 2);  // no channels of it
            k[c] = __builtin_bit_cast(typename O::Frag, load_chunk(kr, d, p.D));
            v[c] = __builtin_bit_cast(typename O::Frag, load_chunk(vr, d, p.D));
        }
    }
    float2 pos = make_float2(0.f, 0.f);
    if (EXTRAS >= kBias && p.slopes) pos = reinterpret_cast<const float2*>(p.k_pos)[(int64_t)w.n * p.Lk + j];
    const bool is_common = key < w.common;
    const int key_code = pad ? 0x7fffffff : key;  // past the last key that any row sees

    // what all of the wave's keys are seen by
    const int doc0 = __builtin_amdgcn_readfirstlane(doc);
    const bool one_doc = __all((doc == doc0) & (doc >= 0)), no_pad = __all(!pad);
    const int wave_last = j_first + wave * 32 + 31;
    const bool masks = p.q_doc || p.causal;

    int t = -1;
    bool clean = true;  // all of the tile's rows count
    Range rr = {0, 0, 1};
    uint4 qx[Tile::kLoads], gx[Tile::kLoads];
    bool pad_x[Tile::kLoads];
    float lse_x = 0.f, delta_x = 0.f, slope_x = 0.f;
    int doc_x = -1, last_x = -1;
    float2 pos_x = make_float2(0.f, 0.f);
#pragma unroll
    for (int a = 0; a < Tile::kLoads; ++a) {
        qx[a] = gx[a] = make_uint4(0, 0, 0, 0);  // what lanes of channels from D on put into LDS
        pad_x[a] = false;
    }
    const float inv_g = 1.f / (float)p.G;
    const T* q_base = static_cast<const T*>(p.q) + w.n * p.qs[0] + w.kv * p.G * p.qs[2];
    const T* g_base = static_cast<const T*>(p.grad_out) + ((int64_t)w.n * p.Lq * p.M + w.kv * p.G) * p.row_width;
    auto query_row = [&](int r) { return q_base + r / p.G * p.qs[1] + r % p.G * p.qs[2]; };
    auto grad_row = [&](int r) { return g_base + ((int64_t)(r / p.G) * p.M + r % p.G) * p.row_width; };
    auto fetch = [&]() {
        t = w.walk.next(lane, w.tile_ranges(p), rr, visits);
        if (t < 0) return;
        // row r of the tile is query i0 + (g0 + r) / G of head (g0 + r) % G of the group
        const int r0 = t * Tile::kRows, i0 = r0 / p.G, g0 = r0 - i0 * p.G;
        clean = r0 + Tile::kRows <= p.R && rr.whole;
        const T* qt = q_base + i0 * p.qs[1];
        const T* gt = g_base + (int64_t)i0 * p.M * p.row_width;
#pragma unroll
        for (int a = 0; a < Tile::kLoads; ++a) {
            const int x = g0 + Tile::row(a), i = small_div(x, inv_g), g = x - i * p.G;
            const bool in = r0 + Tile::row(a) < p.R;
            if (in && Tile::channel() < p.D) {
                qx[a] = load_at(qt, (i * (int)p.qs[1] + g * (int)p.qs[2] + Tile::channel()) * (int)sizeof(T));
                gx[a] = load_at(gt, ((i * p.M + g) * p.row_width + Tile::channel()) * (int)sizeof(T));
            }
            if (!clean) pad_x[a] = !in || (p.q_doc && p.q_doc[(int64_t)w.n * p.Lq + i0 + i] < 0);
        }
        if ((int)threadIdx.x < Tile::kRows) {
            const int x = g0 + (int)threadIdx.x, i = i0 + small_div(x, inv_g), head = w.kv * p.G + x - (i - i0) * p.G;
            lse_x = delta_x = slope_x = 0.f;
            pos_x = make_float2(0.f, 0.f);
            last_x = doc_x = -1;
            if (r0 + (int)threadIdx.x < p.R) {
                const int64_t at = ((int64_t)w.n * p.M + head) * p.Lq + i;
                lse_x = p.lse[at];
                delta_x = p.delta[at];
                doc_x = p.q_doc ? p.q_doc[(int64_t)w.n * p.Lq + i] : 0;
                last_x = p.causal ? max(i + w.off, w.common - 1) : p.Lk - 1;
                if (EXTRAS >= kBias && p.slopes) {
                    slope_x = p.slopes[head] * kLog2e;
                    pos_x = reinterpret_cast<const float2*>(p.q_pos)[(int64_t)w.n * p.Lq + i];
                }
            }
        }
    };
    auto stage = [&](int b) {
        if (!clean) {
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a)
                if (pad_x[a]) qx[a] = gx[a] = make_uint4(0, 0, 0, 0);
        }
        if (masks) {  // sums are over queries and over grad_out
            bool odd = false;
#pragma unroll
            for (int a = 0; a < Tile::kLoads; ++a) {
                odd |= not_finite<T>(qx[a]);
                odd |= not_finite<T>(gx[a]);
            }
            const bool some = __any(odd);
            if (some) {
#pragma unroll
                for (int a = 0; a < Tile::kLoads; ++a) {
                    qx[a] = finite_only<T>(qx[a]);
                    gx[a] = finite_only<T>(gx[a]);
                }
            }
            if (lane == 0) s_odd[b][wave] = some;
        }
#pragma unroll
        for (int a = 0; a < Tile::kLoads; ++a) {
            Tile::put(s_q[b], a, qx[a]);
            Tile::put(s_g[b], a, gx[a]);
        }
        if ((int)threadIdx.x < Tile::kRows) {
            s_lse[b][threadIdx.x] = lse_x == -kInf ? -kInf : kProbShift<T> - lse_x * kLog2e;
            s_delta[b][threadIdx.x] = -delta_x;
            s_doc[b][threadIdx.x] = doc_x;
            s_last[b][threadIdx.x] = doc_x < 0 ? -1 : last_x;
            if (EXTRAS >= kBias) {
                s_slope[b][threadIdx.x] = slope_x;
                s_pos[b][threadIdx.x] = pos_x;
            }
        }
    };

    acc_t gk[DP / 32], gv[DP / 32];
#pragma unroll
    for (int u = 0; u < DP / 32; ++u) gk[u] = gv[u] = acc_t{};
    Odd<DP> odd_k, odd_v;
    odd_k.start(odd_words[0], wave * 32 + (lane & 31), lane, masks);
    odd_v.start(odd_words[1], wave * 32 + (lane & 31), lane, masks);
    // A query that holds an infinity has weights where its scores are capped; the staged copy, which is summed over, is
    // without the infinity. Adds what it gives to the scores of 32 rows from `first` on.
    const T* own_key = static_cast<const T*>(p.k) + w.n * p.ks[0] + j * p.ks[1] + w.kv * p.ks[2];
    auto add_infinities = [&](acc_t& s, int first) {
#pragma unroll 1
        for (int r = 0; r < 16; ++r) {
            const int row = first + block_row(r, h);
            if (row >= p.R) continue;
            const T* qr = query_row(row);
            float more = 0.f;
#pragma unroll 1
            for (int c = 0; c < p.D; ++c) {
                const float x = (float)qr[c];
                if (!(fabsf(x) < kInf)) more += x * (float)own_key[c];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] += i == r ? more : 0.f;
        }
    };
    Carried<T, DP> carried;
    auto body = [&](int b, int r0, int sub, int some, bool partial) {  // the tile's rows from sub on
#pragma unroll
        for (int block = 0; block < Tile::kBlocks; ++block) {
            const int first = sub + block * 32;
            const T* qt = s_q[b] + first * Tile::kStride;
            const T* gt = s_g[b] + first * Tile::kStride;
            acc_t ds;  // the sums of dP begin at -delta
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = s_delta[b][first + block_row(r, h)];
            acc_t s = row_product<T, DP>(qt, Tile::kStride, k, lane, p.D, acc_t{});
            ds = row_product<T, DP>(gt, Tile::kStride, v, lane, p.D, ds);
            float unit = p.scale * kLog2e;
            if constexpr (EXTRAS >= kCap) {
                if (some) add_infinities(s, r0 + first);
                unit = cap_scores<T, EXTRAS>(p, s, &ds);
            }
            if constexpr (EXTRAS >= kBias) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = first + block_row(r, h);
                    const float2 qp = s_pos[b][at];
                    const float dx = qp.x - pos.x, dy = qp.y - pos.y;
                    s[r] = s[r] * unit - s_slope[b][at] * __builtin_amdgcn_sqrtf(dx * dx + dy * dy);
                }
                unit = 1.f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = exp2_of(__builtin_fmaf(s[r], unit, s_lse[b][first + block_row(r, h)]));
                ds[r] *= s[r];
                if constexpr (Carried<T, DP>::kAny) ds[r] *= carried.unit * (1.f / (1 << kProbShift<T>));
            }
            if (partial) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {  // four at a time, as in hide()
                    const int at = first + 8 * g + 4 * h;
                    const int4 l4 = *reinterpret_cast<const int4*>(&s_last[b][at]), d4 = *reinterpret_cast<const int4*>(&s_doc[b][at]);
                    const int last[4] = {l4.x, l4.y, l4.z, l4.w}, row_doc[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool seen = (key_code <= last[e]) & ((row_doc[e] == doc) | is_common);
                        s[4 * g + e] = seen ? s[4 * g + e] : 0.f;
                        ds[4 * g + e] = seen ? ds[4 * g + e] : 0.f;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            carried.keep(ds, gk);
            add_product<T, DP>(gv, s, gt, Tile::kStride, lane);
            add_product<T, DP>(gk, ds, qt, Tile::kStride, lane);
            if (some) {
                odd_v.template note<T>(s, p.D, lane, [&](int r) { return grad_row(r0 + first + r); });
                odd_k.template note<T>(ds, p.D, lane, [&](int r) { return query_row(r0 + first + r); });
            }
        }
    };
    fetch();
    for (int b = 0; ; b ^= 1) {
        if (t < 0) break;
        stage(b);
        // Rows past the last are hidden: their scores may be anything, as a key may hold an infinity. Keys past the last
        // are not written.
        const int r0 = t * Tile::kRows;
        bool whole = r0 + Tile::kRows <= p.R && (!p.causal || wave_last <= r0 / p.G + w.off || wave_last < w.common);
        if (p.q_doc)
            whole = whole && rr.whole && ((one_doc && rr.lo == doc0 && rr.hi == doc0) || (no_pad && wave_last < w.common));
        __syncthreads();  // buffer b is written, and every wave has read the other one, which is next
        fetch();
        int some = 0;
        if (masks) {
#pragma unroll
            for (int i = 0; i < NW; ++i) some |= s_odd[b][i];
        }
#pragma unroll 1
        for (int sub = 0; sub < Tile::kRows; sub += 32 * Tile::kBlocks) body(b, r0, sub, some, !whole);
    }
    if (key >= p.Lk) return;
    const float v_unit = 1.f / (1 << kProbShift<T>);
    float* part = p.part + (((int64_t)w.slab * p.Lk + key) * p.splits + w.split) * 2 * DP;
    const int64_t at = (((int64_t)w.n * p.Lk + key) * p.Mkv + w.kv) * p.D;
#pragma unroll
    for (int u = 0; u < DP / 32; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = u * 32 + 8 * g + 4 * h;
            float x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = carried.taken_out(gk[u][4 * g + e]) * p.scale;
                y[e] = gv[u][4 * g + e] * v_unit;
            }
            odd_k.apply(x, d);
            odd_v.apply(y, d);
            if (p.splits > 1) {
                *reinterpret_cast<float4*>(part + d) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4*>(part + DP + d) = make_float4(y[0], y[1], y[2], y[3]);
            } else {
                store_four(static_cast<T*>(p.grad_k) + at, d, p.D, x);
                store_four(static_cast<T*>(p.grad_v) + at, d, p.D, y);
            }
        }
}

// Adds the splits of a row of grad_q (KV false), or of a key of grad_k and grad_v: DP / 4 lanes per row and result.
template <typename T, int DP, bool KV>
__global__ __launch_bounds__(256) void attn_sum_kernel(AttnParams p) {
    constexpr int kLanes = (KV ? 2 : 1) * DP / 4;
    const int64_t per_slab = KV ? p.Lk : p.R;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
    if (at >= (int64_t)p.N * p.Mkv * per_slab) return;
    const int64_t slab = at / per_slab, n = slab / p.Mkv;
    const int own = (int)(at - slab * per_slab), kv = (int)(slab - n * p.Mkv);
    const int* filled = p.filled + (slab * p.blocks + own / p.own_rows) * p.splits;
    const int e0 = (threadIdx.x % kLanes) * 4;
    const float* part = p.part + at * p.splits * (kLanes * 4) + e0;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < p.splits; s0 += 4) {
        int full[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) full[k] = s0 + k < p.splits ? filled[s0 + k] : 0;
        float4 y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            y[k] = full[k] ? *reinterpret_cast<const float4*>(part + (int64_t)(s0 + k) * (kLanes * 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[0] += y[k].x;
            x[1] += y[k].y;
            x[2] += y[k].z;
            x[3] += y[k].w;
        }
    }
    const bool values = KV && e0 >= DP;
    T* out;
    if constexpr (KV) {
        out = static_cast<T*>(values ? p.grad_v : p.grad_k) + ((n * p.Lk + own) * p.Mkv + kv) * p.D;
    } else {
        const int i = own / p.G;
        out = static_cast<T*>(p.grad_q) + ((n * p.Lq + i) * p.M + kv * p.G + own - i * p.G) * p.D;
    }
    store_four(out, e0 % DP, p.D, x);
}

enum Launch { kRowDelta, kRowGrad, kKeyGrad };

template <typename T, int DP, Launch WHICH, int EXTRAS>
void launch_owners(const AttnParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)xcd_grid((int64_t)p.N * p.Mkv * p.blocks * p.splits));
    if constexpr (WHICH == kKeyGrad) hipLaunchKernelGGL((attn_grad_kv_kernel<T, DP, 4, EXTRAS>), grid, dim3(256), 0, stream, p);
    else if constexpr (WHICH == kRowGrad) hipLaunchKernelGGL((attn_grad_q_kernel<T, DP, 4, EXTRAS>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((attn_delta_kernel<T, DP, 4, EXTRAS>), grid, dim3(256), 0, stream, p);
}

template <typename T, Launch WHICH>
hipError_t launch_typed(const AttnParams& p, hipStream_t stream) {
    return by_channels(p.D, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        constexpr bool KV = WHICH == kKeyGrad;
        const Extras extras = extras_of<T>(p);
        if (extras == kFarCap) {
            if constexpr (sizeof(T) == 2) launch_owners<T, DP, WHICH, kFarCap>(p, stream);
        } else if (extras == kBias) launch_owners<T, DP, WHICH, kBias>(p, stream);
        else if (extras == kCap) launch_owners<T, DP, WHICH, kCap>(p, stream);
        else launch_owners<T, DP, WHICH, kPlain>(p, stream);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.splits == 1) return e;
        const int64_t lanes = (int64_t)p.N * p.Mkv * (KV ? (int64_t)p.Lk * 2 : p.R) * (DP / 4);
        hipLaunchKernelGGL((attn_sum_kernel<T, DP, KV>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, stream, p);
        return hipGetLastError();
    });
}

template <Launch WHICH>
hipError_t launch_grad(const AttnParams& p, int dtype, hipStream_t stream) {
    if (dtype == MSDA_F32) return launch_typed<float, WHICH>(p, stream);
    if (dtype == MSDA_F16) return launch_typed<_Float16, WHICH>(p, stream);
    return launch_typed<bf16_t, WHICH>(p, stream);
}

}  // namespace

hipError_t launch_attn_grad_q(const AttnParams& p, int dtype, hipStream_t stream) {
    return launch_grad<kRowGrad>(p, dtype, stream);
}

hipError_t launch_attn_delta(const AttnParams& p, int dtype, hipStream_t stream) {
    return dtype == MSDA_F16 ? launch_typed<_Float16, kRowDelta>(p, stream) : launch_typed<bf16_t, kRowDelta>(p, stream);
}

hipError_t launch_attn_grad_kv(const AttnParams& p, int dtype, hipStream_t stream) {
    return launch_grad<kKeyGrad>(p, dtype, stream);
}

}  // namespace msda
