// Dense attention, forward.
//   z_ij = cap(scale q_i . k_j) - slope |q_pos_i - k_pos_j|,  lse_i = log sum_j exp z_ij,  out_i = sum_j exp(z_ij - lse_i) v_j
// One pass over the keys with a running maximum and sum (kept in units of log 2 and in fp32): a workgroup
// owns 32 rows per wave, stages one tile of keys and values after the other in LDS (the next tile's loads
// run while a tile is worked on), and skips the tiles of which its rows see nothing. Probabilities
// are rounded to the operands' type for the product with the values, unnormalized (at most 1, times kProbShift's power), while
// their sum is taken before the rounding: the result's error is then the rounding's, averaged over the keys.
// With few rows the keys are split over workgroups, whose partial results a second kernel joins.
// Measured, with the products of the pairs that are seen: bf16, 2 x 4947 rows x 8 heads x 32, padded: 127 us, 276 TFLOP/s,
// bound by the vector work between the products (maximum, exponent, sum and conversion of each pair, which 32
// channels do not outweigh); 2 x 4096 packed causal rows x 16 heads x 128 on 4 key heads, capped: 129 us, 224 TFLOP/s,
// a third of the pairs of its tiles masked; fp32, 3 x 1023 rows over 2999 x 5 x 48: 120 us, 54 TFLOP/s. One row a head,
// 8 x 32 on 8 key heads over 16411 keys x 128: 126 us and 7 to join, 4.3 TB/s (a large copy reaches 5.5).
#include "msda_attn.hpp"

namespace msda {
namespace {

// Waves per SIMD that the registers of a kernel that owns rows have to leave room for. (A lone wave of 128 channels keeps 25
// registers in memory for it, but with one wave per SIMD and none there a token over 16411 keys takes 155 us, not 130.)
constexpr int row_waves(int DP, int NW, size_t element) { return NW == 1 ? (element == 4 && DP > 32 ? 1 : 2) : DP == 32 ? 4 : DP == 64 ? 3 : 2; }

// lse of a row's maximum and sum, both as the kernels hold them.
template <typename T>
__device__ __forceinline__ float lse_of(float m, float l) {
    return l == 0.f ? -kInf : (m + (__builtin_amdgcn_logf(l) - kProbShift<T>)) * kLn2;
}

template <typename T, int DP, int NW, int EXTRAS>
__global__ __launch_bounds__(64 * NW, row_waves(DP, NW, sizeof(T))) void attn_fwd_kernel(AttnParams p) {
    using O = Op<T>;
    using Keys = KeyTiles<T, DP, NW, EXTRAS >= kBias, kValues>;
    using Tile = typename Keys::Tile;
    __shared__ __attribute__((aligned(16))) typename Keys::Shared sh;
    __shared__ uint32_t odd_words[32 * NW * Odd<DP>::kWords];
    Work w(p, true);
    if (!w.any) return;
    const int lane = threadIdx.x & 63, wave = wave_index(), h = lane >> 5;
    Keys keys(sh, p, w, lane);
    if (!w.note_split(p, keys.any())) return;
    const Row32 own = Row32::of<NW>(p, w, wave, lane, EXTRAS >= kBias);
    typename O::Frag q[DP / O::K];
    const T* qr = static_cast<const T*>(p.q) + w.n * p.qs[0] + own.i * p.qs[1] + own.head * p.qs[2];
#pragma unroll
    for (int c = 0; c < DP / O::K; ++c)
        q[c] = __builtin_bit_cast(typename O::Frag, load_chunk(qr, c * O::K + h * (O::K / 2), p.D));

    acc_t o[DP / 32];
#pragma unroll
    for (int u = 0; u < DP / 32; ++u) o[u] = acc_t{};
    float m = -kInf, l = 0.f;
    Odd<DP> odd;
    odd.start(odd_words, wave * 32 + (lane & 31), lane, p.q_doc || p.causal);
    auto body = [&](int b, int j0, int sub, bool partial) {  // the tile's keys from sub on
        acc_t s[Tile::kBlocks];
        float unit = p.scale * kLog2e;  // of the raw scores, left to the exponent where nothing comes between
#pragma unroll
        for (int kb = 0; kb < Tile::kBlocks; ++kb) {
            s[kb] = row_product<T, DP>(sh.k[b] + (sub + kb * 32) * Tile::kStride, Tile::kStride, q, lane, p.D, acc_t{});
            if constexpr (EXTRAS >= kCap) unit = cap_scores<T, EXTRAS>(p, s[kb], nullptr);
            if constexpr (EXTRAS >= kBias) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float2 kp = sh.pos[b][sub + kb * 32 + block_row(r, h)];
                    const float dx = own.pos.x - kp.x, dy = own.pos.y - kp.y;
                    s[kb][r] = s[kb][r] * unit - own.slope * __builtin_amdgcn_sqrtf(dx * dx + dy * dy);
                }
                unit = 1.f;
            }
            if (partial) {
                acc_t x[1] = {s[kb]};
                hide(x, -kInf, sub + kb * 32, h, own.last - j0, own.doc, sh.doc[b]);
                s[kb] = x[0];
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < Tile::kBlocks; ++kb)
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
        const float base = (m == -kInf ? 0.f : m) - kProbShift<T>;  // a row that has seen nothing yet: any
#pragma unroll
        for (int kb = 0; kb < Tile::kBlocks; ++kb) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = exp2_of(__builtin_fmaf(s[kb][r], unit, -base));
                l += s[kb][r];
            }
            add_product<T, DP>(o, s[kb], sh.v[b] + (sub + kb * 32) * Tile::kStride, Tile::kStride, lane);
            keys.note_odd(odd, s[kb], b, j0 + sub + kb * 32);
        }
    };
    keys.fetch();
    for (int b = 0; keys.t >= 0; b ^= Keys::kBuffers - 1) {
        keys.stage(b);
        const bool whole = keys.whole(own);
        const int j0 = keys.t * Tile::kRows;
        __syncthreads();  // buffer b is written, and every wave has read the other one, which is next
        keys.fetch();

#pragma unroll 1
        for (int sub = 0; sub < Tile::kRows; sub += 32 * Tile::kBlocks) body(b, j0, sub, !whole);
        if constexpr (Keys::kBuffers == 1) wave_lds_sync();  // the wave has read the buffer, which is next again
    }
    l = halves_sum(l);
    if (own.row >= p.R) return;
    if (p.splits > 1) {
        const int64_t at = ((int64_t)w.slab * p.R + own.row) * p.splits + w.split;
        float* part = p.part + at * DP;
#pragma unroll
        for (int u = 0; u < DP / 32; ++u)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int d = u * 32 + 8 * g + 4 * h;
                float x[4] = {o[u][4 * g], o[u][4 * g + 1], o[u][4 * g + 2], o[u][4 * g + 3]};
                odd.apply(x, d);
                *reinterpret_cast<float4*>(part + d) = make_float4(x[0], x[1], x[2], x[3]);
            }
        if (h == 0) {
            float2* stats = reinterpret_cast<float2*>(p.part + (int64_t)p.N * p.Mkv * p.R * p.splits * DP);
            stats[at] = make_float2(m, l);
        }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = static_cast<T*>(p.out) + own.at * p.D;
#pragma unroll
    for (int u = 0; u < DP / 32; ++u)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = o[u][4 * g + e] * inv;
            odd.apply(x, u * 32 + 8 * g + 4 * h);
            store_four(out, u * 32 + 8 * g + 4 * h, p.D, x);
        }
    if (p.lse && h == 0) p.lse[own.stat] = lse_of<T>(m, l);
}

// Joins the splits of a row: DP / 4 lanes of four channels each, times `groups` (a power of two, a wave holds whole
// rows) to which the splits are dealt. Loads do not wait for one another: what a split that is not filled holds
// is dropped.
template <typename T, int DP>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnParams p, int groups) {
    constexpr int kLanes = DP / 4;
    const int64_t rows = (int64_t)p.N * p.Mkv * p.R;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / (kLanes * groups);
    if (at >= rows) return;
    const int64_t slab = at / p.R;
    const int lane = threadIdx.x % (kLanes * groups), row = (int)(at - slab * p.R), i = row / p.G;
    const int* filled = p.filled + (slab * p.blocks + row / p.own_rows) * p.splits;
    const int d = lane % kLanes * 4;
    const float2* stats = reinterpret_cast<const float2*>(p.part + rows * p.splits * DP) + at * p.splits;
    const float* part = p.part + at * p.splits * DP + d;
    float m = -kInf, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
    auto take = [&](float m2, float l2, const float (&y)[4]) {
        const float top = fmaxf(m, m2), base = top == -kInf ? 0.f : top;
        const float u = exp2_of(m - base), w = exp2_of(m2 - base);
        m = top;
        l = l * u + l2 * w;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = x[e] * u + y[e] * w;
    };
#pragma unroll 4
    for (int s = lane / kLanes; s < p.splits; s += groups) {
        const bool full = filled[s];
        const float2 ml = stats[s];
        const float4 y4 = *reinterpret_cast<const float4*>(part + (int64_t)s * DP);
        const float y[4] = {full ? y4.x : 0.f, full ? y4.y : 0.f, full ? y4.z : 0.f, full ? y4.w : 0.f};
        take(full ? ml.x : -kInf, full ? ml.y : 0.f, y);
    }
    for (int k = kLanes; k < kLanes * groups; k *= 2) {
        float y[4];
        const float m2 = __shfl_xor(m, k, 64), l2 = __shfl_xor(l, k, 64);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = __shfl_xor(x[e], k, 64);
        take(m2, l2, y);
    }
    if (lane >= kLanes) return;
    const int64_t n = slab / p.Mkv;
    const int head = (int)(slab - n * p.Mkv) * p.G + row - i * p.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= inv;
    store_four(static_cast<T*>(p.out) + ((n * p.Lq + i) * p.M + head) * p.D, d, p.D, x);
    if (p.lse && d == 0) p.lse[(n * p.M + head) * p.Lq + i] = lse_of<T>(m, l);
}

// Documents of the tiles and blocks of each table of a call, one wave for each.
__global__ __launch_bounds__(256) void attn_ranges_kernel(AttnRanges c) {
    const int lane = threadIdx.x & 63;
    int64_t item = (int64_t)blockIdx.x * 4 + wave_index();
    if (item >= (int64_t)c.N * c.per_item) return;
    const int64_t n = item / c.per_item;
    int t = (int)(item - n * c.per_item), k = 0;
    while (t >= c.table[k].count) t -= c.table[k++].count;
    const AttnRanges::Table& x = c.table[k];
    // owners t * size .. of which `group` consecutive ones are of one token
    const int first = (int)((int64_t)t * x.size / x.group), last = (int)(min((int64_t)(t + 1) * x.size, (int64_t)x.tokens * x.group) - 1) / x.group;
    const int* doc = x.doc + n * x.tokens;
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
    if (lane == 0) x.into[n * x.count + t] = make_int4(lo, hi, whole, 0);
}

// Rows that are not whole 16-byte chunks on 16-byte boundaries, copied so that they are: [N, L, H, width] from
// strided [N, L, H, D], the channels from D on zero. A thread writes one chunk.
template <typename T>
__global__ __launch_bounds__(256) void attn_pack_kernel(AttnPack c) {
    constexpr int kPer = 16 / sizeof(T);
    const int chunks = c.width / kPer;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (item >= (int64_t)c.N * c.L * c.H * chunks) return;
    const int64_t row = item / chunks;
    const int d = (int)(item - row * chunks) * kPer;
    const int64_t nl = row / c.H, n = nl / c.L;
    const T* from = static_cast<const T*>(c.from) + n * c.stride[0] + (nl - n * c.L) * c.stride[1] + (row - nl * c.H) * c.stride[2];
    Piece<T, kPer> x;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x.v[i] = d + i < c.D ? from[d + i] : (T)0.f;
    *reinterpret_cast<Piece<T, kPer>*>(static_cast<T*>(c.to) + row * c.width + d) = x;
}

template <typename T, int DP, int EXTRAS>
void launch_rows(const AttnParams& p, int waves, hipStream_t stream) {
    const dim3 grid((unsigned)xcd_grid((int64_t)p.N * p.Mkv * p.blocks * p.splits));
    if (waves == 4) hipLaunchKernelGGL((attn_fwd_kernel<T, DP, 4, EXTRAS>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((attn_fwd_kernel<T, DP, 1, EXTRAS>), grid, dim3(64), 0, stream, p);
}

template <typename T>
hipError_t launch_typed(const AttnParams& p, int waves, hipStream_t stream) {
    return by_channels(p.D, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        const Extras extras = extras_of<T>(p);
        if (extras == kFarCap) {
            if constexpr (sizeof(T) == 2) launch_rows<T, DP, kFarCap>(p, waves, stream);
        } else if (extras == kBias) launch_rows<T, DP, kBias>(p, waves, stream);
        else if (extras == kCap) launch_rows<T, DP, kCap>(p, waves, stream);
        else launch_rows<T, DP, kPlain>(p, waves, stream);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.splits == 1) return e;
        const int64_t rows = (int64_t)p.N * p.Mkv * p.R;
        int groups = 1;  // at most four splits to a lane, where a wave has the lanes
        while (groups < 256 / DP && groups * 4 < p.splits) groups *= 2;
        hipLaunchKernelGGL((attn_join_kernel<T, DP>), dim3((unsigned)((rows * (DP / 4 * groups) + 255) / 256)), dim3(256),
                           0, stream, p, groups);
        return hipGetLastError();
    });
}

}  // namespace

// The kernels' tile: TileOf::kRows.
static int attn_tile(int dtype, int waves, int DP, bool wide) {
    return dtype == MSDA_F32 || waves == 1 ? 32 : wide && DP == 32 ? kWideTile : Op<_Float16>::kTile;
}
int attn_channels(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

AttnPlan attn_plan(const AttnParams& p, int dtype, AttnKernel kernel) {
    const int DP = attn_channels(p.D);
    const int64_t slabs = (int64_t)p.N * p.Mkv, own = kernel == kGradKV ? p.Lk : p.R, across = kernel == kGradKV ? p.R : p.Lk;
    AttnPlan a;
    a.waves = kernel == kForward && own <= 32 ? 1 : 4;
    a.tile = attn_tile(dtype, a.waves, DP, kernel != kForward);
    a.blocks = (int)((own + 32 * a.waves - 1) / (32 * a.waves));
    const int64_t tiles = (across + a.tile - 1) / a.tile, waves = slabs * a.blocks * a.waves;
    // Waves that the card holds at once, by the kernels' registers (a lone wave's by its LDS), where one split's are few;
    // twice as many keep it full while the last workgroups end. With one split each, DETR-encoder self-attention over 4947
    // pixels (2496 waves) took 203, 202 and 248 us in the three kernels, with three 123, 143 and 206.
    const int per_simd = a.waves == 1 ? 2 : DP == 32 ? (kernel == kForward ? 4 : 3) : DP == 64 ? (kernel == kForward ? 3 : 2)
                                                                                   : kernel == kGradKV ? 1 : 2;
    const int64_t room = 1024 * per_simd;
    int64_t splits = waves > 0 ? ((4 * waves < room ? 1 : 2) * room + waves - 1) / waves : 1;
    const bool full = waves >= room;
    // Masks leave some workgroups many tiles and others few. Where a SIMD holds one wave, nothing else runs beside the
    // longest ones, and shorter runs even them out if the runs are long and the workgroups few. The backward, bf16, 4096 tokens
    // of 16 heads of 128 channels on 4 key heads (256 tiles), without and with them: packed causal N = 2 640 us and 517, N = 1 457
    // and 330; packed 942 and 739; causal 1176 and 1040, 736 and 736; padded, where there is nothing to even out, 1500
    // and 1682. On 8 heads of their own (64 tiles) the partial results cost more: packed causal 319 and 452, packed 530 and 753,
    // causal 528 and 664; and with twice the workgroups (9000 packed tokens) 1162 and 1203. The kernels of
    // more waves lose as well (the encoder's step above 433 us -> 536).
    if (per_simd == 1 && tiles >= 128 && waves < 2 * room) splits *= p.q_doc ? 8 : p.causal ? 4 : 1;
    // runs shorter than this do not pay for the workgroup's start and its partial results
    const int64_t least = full ? 16 : 4;
    // and the partial results of all splits have to fit into half a GB
    const int64_t split_bytes = slabs * own * DP * 4 * (kernel == kGradKV ? 2 : 1), most = ((int64_t)512 << 20) / (split_bytes + 1);
    int64_t chunk = (tiles + splits - 1) / splits;
    if (chunk < least) chunk = least;
    if ((tiles + chunk - 1) / chunk > most) chunk = most > 1 ? (tiles + most - 1) / most : tiles;
    a.chunk = (int)(chunk < 1 ? 1 : chunk);
    a.splits = (int)((tiles + a.chunk - 1) / a.chunk);
    if (a.splits < 1) a.splits = 1;
    a.tiles = (int)tiles;
    return a;
}

hipError_t launch_attn_pack(const AttnPack& c, int dtype, hipStream_t stream) {
    const int64_t items = (int64_t)c.N * c.L * c.H * (c.width * dtype_size(dtype) / 16);
    const dim3 grid((unsigned)((items + 255) / 256));
    if (dtype == MSDA_F32) hipLaunchKernelGGL(attn_pack_kernel<float>, grid, dim3(256), 0, stream, c);
    else hipLaunchKernelGGL(attn_pack_kernel<_Float16>, grid, dim3(256), 0, stream, c);  // the bits are copied
    return hipGetLastError();
}

hipError_t launch_attn_ranges(const AttnRanges& c, hipStream_t stream) {
    const int64_t items = (int64_t)c.N * c.per_item;
    hipLaunchKernelGGL(attn_ranges_kernel, dim3((unsigned)((items + 3) / 4)), dim3(256), 0, stream, c);
    return hipGetLastError();
}

hipError_t launch_attn_forward(const AttnParams& p, int dtype, int waves, hipStream_t stream) {
    if (dtype == MSDA_F32) return launch_typed<float>(p, waves, stream);
    if (dtype == MSDA_F16) return launch_typed<_Float16>(p, waves, stream);
    return launch_typed<bf16_t>(p, waves, stream);
}

}  // namespace msda
