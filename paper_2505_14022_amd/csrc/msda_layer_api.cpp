// C ABI of the layer operators (layer norm, rotary positions, dense attention): argument checks and
// launch (host code only).
#include <math.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "msda.h"
#include "msda_layer.h"

using msda::dtype_size;
using msda::fail;
using msda::is_aligned;
using msda::ok;

namespace {

constexpr int64_t kMaxInt = 0x7fffffff;
constexpr int64_t kMaxWorkItems = 0xffffffff;             // of a grid: the runtime takes fewer than 2^32
constexpr int64_t kMaxWorkgroups = kMaxWorkItems / 256;   // of 256

msda_status_t check_dtype(int dtype) {
    if (dtype != MSDA_F32 && dtype != MSDA_F16 && dtype != MSDA_BF16)
        return fail(MSDA_ERROR_INVALID_VALUE, "unknown dtype %d (expected MSDA_F32=0, MSDA_F16=1 or MSDA_BF16=2)", dtype);
    return MSDA_SUCCESS;
}

msda_status_t check_norm(int64_t rows, int64_t C, int dtype) {
    msda_status_t st = check_dtype(dtype);
    if (st != MSDA_SUCCESS) return st;
    if (rows < 0 || C < 1)
        return fail(MSDA_ERROR_INVALID_VALUE, "rows=%lld must be >= 0 and C=%lld >= 1", (long long)rows, (long long)C);
    if (C > MSDA_LAYERNORM_MAX_C)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "C=%lld channels exceeds MSDA_LAYERNORM_MAX_C=%d", (long long)C,
                    MSDA_LAYERNORM_MAX_C);
    if (rows > (INT64_MAX >> 4) / C)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "rows=%lld of C=%lld channels is too large", (long long)rows, (long long)C);
    return MSDA_SUCCESS;
}

// Whether every given row tensor is read in 16-byte pieces.
template <typename... P>
bool norm_pieces(int64_t C, int dtype, P... ptr) {
    return (C * dtype_size(dtype)) % 16 == 0 && (... && is_aligned(ptr, 16));
}

size_t norm_workspace(int64_t rows, int64_t C, int dtype) {
    return rows == 0 ? 0 : (size_t)2 * msda::norm_backward_blocks(rows, C, dtype) * C * sizeof(float);
}

}  // namespace

extern "C" {

msda_status_t msda_layernorm_forward(const void* x, const void* residual, const float* weight, const float* bias,
                                     void* out, void* sum, float* mean, float* rstd, int64_t rows, int64_t C,
                                     float eps, int dtype, void* stream) {
    msda_status_t st = check_norm(rows, C, dtype);
    if (st != MSDA_SUCCESS) return st;
    if (!(eps >= 0.f) || isinf(eps))
        return fail(MSDA_ERROR_INVALID_VALUE, "eps=%g must be finite and >= 0", (double)eps);
    if (rows == 0) return ok();
    if (!x || !out) return fail(MSDA_ERROR_INVALID_VALUE, "x and out must be non-null");
    const int es = dtype_size(dtype);
    if (!is_aligned(x, es) || !is_aligned(residual, es) || !is_aligned(out, es) || !is_aligned(sum, es) ||
        !is_aligned(weight, 4) || !is_aligned(bias, 4) || !is_aligned(mean, 4) || !is_aligned(rstd, 4))
        return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: tensors need the alignment of their elements");
    msda::NormParams p = {};
    p.x = x;
    p.residual = residual;
    p.weight = weight;
    p.bias = bias;
    p.out = out;
    p.sum = sum;
    p.mean = mean;
    p.rstd = rstd;
    p.rows = rows;
    p.C = (int)C;
    p.eps = eps;
    p.vec = norm_pieces(C, dtype, x, residual, (const void*)out, (const void*)sum);
    p.columns = is_aligned(weight, 16) && is_aligned(bias, 16);
    hipError_t e = msda::launch_layernorm_forward(p, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "layer norm launch: %s", hipGetErrorString(e));
    return ok();
}

msda_status_t msda_layernorm_backward_workspace_size(int64_t rows, int64_t C, int dtype, size_t* bytes) {
    if (!bytes) return fail(MSDA_ERROR_INVALID_VALUE, "bytes must be non-null");
    *bytes = 0;
    msda_status_t st = check_norm(rows, C, dtype);
    if (st != MSDA_SUCCESS) return st;
    *bytes = norm_workspace(rows, C, dtype);
    return ok();
}

msda_status_t msda_layernorm_backward(const void* x, const void* residual, const float* weight, const void* grad_out,
                                      const void* grad_sum, const float* mean, const float* rstd, void* grad_x,
                                      float* grad_weight, float* grad_bias, void* workspace, size_t workspace_bytes,
                                      int64_t rows, int64_t C, int dtype, void* stream) {
    msda_status_t st = check_norm(rows, C, dtype);
    if (st != MSDA_SUCCESS) return st;
    const int es = dtype_size(dtype);
    const bool sums = grad_weight || grad_bias;
    if (!is_aligned(grad_weight, 4) || !is_aligned(grad_bias, 4))
        return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: tensors need the alignment of their elements");
    if (rows > 0) {
        if (!x || !grad_out || !mean || !rstd || !grad_x)
            return fail(MSDA_ERROR_INVALID_VALUE, "x, grad_out, mean, rstd and grad_x must be non-null");
        if (!is_aligned(x, es) || !is_aligned(residual, es) || !is_aligned(grad_out, es) || !is_aligned(grad_sum, es) ||
            !is_aligned(grad_x, es) || !is_aligned(weight, 4) || !is_aligned(mean, 4) || !is_aligned(rstd, 4))
            return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: tensors need the alignment of their elements");
        const size_t need = norm_workspace(rows, C, dtype);
        if (sums && (!workspace || workspace_bytes < need))
            return fail(MSDA_ERROR_INVALID_VALUE, "workspace of %zu bytes is smaller than the %zu needed",
                        workspace ? workspace_bytes : (size_t)0, need);
        if (sums && !is_aligned(workspace, 16))
            return fail(MSDA_ERROR_INVALID_VALUE, "workspace must be 16-byte aligned");
    }
    msda::NormParams p = {};
    p.x = x;
    p.residual = residual;
    p.weight = weight;
    p.grad_out = grad_out;
    p.grad_sum = grad_sum;
    p.mean = const_cast<float*>(mean);
    p.rstd = const_cast<float*>(rstd);
    p.grad_x = grad_x;
    p.partial = sums ? static_cast<float*>(workspace) : nullptr;
    p.grad_weight = grad_weight;
    p.grad_bias = grad_bias;
    p.rows = rows;
    p.C = (int)C;
    p.blocks = msda::norm_backward_blocks(rows, C, dtype);
    p.vec = norm_pieces(C, dtype, x, residual, grad_out, grad_sum, (const void*)grad_x);
    p.columns = is_aligned(weight, 16);
    hipError_t e = msda::launch_layernorm_backward(p, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "layer norm backward launch: %s", hipGetErrorString(e));
    return ok();
}

}  // extern "C"

// ---------------------------------------------------------------- rotary positions

namespace {

msda_status_t rotary(const char* in_name, const void* x, const int64_t* x_stride, const float* pos, const float* freqs,
                     const char* out_name, void* out, const int64_t* out_stride, int64_t N, int64_t T, int64_t M,
                     int64_t D, int64_t A, int64_t R, int64_t pos_items, int interleaved, int dtype, float sign,
                     void* stream) {
    msda_status_t st = check_dtype(dtype);
    if (st != MSDA_SUCCESS) return st;
    if (N < 0 || T < 0 || M < 1 || D < 1)
        return fail(MSDA_ERROR_INVALID_VALUE, "N=%lld and T=%lld must be >= 0, M=%lld and D=%lld >= 1", (long long)N,
                    (long long)T, (long long)M, (long long)D);
    if (A < 1 || A > 4) return fail(MSDA_ERROR_INVALID_VALUE, "A=%lld axes: 1 to 4 are taken", (long long)A);
    if (R < 0 || R > D / 2)
        return fail(MSDA_ERROR_INVALID_VALUE, "R=%lld pairs do not fit into D=%lld channels", (long long)R, (long long)D);
    if (pos_items != 1 && pos_items != N)
        return fail(MSDA_ERROR_INVALID_VALUE, "pos_items=%lld must be 1 or N=%lld", (long long)pos_items, (long long)N);
    if (D > MSDA_ROTARY_MAX_D)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "D=%lld channels per head exceeds MSDA_ROTARY_MAX_D=%d", (long long)D,
                    MSDA_ROTARY_MAX_D);
    if (M > 65536 / D)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "M*D of M=%lld, D=%lld exceeds 65536", (long long)M, (long long)D);
    if (N > kMaxInt || T > kMaxInt) return fail(MSDA_ERROR_NOT_SUPPORTED, "N or T exceeds 2^31-1");
    if (N * T == 0) return ok();
    if (!x || !out || (R > 0 && (!pos || !freqs)))
        return fail(MSDA_ERROR_INVALID_VALUE, "%s, pos, freqs and %s must be non-null", in_name, out_name);
    const int es = dtype_size(dtype);
    if (!is_aligned(x, es) || !is_aligned(out, es) || !is_aligned(pos, 4) || !is_aligned(freqs, 4))
        return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: tensors need the alignment of their elements");
    msda::RotaryParams p = {};
    const int64_t whole[3] = {T * M * D, M * D, D}, extent[3] = {N, T, M};
    bool pieces = is_aligned(x, 16) && is_aligned(out, 16);
    for (int i = 0; i < 3; ++i) {
        p.xs[i] = x_stride ? x_stride[i] : whole[i];
        p.os[i] = out_stride ? out_stride[i] : whole[i];
        if (extent[i] > 1 && p.os[i] == 0)
            return fail(MSDA_ERROR_INVALID_VALUE, "%s has a stride of 0 over %lld entries", out_name, (long long)extent[i]);
        // a stride over a single entry is never used
        if (extent[i] > 1) pieces = pieces && (p.xs[i] * es) % 16 == 0 && (p.os[i] * es) % 16 == 0;
    }
    const int64_t per = 16 / es;
    p.x = x;
    p.out = out;
    p.pos = pos;
    p.freqs = freqs;
    p.T = T;
    p.N = (int)N;
    p.M = (int)M;
    p.D = (int)D;
    p.A = (int)A;
    p.R = (int)R;
    p.pos_item = pos_items == N && N > 1 ? T * A : 0;
    p.interleaved = interleaved != 0;
    p.vec = pieces && R % per == 0 && D % per == 0;
    p.sign = sign;
    if (msda::rotary_workgroups(p, dtype) > kMaxWorkgroups)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "T=%lld tokens of M*D=%lld channels are too many for one launch", (long long)T,
                    (long long)(M * D));
    hipError_t e = msda::launch_rotary(p, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "rotary launch: %s", hipGetErrorString(e));
    return ok();
}

}  // namespace

extern "C" {

msda_status_t msda_rotary_forward(const void* x, const int64_t* x_stride, const float* pos, const float* freqs,
                                  void* out, const int64_t* out_stride, int64_t N, int64_t T, int64_t M, int64_t D,
                                  int64_t A, int64_t R, int64_t pos_items, int interleaved, int dtype, void* stream) {
    return rotary("x", x, x_stride, pos, freqs, "out", out, out_stride, N, T, M, D, A, R, pos_items, interleaved, dtype,
                  1.f, stream);
}

msda_status_t msda_rotary_backward(const void* grad_out, const int64_t* grad_out_stride, const float* pos,
                                   const float* freqs, void* grad_x, const int64_t* grad_x_stride, int64_t N, int64_t T,
                                   int64_t M, int64_t D, int64_t A, int64_t R, int64_t pos_items, int interleaved,
                                   int dtype, void* stream) {
    return rotary("grad_out", grad_out, grad_out_stride, pos, freqs, "grad_x", grad_x, grad_x_stride, N, T, M, D, A, R,
                  pos_items, interleaved, dtype, -1.f, stream);
}

}  // extern "C"

// ---------------------------------------------------------------- dense attention

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t round_up(size_t b) { return (b + 255) / 256 * 256; }

msda_status_t check_attention(const msda_attention_t* a) {
    if (!a) return fail(MSDA_ERROR_INVALID_VALUE, "the attention's description must be non-null");
    msda_status_t st = check_dtype(a->dtype);
    if (st != MSDA_SUCCESS) return st;
    if (a->N < 0 || a->Lq < 0 || a->Lk < 0)
        return fail(MSDA_ERROR_INVALID_VALUE, "N=%lld, Lq=%lld and Lk=%lld must be >= 0", (long long)a->N,
                    (long long)a->Lq, (long long)a->Lk);
    if (a->M < 1 || a->Mkv < 1 || a->D < 1 || a->M % a->Mkv != 0)
        return fail(MSDA_ERROR_INVALID_VALUE, "M=%lld, Mkv=%lld and D=%lld must be >= 1 and M a multiple of Mkv",
                    (long long)a->M, (long long)a->Mkv, (long long)a->D);
    if (a->D > MSDA_ATTENTION_MAX_D)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "D=%lld channels per head exceeds MSDA_ATTENTION_MAX_D=%d",
                    (long long)a->D, MSDA_ATTENTION_MAX_D);
    if (!(a->scale > 0.f) || isinf(a->scale))
        return fail(MSDA_ERROR_INVALID_VALUE, "scale=%g must be finite and > 0", (double)a->scale);
    if (!(a->softcap >= 0.f) || isinf(a->softcap))
        return fail(MSDA_ERROR_INVALID_VALUE, "softcap=%g must be finite and >= 0", (double)a->softcap);
    // the kernels' factors, in units of log 2
    const float log2e = 1.4426950408889634f;
    if (isinf(a->scale * log2e))
        return fail(MSDA_ERROR_INVALID_VALUE, "scale=%g times log2(e) must be finite", (double)a->scale);
    if (isinf(a->softcap * log2e) || (a->softcap > 0.f && isinf(2.f * log2e * (a->scale / a->softcap))))
        return fail(MSDA_ERROR_INVALID_VALUE, "softcap=%g and scale=%g: their products with 2 log2(e), and that of scale / softcap, "
                    "must be finite", (double)a->softcap, (double)a->scale);
    if (a->causal && a->Lk < a->Lq)
        return fail(MSDA_ERROR_INVALID_VALUE, "causal needs Lk=%lld >= Lq=%lld", (long long)a->Lk, (long long)a->Lq);
    if (a->M > 32768)  // the rows of a tile lie within 2^31 bytes
        return fail(MSDA_ERROR_NOT_SUPPORTED, "M=%lld heads exceeds 32768", (long long)a->M);
    if (a->N > kMaxInt || a->Lk > kMaxInt - 1024 || a->Lq > (kMaxInt - 1024) / (a->M / a->Mkv))
        return fail(MSDA_ERROR_NOT_SUPPORTED, "N, Lk or Lq * M / Mkv exceeds 2^31");
    // slabs (batch item, key head) and their rows and keys: what is counted from them stays within 64 bits, and
    // check_launches looks at the grids
    const double slabs = (double)a->N * (double)a->Mkv, rows = (double)a->Lq * (double)(a->M / a->Mkv);
    if (slabs > 1073741824.0 || slabs * rows > 8589934592.0 || slabs * (double)a->Lk > 8589934592.0)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "N * Mkv heads of these lengths are too many for one launch");
    for (int i = 0; i < 3; ++i)
        if (a->q_stride[i] < 0 || a->k_stride[i] < 0 || a->v_stride[i] < 0)
            return fail(MSDA_ERROR_INVALID_VALUE, "strides must be >= 0");
    // with empty extents any table may be null; the pointers are not looked at then
    if (a->N > 0 && a->Lq > 0 && a->Lk > 0) {
        if ((a->q_doc != nullptr) != (a->k_doc != nullptr))
            return fail(MSDA_ERROR_INVALID_VALUE, "q_doc and k_doc must be given both or neither");
        if (a->slopes && (!a->q_pos || !a->k_pos))
            return fail(MSDA_ERROR_INVALID_VALUE, "slopes need q_pos and k_pos");
        if (!is_aligned(a->slopes, 4) || !is_aligned(a->q_pos, 8) || !is_aligned(a->k_pos, 8) || !is_aligned(a->q_doc, 4) ||
            !is_aligned(a->k_doc, 4) || !is_aligned(a->prefix, 4))
            return fail(MSDA_ERROR_INVALID_VALUE, "misaligned table: positions need 8 bytes, the others 4");
    }
    return MSDA_SUCCESS;
}

// The kernels' view of a call, and how it is cut up. The workspace's pieces in order: documents of the key tiles
// and row tiles, delta (backward), runs per block, packed copies of q, k, v, out and grad_out, partial results of the splits.
struct Attention {
    msda::AttnParams p = {};
    msda::AttnPlan rows, keys;
    size_t at_ranges[4] = {0, 0, 0, 0}, at_delta = 0, at_filled = 0, at_pack[5] = {0, 0, 0, 0, 0}, at_part = 0, bytes = 0;
    bool pack[5] = {false, false, false, false, false};
    int width = 0;  // of a packed row
};

// Whether rows of D channels with these strides are whole 16-byte pieces on 16-byte boundaries of their base, and
// the rows of a tile (at most 129 tokens of `heads` heads) lie within the 31 bits of the kernels' offsets.
bool row_pieces(const int64_t* stride, int64_t N, int64_t L, int64_t H, int64_t heads, int64_t D, int es) {
    const int64_t extent[3] = {N, L, H};
    bool yes = (D * es) % 16 == 0;
    for (int i = 0; i < 3; ++i) yes = yes && (extent[i] <= 1 || (stride[i] * es) % 16 == 0);
    const double reach = (L > 1 ? 129.0 * fabs((double)stride[1]) : 0.0) + (double)(heads - 1) * fabs((double)stride[2]) + D;
    return yes && reach * es < 2147483648.0;
}

Attention attention_of(const msda_attention_t& a, bool backward) {
    Attention x;
    msda::AttnParams& p = x.p;
    const int es = dtype_size(a.dtype);
    const int64_t G = a.M / a.Mkv, DP = msda::attn_channels((int)a.D), slabs = a.N * a.Mkv;
    p.N = (int)a.N;
    p.Lq = (int)a.Lq;
    p.Lk = (int)a.Lk;
    p.M = (int)a.M;
    p.Mkv = (int)a.Mkv;
    p.G = (int)G;
    p.D = (int)a.D;
    p.R = (int)(a.Lq * G);
    p.causal = a.causal != 0;
    p.scale = a.scale;
    p.softcap = a.softcap;
    for (int i = 0; i < 3; ++i) {
        p.qs[i] = a.q_stride[i];
        p.ks[i] = a.k_stride[i];
        p.vs[i] = a.v_stride[i];
    }
    if (a.Lq > 0 && a.Lk > 0) {
        p.slopes = a.slopes;
        p.q_pos = a.q_pos;
        p.k_pos = a.k_pos;
        p.q_doc = a.q_doc;
        p.k_doc = a.k_doc;
        p.prefix = a.prefix;
    }
    if (a.Lq > 0) x.rows = msda::attn_plan(p, a.dtype, backward ? msda::kGradQ : msda::kForward);
    if (backward && a.Lk > 0) x.keys = msda::attn_plan(p, a.dtype, msda::kGradKV);
    // tables of documents: key tiles and row blocks of one side's kernels, row tiles and key blocks of the other's
    const int counts[4] = {x.rows.tiles, x.rows.blocks, x.keys.tiles, x.keys.blocks};
    size_t at = 0;
    for (int i = 0; i < 4; ++i) {
        x.at_ranges[i] = at;
        if (p.q_doc) at += round_up(sizeof(int4) * a.N * counts[i]);
    }
    x.at_delta = at;
    if (backward) at += round_up(sizeof(float) * a.N * a.M * a.Lq);
    x.at_filled = at;
    size_t filled = 0;
    for (const msda::AttnPlan* plan : {&x.rows, &x.keys})
        if (plan->splits > 1 && (size_t)slabs * plan->blocks * plan->splits > filled)
            filled = (size_t)slabs * plan->blocks * plan->splits;
    at += round_up(sizeof(int) * filled);
    x.width = (int)ceil_div(a.D * es, 16) * 16 / es;
    x.pack[0] = a.unaligned || !row_pieces(a.q_stride, a.N, a.Lq, a.M, G, a.D, es);
    x.pack[1] = a.unaligned || !row_pieces(a.k_stride, a.N, a.Lk, a.Mkv, 1, a.D, es);
    x.pack[2] = a.unaligned || !row_pieces(a.v_stride, a.N, a.Lk, a.Mkv, 1, a.D, es);
    x.pack[3] = x.pack[4] = backward && (a.D * es) % 16 != 0;
    for (int i = 0; i < 5; ++i) {
        x.at_pack[i] = at;
        if (x.pack[i]) at += round_up((size_t)es * a.N * (i == 1 || i == 2 ? a.Lk * a.Mkv : a.Lq * a.M) * x.width);
    }
    x.at_part = at;
    size_t part = 0;
    if (x.rows.splits > 1) part = (size_t)slabs * p.R * x.rows.splits * (DP + (backward ? 0 : 2));
    if (x.keys.splits > 1) {
        const size_t b = (size_t)slabs * p.Lk * x.keys.splits * 2 * DP;
        if (b > part) part = b;
    }
    x.bytes = at + part * sizeof(float);
    return x;
}

// Every launch is one grid: a call that needs a larger one than the runtime takes is refused before any of its kernels is
// enqueued.
msda_status_t check_launches(const Attention& x, const msda_attention_t& a, bool backward) {
    const int64_t slabs = a.N * a.Mkv, DP = msda::attn_channels((int)a.D);
    int64_t most = 0;
    auto launch = [&](int64_t items) { most = items > most ? items : most; };
    const msda::AttnPlan* plans[2] = {&x.rows, &x.keys};
    for (int i = 0; i < 2; ++i) {
        const msda::AttnPlan& plan = *plans[i];
        launch(ceil_div(slabs * plan.blocks * plan.splits, 8) * 8 * 64 * plan.waves);
        // four channels of each result a lane, or in the forward's join up to a wave for a row
        if (plan.splits > 1) launch(i ? slabs * a.Lk * 2 * (DP / 4) : slabs * x.p.R * (backward ? DP / 4 : 64));
    }
    if (x.p.q_doc) launch(a.N * (x.rows.tiles + x.rows.blocks + x.keys.tiles + x.keys.blocks) * 64);
    for (int i = 0; i < 5; ++i)
        if (x.pack[i]) launch(a.N * (i == 1 || i == 2 ? a.Lk * a.Mkv : a.Lq * a.M) * (x.width * dtype_size(a.dtype) / 16));
    if (most + 255 > kMaxWorkItems)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "N * Mkv heads of these lengths are too many for one launch (%lld work items)",
                    (long long)most);
    return MSDA_SUCCESS;
}

// Whether 16-bit rows may have so few keys that their delta is formed with care, in a launch of its own.
bool rows_of_few_keys(const msda_attention_t& a) {
    const int64_t few = msda::kFewKeys;
    return a.dtype != MSDA_F32 && a.Lk > 0 && (a.Lk <= few || a.q_doc || (a.causal && a.Lk - a.Lq < few));
}

msda_status_t check_workspace(const Attention& x, const void* workspace, size_t bytes) {
    if (x.bytes > 0 && (!workspace || bytes < x.bytes))
        return fail(MSDA_ERROR_INVALID_VALUE, "workspace of %zu bytes is smaller than the %zu needed",
                    workspace ? bytes : (size_t)0, x.bytes);
    if (x.bytes > 0 && !is_aligned(workspace, 16))
        return fail(MSDA_ERROR_INVALID_VALUE, "workspace must be 16-byte aligned");
    return MSDA_SUCCESS;
}

msda_status_t check_bases(const msda_attention_t& a, const Attention& x, const void* q, const void* k, const void* v) {
    const int es = dtype_size(a.dtype);
    if (!is_aligned(q, x.pack[0] ? es : 16) || !is_aligned(k, x.pack[1] ? es : 16) || !is_aligned(v, x.pack[2] ? es : 16))
        return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: q, k and v need 16 bytes (their element's where "
                    "they are packed: see msda_attention_t's unaligned)");
    return MSDA_SUCCESS;
}

// Points the kernels at their tensors, and enqueues the copies of those that have to be packed. out and grad_out
// are null in the forward.
hipError_t bind(Attention& x, const msda_attention_t& a, const void* q, const void* k, const void* v, const void* out,
                const void* grad_out, void* workspace, hipStream_t stream) {
    msda::AttnParams& p = x.p;
    char* ws = static_cast<char*>(workspace);
    p.delta = reinterpret_cast<float*>(ws + x.at_delta);
    p.filled = reinterpret_cast<int*>(ws + x.at_filled);
    p.part = reinterpret_cast<float*>(ws + x.at_part);
    p.row_width = x.pack[3] ? x.width : p.D;
    int64_t rows[3] = {a.Lq * a.M * a.D, a.M * a.D, a.D};  // of out and grad_out
    const void* from[5] = {q, k, v, out, grad_out};
    int64_t* stride[5] = {p.qs, p.ks, p.vs, rows, rows};
    for (int i = 0; i < 5; ++i) {
        if (!x.pack[i]) continue;
        const bool of_keys = i == 1 || i == 2;
        msda::AttnPack c = {};
        c.L = of_keys ? a.Lk : a.Lq;
        c.H = (int)(of_keys ? a.Mkv : a.M);
        if (c.L == 0) continue;
        c.from = from[i];
        c.to = ws + x.at_pack[i];
        c.N = p.N;
        c.D = p.D;
        c.width = x.width;
        for (int e = 0; e < 3; ++e) c.stride[e] = stride[i][e];
        hipError_t e = msda::launch_attn_pack(c, a.dtype, stream);
        if (e != hipSuccess) return e;
        from[i] = c.to;
        if (i < 3) {
            stride[i][0] = c.L * c.H * c.width;
            stride[i][1] = (int64_t)c.H * c.width;
            stride[i][2] = c.width;
        }
    }
    p.q = from[0];
    p.k = from[1];
    p.v = from[2];
    p.o = from[3];
    p.grad_out = from[4];
    return hipSuccess;
}

// Enqueues the tables of documents.
hipError_t find_ranges(const Attention& x, void* workspace, hipStream_t stream) {
    const msda::AttnParams& p = x.p;
    if (!p.q_doc) return hipSuccess;
    const msda::AttnPlan &r = x.rows, &k = x.keys;
    msda::AttnRanges c = {{{p.k_doc, nullptr, p.Lk, 1, r.tile, r.tiles},
                           {p.q_doc, nullptr, p.Lq, p.G, 32 * r.waves, r.blocks},
                           {p.q_doc, nullptr, p.Lq, p.G, k.tile, k.tiles},
                           {p.k_doc, nullptr, p.Lk, 1, 32 * k.waves, k.blocks}}, p.N, 0};
    for (int i = 0; i < 4; ++i) {
        c.table[i].into = reinterpret_cast<int4*>(static_cast<char*>(workspace) + x.at_ranges[i]);
        c.per_item += c.table[i].count;
    }
    return msda::launch_attn_ranges(c, stream);
}

// The parameters of the kernels that own rows, or keys.
msda::AttnParams kernel_params(const Attention& x, bool keys, void* workspace) {
    msda::AttnParams p = x.p;
    const msda::AttnPlan& plan = keys ? x.keys : x.rows;
    p.blocks = plan.blocks;
    p.own_rows = 32 * plan.waves;
    p.tiles = plan.tiles;
    p.splits = plan.splits;
    p.chunk = plan.chunk;
    if (p.q_doc) {
        const char* ws = static_cast<const char*>(workspace);
        p.tile_ranges = reinterpret_cast<const int4*>(ws + x.at_ranges[keys ? 2 : 0]);
        p.own_ranges = reinterpret_cast<const int4*>(ws + x.at_ranges[keys ? 3 : 1]);
    }
    return p;
}

}  // namespace

extern "C" {

msda_status_t msda_attention_workspace_size(const msda_attention_t* a, int backward, size_t* bytes) {
    if (!bytes) return fail(MSDA_ERROR_INVALID_VALUE, "bytes must be non-null");
    *bytes = 0;
    msda_status_t st = check_attention(a);
    if (st != MSDA_SUCCESS) return st;
    if (a->N > 0) {
        const Attention x = attention_of(*a, backward != 0);
        if ((st = check_launches(x, *a, backward != 0)) != MSDA_SUCCESS) return st;
        *bytes = x.bytes;
    }
    return ok();
}

msda_status_t msda_attention_forward(const msda_attention_t* a, const void* q, const void* k, const void* v, void* out,
                                     float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    msda_status_t st = check_attention(a);
    if (st != MSDA_SUCCESS) return st;
    if (a->N * a->Lq == 0) return ok();
    if (!q || !out || (a->Lk > 0 && (!k || !v)))
        return fail(MSDA_ERROR_INVALID_VALUE, "q, k, v and out must be non-null");
    if (!is_aligned(out, 16) || !is_aligned(lse, 4))
        return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: out needs 16 bytes, lse 4");
    Attention x = attention_of(*a, false);
    if ((st = check_launches(x, *a, false)) != MSDA_SUCCESS) return st;
    if ((st = check_bases(*a, x, q, k, v)) != MSDA_SUCCESS) return st;
    if ((st = check_workspace(x, workspace, workspace_bytes)) != MSDA_SUCCESS) return st;
    hipError_t e = bind(x, *a, q, k, v, nullptr, nullptr, workspace, (hipStream_t)stream);
    x.p.out = out;
    x.p.lse = lse;
    if (e == hipSuccess) e = find_ranges(x, workspace, (hipStream_t)stream);
    if (e == hipSuccess)
        e = msda::launch_attn_forward(kernel_params(x, false, workspace), a->dtype, x.rows.waves, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "attention launch: %s", hipGetErrorString(e));
    return ok();
}

msda_status_t msda_attention_backward(const msda_attention_t* a, const void* q, const void* k, const void* v,
                                      const void* out, const float* lse, const void* grad_out, void* grad_q,
                                      void* grad_k, void* grad_v, void* workspace, size_t workspace_bytes,
                                      void* stream) {
    msda_status_t st = check_attention(a);
    if (st != MSDA_SUCCESS) return st;
    if (a->N == 0 || (a->Lq == 0 && a->Lk == 0)) return ok();
    if ((a->Lq > 0 && (!q || !out || !lse || !grad_out || !grad_q)) || (a->Lk > 0 && (!k || !v || !grad_k || !grad_v)))
        return fail(MSDA_ERROR_INVALID_VALUE,
                    "q, k, v, out, lse, grad_out, grad_q, grad_k and grad_v must be non-null");
    if (!is_aligned(lse, 4) || !is_aligned(out, 16) || !is_aligned(grad_out, 16) || !is_aligned(grad_q, 16) ||
        !is_aligned(grad_k, 16) || !is_aligned(grad_v, 16))
        return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: out and the gradients need 16 bytes, lse 4");
    Attention x = attention_of(*a, true);
    if ((st = check_launches(x, *a, true)) != MSDA_SUCCESS) return st;
    if ((st = check_bases(*a, x, q, k, v)) != MSDA_SUCCESS) return st;
    if ((st = check_workspace(x, workspace, workspace_bytes)) != MSDA_SUCCESS) return st;
    hipError_t e = bind(x, *a, q, k, v, out, grad_out, workspace, (hipStream_t)stream);
    x.p.lse = const_cast<float*>(lse);
    x.p.grad_q = grad_q;
    x.p.grad_k = grad_k;
    x.p.grad_v = grad_v;
    if (e == hipSuccess) e = find_ranges(x, workspace, (hipStream_t)stream);
    if (e == hipSuccess && a->Lq > 0) {
        msda::AttnParams p = kernel_params(x, false, workspace);
        if (rows_of_few_keys(*a)) {
            msda::AttnParams d = p;
            d.splits = 1;
            d.chunk = d.tiles;
            e = msda::launch_attn_delta(d, a->dtype, (hipStream_t)stream);
            p.delta_known = 1;
        }
        // writes delta otherwise, which grad_k and grad_v need
        if (e == hipSuccess) e = msda::launch_attn_grad_q(p, a->dtype, (hipStream_t)stream);
    }
    if (e == hipSuccess && a->Lk > 0)
        e = msda::launch_attn_grad_kv(kernel_params(x, true, workspace), a->dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "attention backward launch: %s", hipGetErrorString(e));
    return ok();
}

}  // extern "C"
