// C ABI of the serving operators (root-mean-square norm, rows in 8 bits, products of 8-bit integers, paged cache):
// argument checks and launch (host code only).
#include <math.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "msda.h"
#include "msda_checks.h"
#include "msda_serve.h"

using msda::ceil_div;
using msda::check_dtype;
using msda::check_norm;
using msda::dtype_size;
using msda::fail;
using msda::is_aligned;
using msda::kMaxInt;
using msda::kMaxWorkItems;
using msda::norm_pieces;
using msda::ok;

namespace {

const char kMisaligned[] = "misaligned pointer: tensors need the alignment of their elements";

// Root-mean-square norm with a result in the element type (codes null) or in 8 bits.
msda_status_t rms_forward(const void* x, const void* residual, const float* weight, void* out, int8_t* codes, float* scale,
                          void* sum, float* rstd, int64_t rows, int64_t C, float eps, int dtype, msda::RmsResult result,
                          void* stream) {
    msda_status_t st = check_norm(rows, C, dtype);
    if (st != MSDA_SUCCESS) return st;
    if (!(eps >= 0.f) || isinf(eps))
        return fail(MSDA_ERROR_INVALID_VALUE, "eps=%g must be finite and >= 0", (double)eps);
    if (rows == 0) return ok();
    if (result == msda::kNormed ? !x || !out : !x || !codes || !scale)
        return fail(MSDA_ERROR_INVALID_VALUE, result == msda::kNormed ? "x and out must be non-null"
                                                                      : "x, codes and scale must be non-null");
    const int es = dtype_size(dtype);
    if (!is_aligned(x, es) || !is_aligned(residual, es) || !is_aligned(out, es) || !is_aligned(sum, es) ||
        !is_aligned(weight, 4) || !is_aligned(scale, 4) || !is_aligned(rstd, 4))
        return fail(MSDA_ERROR_INVALID_VALUE, kMisaligned);
    msda::RmsParams p = {};
    p.x = x;
    p.residual = residual;
    p.weight = weight;
    p.out = out;
    p.codes = codes;
    p.scale = scale;
    p.sum = sum;
    p.rstd = rstd;
    p.rows = rows;
    p.C = (int)C;
    p.eps = eps;
    p.vec = norm_pieces(C, dtype, x, residual, (const void*)out, (const void*)sum) && is_aligned(codes, 8);
    p.columns = is_aligned(weight, 16);
    hipError_t e = msda::launch_rms_forward(p, result, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "root-mean-square norm launch: %s", hipGetErrorString(e));
    return ok();
}

size_t rms_workspace(int64_t rows, int64_t C, int dtype) {
    return rows == 0 ? 0 : (size_t)msda::norm_backward_blocks(rows, C, dtype) * C * sizeof(float);
}

}  // namespace

extern "C" {

msda_status_t msda_rmsnorm_forward(const void* x, const void* residual, const float* weight, void* out, void* sum,
                                   float* rstd, int64_t rows, int64_t C, float eps, int dtype, void* stream) {
    return rms_forward(x, residual, weight, out, nullptr, nullptr, sum, rstd, rows, C, eps, dtype, msda::kNormed, stream);
}

msda_status_t msda_rmsnorm_quantize(const void* x, const void* residual, const float* weight, int8_t* codes, float* scale,
                                    void* sum, int64_t rows, int64_t C, float eps, int dtype, void* stream) {
    return rms_forward(x, residual, weight, nullptr, codes, scale, sum, nullptr, rows, C, eps, dtype, msda::kNormedCodes,
                       stream);
}

msda_status_t msda_quantize_rows(const void* x, int8_t* codes, float* scale, int64_t rows, int64_t C, int dtype,
                                 void* stream) {
    return rms_forward(x, nullptr, nullptr, nullptr, codes, scale, nullptr, nullptr, rows, C, 0.f, dtype, msda::kCodes,
                       stream);
}

msda_status_t msda_rmsnorm_backward_workspace_size(int64_t rows, int64_t C, int dtype, size_t* bytes) {
    if (!bytes) return fail(MSDA_ERROR_INVALID_VALUE, "bytes must be non-null");
    *bytes = 0;
    msda_status_t st = check_norm(rows, C, dtype);
    if (st != MSDA_SUCCESS) return st;
    *bytes = rms_workspace(rows, C, dtype);
    return ok();
}

msda_status_t msda_rmsnorm_backward(const void* x, const void* residual, const float* weight, const void* grad_out,
                                    const void* grad_sum, const float* rstd, void* grad_x, float* grad_weight,
                                    void* workspace, size_t workspace_bytes, int64_t rows, int64_t C, int dtype,
                                    void* stream) {
    msda_status_t st = check_norm(rows, C, dtype);
    if (st != MSDA_SUCCESS) return st;
    const int es = dtype_size(dtype);
    if (!is_aligned(grad_weight, 4)) return fail(MSDA_ERROR_INVALID_VALUE, kMisaligned);
    if (rows > 0) {
        if (!x || !grad_out || !rstd || !grad_x)
            return fail(MSDA_ERROR_INVALID_VALUE, "x, grad_out, rstd and grad_x must be non-null");
        if (!is_aligned(x, es) || !is_aligned(residual, es) || !is_aligned(grad_out, es) || !is_aligned(grad_sum, es) ||
            !is_aligned(grad_x, es) || !is_aligned(weight, 4) || !is_aligned(rstd, 4))
            return fail(MSDA_ERROR_INVALID_VALUE, kMisaligned);
        const size_t need = rms_workspace(rows, C, dtype);
        if (grad_weight && (!workspace || workspace_bytes < need))
            return fail(MSDA_ERROR_INVALID_VALUE, "workspace of %zu bytes is smaller than the %zu needed",
                        workspace ? workspace_bytes : (size_t)0, need);
        if (grad_weight && !is_aligned(workspace, 16))
            return fail(MSDA_ERROR_INVALID_VALUE, "workspace must be 16-byte aligned");
    }
    msda::RmsParams p = {};
    p.x = x;
    p.residual = residual;
    p.weight = weight;
    p.grad_out = grad_out;
    p.grad_sum = grad_sum;
    p.rstd = const_cast<float*>(rstd);
    p.grad_x = grad_x;
    p.partial = grad_weight ? static_cast<float*>(workspace) : nullptr;
    p.grad_weight = grad_weight;
    p.rows = rows;
    p.C = (int)C;
    p.blocks = msda::norm_backward_blocks(rows, C, dtype);
    p.vec = norm_pieces(C, dtype, x, residual, grad_out, grad_sum, (const void*)grad_x);
    p.columns = is_aligned(weight, 16);
    hipError_t e = msda::launch_rms_backward(p, dtype, (hipStream_t)stream);
    if (e != hipSuccess)
        return fail(MSDA_ERROR_LAUNCH_FAILED, "root-mean-square norm backward launch: %s", hipGetErrorString(e));
    return ok();
}

// ---------------------------------------------------------------- matrix product of 8-bit integers

msda_status_t msda_quantized_matmul(const int8_t* a, const int8_t* b, const float* a_scale, const float* b_scale,
                                    const float* bias, void* out, int64_t T, int64_t K, int64_t O, int dtype,
                                    void* stream) {
    msda_status_t st = check_dtype(dtype);
    if (st != MSDA_SUCCESS) return st;
    if (T < 0 || O < 0 || K < 1)
        return fail(MSDA_ERROR_INVALID_VALUE, "T=%lld and O=%lld must be >= 0 and K=%lld >= 1", (long long)T, (long long)O,
                    (long long)K);
    if (K > MSDA_QUANTIZED_MAX_K)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "K=%lld exceeds MSDA_QUANTIZED_MAX_K=%d: sums would not fit into 32 bits",
                    (long long)K, MSDA_QUANTIZED_MAX_K);
    if (T > kMaxInt - 1024 || O > kMaxInt - 1024) return fail(MSDA_ERROR_NOT_SUPPORTED, "T or O exceeds 2^31 - 1024");
    if (T * O == 0) return ok();
    if (!a || !b || !a_scale || !b_scale || !out)
        return fail(MSDA_ERROR_INVALID_VALUE, "a, b, a_scale, b_scale and out must be non-null");
    if (!is_aligned(a_scale, 4) || !is_aligned(b_scale, 4) || !is_aligned(bias, 4) || !is_aligned(out, dtype_size(dtype)))
        return fail(MSDA_ERROR_INVALID_VALUE, kMisaligned);
    msda::ProductParams p = {};
    p.a = a;
    p.b = b;
    p.a_scale = a_scale;
    p.b_scale = b_scale;
    p.bias = bias;
    p.out = out;
    p.T = (int)T;
    p.K = (int)K;
    p.O = (int)O;
    p.pieces = K % 16 == 0 && is_aligned(a, 16) && is_aligned(b, 16);
    p.wide = (O * dtype_size(dtype)) % 16 == 0 && is_aligned(out, 16);
    const msda::ProductPlan plan = msda::product_plan(p);
    if (plan.workgroups > kMaxWorkItems / (64 * plan.waves))
        return fail(MSDA_ERROR_NOT_SUPPORTED, "T=%lld rows of O=%lld channels are too many for one launch", (long long)T,
                    (long long)O);
    hipError_t e = msda::launch_product(p, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "product launch: %s", hipGetErrorString(e));
    return ok();
}

}  // extern "C"

// ---------------------------------------------------------------- paged cache

namespace {

msda_status_t check_cache(const msda_cache_t* c, int64_t T) {
    if (!c) return fail(MSDA_ERROR_INVALID_VALUE, "the cache's description must be non-null");
    if (c->N < 0 || T < 0 || c->pages < 0 || c->width < 0)
        return fail(MSDA_ERROR_INVALID_VALUE, "N=%lld, T=%lld, pages=%lld and width=%lld must be >= 0", (long long)c->N,
                    (long long)T, (long long)c->pages, (long long)c->width);
    if (c->Mkv < 1 || c->D < 1)
        return fail(MSDA_ERROR_INVALID_VALUE, "Mkv=%lld and D=%lld must be >= 1", (long long)c->Mkv, (long long)c->D);
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128 && c->page_size != 256)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "page_size=%lld: 16, 32, 64, 128 and 256 are taken", (long long)c->page_size);
    if (c->D % 16 != 0 || c->D > MSDA_CACHE_MAX_D)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "D=%lld must be a multiple of 16, at most MSDA_CACHE_MAX_D=%d", (long long)c->D,
                    MSDA_CACHE_MAX_D);
    if (c->Mkv > 65536) return fail(MSDA_ERROR_NOT_SUPPORTED, "Mkv=%lld heads exceeds 65536", (long long)c->Mkv);
    if (c->N >= 1 << 24) return fail(MSDA_ERROR_NOT_SUPPORTED, "N=%lld sequences reaches 2^24", (long long)c->N);
    if (T > kMaxInt - 1024) return fail(MSDA_ERROR_NOT_SUPPORTED, "T=%lld exceeds 2^31 - 1024", (long long)T);
    if (c->pages > kMaxInt) return fail(MSDA_ERROR_NOT_SUPPORTED, "pages=%lld exceeds 2^31 - 1", (long long)c->pages);
    if (c->width > (kMaxInt - 1024) / c->page_size)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "width=%lld pages of page_size=%lld exceed 2^31 - 1024 tokens", (long long)c->width,
                    (long long)c->page_size);
    if (c->N > 1 && c->table_stride < c->width)
        return fail(MSDA_ERROR_INVALID_VALUE, "table_stride=%lld is smaller than width=%lld", (long long)c->table_stride,
                    (long long)c->width);
    if (!c->start && T != c->N)
        return fail(MSDA_ERROR_INVALID_VALUE, "without start every sequence has one token: T=%lld must be N=%lld", (long long)T,
                    (long long)c->N);
    return MSDA_SUCCESS;
}

msda_status_t check_cache_pointers(const msda_cache_t* c) {
    if (!c->length || (c->width > 0 && !c->table) || (c->pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)))
        return fail(MSDA_ERROR_INVALID_VALUE, "k, v, k_scale, v_scale, table and length of the cache must be non-null");
    if (!is_aligned(c->k, 16) || !is_aligned(c->v, 16))
        return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: the cache's k and v need 16 bytes");
    if (!is_aligned(c->k_scale, 4) || !is_aligned(c->v_scale, 4) || !is_aligned(c->table, 4) || !is_aligned(c->length, 4) ||
        !is_aligned(c->start, 4))
        return fail(MSDA_ERROR_INVALID_VALUE, kMisaligned);
    return MSDA_SUCCESS;
}

msda::Cache cache_of(const msda_cache_t& c, int64_t T) {
    msda::Cache x = {};
    x.k = c.k;
    x.v = c.v;
    x.k_scale = c.k_scale;
    x.v_scale = c.v_scale;
    x.table = c.table;
    x.length = c.length;
    x.start = c.start;
    x.table_stride = c.table_stride;
    x.N = (int)c.N;
    x.T = (int)T;
    x.pages = (int)c.pages;
    x.page = (int)c.page_size;
    while ((1 << x.page_shift) < x.page) ++x.page_shift;
    x.Mkv = (int)c.Mkv;
    x.D = (int)c.D;
    x.width = c.pages > 0 ? (int)c.width : 0;  // without a page no token exists
    return x;
}

// Whether rows of tokens and heads with these strides are whole 16-byte pieces.
bool token_pieces(const void* x, const int64_t* stride, int64_t T, int64_t heads, int es) {
    return is_aligned(x, 16) && (T <= 1 || (stride[0] * es) % 16 == 0) && (heads <= 1 || (stride[1] * es) % 16 == 0);
}

// The attention's view of a call, all but the tensors.
msda::CacheAttnParams attention_of(const msda_cache_t& c, int64_t T, int64_t M, int dtype, msda::CacheAttnPlan* plan) {
    msda::CacheAttnParams p = {};
    p.c = cache_of(c, T);
    p.M = (int)M;
    p.G = (int)(M / c.Mkv);
    *plan = msda::cache_attn_plan(p, dtype);
    p.group = plan->group;
    p.groups = plan->groups;
    p.tokens = plan->tokens;
    p.blocks = (int)plan->blocks;
    p.splits = plan->splits;
    p.run = plan->run;
    return p;
}

msda_status_t check_cache_attention(const msda_cache_t* c, int64_t T, int64_t M, int dtype) {
    msda_status_t st = check_dtype(dtype);
    if (st == MSDA_SUCCESS) st = check_cache(c, T);
    if (st != MSDA_SUCCESS) return st;
    if (M < 1 || M % c->Mkv != 0)
        return fail(MSDA_ERROR_INVALID_VALUE, "M=%lld must be a multiple of Mkv=%lld", (long long)M, (long long)c->Mkv);
    if (M > 65536) return fail(MSDA_ERROR_NOT_SUPPORTED, "M=%lld heads exceeds 65536", (long long)M);
    // work items of the largest launch, in blocks of at least one token
    if (((double)T + (double)c->N) * (double)M > 16777215.0 * 16.0)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "T=%lld tokens of M=%lld heads are too many for one launch", (long long)T,
                    (long long)M);
    return MSDA_SUCCESS;
}

msda_status_t check_cache_launch(const msda::CacheAttnPlan& plan) {
    if (plan.workgroups > kMaxWorkItems / 256)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "the call's tokens and heads are too many for one launch (%lld workgroups)",
                    (long long)plan.workgroups);
    return MSDA_SUCCESS;
}

}  // namespace

extern "C" {

msda_status_t msda_cache_append(const msda_cache_t* cache, const void* k, const int64_t* k_stride, const void* v,
                                const int64_t* v_stride, const float* pos, const float* freqs, int64_t T, int64_t A,
                                int64_t R, int interleaved, int dtype, void* stream) {
    msda_status_t st = check_dtype(dtype);
    if (st == MSDA_SUCCESS) st = check_cache(cache, T);
    if (st != MSDA_SUCCESS) return st;
    if (A < 1 || A > 4) return fail(MSDA_ERROR_INVALID_VALUE, "A=%lld axes: 1 to 4 are taken", (long long)A);
    if (!pos && A != 1)
        return fail(MSDA_ERROR_INVALID_VALUE, "without pos, a token's place is its position on one axis, not on A=%lld", (long long)A);
    if (R < 0 || R > cache->D / 2)
        return fail(MSDA_ERROR_INVALID_VALUE, "R=%lld pairs do not fit into D=%lld channels", (long long)R, (long long)cache->D);
    if (!k_stride || !v_stride) return fail(MSDA_ERROR_INVALID_VALUE, "k_stride and v_stride must be non-null");
    for (int i = 0; i < 2; ++i)
        if (k_stride[i] < 0 || v_stride[i] < 0) return fail(MSDA_ERROR_INVALID_VALUE, "strides must be >= 0");
    msda::AppendParams p = {};
    p.c = cache_of(*cache, T);
    if (msda::append_workgroups(p) > kMaxWorkItems / 256)
        return fail(MSDA_ERROR_NOT_SUPPORTED, "T=%lld tokens of N=%lld sequences and Mkv=%lld heads are too many for one launch",
                    (long long)T, (long long)cache->N, (long long)cache->Mkv);
    if (T == 0 || cache->N == 0 || cache->pages == 0 || cache->width == 0) return ok();
    if (!k || !v || (R > 0 && !freqs)) return fail(MSDA_ERROR_INVALID_VALUE, "k, v and freqs must be non-null");
    if ((st = check_cache_pointers(cache)) != MSDA_SUCCESS) return st;
    const int es = dtype_size(dtype);
    if (!is_aligned(k, es) || !is_aligned(v, es) || !is_aligned(pos, 4) || !is_aligned(freqs, 4))
        return fail(MSDA_ERROR_INVALID_VALUE, kMisaligned);
    p.k = k;
    p.v = v;
    for (int i = 0; i < 2; ++i) {
        p.ks[i] = k_stride[i];
        p.vs[i] = v_stride[i];
    }
    p.pos = pos;
    p.freqs = freqs;
    p.A = (int)A;
    p.R = (int)R;
    p.interleaved = interleaved != 0;
    p.vec = R % (16 / es) == 0 && token_pieces(k, k_stride, T, cache->Mkv, es) && token_pieces(v, v_stride, T, cache->Mkv, es);
    hipError_t e = msda::launch_append(p, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "cache append launch: %s", hipGetErrorString(e));
    return ok();
}

msda_status_t msda_cache_attention_workspace_size(const msda_cache_t* cache, int64_t T, int64_t M, int dtype,
                                                  size_t* bytes) {
    if (!bytes) return fail(MSDA_ERROR_INVALID_VALUE, "bytes must be non-null");
    *bytes = 0;
    msda_status_t st = check_cache_attention(cache, T, M, dtype);
    if (st != MSDA_SUCCESS) return st;
    if (T == 0 || cache->N == 0) return ok();
    msda::CacheAttnPlan plan;
    attention_of(*cache, T, M, dtype, &plan);
    if ((st = check_cache_launch(plan)) != MSDA_SUCCESS) return st;
    *bytes = plan.bytes;
    return ok();
}

msda_status_t msda_cache_attention(const msda_cache_t* cache, const void* q, const int64_t* q_stride, void* out,
                                   float* lse, int64_t T, int64_t M, float scale, float softcap, int causal, int dtype,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    msda_status_t st = check_cache_attention(cache, T, M, dtype);
    if (st != MSDA_SUCCESS) return st;
    if (!(scale > 0.f) || !(scale < 1e38f)) return fail(MSDA_ERROR_INVALID_VALUE, "scale=%g must be > 0 and below 1e38", (double)scale);
    if (!(softcap >= 0.f) || !(softcap < 1e38f))
        return fail(MSDA_ERROR_INVALID_VALUE, "softcap=%g must be >= 0 and below 1e38", (double)softcap);
    if (softcap > 0.f && !(softcap > 1e-37f))
        return fail(MSDA_ERROR_INVALID_VALUE, "softcap=%g: its inverse has to be finite (0: scores are not capped)", (double)softcap);
    if (!q_stride) return fail(MSDA_ERROR_INVALID_VALUE, "q_stride must be non-null");
    if (q_stride[0] < 0 || q_stride[1] < 0) return fail(MSDA_ERROR_INVALID_VALUE, "strides must be >= 0");
    if (T == 0 || cache->N == 0) return ok();
    msda::CacheAttnPlan plan;
    msda::CacheAttnParams p = attention_of(*cache, T, M, dtype, &plan);
    if ((st = check_cache_launch(plan)) != MSDA_SUCCESS) return st;
    if (!q || !out) return fail(MSDA_ERROR_INVALID_VALUE, "q and out must be non-null");
    if ((st = check_cache_pointers(cache)) != MSDA_SUCCESS) return st;
    const int es = dtype_size(dtype);
    if (!is_aligned(q, es) || !is_aligned(lse, 4)) return fail(MSDA_ERROR_INVALID_VALUE, kMisaligned);
    if (!is_aligned(out, 16)) return fail(MSDA_ERROR_INVALID_VALUE, "misaligned pointer: out needs 16 bytes");
    if (plan.bytes > 0 && (!workspace || workspace_bytes < plan.bytes))
        return fail(MSDA_ERROR_INVALID_VALUE, "workspace of %zu bytes is smaller than the %zu needed",
                    workspace ? workspace_bytes : (size_t)0, plan.bytes);
    if (plan.bytes > 0 && !is_aligned(workspace, 16))
        return fail(MSDA_ERROR_INVALID_VALUE, "workspace must be 16-byte aligned");
    p.q = q;
    p.out = out;
    p.lse = lse;
    p.qs[0] = q_stride[0];
    p.qs[1] = q_stride[1];
    p.part = static_cast<float*>(workspace);
    p.causal = causal != 0;
    p.vec = token_pieces(q, q_stride, T, M, es);
    p.scale = scale;
    p.softcap = softcap;
    if (softcap > 0.f) {
        const float log2e = 1.4426950408889634f;
        p.cap_unit = softcap * log2e;
        p.cap_inverse = 1.f / softcap;
        p.cap_exponent = 2.f * log2e / softcap;
    }
    hipError_t e = msda::launch_cache_attn(p, plan, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(MSDA_ERROR_LAUNCH_FAILED, "cache attention launch: %s", hipGetErrorString(e));
    return ok();
}

}  // extern "C"
