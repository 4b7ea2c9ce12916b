// Internal interface between the serving operators' C ABI (msda_serve_api.cpp) and their HIP kernels.
#pragma once

#include "msda_layer.h"

namespace msda {

// ---------------------------------------------------------------- root-mean-square norm, rows in 8 bits

struct RmsParams {
    const void *x, *residual;   // [rows, C] dtype; residual may be null
    const float* weight;        // [C] or null
    void *out, *sum;            // forward; sum may be null
    int8_t* codes;              // in 8 bits: codes and their rows' scales
    float* scale;
    const void *grad_out, *grad_sum;  // backward; grad_sum may be null
    void* grad_x;
    float* rstd;                // [rows]; may be null in the forward
    float* partial;             // backward: [blocks][C] partial sums of grad_weight, or null
    float* grad_weight;
    int64_t rows;
    int C, blocks;
    float eps;
    bool vec;                   // rows are whole 16-byte pieces, 16-byte aligned, and their codes 8-byte aligned
    bool columns;               // weight is 16-byte aligned
};
enum RmsResult { kNormed, kNormedCodes, kCodes };
hipError_t launch_rms_forward(const RmsParams& p, RmsResult result, int dtype, hipStream_t stream);
hipError_t launch_rms_backward(const RmsParams& p, int dtype, hipStream_t stream);

// ---------------------------------------------------------------- matrix product of 8-bit integers

struct ProductParams {
    const int8_t *a, *b;        // [T, K], [O, K]
    const float *a_scale, *b_scale, *bias;  // [T], [O], [O] or null
    void* out;                  // [T, O] dtype
    int T, K, O;
    bool pieces;                // rows of a and b are whole 16-byte pieces on 16-byte boundaries
    bool wide;                  // rows of out are whole 16-byte pieces on 16-byte boundaries
};
// How a product is cut up: rows of a and of b to a workgroup.
struct ProductPlan {
    int tokens, channels, waves;
    int64_t workgroups;
};
ProductPlan product_plan(const ProductParams& p);
hipError_t launch_product(const ProductParams& p, int dtype, hipStream_t stream);

// ---------------------------------------------------------------- paged cache

// The kernels' view of msda_cache_t.
struct Cache {
    int8_t *k, *v;              // [pages, Mkv, page, D]
    float *k_scale, *v_scale;   // [pages, Mkv]
    const int *table, *length, *start;
    int64_t table_stride;
    int N, T, pages, page, page_shift, Mkv, D, width;
};

struct AppendParams {
    Cache c;
    const void *k, *v;
    int64_t ks[2], vs[2];       // strides in elements: token, head
    const float *pos, *freqs;
    int A, R;
    bool interleaved, vec;      // vec: 16-byte pieces of channels
};
int64_t append_workgroups(const AppendParams& p);
hipError_t launch_append(const AppendParams& p, int dtype, hipStream_t stream);

// Query heads that share a key head are packed: row r of a block of a sequence's tokens is head r % group of those that
// the block takes of token r / group.
struct CacheAttnParams {
    Cache c;
    const void* q;
    void* out;
    float* lse;                 // [T, M] or null
    int64_t qs[2];
    float* part;                // partial results of the splits
    int M, G;
    int group, groups;          // heads of a block, and blocks of heads of a key head
    int tokens;                 // of a block
    int blocks;                 // of tokens, of all sequences
    int splits, run;            // runs of `run` tokens of the sequence, one to each of `splits` workgroups
    int causal;
    bool vec;                   // queries are read in 16-byte pieces
    float scale, softcap;
    float cap_unit, cap_inverse, cap_exponent;  // softcap log2(e), 1 / softcap, 2 log2(e) / softcap
};
struct CacheAttnPlan {
    int rows;                   // of a workgroup, shared by its waves: 16, 32 or 48
    int group, groups, tokens, splits, run;
    int64_t blocks, workgroups;
    size_t bytes;               // of the workspace
};
CacheAttnPlan cache_attn_plan(const CacheAttnParams& p, int dtype);
hipError_t launch_cache_attn(const CacheAttnParams& p, const CacheAttnPlan& plan, int dtype, hipStream_t stream);

}  // namespace msda
