// Internal interface between the layer operators' C ABI (msda_layer_api.cpp) and their HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "msda.h"

namespace msda {

// Errors of all entry points (msda_api.cpp): fail() keeps the message for msda_last_error().
msda_status_t fail(msda_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
msda_status_t ok();

inline bool is_aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int dtype_size(int dtype) { return dtype == MSDA_F32 ? 4 : 2; }

// ---------------------------------------------------------------- layer norm

struct NormParams {
    const void *x, *residual;   // [rows, C] dtype; residual may be null
    const float *weight, *bias; // [C] or null
    void *out, *sum;            // forward; sum may be null
    const void *grad_out, *grad_sum;  // backward; grad_sum may be null
    void* grad_x;
    float *mean, *rstd;         // [rows]; may be null in the forward
    float* partial;             // backward: [2][blocks][C] partial sums of grad_weight and grad_bias, or null
    float *grad_weight, *grad_bias;   // may be null
    int64_t rows;
    int C, blocks;
    float eps;
    bool vec;                   // rows are whole 16-byte pieces, 16-byte aligned
    bool columns;               // weight and bias are 16-byte aligned
};

// Workgroups of the backward kernel, each with a row of partial sums.
int norm_backward_blocks(int64_t rows, int64_t C, int dtype);
hipError_t launch_layernorm_forward(const NormParams& p, int dtype, hipStream_t stream);
hipError_t launch_layernorm_backward(const NormParams& p, int dtype, hipStream_t stream);
// Sums over `blocks` rows of `partial` [2][blocks][C] (or [blocks][C] without `second`), and zeros; either result may be null.
hipError_t launch_column_sums(const float* partial, float* first, float* second, int C, int blocks, hipStream_t stream);
hipError_t launch_column_zeros(float* first, float* second, int C, hipStream_t stream);

// ---------------------------------------------------------------- rotary positions

struct RotaryParams {
    const void* x;
    void* out;
    const float *pos, *freqs;
    int64_t xs[3], os[3];       // strides in elements: batch item, token, head
    int64_t T, pos_item;        // pos_item: elements between the positions of two batch items (0: shared)
    int N, M, D, A, R;
    bool interleaved, vec;      // vec: 16-byte pieces of pairs and of copied channels
    float sign;                 // 1 forward, -1 backward
};
int64_t rotary_workgroups(const RotaryParams& p, int dtype);  // of a launch for one batch item
hipError_t launch_rotary(const RotaryParams& p, int dtype, hipStream_t stream);

// ---------------------------------------------------------------- dense attention

// The query heads that share a key head are packed: "row" r of a slab (batch item, key head) is query
// r / G of query head kv * G + r % G, so that shared keys are read once for all of them and a single token
// of G heads fills G rows of a matrix product.
struct AttnParams {
    const void *q, *k, *v, *o, *grad_out;  // o: the forward's result (backward)
    void *out, *grad_q, *grad_k, *grad_v;
    float* lse;                  // [N, M, Lq]; written by the forward (or null), read by the backward
    float* delta;                // [N, M, Lq]: sum over channels of grad_out * o (backward)
    const float *slopes, *q_pos, *k_pos;
    const int *q_doc, *k_doc, *prefix;
    const int4 *own_ranges, *tile_ranges;  // documents of the kernel's blocks [N, blocks] and tiles [N, tiles], or null
    float* part;                  // partial results of the splits
    int* filled;                  // [slabs, blocks, splits]: whether a split has a partial result
    int64_t qs[3], ks[3], vs[3];  // strides in elements: batch item, token, head
    int N, Lq, Lk, M, Mkv, G, D;
    int R;                        // rows of a slab: Lq * G
    int row_width;                // elements from one row of o and grad_out to the next (D, or more where they were packed)
    int blocks, own_rows;         // workgroups of a slab's owners, and the owners of each
    int tiles, chunk, splits;     // tiles of the other axis, in runs of `chunk` for each of `splits` workgroups
    int causal;
    int delta_known;              // grad_q reads delta (of launch_attn_delta), which it writes otherwise
    float scale, softcap;
};

// A copy of a strided tensor in rows of `width` elements, whole 16-byte pieces.
struct AttnPack {
    const void* from;
    void* to;
    int64_t stride[3];
    int64_t L;
    int N, H, D, width;
};

// How a kernel is cut up: waves per workgroup, rows or keys per tile of the other axis, workgroups per slab, and the
// runs of tiles that the workgroups of a block share. Workgroups own rows (forward, grad_q) or keys (grad_k and grad_v).
enum AttnKernel { kForward, kGradQ, kGradKV };
struct AttnPlan {
    int waves = 1, tile = 32, blocks = 0, tiles = 0, splits = 1, chunk = 1;
};
AttnPlan attn_plan(const AttnParams& p, int dtype, AttnKernel kernel);
int attn_channels(int D);  // channels that the kernels hold: 32, 64 or 128
hipError_t launch_attn_pack(const AttnPack& c, int dtype, hipStream_t stream);
// The documents of runs of `size` owners (keys, or rows of `group` heads to a token) of each batch item: the smallest
// and largest that are not padding, and whether none is.
struct AttnRanges {
    struct Table {
        const int* doc;  // [N, tokens]
        int4* into;      // [N, count]
        int tokens, group, size, count;
    } table[4];
    int N, per_item;     // per_item: the counts' sum
};
hipError_t launch_attn_ranges(const AttnRanges& c, hipStream_t stream);
hipError_t launch_attn_forward(const AttnParams& p, int dtype, int waves, hipStream_t stream);
constexpr int kFewKeys = 64;  // rows of at most so many have their delta formed with care
hipError_t launch_attn_delta(const AttnParams& p, int dtype, hipStream_t stream);  // 16-bit types; splits == 1
hipError_t launch_attn_grad_q(const AttnParams& p, int dtype, hipStream_t stream);
hipError_t launch_attn_grad_kv(const AttnParams& p, int dtype, hipStream_t stream);

}  // namespace msda
