// What the checks of the layer operators' and the serving operators' C ABI share (host code only).
#pragma once

#include "msda_layer.h"

namespace msda {
namespace {

constexpr int64_t kMaxInt = 0x7fffffff;
constexpr int64_t kMaxWorkItems = 0xffffffff;             // of a grid: the runtime takes fewer than 2^32
constexpr int64_t kMaxWorkgroups = kMaxWorkItems / 256;   // of 256

inline msda_status_t check_dtype(int dtype) {
    if (dtype != MSDA_F32 && dtype != MSDA_F16 && dtype != MSDA_BF16)
        return fail(MSDA_ERROR_INVALID_VALUE, "unknown dtype %d (expected MSDA_F32=0, MSDA_F16=1 or MSDA_BF16=2)", dtype);
    return MSDA_SUCCESS;
}

inline msda_status_t check_norm(int64_t rows, int64_t C, int dtype) {
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

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace
}  // namespace msda
