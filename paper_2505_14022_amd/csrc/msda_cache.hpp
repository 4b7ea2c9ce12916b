// What the kernels of the paged cache share: which sequence a workgroup belongs to, and its tokens.
//
// The call's tokens are packed, and how many each sequence has is known on the device alone. Sequence n gets the
// workgroups from first(n) = start[n] / size + extra * n on, of which there are enough for its tokens: with c of them,
// (start[n] + c) / size - start[n] / size + extra >= c / size + extra (rounded down). So the grid follows from T and N,
// and a workgroup finds its sequence by a search of 64 places at a time; those that are left over end at once.
#pragma once

#include "msda_layer.hpp"
#include "msda_serve.h"

namespace msda {
namespace {

__device__ __forceinline__ int start_of(const Cache& c, int n) { return c.start ? min(max(c.start[n], 0), c.T) : n; }

// A workgroup's sequence (-1: none), and which of the sequence's workgroups it is.
struct Place {
    int n, block;
};
__device__ __forceinline__ Place find_place(const Cache& c, int b, int size, int extra, int lane) {
    auto first = [&](int n) { return start_of(c, n) / size + extra * n; };
    int lo = 0, hi = c.N;  // the sequence is one of lo .. hi - 1, if any
    while (true) {
        const int step = (hi - lo + 63) / 64, n = lo + lane * step;
        const uint64_t below = __ballot(n < hi && first(n) <= b);
        if (below == 0) return {-1, 0};
        lo += (63 - __builtin_clzll(below)) * step;
        if (step == 1) break;
        hi = min(hi, lo + step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    return {lo, b - first(lo)};
}

// The tokens of a sequence: in all, the call's first one, how many there are of the call's, and the first one's place.
struct Tokens {
    int length, start, count, first;
    __device__ __forceinline__ Tokens(const Cache& c, int n) {
        length = max(c.length[n], 0);
        start = start_of(c, n);
        count = c.start ? max(start_of(c, n + 1) - start, 0) : 1;
        first = length - count;
    }
};

// The page of a sequence's tokens page * column .., or -1.
__device__ __forceinline__ int page_at(const Cache& c, int n, int column) {
    if (column < 0 || column >= c.width) return -1;
    const int page = c.table[n * c.table_stride + column];
    return page >= 0 && page < c.pages ? page : -1;
}

// Workgroups of `size` tokens, or fewer at a sequence's ends: see above.
inline int64_t place_count(const Cache& c, int size, int extra) {
    return c.start ? (int64_t)c.T / size + (int64_t)extra * c.N : c.N;
}

}  // namespace
}  // namespace msda
