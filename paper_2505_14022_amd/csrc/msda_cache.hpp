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

// A workgroup's sequence, which of the sequence's workgroups it is, and the sequence's tokens: in all, the call's first one, how
// many there are of the call's, and the first one's place. What the last look takes of every candidate is the sequence's
// all: nothing more is read for it.
struct Place {
    int n, block;  // n < 0: none
    int length, start, count, first;
};
__device__ __forceinline__ Place find_place(const Cache& c, int b, int size, int extra, int lane) {
    auto at = [&](int n) { return min(max(c.start[n], 0), c.T); };
    Place x = {-1, 0, 0, 0, 0, 0};
    if (!c.start) {  // a token and a workgroup each
        x.n = b;
        x.length = max(c.length[b], 0);
        x.start = b;
        x.count = 1;
        x.first = x.length - 1;
        return x;
    }
    int lo = 0, hi = c.N;  // the sequence is one of lo .. hi - 1, if any
    while (true) {
        const int step = (hi - lo + 63) / 64, n = lo + lane * step;
        int start = 0, next = 0, length = 0;
        if (n < hi) {
            start = at(n);
            if (step == 1) {
                next = at(n + 1);
                length = max(c.length[n], 0);
            }
        }
        const uint64_t below = __ballot(n < hi && start / size + extra * n <= b);
        if (below == 0) return x;
        const int winner = 63 - __builtin_clzll(below);
        lo += winner * step;
        if (step == 1) {
            x.n = __builtin_amdgcn_readfirstlane(lo);
            x.start = __builtin_amdgcn_readlane(start, winner);
            x.length = __builtin_amdgcn_readlane(length, winner);
            x.count = max(__builtin_amdgcn_readlane(next, winner) - x.start, 0);
            x.first = x.length - x.count;
            x.block = b - (x.start / size + extra * x.n);
            return x;
        }
        hi = min(hi, lo + step);
    }
}

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
