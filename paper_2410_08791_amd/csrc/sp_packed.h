// Packed batches: the rows of n sequences of different lengths lie one behind the other, rows cu[r] .. cu[r + 1] - 1 are
// sequence r's.  What the kernels over such rows share.
#pragma once
#include "sp_common.h"

// A block of QB rows of one sequence.
struct PackedBlock {
    int row0, len;       // the sequence's first row and its length, inside [0, T] whatever cu holds
    int blk;             // block of the sequence; blk * QB >= len: none
};

// Slot j of the packed blocks.  Sequence r owns the slots cu[r] / QB + r .. cu[r + 1] / QB + r: at least ceil(len / QB) of
// them for any start, and T / QB + n slots in all, a number that the host knows without the lengths.  (A list of blocks
// built by a launch of its own would cost that launch; at most one slot of a sequence is left over here, and its
// work-group ends at once.)  A sequence's last block comes first: under a causal mask it has the most keys.
// The whole wave looks: one load of cu finds the sequence and its rows among 63 (each further dependent load costs every
// work-group the better part of a microsecond), two more its rows among kPackedMaxSeqs.
template <int QB>
__device__ __forceinline__ PackedBlock packed_block(const int* __restrict__ cu, int n, int T, int j) {
    const int lane = threadIdx.x & 63;
    auto key = [&](int row, int r) { return row / QB + r; };
    // the last of 64 candidates that begins at j or before; the first where cu does not ascend and none does
    auto last = [](bool at_or_before) { return max((int)__popcll(__ballot(at_or_before)) - 1, 0); };
    PackedBlock p;
    int r, end;
    if (n < 64) {
        const int row = min(max(cu[min(lane, n)], 0), T);
        r = __builtin_amdgcn_readfirstlane(last(lane < n && key(row, lane) <= j));
        p.row0 = __builtin_amdgcn_readlane(row, r);
        end = __builtin_amdgcn_readlane(row, r + 1);
    } else {
        auto at = [&](int i) { return min(max(cu[i], 0), T); };
        const int step = (n + 63) / 64;
        r = last(lane * step < n && key(at(lane * step), lane * step) <= j) * step;
        if (step > 1) r += last(lane < step && r + lane < n && key(at(r + lane), r + lane) <= j);
        r = __builtin_amdgcn_readfirstlane(r);
        p.row0 = at(r);
        end = at(r + 1);
    }
    p.len = max(end - p.row0, 0);
    const int first = p.row0 / QB + r, slots = (p.row0 + p.len) / QB + 1 - p.row0 / QB;
    p.blk = slots - 1 - (j - first);
    if (p.blk < 0 || j < first) { p.blk = 0; p.len = 0; }      // cu does not ascend: no such block
    return p;
}
