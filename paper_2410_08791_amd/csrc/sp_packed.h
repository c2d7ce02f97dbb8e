// Packed batches: the rows of n sequences of different lengths lie one behind the other, rows cu[r] .. cu[r + 1] - 1 are
// sequence r's.  What the kernels over such rows share.
#pragma once
#include "sp_common.h"

// A block of QB rows of one sequence.
struct PackedBlock {
    int row0, len;       // the sequence's first row and its length, inside [0, T] whatever cu holds
    int blk;             // block of the sequence; blk * QB >= len: none
};

// Slot j of the packed blocks, T / QB + n of them at the most for any lengths: a number that the host knows without them.
//
// Fewer than 64 sequences: the blocks of the longest sequence come first, its last one (under a causal mask the one with the
// most keys) before the others, and so on down to the shortest, so that work-groups start in about the order of their
// work and the chip empties evenly; the slots left over end at once.  (In the order of the rows the backward took 109 us for
// 105 over 12 sequences, 16 heads of 128, and 52.8 for 51.8 over 9, 32/8 heads of 64; 40 sequences under no mask took the
// same.  With many short sequences the search costs more than the order brings: 60 of 20 to 400 rows, 32/8 heads of 128, forward 117 us and
// backward 278, 105 and 268 in the order of the rows; 16 heads of 64 40.4 and 119, 39.0 and 106.)  The whole wave looks: one load of cu -- each further dependent load would cost every work-group the better part
// of a microsecond -- then lane r adds up the blocks of the sequences in front of sequence r.
//
// More: in the order of the rows.  Sequence r owns the slots cu[r] / QB + r .. cu[r + 1] / QB + r, at least ceil(len / QB)
// of them for any start; three loads find one among kPackedMaxSeqs.
template <int QB>
__device__ __forceinline__ PackedBlock packed_block(const int* __restrict__ cu, int n, int T, int j) {
    const int lane = threadIdx.x & 63;
    PackedBlock p{0, 0, 0};
    if (n < 64) {
        const int row = min(max(cu[min(lane, n)], 0), T), next = __shfl_down(row, 1, 64);
        const int len = lane < n ? max(next - row, 0) : 0, blocks = (len + QB - 1) / QB;
        const int key = blocks << 6 | (63 - lane);                     // more blocks first, then the earlier; T / 32 * heads < 2^23
        int first = 0;
        for (int i = 0; i < n; i += 8)                                 // a lane behind the n has no blocks
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int other = __builtin_amdgcn_readlane(key, i + k);
                first += other > key ? other >> 6 : 0;
            }
        const unsigned long long mine = __ballot(j >= first && j - first < blocks);
        if (!mine) return p;
        const int r = __builtin_ctzll(mine);
        p.row0 = __builtin_amdgcn_readlane(row, r);
        p.len = __builtin_amdgcn_readlane(len, r);
        p.blk = __builtin_amdgcn_readlane(blocks, r) - 1 - (j - __builtin_amdgcn_readlane(first, r));
        return p;
    }
    auto at = [&](int i) { return min(max(cu[i], 0), T); };
    auto key = [&](int r) { return at(r) / QB + r; };
    // the last of 64 candidates that begins at j or before; the first where cu does not ascend and none does
    auto last = [](bool at_or_before) { return max((int)__popcll(__ballot(at_or_before)) - 1, 0); };
    const int step = (n + 63) / 64;
    int r = last(lane * step < n && key(lane * step) <= j) * step;
    if (step > 1) r += last(lane < step && r + lane < n && key(r + lane) <= j);
    r = __builtin_amdgcn_readfirstlane(r);
    p.row0 = at(r);
    p.len = max(at(r + 1) - p.row0, 0);
    const int begin = p.row0 / QB + r, slots = (p.row0 + p.len) / QB + 1 - p.row0 / QB;
    p.blk = slots - 1 - (j - begin);
    if (p.blk < 0 || j < begin) { p.blk = 0; p.len = 0; }      // cu does not ascend: no such block
    return p;
}
