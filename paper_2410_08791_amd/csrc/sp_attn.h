// LDS tiles of the attention kernels (forward: described in k_attn.hip).
#pragma once
#include "sp_gemm.h"

constexpr int KB = 64;    // keys per LDS tile

// NW = waves per work-group: a work-group handles NW * 32 queries of one head.
template <int HD, int NW>
struct AttnCfg {
    static constexpr int QB = NW * 32;              // queries per work-group
    static constexpr int NKS = HD / 16;             // MFMA k-steps over head_dim
    static constexpr int NMT = (HD + 31) / 32;      // 32-row tiles of O^T
    static constexpr int HDP = NMT * 32;
    static constexpr int ROWB = HD == 80 ? 192 : HD * 2;   // bytes per key / value row in LDS
    static constexpr int CPR = HD / 8;                     // 16-byte chunks of a row that hold data
    static constexpr int TILE_BYTES = KB * ROWB;           // one K or one V tile
    static constexpr int STAGE = 2 * TILE_BYTES;           // K tile, then V tile
    static constexpr int NINST = STAGE / 1024;             // 1 KiB load instructions per stage
    static constexpr int NLOAD = (NINST + NW - 1) / NW;    // per wave (the last wave may have fewer)
    // head_dim 80: the rows 80..95 of the third O^T tile are padding.  In k_attn.hip the V tiles' padding
    // elements are set to 1.0 once and never loaded over, so row 80 of O^T accumulates the sum of
    // the (bf16) probabilities: the softmax denominator comes out of the matrix pipe, which idles
    // most of the time there, instead of 32 additions per lane and tile on the vector pipe, which
    // is the one that bounds that kernel.  (k_attn_packed.hip loads zeros there and sums the unrounded probabilities.)
    static constexpr bool ONES_ROW = HDP > HD;
    static_assert(STAGE % 1024 == 0 && TILE_BYTES % 1024 == 0, "whole load instructions per tile");
    static_assert(HDP * 2 <= ROWB, "the fragment reads of a padded head_dim stay inside the row");
    __device__ static int k_swz(int row) { return HD == 128 ? (row & 15) : HD == 64 ? ((row >> 1) & 7) : ((row >> 2) & 3); }
    // in 64-byte blocks
    __device__ static int v_swz(int row) { return HD == 128 ? (row & 3) : HD == 64 ? ((row >> 1) & 1) : 0; }
};

// A 64-row token tile in LDS: rows of ROWB bytes (head_dim 80: 192; the padding holds nothing that counts: k_attn_bwd.hip never loads it, the packed kernels load zeros), the 16-byte
// chunk c of row r at position c ^ swz(r).  swz serves both readers: the 16 rows of a straight 16-byte read
// fall on all banks, and the four consecutive rows of a transposing read in different 64-byte blocks.  It has
// period 16 in r, and r + 8 flips exactly bit 1 (the hi half of a transposed fragment: address ^ 32).
template <int HD>
struct TokTile {
    static constexpr int ROWB = HD == 80 ? 192 : HD * 2, CPR = HD / 8;
    static constexpr int NKS = HD / 16, NMT = (HD + 31) / 32;
    static constexpr int ROWS = 64, BYTES = ROWS * ROWB;
    __device__ static int swz(int r) {
        return HD == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : HD == 64 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : (r >> 2) & 3;
    }
    // lane part of the straight fragment of k-step ks: row l32, head-dimension elements 16 ks + 8 half ..
    __device__ static int row_pos(int ks, int l32, int half) { return l32 * ROWB + (((2 * ks + half) ^ swz(l32)) << 4); }
    __device__ static bf16x8_t row_frag(const unsigned char* p) { return *reinterpret_cast<const bf16x8_t*>(p); }
    // Transposed MFMA operand: the lane ends up with head-dimension row (lane & 31) of the 32-row block mt and
    // the eight tokens 4*half + {0..3} and 8 + 4*half + {0..3} of a 16-token step -- the token order in which
    // the score tiles hold their bf16 operands.  ds_read_b64_tr_b16 works on groups of 16 lanes: lane s
    // supplies the address of four values of one token row, lane i receives element i%4 of the blocks
    // supplied by lanes i/4, i/4+4, i/4+8, i/4+12.
    __device__ static int tr_pos(int mt, int lane) {
        const int s16 = lane & 15, row = 4 * (lane >> 5) + (s16 >> 2);
        const int chunk = mt * 4 + 2 * ((lane >> 4) & 1) + ((s16 & 3) >> 1);
        return row * ROWB + ((chunk ^ swz(row)) << 4) + (s16 & 1) * 8;
    }
    __device__ static bf16x8_t tr_frag(const unsigned char* step, int pos) {
        const s16x4_t lo = sp_tr_read((lds_s16x4_ptr)(step + pos));
        const s16x4_t hi = sp_tr_read((lds_s16x4_ptr)(step + (pos ^ 32) + 8 * ROWB));
        return __builtin_bit_cast(bf16x8_t, s16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
};
