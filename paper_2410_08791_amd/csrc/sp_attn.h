// LDS tiles of the attention forward kernels (described in k_attn.hip).
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
    // head_dim 80: the rows 80..95 of the third O^T tile are padding.  The V tiles' padding
    // elements are set to 1.0 once and never loaded over, so row 80 of O^T accumulates the sum of
    // the (bf16) probabilities: the softmax denominator comes out of the matrix pipe, which idles
    // most of the time here, instead of 32 additions per lane and tile on the vector pipe, which
    // is the one that bounds this kernel.
    static constexpr bool ONES_ROW = HDP > HD;
    static_assert(STAGE % 1024 == 0 && TILE_BYTES % 1024 == 0, "whole load instructions per tile");
    static_assert(HDP * 2 <= ROWB, "the fragment reads of a padded head_dim stay inside the row");
    __device__ static int k_swz(int row) { return HD == 128 ? (row & 15) : HD == 64 ? ((row >> 1) & 7) : ((row >> 2) & 3); }
    // in 64-byte blocks
    __device__ static int v_swz(int row) { return HD == 128 ? (row & 3) : HD == 64 ? ((row >> 1) & 1) : 0; }
};
