// Attention over packed prompts: o = softmax(q k^T / sqrt(hd) + mask) v inside each of n sequences whose rows lie one
// behind the other, causal or bidirectional, grouped heads, head_dim in {64, 80, 128}.
//
// The products, the LDS tiles and the softmax in base 2 with a lazily moving reference are those of k_attn.hip.  A wave
// owns MQ blocks of 32 queries; each key or value fragment that it reads from LDS serves all of them.  The denominator
// is the fp32 sum of the unrounded probabilities at every head_dim, so that the log-sum-exp is as exact as fp32 allows.
// A row of scores that are all -inf gives NaN, as the definition does (0 / 0).
#include "sp_attn.h"
#include "sp_packed.h"

namespace {

// One tile of 64 keys for one wave's MQ x 32 queries.
template <int HD, int NW, int MQ, bool MASK>
__device__ __forceinline__ void packed_tile(const unsigned char* sK, const unsigned char* sV, const int* kpos, const int* vpos,
                                            const bf16x8_t (*qf)[HD / 16], f32x16_t (*oacc)[(HD + 31) / 32], float* m_run, float* l_run,
                                            int key0, int len, int causal, int qi, int half, float scale_log2e) {
    typedef AttnCfg<HD, NW> C;
    f32x16_t sacc[MQ][2];
#pragma unroll
    for (int m = 0; m < MQ; ++m)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) sacc[m][t][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(sK + t * 32 * C::ROWB + kpos[ks]);
#pragma unroll
            for (int m = 0; m < MQ; ++m) sacc[m][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[m][ks], sacc[m][t], 0, 0, 0);
        }
    bf16x8_t pf[MQ][2][2];
#pragma unroll
    for (int m = 0; m < MQ; ++m) {
        if (MASK) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = key0 + t * 32 + (e >> 2) * 8 + half * 4 + (e & 3);
                    if (key >= len || (causal && key > qi + 32 * m)) sacc[m][t][e] = -INFINITY;
                }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sacc[m][t][e]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        // the reference starts at the lowest finite value: a tile without a visible key then has probabilities 0
        const bool move = (mx - m_run[m]) * scale_log2e > 8.0f;
        const float m_new = move ? mx : m_run[m];
        const float alpha = move ? __builtin_amdgcn_exp2f((m_run[m] - m_new) * scale_log2e) : 1.0f;
        const float m_scaled = m_new * scale_log2e;
        m_run[m] = m_new;
        float psum = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(sacc[m][t][j * 8 + e], scale_log2e, -m_scaled));
                    psum += p;
                    pf[m][t][j][e] = (__bf16)p;      // at most 256: half a step of bf16, as every operand of the products
                }
        l_run[m] = l_run[m] * alpha + psum;
        if (__any(move)) {
#pragma unroll
            for (int t = 0; t < C::NMT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[m][t][e] *= alpha;
        }
    }
#pragma unroll
    for (int tj = 0; tj < 4; ++tj)
#pragma unroll
        for (int mt = 0; mt < C::NMT; ++mt) {
            const unsigned char* vp = sV + ((tj >> 1) * 32 + 16 * (tj & 1)) * C::ROWB + vpos[mt];
            const s16x4_t lo = sp_tr_read((lds_s16x4_ptr)(vp));
            const s16x4_t hi = sp_tr_read((lds_s16x4_ptr)(vp + 8 * C::ROWB));
            const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, s16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
#pragma unroll
            for (int m = 0; m < MQ; ++m) oacc[m][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[m][tj >> 1][tj & 1], oacc[m][mt], 0, 0, 0);
        }
}

template <int HD, int NW, int MQ>
__global__ __launch_bounds__(NW * 64, MQ == 1 ? 2 : 1) void attn_packed_kernel(const bf16_t* __restrict__ qkv, const int* __restrict__ cu,
                                                                              bf16_t* __restrict__ o, float* __restrict__ lse, int n,
                                                                              int T, int slots, int Hq, int Hkv, int causal,
                                                                              float scale_log2e) {
    typedef AttnCfg<HD, NW> C;
    constexpr int QB = NW * MQ * 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_packed[];     // two stages of {K tile, V tile}
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    // An XCD works through a contiguous range of (head, slot): a head's keys and values come through one L2, and every XCD
    // gets its share of the long sequences, which it would not if the range ran over the sequences first.
    const int job = xcd_remap(blockIdx.x, gridDim.x);
    const int h = job / slots;
    const PackedBlock pb = packed_block<QB>(cu, n, T, job - h * slots);
    if (pb.blk * QB >= pb.len) return;
    const int len = pb.len, ld = (Hq + 2 * Hkv) * HD;
    const size_t tok0 = pb.row0;
    [[maybe_unused]] const bf16_t* kbase = qkv + tok0 * ld + (size_t)(Hq + h / (Hq / Hkv)) * HD;
    int ld_col[C::NLOAD], ld_row[C::NLOAD];
    bool ld_on[C::NLOAD];
#pragma unroll
    for (int i = 0; i < C::NLOAD; ++i) {
        const int off = (wave * C::NLOAD + i) * 1024 + lane * 16;
        const bool isv = off >= C::TILE_BYTES;
        const int rel = off - (isv ? C::TILE_BYTES : 0);
        const int row = rel / C::ROWB, pos = (rel % C::ROWB) >> 4;
        const int c = isv ? pos ^ (C::v_swz(row) << 2) : pos ^ C::k_swz(row);
        ld_on[i] = c < C::CPR;
        ld_row[i] = row;
        ld_col[i] = (isv ? Hkv * HD : 0) + (c < C::CPR ? c : 0) * 8;
    }
    auto issue = [&](int kt) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
        for (int i = 0; i < C::NLOAD; ++i)
            if (wave * C::NLOAD + i < C::NINST && ld_on[i])
                __builtin_amdgcn_global_load_lds(kbase + ((size_t)min(kt * KB + ld_row[i], len - 1) * ld + ld_col[i]),
                                                 (lds_void_ptr)(smem_packed + (kt & 1) * C::STAGE + (wave * C::NLOAD + i) * 1024), 16, 0, 0);
#endif
    };
    int kpos[C::NKS], vpos[C::NMT];
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) kpos[ks] = l32 * C::ROWB + (((2 * ks + half) ^ C::k_swz(l32)) << 4);
    const int rowv = half * 4 + ((lane & 15) >> 2);
#pragma unroll
    for (int mt = 0; mt < C::NMT; ++mt) vpos[mt] = rowv * C::ROWB + ((mt ^ C::v_swz(rowv)) << 6) + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);

    const int q0 = pb.blk * QB, wq0 = q0 + wave * (MQ * 32), qi = wq0 + l32;
    bf16x8_t qf[MQ][C::NKS];
#pragma unroll
    for (int m = 0; m < MQ; ++m) {
        const bf16_t* qp = qkv + (tok0 + min(qi + 32 * m, len - 1)) * ld + h * HD + half * 8;
#pragma unroll
        for (int ks = 0; ks < C::NKS; ++ks) qf[m][ks] = *reinterpret_cast<const bf16x8_t*>(qp + ks * 16);
    }
    f32x16_t oacc[MQ][C::NMT];
    float m_run[MQ], l_run[MQ];
#pragma unroll
    for (int m = 0; m < MQ; ++m) {
        m_run[m] = -3.402823466e38f;
        l_run[m] = 0.f;
#pragma unroll
        for (int t = 0; t < C::NMT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) oacc[m][t][e] = 0.f;
    }
    const int k_end = causal ? min(len, q0 + QB) : len;
    const int ntiles = (k_end + KB - 1) / KB;
    auto landed = [&] {     // this wave's loads; behind the barrier every wave's, and every wave is done with the other stage
        __builtin_amdgcn_s_waitcnt(sp_waitcnt(0, 15));
        asm volatile("" ::: "memory");
        __syncthreads();
    };
    issue(0);
    landed();
    for (int kt = 0; kt < ntiles; ++kt) {
        const int key0 = kt * KB;
        if (kt + 1 < ntiles) issue(kt + 1);
        const unsigned char* sK = smem_packed + (kt & 1) * C::STAGE;
        // wave-uniform: no key of the tile is visible to the wave, no query of the wave exists
        if (!((causal && key0 > wq0 + MQ * 32 - 1) || wq0 >= len)) {
            if ((causal && key0 + KB - 1 > wq0) || key0 + KB > len)
                packed_tile<HD, NW, MQ, true>(sK, sK + C::TILE_BYTES, kpos, vpos, qf, oacc, m_run, l_run, key0, len, causal, qi, half, scale_log2e);
            else
                packed_tile<HD, NW, MQ, false>(sK, sK + C::TILE_BYTES, kpos, vpos, qf, oacc, m_run, l_run, key0, len, causal, qi, half, scale_log2e);
        }
        if (kt + 1 < ntiles) landed();
    }
#pragma unroll
    for (int m = 0; m < MQ; ++m) {
        const float l = l_run[m] + __shfl_xor(l_run[m], 32, 64);
        const int q = qi + 32 * m;
        if (q >= len) continue;
        const float inv = 1.0f / l;
        bf16_t* op = o + (tok0 + q) * (size_t)(Hq * HD) + h * HD;
#pragma unroll
        for (int mt = 0; mt < C::NMT; ++mt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int e0 = mt * 32 + g * 8 + half * 4;
                if (e0 < HD)
                    *reinterpret_cast<uint2*>(op + e0) =
                        make_uint2(pack_bf2(oacc[m][mt][g * 4] * inv, oacc[m][mt][g * 4 + 1] * inv),
                                   pack_bf2(oacc[m][mt][g * 4 + 2] * inv, oacc[m][mt][g * 4 + 3] * inv));
            }
        if (lse && half == 0) lse[(size_t)h * T + tok0 + q] = m_run[m] * scale_log2e * 0.69314718055994530942f + logf(l);
    }
}

template <int HD, int NW, int MQ>
hipError_t launch_packed(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* lse, const PackedShape& a) {
    constexpr int LDS = 2 * AttnCfg<HD, NW>::STAGE;
    static LdsLimitOnce lds_limit;
    hipError_t e = lds_limit.set(reinterpret_cast<const void*>(attn_packed_kernel<HD, NW, MQ>), LDS);
    if (e != hipSuccess) return e;
    const int slots = a.T / (NW * MQ * 32) + a.n;
    attn_packed_kernel<HD, NW, MQ><<<dim3((unsigned)((long)slots * a.Hq)), NW * 64, LDS, st>>>(qkv, a.cu, o, lse, a.n, a.T, slots, a.Hq, a.Hkv,
                                                                                               a.causal, 1.4426950408889634f / sqrtf((float)HD));
    return hipGetLastError();
}

}  // namespace

hipError_t spk_launch_attention_packed(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* lse, const PackedShape& a) {
    switch (a.hd) {
        case 64: return launch_packed<64, 4, 1>(st, qkv, o, lse, a);
        case 80: return launch_packed<80, 4, 1>(st, qkv, o, lse, a);
        case 128: return launch_packed<128, 4, 1>(st, qkv, o, lse, a);
        default: return hipErrorInvalidValue;
    }
}
