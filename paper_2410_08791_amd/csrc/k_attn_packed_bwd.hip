// Backward of the attention over packed prompts: dq, dk, dv from q, k, v, dO, the forward's log-sum-exp and
// delta = rowsum(dO * O), without atomics, in one launch (behind a small one for -delta) of two kinds of work-groups that
// do not depend on one another:
//   dk/dv -- a work-group owns 32 KG keys of one key/value head and walks the queries of every query head that shares it;
//   dq    -- a work-group owns 128 queries of one head and walks the keys.
// P = exp(s - lse), dS = P (dP - delta), dP = dO V^T (in dk/dv its sums begin at -delta); layouts and tiles are those of k_attn_bwd.hip.
//
// What bounds it: 7 products of 2 hd flops per pair of a query and a key on the matrix pipe and the arithmetic of P and dS on the
// vector pipe, in chains that two waves per SIMD do not fill; batches of few long sequences wait for their longest one.  No unit is
// full.  At head_dim 128 the eight waves of a CU take 40 KB each out of LDS for the 32 MFMAs of 32 keys and 32 queries in dk/dv (the keys
// have no room in registers), 1280 cycles of LDS beside 2048 of the matrix pipes; over 12 documents, 16 heads of 128, the matrix
// pipes are busy in 38 % of the cycles, the LDS in 24, vector instructions issue in 33; 9 documents, 32/8 heads of 64: 25, 16 and 35 %.  Every
// wave therefore reads its fragments a few MFMAs ahead, in an order that the source fixes, and works P beside the MFMAs
// of dP, and dS beside those of dV (dk/dv) or of the next 32 keys' scores (dq).  One launch: a short batch has too few
// blocks of either kind to fill the chip.  Four waves each, two work-groups per CU: with one of eight, nothing covered
// the other's first loads and last stores.
#include "sp_attn.h"
#include "sp_packed.h"

namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bf16x8_t lds_b128(const unsigned char* __restrict__ p) { return *reinterpret_cast<const bf16x8_t*>(p); }
__device__ __forceinline__ float4 lds_f4(const float* __restrict__ p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ uint32_t pack2(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)a, (__bf16)b}); }

constexpr int BWD_WAVES = 4;
// The one of n steps that share out `total` items evenly which takes item e.
constexpr int step_of(int e, int n, int total) {
    int i = 0;
    while (e >= total * (i + 1) / n) ++i;
    return i;
}
constexpr float LOG2E = 1.4426950408889634f;

// Fragments of the token tiles (TokTile) of a stage: the lane's addresses in the stage's first tile, the k-step or 32-row
// block on top; what lies further on in the stage is a constant, which the read takes as its offset.
template <int HD>
struct FragAt {
    typedef TokTile<HD> T;
    int r0, r1, t0;
    __device__ void init(int lane) {
        r0 = T::row_pos(0, lane & 31, lane >> 5);
        r1 = T::row_pos(1, lane & 31, lane >> 5);
        t0 = T::tr_pos(0, lane);
    }
    // rows of 128 and 256 bytes: an exclusive or; of 192: two k-steps of four chunks, or a block, are an offset
    __device__ __forceinline__ bf16x8_t row(const unsigned char* smem, int base, int ks, int off) const {
        return lds_b128(smem + (HD != 80 ? (base + r0) ^ (ks << 5) : base + ((ks & 1) ? r1 : r0) + (ks >> 1) * 64) + off);
    }
    __device__ __forceinline__ bf16x8_t tr(const unsigned char* smem, int base, int mt, int off) const {
        const int a = HD != 80 ? (base + t0) ^ (mt << 6) : base + t0 + mt * 64;
        const s16x4_t lo = sp_tr_read((lds_s16x4_ptr)(smem + a + off));
        const s16x4_t hi = sp_tr_read((lds_s16x4_ptr)(smem + (a ^ 32) + off + 8 * T::ROWB));
        return __builtin_bit_cast(bf16x8_t, s16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    }
};

// Loads of a tile of ROWS token rows by a work-group, straight into LDS.  Rows past those that exist and the padding of
// 192-byte rows lie outside the buffer that the load is given and land as zeros.
template <int HD, int ROWS>
struct TileLoad {
    typedef TokTile<HD> T;
    static constexpr int BYTES = ROWS * T::ROWB, NINST = BYTES / 1024, NI = (NINST + BWD_WAVES - 1) / BWD_WAVES;
    static_assert(BYTES % 1024 == 0 && NINST % NI == 0, "whole load instructions; a wave has NI of them or none, which the waits count on");
    int row[NI], col[NI];
    __device__ void init(int wave, int lane) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int off = (wave * NI + i) * 1024 + lane * 16;
            row[i] = off / T::ROWB;
            const int c = ((off % T::ROWB) >> 4) ^ T::swz(row[i]);
            col[i] = c < T::CPR ? c * 16 : -1;
        }
    }
    __device__ __forceinline__ void issue(unsigned char* dst, int wave, const bf16_t* src, int ld, int rows) const {
#if defined(__HIP_DEVICE_COMPILE__)
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(src), 0, min(rows, ROWS) * ld * 2, 0x00020000);
#pragma unroll
        for (int i = 0; i < NI; ++i)
            if (NINST % BWD_WAVES == 0 || wave * NI + i < NINST)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_ptr)(dst + (wave * NI + i) * 1024), 16,
                                                         col[i] < 0 ? -1 : row[i] * ld * 2 + col[i], 0, 0, 0);
#endif
    }
};

template <int HD>
constexpr int STAGES = HD == 128 ? 2 : 3;     // tiles under way: the one that is worked, and those that are loading
// A wave's loads but the last IN_FLIGHT have landed; behind the barrier every wave's have.
template <int IN_FLIGHT>
__device__ __forceinline__ void landed() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(sp_waitcnt(IN_FLIGHT, 15));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ f32x16_t zeros() {
    f32x16_t z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    return z;
}

struct BwdDev {
    const bf16_t *qkv, *dO;
    const float *lse, *minus_delta;
    bf16_t* dqkv;
    const int* cu;
    int n, T, Hq, Hkv, causal;
    float scale, scale_log2e;
};

__device__ __forceinline__ int near_heads(int i, int heads) { return heads & 7 ? i : (i & 7) * (heads >> 3) + (i >> 3); }

// -------------------------------------------------------------------------------------------------- dq
template <int HD>
struct DqCfg {
    typedef TokTile<HD> T;
    static constexpr int STAGE = 2 * T::BYTES, LDS = STAGES<HD> * STAGE;      // {K, V} of 64 keys
};

template <int HD>
__device__ __forceinline__ void dq_group(const BwdDev& g, unsigned char* smem, int id) {
    typedef TokTile<HD> T;
    typedef DqCfg<HD> C;
    constexpr int KEYS = T::ROWS, NK = T::NKS, NV = 2 * T::NMT, PF = 3;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int Hq = g.Hq, Hkv = g.Hkv, grp = Hq / Hkv, ld = (Hq + 2 * Hkv) * HD;
    const int slot = id / Hq, h = near_heads(id - slot * Hq, Hq);
    const PackedBlock pb = packed_block<128>(g.cu, g.n, g.T, slot);
    const int q0 = pb.blk * 128, len = pb.len;
    if (q0 >= len) return;
    const int wq0 = q0 + wave * 32, qi = wq0 + l32;
    const size_t tok0 = pb.row0, row0 = (size_t)h * g.T + tok0;
    const int qr = min(qi, len - 1);
    const bf16_t* kbase = g.qkv + tok0 * ld + (size_t)(Hq + h / grp) * HD;
    const bf16_t* vbase = kbase + (size_t)Hkv * HD;
    const int ntiles = ((g.causal ? min(len, q0 + 128) : len) + KEYS - 1) / KEYS;
    const int mine = wq0 >= len ? 0 : ((g.causal ? min(len, wq0 + 32) : len) + KEYS - 1) / KEYS;
    TileLoad<HD, KEYS> tl;
    tl.init(wave, lane);
    auto issue = [&](int t) __attribute__((always_inline)) {
        unsigned char* st = smem + t % STAGES<HD> * C::STAGE;
        tl.issue(st, wave, kbase + (size_t)t * KEYS * ld, ld, len - t * KEYS);
        tl.issue(st + T::BYTES, wave, vbase + (size_t)t * KEYS * ld, ld, len - t * KEYS);
    };
    bf16x8_t qf[NK], dof[NK];
    {
        const bf16_t* qp = g.qkv + (tok0 + qr) * ld + h * HD + half * 8;
        const bf16_t* dp = g.dO + (tok0 + qr) * (size_t)(Hq * HD) + h * HD + half * 8;
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
            qf[ks] = *reinterpret_cast<const bf16x8_t*>(qp + ks * 16);
            dof[ks] = *reinterpret_cast<const bf16x8_t*>(dp + ks * 16);
        }
    }
    const float lse_q = g.lse[row0 + qr] * LOG2E, minus_delta = g.minus_delta[row0 + qr];
    issue(0);
    if (STAGES<HD> > 2 && ntiles > 1) issue(1);
    FragAt<HD> at;
    at.init(lane);
    f32x16_t acc[T::NMT];
#pragma unroll
    for (int t = 0; t < T::NMT; ++t) acc[t] = zeros();

    auto mask_scores = [&](f32x16_t& s, int key0) __attribute__((always_inline)) {
        const int last = min(len - 1, g.causal ? qi : len - 1) - key0 - 4 * half;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = (e >> 2) * 8 + (e & 3) <= last ? s[e] : -INFINITY;
    };
    // 32 keys: dP beside P (which takes the place of the scores), from the V rows at base_v
    auto probs = [&](f32x16_t& s, f32x16_t& dp, int base, int off) __attribute__((always_inline)) {
        bf16x8_t vf[NK];
#pragma unroll
        for (int i = 0; i < PF; ++i) vf[i] = at.row(smem, base, i, off);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            if (i + PF < NK) vf[i + PF] = at.row(smem, base, i + PF, off);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], dof[i], i ? dp : zeros(), 0, 0, 0);
#pragma unroll
            for (int e = 16 * i / NK; e < 16 * (i + 1) / NK; ++e) {
                float p = __builtin_amdgcn_exp2f(fmaf(s[e], g.scale_log2e, -lse_q));
                asm volatile("" : "+v"(p));
                s[e] = p;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // dS of 32 keys (P in s) beside the next scores, if any, from the K rows at base_k
    auto grads = [&](const f32x16_t& s, const f32x16_t& dp, u32x4_t (&ds)[2], f32x16_t& s_next, int base, int off, bool next) __attribute__((always_inline)) {
        bf16x8_t kf[NK];
        if (next) {
#pragma unroll
            for (int i = 0; i < PF; ++i) kf[i] = at.row(smem, base, i, off);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            if (next) {
                if (i + PF < NK) kf[i + PF] = at.row(smem, base, i + PF, off);
                s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i], i ? s_next : zeros(), 0, 0, 0);
            }
#pragma unroll
            for (int e = 8 * i / NK; e < 8 * (i + 1) / NK; ++e) {
                uint32_t w = pack2(s[2 * e] * (dp[2 * e] + minus_delta), s[2 * e + 1] * (dp[2 * e + 1] + minus_delta));
                asm volatile("" : "+v"(w));
                ds[e >> 2][e & 3] = w;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto output = [&](const u32x4_t (&ds)[2], int base, int off) __attribute__((always_inline)) {
        bf16x8_t tf[NV];
        auto read = [&](int i) __attribute__((always_inline)) { tf[i] = at.tr(smem, base, i % T::NMT, off + 16 * (i / T::NMT) * T::ROWB); };
#pragma unroll
        for (int i = 0; i < PF; ++i) read(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i + PF < NV) read(i + PF);
            acc[i % T::NMT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tf[i], __builtin_bit_cast(bf16x8_t, ds[i / T::NMT]), acc[i % T::NMT], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto tile = [&](int t, bool mask) __attribute__((always_inline)) {
        constexpr int HALF = 32 * T::ROWB;
        const int st = t % STAGES<HD> * C::STAGE;
        f32x16_t sa, sb, dp;
        u32x4_t ds[2];
        {
            bf16x8_t kf[NK];
#pragma unroll
            for (int i = 0; i < NK; ++i) kf[i] = at.row(smem, st, i, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NK; ++i) sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i], i ? sa : zeros(), 0, 0, 0);
        }
        if (mask) mask_scores(sa, t * KEYS);
        probs(sa, dp, st, T::BYTES);
        grads(sa, dp, ds, sb, st, HALF, true);
        output(ds, st, 0);
        if (mask) mask_scores(sb, t * KEYS + 32);
        probs(sb, dp, st, T::BYTES + HALF);
        grads(sb, dp, ds, sa, st, 0, false);
        output(ds, st, HALF);
    };
    // one barrier per tile for every wave; the diagonal and a ragged end lie in a wave's last tile
    int t = 0;
    auto enter = [&]() __attribute__((always_inline)) {
        if (STAGES<HD> > 2 && t + 1 < ntiles) landed<2 * TileLoad<HD, KEYS>::NI>();
        else landed<0>();
        if (t + STAGES<HD> - 1 < ntiles) issue(t + STAGES<HD> - 1);
    };
    enter();
    if (mine > 0) {
        while (t + 1 < mine) {
            tile(t, false);
            ++t;
            enter();
        }
        tile(t, true);
    }
    while (t + 1 < ntiles) {
        ++t;
        enter();
    }
    if (qi < len) {
        bf16_t* op = g.dqkv + (tok0 + qi) * ld + h * HD;
#pragma unroll
        for (int mt = 0; mt < T::NMT; ++mt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int e0 = mt * 32 + k * 8 + half * 4;
                if (e0 < HD)
                    *reinterpret_cast<uint2*>(op + e0) = make_uint2(pack2(acc[mt][k * 4] * g.scale, acc[mt][k * 4 + 1] * g.scale),
                                                                    pack2(acc[mt][k * 4 + 2] * g.scale, acc[mt][k * 4 + 3] * g.scale));
            }
    }
}

// ---------------------------------------------------------------------------------------------- dk, dv
// Wave w takes the 32 keys of group w % KG (one key per lane as the B operand of S = Q K^T and dP = dO V^T) against the 32
// queries of part w / KG of each tile; the parts' sums are added through LDS at the end.
template <int HD, int KG>
struct DkvCfg {
    typedef TokTile<HD> T;
    static constexpr int SUBS = BWD_WAVES / KG, ROWS = 32 * SUBS, KEYS = 32 * KG;
    static constexpr bool K_IN_LDS = HD == 128;       // K fragments would not fit beside the accumulators
    static constexpr int TILE = ROWS * T::ROWB, STAGE = 2 * TILE;
    // k-steps of the keys that are kept there, 32 keys of a k-step in the order of a wave's lanes; all, or all but one where
    // two work-groups fit a CU only so: that one is read again for every tile
    static constexpr int KSTEP = KEYS * 32, KIN = !K_IN_LDS ? 0 : 2 * STAGE + T::NKS * KSTEP + 4 * ROWS * 4 <= 80 * 1024 ? T::NKS : T::NKS - 1;
    static constexpr int KBYTES = KIN * KSTEP;
    static constexpr int bytes(int stages) { return stages * STAGE + KBYTES + stages * 2 * ROWS * 4; }
    static constexpr int STG = HD == 128 || bytes(3) > 80 * 1024 ? 2 : 3;
    static constexpr int LDS = std::max(bytes(STG), SUBS > 1 ? (SUBS - 1) * KG * T::NMT * 16 * 256 : 0);
};

template <int HD, int KG>
__device__ __forceinline__ void dkv_group(const BwdDev& g, unsigned char* smem, int id) {
    typedef TokTile<HD> T;
    typedef DkvCfg<HD, KG> C;
    constexpr int NK = T::NKS, NV = 2 * T::NMT, PF = HD == 128 ? 2 : 3;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5, kg = wave % KG, sub = wave / KG;
    const int Hq = g.Hq, Hkv = g.Hkv, grp = Hq / Hkv, ld = (Hq + 2 * Hkv) * HD, ld_do = Hq * HD;
    const int slot = id / Hkv, kvh = near_heads(id - slot * Hkv, Hkv);
    const PackedBlock pb = packed_block<C::KEYS>(g.cu, g.n, g.T, slot);
    const int len = pb.len;
    if (pb.blk * C::KEYS >= len) return;
    // under a causal mask the first block has the most queries
    const int blk = g.causal ? (len - 1) / C::KEYS - pb.blk : pb.blk;
    const int k0 = blk * C::KEYS, wk0 = k0 + kg * 32, kj = wk0 + l32;
    const size_t tok0 = pb.row0;
    const bf16_t* kbase = g.qkv + tok0 * ld + (size_t)(Hq + kvh) * HD;
    const bf16_t* vbase = kbase + (size_t)Hkv * HD;
    unsigned char* sKeys = smem + C::STG * C::STAGE;
    float* rowvals = reinterpret_cast<float*>(smem + C::STG * C::STAGE + C::KBYTES);       // [stage][lse | -delta][ROWS]

    // the tiles in walking order: (query head of the group, ROWS queries)
    const int q_begin = g.causal ? k0 / C::ROWS * C::ROWS : 0;
    const int per_head = (len - q_begin + C::ROWS - 1) / C::ROWS, n_tiles = grp * per_head;
    TileLoad<HD, C::ROWS> tl;
    tl.init(wave, lane);
    constexpr int NR = (C::ROWS + 63) / 64;           // load instructions of a tile's row values
    int f_head = 0, f_q = q_begin;                    // of the tile fetched next
    auto fetch = [&](int stage) __attribute__((always_inline)) {
        const int h = kvh * grp + f_head;
        unsigned char* st = smem + stage * C::STAGE;
        tl.issue(st, wave, g.qkv + (tok0 + f_q) * ld + (size_t)h * HD, ld, len - f_q);
        tl.issue(st + C::TILE, wave, g.dO + (tok0 + f_q) * ld_do + (size_t)h * HD, ld_do, len - f_q);
        // wave 0 the rows' log-sum-exps, wave 1 their -deltas
#if defined(__HIP_DEVICE_COMPILE__)
        if (wave < 2 && lane < C::ROWS) {
            const float* src = (wave ? g.minus_delta : g.lse) + (size_t)h * g.T + tok0 + f_q;
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(src), 0, min(len - f_q, C::ROWS) * 4, 0x00020000);
#pragma unroll
            for (int i = 0; i < NR; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_ptr)(rowvals + (stage * 2 + wave) * C::ROWS + i * 64), 4,
                                                         (i * 64 + lane) * 4, 0, 0, 0);
        }
#endif
        f_q += C::ROWS;
        if (f_q >= len) { f_q = q_begin; ++f_head; }
    };
    if (C::K_IN_LDS) {
#if defined(__HIP_DEVICE_COMPILE__)
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(kbase + (size_t)k0 * ld), 0, min(len - k0, C::KEYS) * ld * 2, 0x00020000);
#pragma unroll
        for (int i = 0; i < (C::KIN * KG + BWD_WAVES - 1) / BWD_WAVES; ++i) {
            const int j = wave + i * BWD_WAVES;
            if (j < C::KIN * KG)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_ptr)(sKeys + j * 1024), 16, (j % KG * 32 + l32) * ld * 2 + half * 16,
                                                         j / KG * 32, 0, 0);
        }
#endif
    }
    bf16x8_t kf_reg[NK], vf[NK];                      // kf_reg: of the k-steps that are not in LDS
    const size_t krow = (size_t)min(kj, len - 1) * ld + half * 8;
#pragma unroll
    for (int ks = 0; ks < NK; ++ks) {
        if (!C::K_IN_LDS) kf_reg[ks] = *reinterpret_cast<const bf16x8_t*>(kbase + krow + ks * 16);
        vf[ks] = *reinterpret_cast<const bf16x8_t*>(vbase + krow + ks * 16);
    }
    // The k-step that is neither in LDS nor, but between two tiles, in registers: its load lands with the next tile's.
    auto k_again = [&]() __attribute__((always_inline)) {
        size_t row = krow;
        asm volatile("" : "+v"(row));                 // not the load before
        kf_reg[NK - 1] = *reinterpret_cast<const bf16x8_t*>(kbase + row + (NK - 1) * 16);
    };
    if constexpr (C::K_IN_LDS && C::KIN < NK) k_again();
    FragAt<HD> at;
    at.init(lane);
    f32x16_t dk[T::NMT], dv[T::NMT];
#pragma unroll
    for (int t = 0; t < T::NMT; ++t) { dk[t] = zeros(); dv[t] = zeros(); }

    fetch(0);
    if (C::STG > 2 && n_tiles > 1) fetch(1);
    int qs = q_begin + sub * 32;                      // this wave's first query of the tile
    constexpr int NL = 2 * TileLoad<HD, C::ROWS>::NI; // a wave's loads of a tile, without the row values
    for (int tile = 0, stage = 0; tile < n_tiles; ++tile) {
        // the tile is there; everybody is done with the one before it, whose stage the next fetch takes
        if (C::STG == 2 || tile + 1 == n_tiles) landed<0>();
        else if (wave < 2) landed<NL + NR>();
        else landed<NL>();
        if (tile + C::STG - 1 < n_tiles) fetch(stage ? stage - 1 : C::STG - 1);
        const int q_at = stage * C::STAGE + sub * 32 * T::ROWB;
        const float* lrow = rowvals + stage * 2 * C::ROWS + sub * 32 + half * 4;
        // wave-uniform skips: every query of the part precedes this wave's keys, none exists, no key exists
        if (!(qs >= len || wk0 >= len || (g.causal && qs + 31 < wk0))) {
            f32x16_t s, dp;
            u32x4_t pw[2], ds[2];
            bf16x8_t qf[NK], kf[NK], df[NK], tv[NV], tk[NV];
            float4 l4[4];
            auto read_s = [&](int i) __attribute__((always_inline)) {
                qf[i] = at.row(smem, q_at, i, 0);
                kf[i] = i < C::KIN ? lds_b128(sKeys + i * C::KSTEP + kg * 1024 + lane * 16) : kf_reg[i];
            };
            auto read_p = [&](int i) __attribute__((always_inline)) { df[i] = at.row(smem, q_at, i, C::TILE); };
            auto read_v = [&](int i) __attribute__((always_inline)) { tv[i] = at.tr(smem, q_at, i % T::NMT, C::TILE + 16 * (i / T::NMT) * T::ROWB); };
            auto read_k = [&](int i) __attribute__((always_inline)) { tk[i] = at.tr(smem, q_at, i % T::NMT, 16 * (i / T::NMT) * T::ROWB); };
            // Four phases of MFMAs.  Each reads its fragments PF ahead, and with its last MFMAs the first ones of the next phase.
            // S:
#pragma unroll
            for (int i = 0; i < PF; ++i) read_s(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                if (i + PF < NK) read_s(i + PF);
                else read_p(i + PF - NK);
                if (i + 1 == NK) l4[0] = lds_f4(lrow);
                if (i + 2 >= NK) {                        // dP begins at -delta
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float4 d = lds_f4(lrow + C::ROWS + ((i + 2 - NK) * 2 + k) * 8);
                        const int e = ((i + 2 - NK) * 2 + k) * 4;
                        dp[e] = d.x; dp[e + 1] = d.y; dp[e + 2] = d.z; dp[e + 3] = d.w;
                    }
                }
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[i], kf[i], i ? s : zeros(), 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if ((g.causal && qs < wk0 + 31) || qs + 32 > len) {
                // element e is query qs + 4 half + (e >> 2) * 8 + (e & 3)
                const int first = (g.causal ? kj : 0) - qs - 4 * half, end = len - qs - 4 * half;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int q = (e >> 2) * 8 + (e & 3);
                    s[e] = q >= first && q < end ? s[e] : -INFINITY;
                }
            }
            if constexpr (C::K_IN_LDS && C::KIN < NK) k_again();
            // dP beside P, which takes the place of the scores; row values a step ahead of their use: registers are short here
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                if (i + PF < NK) read_p(i + PF);
                else read_v(i + PF - NK);
#pragma unroll
                for (int k = 1; k < 4; ++k)
                    if (step_of(2 * k, NK, 8) == i + 1) l4[k] = lds_f4(lrow + k * 8);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(df[i], vf[i], dp, 0, 0, 0);
#pragma unroll
                for (int e = 8 * i / NK; e < 8 * (i + 1) / NK; ++e) {
                    const float4 l = l4[e >> 1];
                    const float a = __builtin_amdgcn_exp2f(fmaf(s[2 * e], g.scale_log2e, -LOG2E * ((e & 1) ? l.z : l.x)));
                    const float b = __builtin_amdgcn_exp2f(fmaf(s[2 * e + 1], g.scale_log2e, -LOG2E * ((e & 1) ? l.w : l.y)));
                    uint32_t w = pack2(a, b);
                    asm volatile("" : "+v"(w));
                    pw[e >> 2][e & 3] = w;
                    s[2 * e] = a;
                    s[2 * e + 1] = b;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // dV beside dS
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i + PF < NV) read_v(i + PF);
                else read_k(i + PF - NV);
                dv[i % T::NMT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tv[i], __builtin_bit_cast(bf16x8_t, pw[i / T::NMT]), dv[i % T::NMT], 0, 0, 0);
#pragma unroll
                for (int e = 8 * i / NV; e < 8 * (i + 1) / NV; ++e) {
                    uint32_t w = pack2(s[2 * e] * dp[2 * e], s[2 * e + 1] * dp[2 * e + 1]);
                    asm volatile("" : "+v"(w));
                    ds[e >> 2][e & 3] = w;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // dK
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i + PF < NV) read_k(i + PF);
                dk[i % T::NMT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tk[i], __builtin_bit_cast(bf16x8_t, ds[i / T::NMT]), dk[i % T::NMT], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        qs += C::ROWS;
        if (qs - sub * 32 >= len) qs = q_begin + sub * 32;
        stage = stage + 1 == C::STG ? 0 : stage + 1;
    }
    // The parts' sums meet in LDS: dK in part 0, dV in the next, added in the order of the parts.
    if (C::SUBS > 1) landed<0>();
    float4* x = reinterpret_cast<float4*>(smem) + lane;
    auto place = [&](int s, int owner) { return ((s < owner ? s : s - 1) * KG + kg) * (T::NMT * 4 * 64); };
    auto give = [&](const f32x16_t* a, int owner) __attribute__((always_inline)) {
        if (sub == owner) return;
#pragma unroll
        for (int t = 0; t < T::NMT; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                x[place(sub, owner) + (t * 4 + k) * 64] = make_float4(a[t][k * 4], a[t][k * 4 + 1], a[t][k * 4 + 2], a[t][k * 4 + 3]);
    };
    auto take = [&](const f32x16_t* a, int owner, int col, float f) __attribute__((always_inline)) {
        if (sub != owner || kj >= len) return;
        bf16_t* out = g.dqkv + (tok0 + kj) * ld + (size_t)(Hq + col + kvh) * HD;
#pragma unroll
        for (int t = 0; t < T::NMT; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < C::SUBS; ++s) {
                    const float4 o = s == owner ? make_float4(a[t][k * 4], a[t][k * 4 + 1], a[t][k * 4 + 2], a[t][k * 4 + 3])
                                                : x[place(s, owner) + (t * 4 + k) * 64];
                    v[0] += o.x; v[1] += o.y; v[2] += o.z; v[3] += o.w;
                }
                const int e0 = t * 32 + k * 8 + half * 4;
                if (e0 < HD) *reinterpret_cast<uint2*>(out + e0) = make_uint2(pack2(v[0] * f, v[1] * f), pack2(v[2] * f, v[3] * f));
            }
    };
    if (C::SUBS > 1) { give(dk, 0); sp_lds_barrier(); }
    take(dk, 0, 0, g.scale);
    if (C::SUBS > 1) { sp_lds_barrier(); give(dv, 1); sp_lds_barrier(); }
    take(dv, C::SUBS > 1 ? 1 : 0, Hkv, 1.0f);
}

// -delta = -rowsum(dO * O), [Hq][T].  HBM-bound: LANES lanes per (token, head), which lie side by side in dO and O, and four such
// rows on their way per lane.
template <int HD>
__global__ __launch_bounds__(256) void minus_delta_kernel(const bf16_t* __restrict__ dO, const bf16_t* __restrict__ o, float* __restrict__ minus_delta,
                                                          int T, int Hq) {
    constexpr int LANES = HD == 64 ? 8 : 16, PER = 256 / LANES, BATCH = 4;
    const int sub = threadIdx.x % LANES, total = T * Hq, first = (int)blockIdx.x * (PER * BATCH) + threadIdx.x / LANES;
    u32x4_t a[BATCH], b[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
        const size_t at = (size_t)min(first + i * PER, total - 1) * HD + min(sub * 8, HD - 8);
        a[i] = *reinterpret_cast<const u32x4_t*>(dO + at);
        b[i] = *reinterpret_cast<const u32x4_t*>(o + at);
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) s = fmaf(bf_hi(a[i][k]), bf_hi(b[i][k]), fmaf(bf_lo(a[i][k]), bf_lo(b[i][k]), s));
        if (sub * 8 >= HD) s = 0.f;
#pragma unroll
        for (int x = LANES / 2; x > 0; x >>= 1) s += __shfl_xor(s, x, 64);
        const int it = first + i * PER;
        if (sub == 0 && it < total) {
            const int tok = it / Hq, h = it - tok * Hq;
            minus_delta[(size_t)h * T + tok] = -s;
        }
    }
}

template <int HD, int KG>
__global__ __launch_bounds__(BWD_WAVES * 64, 2) void attn_packed_bwd_kernel(BwdDev g, int dkv_groups) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_bwd[];
    if ((int)blockIdx.x < dkv_groups) dkv_group<HD, KG>(g, smem_bwd, blockIdx.x);
    else dq_group<HD>(g, smem_bwd, blockIdx.x - dkv_groups);
}

template <int HD, int KG>
hipError_t launch_bwd(hipStream_t st, const PackedBwdArgs& b, const PackedShape& a) {
    constexpr int LDS = std::max(DqCfg<HD>::LDS, DkvCfg<HD, KG>::LDS);
    static LdsLimitOnce lim;
    hipError_t e = lim.set(reinterpret_cast<const void*>(attn_packed_bwd_kernel<HD, KG>), LDS);
    if (e != hipSuccess) return e;
    const float scale = 1.0f / sqrtf((float)HD);
    const BwdDev g{b.qkv, b.dO, b.lse, b.minus_delta, b.dqkv, a.cu, a.n, a.T, a.Hq, a.Hkv, a.causal, scale, scale * LOG2E};
    const long slots = (long)a.T / 128 + a.n;
    const long kv = (((long)a.T / (32 * KG) + a.n) * a.Hkv + 7) / 8 * 8;         // ids of either kind begin on the first XCD
    attn_packed_bwd_kernel<HD, KG><<<dim3((unsigned)(kv + slots * a.Hq)), BWD_WAVES * 64, LDS, st>>>(g, (int)kv);
    return hipGetLastError();
}

// Keys of a dk/dv work-group.  Its chain is the queries of all heads that share them, 32 at a time: with 128 keys per group that
// is what a batch of few groups waits for, with fewer the waves share out the queries and the chain is a half or a quarter.
// But each group loads all queries.  us for 128, 64, 32 keys under a causal mask, inputs in the caches (groups of 128 keys in brackets):
//   head_dim 64:  900 + 200 tokens, 8/4 heads (40) 52 30 22;  3 x 2000, 8/2 (98) 198 108 80;  3000, 8/8 (192) 80 58 68;
//                 8 x 512, 16/16 (640) 42.2 42.5 52.8;  12 x 300, 32/32 (1280) 57 61 83
//   head_dim 80:  1500 + 300, 8/2 (32) 160 89 57;  6 x 700, 32/8 (304) 103 92 146;  8 x 577, 16/16 (704) 59 63 112; 4 x 1000,
//                 8/8 (280), where the chain is one head, 41 46 62
//   head_dim 128: 3 x 2000, 8/2 (98) 266 165;  3000, 8/8 (192) 114 91;  4000, 32/8 (256) 607 438;  6 x 700, 32/8 (304) 131 127;
//                 20 x 200, 32/8 (408) 80 85;  4 x 2048, 64/8 (544) 984 1009;  3000, 12/12 (288) 127 118; 1541 + 1026 + 400, 16/16
//                 (416) 77 85
template <int HD>
hipError_t launch_hd(hipStream_t st, const PackedBwdArgs& b, const PackedShape& a) {
    const int per_group = 4 * (HD == 64 ? 32 : 16);
    minus_delta_kernel<HD><<<(unsigned)(((long)a.T * a.Hq + per_group - 1) / per_group), 256, 0, st>>>(b.dO, b.o, b.minus_delta, a.T, a.Hq);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const long groups = ((long)a.T / 128 + a.n) * a.Hkv;
    if (HD == 128) return groups <= (a.Hq > a.Hkv ? 400 : 288) ? launch_bwd<HD, 2>(st, b, a) : launch_bwd<HD, 4>(st, b, a);
    if constexpr (HD != 128)
        if (groups <= (HD == 64 ? 128 : 64)) return launch_bwd<HD, 1>(st, b, a);
    if (HD == 64 ? groups <= 640 : groups <= 512 && a.Hq > a.Hkv) return launch_bwd<HD, 2>(st, b, a);
    return launch_bwd<HD, 4>(st, b, a);
}

}  // namespace

hipError_t spk_launch_attention_packed_bwd(hipStream_t st, const PackedBwdArgs& b, const PackedShape& a) {
    switch (a.hd) {
        case 64: return launch_hd<64>(st, b, a);
        case 80: return launch_hd<80>(st, b, a);
        case 128: return launch_hd<128>(st, b, a);
        default: return hipErrorInvalidValue;
    }
}
