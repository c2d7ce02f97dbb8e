// Attention over packed prompts: o = softmax(q k^T / sqrt(hd) + mask) v inside each of n sequences whose rows lie one
// behind the other, causal or bidirectional, grouped heads, head_dim in {64, 80, 128}.
//
// As in k_attn.hip the scores are formed transposed, S^T = K Q^T (v_mfma_f32_32x32x16_bf16: a lane holds one query and 16 keys
// of a 32-key step), and the probabilities in bf16 are the B operand of O^T = V^T P^T as they stand; tiles of 64 keys come
// by LDS-DMA and V^T out of the transposing LDS read.
//
// What bounds such a kernel: the softmax arithmetic takes as many cycles on the vector pipe as the products take on the matrix pipe (at
// head_dim 64 nearly twice as many), and the two or three waves of a SIMD do not hide one behind the other.  No unit is full: over
// 5241 tokens, 64/8 heads of 128, the matrix pipes are busy in 48 % of the cycles, vector instructions issue in 55 %, the LDS
// works in 24 % (it reads 256 bytes a cycle, a wave needs 1 KB per MFMA of 32); 3 x 3000, 32/8 heads of 64: 38, 72 and 19 %; 40
// images, 16 heads of 80: 25, 56 and 13 %.
//
// The denominator is the fp32 sum of the unrounded probabilities, so that the log-sum-exp is as exact as fp32 allows.  A
// row of scores that are all -inf gives NaN, as the definition does (0 / 0).
#include "sp_attn.h"
#include "sp_packed.h"

namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bf16x8_t lds_frag(const unsigned char* __restrict__ p) { return *reinterpret_cast<const bf16x8_t*>(p); }

__device__ __forceinline__ f32x16_t zeros() {
    f32x16_t z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    return z;
}

// Maximum of a value over the two half-waves.
__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

constexpr int NW = 4;                    // waves of a work-group
template <int HD>
struct PackedCfg {
    typedef AttnCfg<HD, NW> C;
    static constexpr int STAGES = 2;
    static constexpr int LDS = STAGES * C::STAGE;
    static_assert(LDS <= 160 * 1024, "fits the LDS");
};

template <int HD>
__global__ __launch_bounds__(64 * NW, HD == 128 ? 2 : 3) void attn_packed_kernel(const bf16_t* __restrict__ qkv, const int* __restrict__ cu,
                                                           bf16_t* __restrict__ o, float* __restrict__ lse, int n, int T,
                                                           int Hq, int Hkv, int causal, float scale_log2e) {
    typedef typename PackedCfg<HD>::C C;
    constexpr int QB = C::QB;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_packed[];     // stages of {K tile, V tile}
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    // Slots first, a slot's heads side by side: work-groups then start in the order of a sequence's blocks, longest first,
    // for all heads, and what is left for the end is short.  (Head after head, the last head's longest block started when
    // everything else was all but done.)  Ids go round the eight XCDs, each with its own L2: an XCD gets neighbouring heads,
    // which share keys and values.
    const int slot = blockIdx.x / Hq, hi = blockIdx.x - slot * Hq;
    const int h = Hq & 7 ? hi : (hi & 7) * (Hq >> 3) + (hi >> 3);
    const PackedBlock pb = packed_block<QB>(cu, n, T, slot);
    if (pb.blk * QB >= pb.len) return;
    const int len = pb.len, ld = (Hq + 2 * Hkv) * HD;
    const size_t tok0 = pb.row0;
    [[maybe_unused]] const bf16_t* kbase = qkv + tok0 * ld + (size_t)(Hq + h / (Hq / Hkv)) * HD;
    // Instruction i of a wave lands at byte (wave * NLOAD + i) * 1024 + lane * 16 of a stage; the lane fetches the chunk that the
    // swizzle puts there, as a byte offset from the tile's first key.  Rows behind the sequence and the padding of the
    // 192-byte rows lie outside the buffer that a load is given and land as zeros.
    uint32_t ld_off[C::NLOAD];
#pragma unroll
    for (int i = 0; i < C::NLOAD; ++i) {
        const int off = (wave * C::NLOAD + i) * 1024 + lane * 16;
        const bool isv = off >= C::TILE_BYTES;
        const int rel = off - (isv ? C::TILE_BYTES : 0);
        const int row = rel / C::ROWB, pos = (rel % C::ROWB) >> 4;
        const int c = isv ? pos ^ (C::v_swz(row) << 2) : pos ^ C::k_swz(row);
        ld_off[i] = c < C::CPR ? (uint32_t)(row * ld + (isv ? Hkv * HD : 0) + c * 8) * 2 : 0xffffffffu;
    }
    auto issue = [&](int kt, int stage) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(kbase + (size_t)kt * KB * ld), 0, min(len - kt * KB, KB) * ld * 2,
                                                            0x00020000);
#pragma unroll
        for (int i = 0; i < C::NLOAD; ++i)
            if (wave * C::NLOAD + i < C::NINST)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_ptr)(smem_packed + stage * C::STAGE + (wave * C::NLOAD + i) * 1024), 16,
                                                         ld_off[i], 0, 0, 0);
#endif
    };
    // Lane parts of the fragment addresses.  Rows of 128 and 256 bytes: a k-step, or a 32-row block of V^T, is an exclusive or
    // on top; rows of 192: two k-steps of four chunks are an offset.
    constexpr bool XOR = HD != 80;
    const int kp0 = l32 * C::ROWB + ((half ^ C::k_swz(l32)) << 4), kp1 = l32 * C::ROWB + (((2 | half) ^ C::k_swz(l32)) << 4);
    // Addresses are of the stage at `base`; what lies further on in it is a constant on top, which the read takes as its offset.
    auto k_at = [&](int base, int ks) { return smem_packed + (XOR ? (base + kp0) ^ (ks << 5) : base + ((ks & 1) ? kp1 : kp0) + (ks >> 1) * 64); };
    const int rowv = half * 4 + ((lane & 15) >> 2);
    const int vp0 = rowv * C::ROWB + (C::v_swz(rowv) << 6) + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    auto v_at = [&](int base, int mt) { return smem_packed + (XOR ? (base + vp0) ^ (mt << 6) : base + vp0 + mt * 64); };

    const int q0 = pb.blk * QB, wq0 = q0 + wave * 32, qi = wq0 + l32;
    bf16x8_t qf[C::NKS];
    {
        const bf16_t* qp = qkv + (tok0 + min(qi, len - 1)) * ld + h * HD + half * 8;
#pragma unroll
        for (int ks = 0; ks < C::NKS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(qp + ks * 16);
    }
    f32x16_t oacc[C::NMT];
    float m_run = -3.402823466e38f, l_run = 0.f;       // finite: a step without a visible key then has probabilities 0
#pragma unroll
    for (int t = 0; t < C::NMT; ++t) oacc[t] = zeros();
    const int ntiles = ((causal ? min(len, q0 + QB) : len) + KB - 1) / KB;               // of the work-group
    const int mine = wq0 >= len ? 0 : ((causal ? min(len, wq0 + 32) : len) + KB - 1) / KB;   // of this wave

    // Scores of a tile's first 32 keys, nothing beside them: all fragments are on their way before the first MFMA.
    auto scores = [&](int base, f32x16_t& s) __attribute__((always_inline)) {
        bf16x8_t kf[C::NKS];
#pragma unroll
        for (int ks = 0; ks < C::NKS; ++ks) kf[ks] = lds_frag(k_at(base, ks));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < C::NKS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], ks ? s : zeros(), 0, 0, 0);
    };
    f32x16_t sa, sb;
    float mx;                                // mx: of the lane's 16 scores of the next step
    // Masks the scores of the 32 keys from key0 on, moves the references that they ask for, and rescales what was summed up to them.
    auto settle = [&](f32x16_t& s, int key0, bool mask) __attribute__((always_inline)) {
        if (mask) {
            // element e is key key0 + 4 half + (e >> 2) * 8 + (e & 3)
            const int last = min(len - 1, causal ? qi : len - 1) - key0 - 4 * half;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = (e >> 2) * 8 + (e & 3) <= last ? s[e] : -INFINITY;
            mx = s[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
        }
        const float top = half_max(mx);
        // the reference follows the maximum lazily, see k_attn.hip
        const bool move = (top - m_run) * scale_log2e > 8.0f;
        const float m_new = move ? top : m_run;
        float alpha = move ? __builtin_amdgcn_exp2f((m_run - m_new) * scale_log2e) : 1.0f;
        m_run = m_new;
        if (__any(move)) {
            asm volatile("" : "+v"(alpha));          // keeps the products here: speculated they cost their time in every step, and 64 registers
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < C::NMT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[t][e] *= alpha;
        }
    };
    // One step of 32 keys, settled scores s: the next step's scores beside the probabilities of this one, then its output beside
    // the maximum of the next.  The order is the source's: fragments are read PF ahead of the MFMA that takes them, and each
    // MFMA is followed by its share of the vector arithmetic (left to the compiler, every read was waited for at once; the
    // empty asm statements keep it from sinking the arithmetic to its use).
    auto step = [&](f32x16_t& s, f32x16_t& s_next, int base, int off_v, int off_k, bool next) __attribute__((always_inline)) {
        constexpr int NK = C::NKS, NV = 2 * C::NMT, PF = NK < 5 ? NK : 5;
        u32x4_t p[2];
        bf16x8_t kf[NK], vf[NV];
        const float m_scaled = m_run * scale_log2e;
        float sum = 0.f;
        auto kread = [&](int i) __attribute__((always_inline)) { kf[i] = lds_frag(k_at(base, i) + off_k); };
        auto vread = [&](int i) __attribute__((always_inline)) {
            const unsigned char* vp = v_at(base, i % C::NMT) + off_v + 16 * (i / C::NMT) * C::ROWB;
            const s16x4_t lo = sp_tr_read((lds_s16x4_ptr)(vp));
            const s16x4_t hi = sp_tr_read((lds_s16x4_ptr)(vp + 8 * C::ROWB));
            vf[i] = __builtin_bit_cast(bf16x8_t, s16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        };
#pragma unroll
        for (int i = 0; i < PF; ++i)
            if (next) kread(i);
        // Ahead of the wave that shares the SIMD until half of the output is done: the two then work different parts (2 x 2000
        // tokens, 32/8 heads: 77 us for 83; 64/8 heads over 5241: 274 for 279).  Three waves to a SIMD, at head_dim 64 and 80,
        // lose by it (40 sequences of 52 to 571, 16 heads of 80: 41.6 for 40.9).
        if constexpr (HD == 128) __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            if (i + PF >= NK) vread(i + PF - NK);
            else if (next) kread(i + PF);
            if (next) s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i], i ? s_next : zeros(), 0, 0, 0);
#pragma unroll
            for (int e = 8 * i / NK; e < 8 * (i + 1) / NK; ++e) {
                const float v = __builtin_amdgcn_exp2f(fmaf(s[2 * e], scale_log2e, -m_scaled));
                const float w = __builtin_amdgcn_exp2f(fmaf(s[2 * e + 1], scale_log2e, -m_scaled));
                sum += v + w;
                uint32_t pw = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)v, (__bf16)w});      // at most 256: half a step of bf16, as every operand of the products
                asm volatile("" : "+v"(pw));
                p[e >> 2][e & 3] = pw;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        l_run += sum;
        if (next) mx = s_next[0];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (HD == 128)
                if (i == NV / 2) __builtin_amdgcn_s_setprio(0);
            if (i + PF < NV) vread(i + PF);
            oacc[i % C::NMT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], __builtin_bit_cast(bf16x8_t, p[i / C::NMT]), oacc[i % C::NMT], 0, 0, 0);
            if (next) {
#pragma unroll
                for (int e = 16 * i / NV; e < 16 * (i + 1) / NV; ++e) mx = fmaxf(mx, s_next[e]);
                asm volatile("" : "+v"(mx));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr int HALF = 32 * C::ROWB;
    // A tile, the scores of whose first half are there; the second half's come beside its softmax.  (To take the next
    // tile's first scores beside the second half as well needs a third stage: one work-group of eight waves per CU instead of
    // two of four, 333 us for the 274 of 64/8 heads of 128 over 3333 + 130 + 1 + 1777 tokens.)
    auto body = [&](int cur, int key0, bool mask) __attribute__((always_inline)) {
        settle(sa, key0, mask);
        step(sa, sb, cur, C::TILE_BYTES, HALF, true);
        settle(sb, key0 + 32, mask);
        step(sb, sa, cur, C::TILE_BYTES + HALF, 0, false);
    };
    auto enter = [&](int kt) __attribute__((always_inline)) {
        // tile kt has landed, this wave's part by the wait, everybody's by the barrier; and everybody is done with tile kt - 1,
        // whose stage tile kt + 1 takes
        __builtin_amdgcn_s_waitcnt(sp_waitcnt(0, 15));
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (kt + 1 < ntiles) issue(kt + 1, (kt + 1) & 1);
    };
    issue(0, 0);
    // One barrier per tile for every wave, whatever it has to do in it.  The diagonal and a ragged end lie in a wave's last
    // tile: it alone is masked, outside the loop.
    int kt = 0;
    enter(0);
    if (mine > 0) {
        auto begin = [&]() __attribute__((always_inline)) {
            scores((kt & 1) * C::STAGE, sa);
            mx = sa[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sa[e]);
        };
        begin();
        for (; kt + 1 < mine;) {
            body((kt & 1) * C::STAGE, kt * KB, false);
            enter(++kt);
            begin();
        }
        body((kt & 1) * C::STAGE, kt * KB, true);
    }
    while (kt + 1 < ntiles) {
        enter(++kt);
    }
    const float l = l_run + __shfl_xor(l_run, 32, 64);
    if (qi >= len) return;
    const float inv = 1.0f / l;
    bf16_t* op = o + (tok0 + qi) * (size_t)(Hq * HD) + h * HD;
#pragma unroll
    for (int mt = 0; mt < C::NMT; ++mt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int e0 = mt * 32 + g * 8 + half * 4;
            if (e0 < HD)
                *reinterpret_cast<uint2*>(op + e0) = make_uint2(pack_bf2(oacc[mt][g * 4] * inv, oacc[mt][g * 4 + 1] * inv),
                                                                pack_bf2(oacc[mt][g * 4 + 2] * inv, oacc[mt][g * 4 + 3] * inv));
        }
    if (lse && half == 0) lse[(size_t)h * T + tok0 + qi] = m_run * scale_log2e * 0.69314718055994530942f + logf(l);
}

// The same for batches of few blocks: a work-group has 32 queries of one head and its four waves share out the keys, wave w
// the steps of 32 keys w, w + 4, ...  A wave loads its steps into two LDS buffers of its own and waits for nobody; at the
// end the waves' outputs, sums and maxima meet in LDS and are added in wave order.  What bounds such a batch is the chain
// of one wave, which is a quarter as long so.
template <int HD>
struct SplitCfg {
    typedef AttnCfg<HD, 1> C;
    static constexpr int WAVES = 4, TILE = 32 * C::ROWB, BUF = 2 * TILE;        // K rows, then V rows
    static constexpr int NI = BUF / 1024;                                      // load instructions of a step
    static constexpr int MERGE = WAVES * (C::NMT * 16 + 2) * 64 * 4, LOOP = WAVES * 2 * BUF;
    static constexpr int LDS = MERGE > LOOP ? MERGE : LOOP;
    static_assert(TILE % 1024 == 0 && LDS <= 160 * 1024, "whole load instructions, and they fit the LDS");
};

template <int HD>
__global__ __launch_bounds__(256, 1) void attn_packed_split_kernel(const bf16_t* __restrict__ qkv, const int* __restrict__ cu,
                                                                 bf16_t* __restrict__ o, float* __restrict__ lse, int n, int T, int Hq,
                                                                 int Hkv, int causal, float scale_log2e) {
    typedef SplitCfg<HD> G;
    typedef typename G::C C;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_split[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int slot = blockIdx.x / Hq, hi = blockIdx.x - slot * Hq;
    const int h = Hq & 7 ? hi : (hi & 7) * (Hq >> 3) + (hi >> 3);
    const PackedBlock pb = packed_block<32>(cu, n, T, slot);
    const int len = pb.len, q0 = pb.blk * 32, qi = q0 + l32, ld = (Hq + 2 * Hkv) * HD;
    if (q0 >= len) return;
    const size_t tok0 = pb.row0;
    [[maybe_unused]] const bf16_t* kbase = qkv + tok0 * ld + (size_t)(Hq + h / (Hq / Hkv)) * HD;
    const int steps = ((causal ? min(len, q0 + 32) : len) + 31) / 32;
    auto issue = [&](int i) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(kbase + (size_t)i * 32 * ld), 0, min(len - i * 32, 32) * ld * 2,
                                                            0x00020000);
#pragma unroll
        for (int k = 0; k < G::NI; ++k) {
            const bool isv = k * 1024 >= G::TILE;
            const int rel = k * 1024 + lane * 16 - (isv ? G::TILE : 0), row = rel / C::ROWB, pos = (rel % C::ROWB) >> 4;
            const int c = isv ? pos ^ (C::v_swz(row) << 2) : pos ^ C::k_swz(row);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_ptr)(smem_split + (wave * 2 + ((i >> 2) & 1)) * G::BUF + k * 1024), 16,
                                                     c < C::CPR ? (row * ld + (isv ? Hkv * HD : 0) + c * 8) * 2 : -1, 0, 0, 0);
        }
#endif
    };
    if (wave < steps) issue(wave);
    bf16x8_t qf[C::NKS];
    {
        const bf16_t* qp = qkv + (tok0 + min(qi, len - 1)) * ld + h * HD + half * 8;
#pragma unroll
        for (int ks = 0; ks < C::NKS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(qp + ks * 16);
    }
    const int rowv = half * 4 + ((lane & 15) >> 2);
    f32x16_t acc[C::NMT];
#pragma unroll
    for (int t = 0; t < C::NMT; ++t) acc[t] = zeros();
    float m_run = -3.402823466e38f, l_run = 0.f;       // finite: a wave may hold no key that a query sees
    for (int i = wave; i < steps; i += G::WAVES) {
        // the last user of the other buffer has read it: every fragment went into an MFMA
        if (i + G::WAVES < steps) {
            issue(i + G::WAVES);
            __builtin_amdgcn_s_waitcnt(sp_waitcnt(G::NI, 15));
        } else {
            __builtin_amdgcn_s_waitcnt(sp_waitcnt(0, 15));
        }
        asm volatile("" ::: "memory");
        const unsigned char* sK = smem_split + (wave * 2 + ((i >> 2) & 1)) * G::BUF;
        bf16x8_t kf[C::NKS];
#pragma unroll
        for (int ks = 0; ks < C::NKS; ++ks) kf[ks] = lds_frag(sK + l32 * C::ROWB + (((2 * ks + half) ^ C::k_swz(l32)) << 4));
        s16x4_t lo[2 * C::NMT], hi4[2 * C::NMT];
#pragma unroll
        for (int k = 0; k < 2 * C::NMT; ++k) {
            const int mt = k % C::NMT, j = k / C::NMT;
            const unsigned char* vp = sK + G::TILE + (rowv + 16 * j) * C::ROWB + ((mt ^ C::v_swz(rowv)) << 6) + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
            lo[k] = sp_tr_read((lds_s16x4_ptr)(vp));
            hi4[k] = sp_tr_read((lds_s16x4_ptr)(vp + 8 * C::ROWB));
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x16_t s;
#pragma unroll
        for (int ks = 0; ks < C::NKS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], ks ? s : zeros(), 0, 0, 0);
        if (i * 32 + 32 > len || (causal && i * 32 + 31 > q0)) {
            const int last = min(len - 1, causal ? qi : len - 1) - i * 32 - 4 * half;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = (e >> 2) * 8 + (e & 3) <= last ? s[e] : -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
        const float top = half_max(mx);
        const bool move = (top - m_run) * scale_log2e > 8.0f;
        const float m_new = move ? top : m_run;
        float alpha = move ? __builtin_amdgcn_exp2f((m_run - m_new) * scale_log2e) : 1.0f;
        m_run = m_new;
        if (__any(move)) {
            asm volatile("" : "+v"(alpha));
            l_run *= alpha;
#pragma unroll
            for (int t = 0; t < C::NMT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[t][e] *= alpha;
        }
        u32x4_t p[2];
        const float m_scaled = m_new * scale_log2e;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = __builtin_amdgcn_exp2f(fmaf(s[2 * e], scale_log2e, -m_scaled));
            const float w = __builtin_amdgcn_exp2f(fmaf(s[2 * e + 1], scale_log2e, -m_scaled));
            sum += v + w;
            p[e >> 2][e & 3] = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)v, (__bf16)w});
        }
        l_run += sum;
#pragma unroll
        for (int k = 0; k < 2 * C::NMT; ++k) {
            const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, s16x8_t{lo[k][0], lo[k][1], lo[k][2], lo[k][3], hi4[k][0], hi4[k][1], hi4[k][2], hi4[k][3]});
            acc[k % C::NMT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8_t, p[k / C::NMT]), acc[k % C::NMT], 0, 0, 0);
        }
    }
    const float l = l_run + __shfl_xor(l_run, 32, 64);
    __syncthreads();                          // the buffers are free
    float4* rows = reinterpret_cast<float4*>(smem_split);                        // [wave][group of four rows][lane]
    float* ml = reinterpret_cast<float*>(smem_split) + G::WAVES * C::NMT * 16 * 64;      // [wave][maximum, sum][lane]
#pragma unroll
    for (int t = 0; t < C::NMT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            rows[((wave * C::NMT + t) * 4 + k) * 64 + lane] = make_float4(acc[t][k * 4], acc[t][k * 4 + 1], acc[t][k * 4 + 2], acc[t][k * 4 + 3]);
    ml[(wave * 2) * 64 + lane] = m_run;
    ml[(wave * 2 + 1) * 64 + lane] = l;
    __syncthreads();
    float M = ml[lane], f[G::WAVES], L = 0.f;
#pragma unroll
    for (int w = 1; w < G::WAVES; ++w) M = fmaxf(M, ml[w * 2 * 64 + lane]);
#pragma unroll
    for (int w = 0; w < G::WAVES; ++w) {
        f[w] = __builtin_amdgcn_exp2f((ml[w * 2 * 64 + lane] - M) * scale_log2e);
        L = fmaf(f[w], ml[(w * 2 + 1) * 64 + lane], L);
    }
    if (qi >= len) return;
    const float inv = 1.0f / L;
    bf16_t* op = o + (tok0 + qi) * (size_t)(Hq * HD) + h * HD;
#pragma unroll
    for (int i = 0; i < C::NMT; ++i) {
        const int grp = wave + G::WAVES * i, e0 = grp * 8 + half * 4;            // group of eight rows, four a lane
        if (e0 >= HD) continue;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < G::WAVES; ++w) {
            const float4 r = rows[(w * C::NMT * 4 + grp) * 64 + lane];
            v[0] = fmaf(f[w], r.x, v[0]); v[1] = fmaf(f[w], r.y, v[1]); v[2] = fmaf(f[w], r.z, v[2]); v[3] = fmaf(f[w], r.w, v[3]);
        }
        *reinterpret_cast<uint2*>(op + e0) = make_uint2(pack_bf2(v[0] * inv, v[1] * inv), pack_bf2(v[2] * inv, v[3] * inv));
    }
    if (lse && wave == 0 && half == 0) lse[(size_t)h * T + tok0 + qi] = M * scale_log2e * 0.69314718055994530942f + logf(L);
}

template <int HD>
hipError_t launch_split(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* lse, const PackedShape& a) {
    typedef SplitCfg<HD> G;
    static LdsLimitOnce lds_limit;
    hipError_t e = lds_limit.set(reinterpret_cast<const void*>(attn_packed_split_kernel<HD>), G::LDS);
    if (e != hipSuccess) return e;
    const long slots = (long)a.T / 32 + a.n;
    attn_packed_split_kernel<HD><<<dim3((unsigned)(slots * a.Hq)), 256, G::LDS, st>>>(qkv, a.cu, o, lse, a.n, a.T, a.Hq, a.Hkv, a.causal,
                                                                                     1.4426950408889634f / sqrtf((float)HD));
    return hipGetLastError();
}

template <int HD>
hipError_t launch_packed(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* lse, const PackedShape& a) {
    typedef PackedCfg<HD> G;
    static LdsLimitOnce lds_limit;
    hipError_t e = lds_limit.set(reinterpret_cast<const void*>(attn_packed_kernel<HD>), G::LDS);
    if (e != hipSuccess) return e;
    const int slots = a.T / G::C::QB + a.n;
    attn_packed_kernel<HD><<<dim3((unsigned)((long)slots * a.Hq)), 64 * NW, G::LDS, st>>>(qkv, a.cu, o, lse, a.n, a.T, a.Hq, a.Hkv,
                                                                                             a.causal, 1.4426950408889634f / sqrtf((float)HD));
    return hipGetLastError();
}

// Shared-out keys while the 32-query groups are few: one per CU at head_dim 80, two else, and some more where the sequences are
// long on average (their first blocks have few keys under a causal mask).  us, 128 queries and 32 (groups of 32), inputs in the
// caches / out of memory:
//   head_dim 64:  5 prompts of 1 to 128 tokens, 4 heads (56) 5.9 4.6 / 5.8 4.4;  3000 tokens, 4 heads (376) 40 20 / 40 21;  2 x 1000,
//                 16 heads (1024) 17.7 16.8 / 18.3 21.8;  30 x 100, 8 heads (984) 6.5 9.8 / 7.5 11.0;  3000, 16 heads (1504) 42 41 / 42 48
//   head_dim 80, no mask:  257 tokens, 16 heads (144) 9.6 6.6 / 9.8 6.9;  4 x 257 (576) 9.9 16.5 / 10.6 17.4
//   head_dim 128: 2 x 1000, 8 heads (512) 24 17 / 25 20;  3000, 8 heads (752) 60 45 / 60 47;  3 x 500, 16 heads (784) 15.6 19.4 / 17.1 23.0;
//                 3000, 16 heads (1504) 64 80 / 66 85
// Out of memory, over some 250 shapes each (1 to 8 sequences of 64 to 3000, 128 to 1536 groups), the choice costs 1.7 % on average at head_dim
// 64, 2 (causal) and 4 at 128, 1.7 (no mask) and 8 (causal) at 80 against always the quicker form.  It loses most under a causal mask at
// head_dim 80 with few long sequences, up to 2.2 times, and with a mean length just over 1000, where the bound rises at once.
template <int HD>
hipError_t launch_hd(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* lse, const PackedShape& a) {
    const long groups = ((long)a.T / 32 + a.n) * a.Hq;
    const bool lengthy = a.T / a.n >= 1000;
    const long most = HD == 80 ? 256 : !lengthy ? 512 : HD == 64 ? 1024 : 768;
    return groups <= most ? launch_split<HD>(st, qkv, o, lse, a) : launch_packed<HD>(st, qkv, o, lse, a);
}

}  // namespace

hipError_t spk_launch_attention_packed(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* lse, const PackedShape& a) {
    switch (a.hd) {
        case 64: return launch_hd<64>(st, qkv, o, lse, a);
        case 80: return launch_hd<80>(st, qkv, o, lse, a);
        case 128: return launch_hd<128>(st, qkv, o, lse, a);
        default: return hipErrorInvalidValue;
    }
}
