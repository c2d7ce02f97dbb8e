// A block cache of keys and values in 8 bits: appending to it and single-query attention over it.
//
// One layer's cache is a pool of blocks of BS = 16, 32 or 64 tokens:
//   k8 [blocks][Hkv][BS][hd]   e4m3, a token's head-dimension elements contiguous
//   v8 [blocks][Hkv][hd][BS]   e4m3, an element's tokens contiguous
//   scales fp32 [blocks][Hkv][2]   of a block's keys and values: what is stored is e4m3(x / scale).
// A scale is 2^e, the smallest e >= -126 with max |x| <= 448 * 2^e (448 = the largest e4m3 value).  A power of two costs
// nothing against max / 448 (e4m3 is a floating type: its relative step is the same at every magnitude) and buys
// exactness: x / scale and code * scale are exact, so a stored value is off by the one rounding to e4m3 (half a step,
// 2^-4 relative, 2^-10 scale below 2^-6 scale), and a block whose scale grows while it fills is re-coded by an exact
// shift of the exponent (a second rounding only where a code falls below the normal range).
#include "sp_attn.h"
#include "sp_kernels.h"

namespace {

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float exp2_bits(int biased) { return __uint_as_float((uint32_t)biased << 23); }

// ---------------------------------------------------------------------------------------------- append
// A run is a maximal row of tokens with consecutive slots inside one block.  The keys, and apart from them the values, of one
// block and head are written by one wave or work-group, run after run in the order of the rows, and nobody else touches
// them: a row whose block occurs in the 64 rows before it leaves the block to whoever met it first.
// NL lanes work a run in parts of GROUPS * TPL positions: lane (rg, ch) has TPL neighbouring positions of the elements
// 8 ch .. 8 ch + 7, so that a row of keys leaves in pieces of 8 bytes, and the transposition that the value layout needs
// happens inside the lane.  Between the largest value and the coding a run of one part stays in registers; a longer one is
// read again, out of the cache.
// HBM-bound for prompts (4 bytes read and 2 written per token, head and element), latency-bound for single tokens: their
// block is read again only where its scale grows.

// m tokens from row t on go to the positions off .. of a block.  NL == 256: by the whole work-group, `tops` its four words of LDS.
template <int HD, int BS, int NL>
__device__ __forceinline__ void store_run(const bf16_t* __restrict__ qkv, int ld, int Hq, const Kv8Cache& c, int h, int isv, int t, int m,
                                          int block, int off, int* tops) {
    constexpr int LPR = HD / 8, GROUPS = NL / LPR;                          // lanes per row, rows at a time
    constexpr int TPL = BS >= 4 * GROUPS ? 4 : BS > GROUPS ? BS / GROUPS : 1, PART = GROUPS * TPL;
    const int id = NL == 64 ? threadIdx.x & 63 : threadIdx.x, lane = threadIdx.x & 63;
    // A work-group's wave has all positions of a part for a quarter of the elements of values, whose rows lie along the positions
    // (with a quarter of the positions instead, as for keys, four waves wrote 16 bytes each of a line: 16.0 us for 13.7 over 7 k
    // tokens, 8 heads of 128).
    constexpr int CPW = LPR / 4;
    const bool by_elements = NL > 64 && isv;
    const int rg = by_elements ? lane / CPW : id / LPR, ch = by_elements ? (threadIdx.x >> 6) * CPW + lane % CPW : id % LPR;
    const size_t bh = (size_t)block * c.Hkv + h;
    const bf16_t* src = qkv + (size_t)t * ld + (size_t)(Hq + isv * c.Hkv + h) * HD + ch * 8;
    float* sp = c.scales + bh * 2 + isv;
    const int e_old = off ? min(max((int)((__float_as_uint(*sp) >> 23) & 255), 1), 253) : 0;
    u32x4_t x[TPL];
    const int from = off / PART, to = (off + m - 1) / PART;      // parts that hold new tokens
    auto load = [&](int part) {
#pragma unroll
        for (int i = 0; i < TPL; ++i) {
            const int p = part * PART + rg * TPL + i - off;      // token of the run
            x[i] = u32x4_t{0, 0, 0, 0};
            if (p >= 0 && p < m) x[i] = *reinterpret_cast<const u32x4_t*>(src + (size_t)p * ld);
        }
    };
    uint32_t big = 0;
    for (int part = from; part <= to; ++part) {
        load(part);
#pragma unroll
        for (int i = 0; i < TPL; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const u16x2_t a = __builtin_bit_cast(u16x2_t, x[i][k] & 0x7fff7fffu);
                big = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, big), a));
            }
    }
    auto over_lanes = [&](int v) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
        if (NL > 64) {
            __syncthreads();
            if (lane == 0) tops[threadIdx.x >> 6] = v;
            __syncthreads();
            v = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
        }
        return v;
    };
    int top = over_lanes(max((int)(big & 0xffff), (int)(big >> 16)));
    const bool odd = top >= 0x7f80;                              // infinities or NaN among them: stored as NaN, the scale is the others'
    if (odd) {
        top = 0;
        for (int part = from; part <= to; ++part) {
            load(part);
#pragma unroll
            for (int i = 0; i < TPL; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int lo = x[i][k] & 0x7fff, hi = (x[i][k] >> 16) & 0x7fff;
                    top = max(top, max(lo < 0x7f80 ? lo : 0, hi < 0x7f80 ? hi : 0));
                }
        }
        top = over_lanes(top);
    }
    // biased exponent of the scale: 1.75 * 2^8 is the largest code
    int e = max((top >> 7) - 8 + ((top & 127) > 96 ? 1 : 0), 1);
    e = max(e, e_old);
    const bool grow = off && e > e_old;
    const float inv = exp2_bits(254 - e), shift = exp2_bits(max(127 + e_old - e, 0));
    if (id == 0 && e != e_old) *sp = exp2_bits(e);               // everybody has read the old one: the work-group met in over_lanes
    auto code4 = [&](uint32_t w0, uint32_t w1) {                 // four bf16 values
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(w0) * inv, bf_hi(w0) * inv, 0, false);
        r = __builtin_amdgcn_cvt_pk_fp8_f32(bf_lo(w1) * inv, bf_hi(w1) * inv, r, true);
        if (odd) {
            const uint32_t w[2] = {w0, w1};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t v = w[k >> 1] >> (16 * (k & 1));
                if ((v & 0x7fff) >= 0x7f80) r = (r & ~(255u << (8 * k))) | ((127u | (v >> 8 & 128u)) << (8 * k));
            }
        }
        return (uint32_t)r;
    };
    auto recode4 = [&](uint32_t w) {
        const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(a.x * shift, a.y * shift, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b.x * shift, b.y * shift, r, true);
    };
    for (int part = grow ? 0 : from; part <= to; ++part) {
        if (from != to || grow) load(part);
        const int p0 = part * PART + rg * TPL;
        if (!isv) {
            uint8_t* dst = c.k8 + bh * (BS * HD) + ch * 8;
#pragma unroll
            for (int i = 0; i < TPL; ++i) {
                const int p = p0 + i;
                uint32_t* d = reinterpret_cast<uint32_t*>(dst + p * HD);
                if (p >= off && p < off + m) {
                    *reinterpret_cast<uint2*>(d) = make_uint2(code4(x[i][0], x[i][1]), code4(x[i][2], x[i][3]));
                } else if (grow && p < off) {
                    const uint2 o = *reinterpret_cast<const uint2*>(d);
                    *reinterpret_cast<uint2*>(d) = make_uint2(recode4(o.x), recode4(o.y));
                }
            }
            continue;
        }
        uint8_t* dst = c.v8 + bh * (BS * HD) + (size_t)ch * 8 * BS + p0;
        uint32_t y[TPL][2];
#pragma unroll
        for (int i = 0; i < TPL; ++i) { y[i][0] = code4(x[i][0], x[i][1]); y[i][1] = code4(x[i][2], x[i][3]); }
        if (NL == 64 && m == 1 && !grow) {
            // A single token: a byte of every element's row.  Neighbouring lanes take neighbouring elements, whose rows share
            // lines (8 stores by the 16 lanes that have the token, each to 16 lines: 6.5 us for 5.8, 64 tokens, 32 heads of 128).
            uint32_t t0 = y[0][0], t1 = y[0][1];
#pragma unroll
            for (int i = 1; i < TPL; ++i)
                if (off % TPL == i) { t0 = y[i][0]; t1 = y[i][1]; }
            uint8_t* row = c.v8 + bh * (BS * HD) + off;
#pragma unroll
            for (int j = 0; j < HD / 64; ++j) {
                const int el = j * 64 + lane, from_lane = (off % PART / TPL) * LPR + el / 8;
                const uint32_t w0 = __shfl(t0, from_lane, 64), w1 = __shfl(t1, from_lane, 64);
                row[el * BS] = (uint8_t)((el & 4 ? w1 : w0) >> (8 * (el & 3)));
            }
            continue;
        }
        if (p0 >= off && p0 + TPL <= off + m) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                uint32_t w = 0;
#pragma unroll
                for (int i = 0; i < TPL; ++i) w |= ((y[i][k >> 2] >> (8 * (k & 3))) & 255u) << (8 * i);
                if constexpr (TPL == 4) *reinterpret_cast<uint32_t*>(dst + k * BS) = w;
                else if constexpr (TPL == 2) *reinterpret_cast<uint16_t*>(dst + k * BS) = (uint16_t)w;
                else dst[k * BS] = (uint8_t)w;
            }
        } else if (p0 < off + m && p0 + TPL > (grow ? 0 : off)) {
#pragma unroll
            for (int i = 0; i < TPL; ++i) {
                const int p = p0 + i;
                if (p >= off && p < off + m) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) dst[k * BS + i] = (uint8_t)(y[i][k >> 2] >> (8 * (k & 3)));
                } else if (grow && p < off) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) dst[k * BS + i] = (uint8_t)recode4(dst[k * BS + i]);
                }
            }
        }
    }
}

// ROWS == 1: a wave per row.  ROWS == 64: a work-group per 64 rows; where fewer than four blocks begin in them, as in a prompt, it
// works each run as a whole, else every wave takes every fourth block.  What a run needs to know comes from the slots alone.
template <int HD, int BS, int ROWS>
__global__ __launch_bounds__(256) void kv8_append_kernel(const bf16_t* __restrict__ qkv, const int* __restrict__ slots, int T, int Hq, Kv8Cache c) {
    __shared__ int tops[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ld = (Hq + 2 * c.Hkv) * HD, limit = c.blocks * BS;
    const int isv = blockIdx.y & 1, h = blockIdx.y >> 1;
    const int begin = ROWS == 1 ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x * 64;         // T <= 2^30
    if (begin >= T) return;
    auto slot_at = [&](int row) { return row >= 0 && row < T ? slots[row] : -1; };
    // the rows begin - 64 .. begin - 1, begin .. begin + 63 and begin + 64 .. begin + 127
    const int before = slot_at(begin - 64 + lane), from = slot_at(begin + lane), after = slot_at(begin + 64 + lane);
    const int last_before = __builtin_amdgcn_readlane(before, 63), left = __shfl_up(from, 1, 64), prev = lane ? left : last_before;
    // the slots of row and the 63 behind it, `at` its place behind `begin`; out of the registers where they hold them all
    auto ahead = [&](int at, int row) {
        const int a = __shfl(from, (at + lane) & 63, 64), b = __shfl(after, (at + lane) & 63, 64);
        return at > 64 ? slot_at(row + lane) : at + lane < 64 ? a : b;
    };
    // rows that begin a run, and of those the ones whose block does not occur in the 64 rows in front of them
    unsigned long long first = __ballot(lane < ROWS && from >= 0 && from < limit && (prev != from - 1 || from % BS == 0));
    for (unsigned long long todo = first; todo; todo &= todo - 1) {
        const int i = __builtin_ctzll(todo), block = __builtin_amdgcn_readlane(from, i) / BS;
        const int in_front = lane >= i ? before : from;
        if (__any(in_front >= 0 && in_front / BS == block)) first &= ~(1ull << i);
    }
    const bool together = ROWS > 1 && __popcll(first) < 4;
    for (int turn = 0; first; first &= first - 1, ++turn) {
        if (ROWS > 1 && !together && (turn & 3) != wave) continue;
        int at = __builtin_ctzll(first), t = begin + at, s = __builtin_amdgcn_readlane(from, at);
        const int block = s / BS;
        for (;;) {
            const int off = s % BS;
            // the row's slots follow one another up to the end of the block
            const int slot = ahead(at, t);                                           // by all lanes: it shuffles
            const bool in = lane == 0 || (lane < BS - off && slot == s + lane);      // m >= 1: the loop moves on
            const unsigned long long miss = ~__ballot(in);
            const int m = miss ? __builtin_ctzll(miss) : 64;
            if (together) store_run<HD, BS, 256>(qkv, ld, Hq, c, h, isv, t, m, block, off, tops);
            else store_run<HD, BS, 64>(qkv, ld, Hq, c, h, isv, t, m, block, off, nullptr);
            // the block's next run, if the 64 rows that follow have one; it reads what this one wrote
            at += m;
            const int next = ahead(at, t + m);
            const unsigned long long more = __ballot(next >= 0 && next / BS == block);
            if (!more) break;
            const int gap = __builtin_ctzll(more);
            t += m + gap;
            at += gap;
            s = slots[t];
            __threadfence_block();
            if (together) __syncthreads();
        }
    }
}

template <int HD, int BS>
hipError_t launch_append_bs(hipStream_t st, const bf16_t* qkv, const int* slots, int T, int Hq, const Kv8Cache& c) {
    // The host cannot tell single tokens, which want a wave per row (a work-group of 64 rows works their blocks four at a time), from
    // prompts, which want the work-group: few (row, head) pairs are taken for the former.  us by rows and by work-groups of 64 rows, pairs
    // times two in brackets:  single tokens, 64 of 32 heads of 128 (4096) 5.9 41, 256 (16384) 19 48, 512 of 32 heads of 64
    // (32768) 24 49;  prompts of 8 heads of 128, 300 tokens (4800) 8.8 4.7, 1000 (16000) 12.0 5.6, 1500 (24000) 12.1 6.0;
    // 300 tokens, 32 heads of 128, blocks of 16 (19200) 7.3 8.7.
    const bool wave_per_row = (long)T * c.Hkv * 2 <= 16384;
    if (wave_per_row) kv8_append_kernel<HD, BS, 1><<<dim3((unsigned)((T + 3) / 4), c.Hkv * 2), 256, 0, st>>>(qkv, slots, T, Hq, c);
    else kv8_append_kernel<HD, BS, 64><<<dim3((unsigned)((T + 63) / 64), c.Hkv * 2), 256, 0, st>>>(qkv, slots, T, Hq, c);
    return hipGetLastError();
}

template <int HD>
hipError_t launch_append(hipStream_t st, const bf16_t* qkv, const int* slots, int T, int Hq, const Kv8Cache& c) {
    switch (c.block_size) {
        case 16: return launch_append_bs<HD, 16>(st, qkv, slots, T, Hq, c);
        case 32: return launch_append_bs<HD, 32>(st, qkv, slots, T, Hq, c);
        case 64: return launch_append_bs<HD, 64>(st, qkv, slots, T, Hq, c);
        default: return hipErrorInvalidValue;
    }
}

// ------------------------------------------------------------------------------------------- attention
// o = softmax(q K^T / sqrt(hd)) V for one query per request over its first kv_len positions.
//
// HBM-bound: 2 Hkv hd bytes per position.  A wave walks 64 positions at a time on its own, 16 loads of 16 bytes per lane
// in flight at hd 128.  Both products are v_mfma_f32_16x16x32_bf16 on codes converted to bf16 (exact), the query heads
// that share a key/value head being the 16 columns: S^T = K Q^T, then O^T = V^T P^T.  In the accumulators of S^T a lane
// (column r = head, row group g) holds four rows of a 16-row tile; the rows of the four tiles are assigned to positions so
// that these are the positions 16 g .. 16 g + 15, in the order in which the lane's bytes of a V row come: P^T in bf16 is
// then the B operand as it stands, K and V are read as they lie, and all that a lane weighs belongs to one block -- one
// key scale, which multiplies its scores, and one value scale, which the conversion applies.
constexpr int NW8 = 4;
constexpr float LOWEST = -3.402823466e38f;        // finite: the weight of a score of -inf is then 0

__device__ __forceinline__ bf16x8_t bf16_of_codes(uint32_t a, uint32_t b, float scale) {
    union { bf16x2_t p[4]; bf16x8_t v; } u;
    u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
    u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
    u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return u.v;
}

template <int HD>
__global__ __launch_bounds__(NW8 * 64, 3) void kv8_attn_kernel(const bf16_t* __restrict__ qkv, Kv8Cache c, const int* __restrict__ table,
                                                            const int* __restrict__ kv_len, bf16_t* __restrict__ o,
                                                            float* __restrict__ part, int lbs, int max_blocks, int Hq, int splits,
                                                            int per, float scale_log2e) {
    constexpr int NJ = HD / 64, NT = HD / 16;
    __shared__ __attribute__((aligned(16))) float buf[NW8][16][HD + 4];
    __shared__ float wm[NW8][16], wl[NW8][16];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int Hkv = c.Hkv, grp = Hq / Hkv, ngb = (grp + 15) / 16;
    // Heads first: ids go round the eight XCDs, and heads have the same work, which requests and pieces have not (with the
    // pieces first, eight of them to a request, one XCD had all the first pieces and another all the last: 89 us for 64
    // requests of 300 to 6000 positions, 8 heads of 128; so 57).  Last pieces, which may be empty, come last.
    const int hk = blockIdx.x / ngb, h0 = (blockIdx.x % ngb) * 16, b = blockIdx.y, split = blockIdx.z;
    const int bs = 1 << lbs;
    const int s0 = split * per;
    const int heads = min(grp - h0, 16);
    const int hq = hk * grp + h0;

    bf16x8_t qf[NJ][2];
    {
        const bf16_t* qp = qkv + (size_t)b * ((Hq + 2 * Hkv) * HD) + (size_t)(hq + min(r, heads - 1)) * HD + g * 16;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int s = 0; s < 2; ++s) qf[j][s] = *reinterpret_cast<const bf16x8_t*>(qp + j * 64 + s * 8);
    }
    const int* row = table + (size_t)b * max_blocks;
    // What a step of 64 positions at t0 reads: its entries of the table first, one step ahead of the rest (K: of the group
    // that this lane's row of a score tile belongs to, V: of the lane's own group; nothing where there are no positions or
    // the entry is no block).
    // An entry behind the last position may be anything: what it leads to is inside the pool and is not looked at.  (Its
    // load does not wait for kv_len then.)
    auto entry = [&](int t0, int x) { return row[min((t0 + 16 * x) >> lbs, max_blocks - 1)]; };
    u32x4_t kw[4][NJ], vw[NT];
    auto load_k = [&](int t0, int k) {
        const size_t blk = (size_t)((unsigned)k < (unsigned)c.blocks ? k : 0) * Hkv + hk;
        const uint8_t* kp = c.k8 + (blk << lbs) * HD + (((t0 + 16 * (r >> 2)) & (bs - 1)) + (r & 3)) * HD + g * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < NJ; ++j) kw[t][j] = *reinterpret_cast<const u32x4_t*>(kp + t * 4 * HD + j * 64);
    };
    float2 sc;
    auto load_v = [&](int t0, int k) {
        const size_t blk = (size_t)((unsigned)k < (unsigned)c.blocks ? k : 0) * Hkv + hk;
        const uint8_t* vp = c.v8 + (blk << lbs) * HD + (r << lbs) + ((t0 + 16 * g) & (bs - 1));
        sc = *reinterpret_cast<const float2*>(c.scales + blk * 2);
#pragma unroll
        for (int t = 0; t < NT; ++t) vw[t] = *reinterpret_cast<const u32x4_t*>(vp + ((t * 16) << lbs));
    };
    f32x4_t acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m_run = LOWEST, l_run = 0.f;
    int seen = 0;                          // this lane has met a position
    constexpr int STEP = NW8 * 64;
    int t0 = s0 + w * 64;
    int ev = entry(t0, g), ek = entry(t0, r >> 2), ek_next = entry(t0 + STEP, r >> 2), ev_next = entry(t0 + STEP, g);
    const int n = min(max(kv_len[b], 0), max_blocks << lbs), s1 = min(n, s0 + per);
    if (s0 >= n && split > 0) return;      // the combination reads ceil(n / per) pieces, at least one
    if (t0 < s1) {
        load_k(t0, ek);
        load_v(t0, ev);
    }
    for (; t0 < s1; t0 += STEP) {
        // Loads return in order: the entries of the step after next go out in front of the next step's rows, so that waiting for
        // them does not wait for those.
        const int ek_after = entry(t0 + 2 * STEP, r >> 2), ev_after = entry(t0 + 2 * STEP, g);
        __builtin_amdgcn_sched_barrier(0);
        f32x4_t s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of_codes(kw[t][j][0], kw[t][j][1], 1.0f), qf[j][0], s[t], 0, 0, 0);
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of_codes(kw[t][j][2], kw[t][j][3], 1.0f), qf[j][1], s[t], 0, 0, 0);
            }
        }
        // the next step's keys are on their way while this step's softmax and values are worked, its values during the
        // next step's keys
        const bool more = t0 + STEP < s1;
        if (more) load_k(t0 + STEP, ek_next);
        const bool ok = (unsigned)ev < (unsigned)c.blocks;
        const int left = ok ? min(max(n - (t0 + 16 * g), 0), 16) : 0;      // positions of this lane's 16
        seen |= left;
        const float sk = sc.x * scale_log2e, sv = left ? sc.y : 1.0f;
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = t * 4 + i < left ? s[t][i] * sk : -INFINITY;
                mx = fmaxf(mx, s[t][i]);
            }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m_run, mx);
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        bf16x8_t pf[2];
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(s[t][i] - m_new);
                sum += p;
                pf[t >> 1][(t & 1) * 4 + i] = (__bf16)p;
            }
        l_run = fmaf(l_run, alpha, sum);
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] *= alpha;
        if (__any(left < 16)) {
            // what lies behind the last position is whatever the block held before, NaN codes included
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int live = min(max(left - 4 * k, 0), 4);
                    vw[t][k] &= live == 4 ? 0xffffffffu : (1u << (8 * live)) - 1;
                }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of_codes(vw[t][0], vw[t][1], sv), pf[0], acc[t], 0, 0, 0);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of_codes(vw[t][2], vw[t][3], sv), pf[1], acc[t], 0, 0, 0);
        }
        if (more) load_v(t0 + STEP, ev_next);
        ev = ev_next; ev_next = ev_after; ek_next = ek_after;
    }
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4_t*>(&buf[w][r][t * 16 + 4 * g]) = acc[t];
    // No positions and no weight are different states: scores that are all -inf leave the lowest finite maximum and a sum of 0, which
    // gives NaN as the definition does (0 / 0); without positions the maximum is -inf, and if everybody's is, o is 0.
    const bool met = __any(seen);
    if (g == 0) { wm[w][r] = met ? m_run : -INFINITY; wl[w][r] = l_run; }
    __syncthreads();
    for (int i = threadIdx.x; i < heads * HD; i += NW8 * 64) {
        const int head = i / HD, d = i % HD;
        float M = wm[0][head];
#pragma unroll
        for (int k = 1; k < NW8; ++k) M = fmaxf(M, wm[k][head]);
        float L = 0.f, a = 0.f;
        const float top = fmaxf(M, LOWEST);
#pragma unroll
        for (int k = 0; k < NW8; ++k) {
            const float f = __builtin_amdgcn_exp2f(wm[k][head] - top);
            L = fmaf(f, wl[k][head], L);
            a = fmaf(f, buf[k][head][d], a);
        }
        if (splits == 1) {
            o[((size_t)b * Hq + hq + head) * HD + d] = f2bf(M == -INFINITY ? 0.f : a / L);
        } else {
            float* pr = part + (((size_t)b * Hq + hq + head) * splits + split) * (HD + 2);
            pr[d] = a;
            if (d == 0) { pr[HD] = M; pr[HD + 1] = L; }
        }
    }
}

// o from the pieces of a request's positions: NW waves share out the pieces of a head, eight rows in flight each (one chain
// of dependent loads per piece took 31 us for 59 pieces), and add up in wave order.  Four waves per head from 17 pieces on: up to
// 16 it makes no difference of 3 % either way, for 24 pieces attention and combination take 12.1 us instead of 12.3, for 40 15.2 instead
// of 16.5, for 63 8.3 instead of 10.7 (32 heads of 128; 63: 4 of 64).
template <int HD, int NW>
__global__ __launch_bounds__(256) void kv8_combine_kernel(const float* __restrict__ part, const int* __restrict__ kv_len,
                                                          bf16_t* __restrict__ o, int splits, int per, int most, int Hq) {
    constexpr int E = HD / 64, BATCH = 8, HEADS = 4 / NW;
    __shared__ float sums[4][HD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave % NW;
    const int hq = blockIdx.x * HEADS + wave / NW, b = blockIdx.y;
    const int pieces = hq < Hq ? max((min(max(kv_len[b], 0), most) + per - 1) / per, 1) : 0;
    const float* p = part + ((size_t)b * Hq + hq) * splits * (HD + 2);
    auto ml_of = [&](int s) { return s < pieces ? *reinterpret_cast<const float2*>(p + (size_t)s * (HD + 2) + HD) : make_float2(-INFINITY, 0.f); };
    float M = -INFINITY, L = 0.f;
    for (int s = lane; s < pieces; s += 64) M = fmaxf(M, ml_of(s).x);
    M = wave_max(M);                   // -inf: no piece has positions
    const float top = fmaxf(M, LOWEST);
    for (int s = lane; s < pieces; s += 64) {
        const float2 ml = ml_of(s);
        L = fmaf(__builtin_amdgcn_exp2f(ml.x - top), ml.y, L);
    }
    L = wave_sum(L);
    float a[E] = {};
    for (int s0 = w; s0 < pieces; s0 += NW * BATCH) {
        float v[BATCH][E], f[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int s = min(s0 + NW * k, pieces - 1);
#pragma unroll
            for (int e = 0; e < E; ++e) v[k][e] = p[(size_t)s * (HD + 2) + lane + 64 * e];
            f[k] = ml_of(s0 + NW * k).x;
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (s0 + NW * k < pieces) {
#pragma unroll
                for (int e = 0; e < E; ++e) a[e] = fmaf(__builtin_amdgcn_exp2f(f[k] - top), v[k][e], a[e]);
            }
    }
    const float inv = M == -INFINITY ? 0.f : 1.0f / L;
    if (NW == 1) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (hq < Hq) o[((size_t)b * Hq + hq) * HD + lane + 64 * e] = f2bf(a[e] * inv);
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sums[wave][lane + 64 * e] = a[e];
    __syncthreads();
    if (threadIdx.x < HD) {
        const float v = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
        o[((size_t)b * Hq + hq) * HD + threadIdx.x] = f2bf(v * inv);
    }
}

// Pieces of 768 positions where that is three rounds of work-groups and more (three live on a CU), of 512 where it fills the
// chip, else of 256; none where the heads alone fill the chip and nobody has more than 1024 positions (the second launch
// would cost more).  The table's width stands for the lengths, which the host does not know.  us without the combination's 4 to 5, 64
// requests of 300 to 6000 positions with 8 heads of 128 in pieces of 256, 512, 768, 1024, 1536: 66.1 58.8 57.6 59.0 61.7;  30011 and
// 17003 positions: 20.5 19.2 20.0 19.4 23.3.  With it, tables as wide as the lengths, the rule's choice first:  4 x 2000, 8 heads of 128, 256
// 9.5, 512 10.6, 1024 13.5;  16 x 2000 256 20.7, 512 18.9, 1024 19.2;  4 x 20000 512 36.7, 256 40.4, 1024 37.5;  64 x 700, 32 heads 1024 64.8,
// 256 74.1;  64 x 1000, 8 heads of 64 1024 15.0, 512 18.1.  It loses where one piece is enough and the heads do not fill the chip (500
// positions, 8 heads: 256 7.1, 512 5.7;  32 x 1000, 8 heads: 256 20.8, 1024 16.2) and in the largest batches (32 x 8000: 768 105.9, 1536 99.4).
struct Kv8Plan { int splits, per; };

Kv8Plan plan_kv8(int B, int max_blocks, int block_size, int Hq, int Hkv) {
    const long most = (long)max_blocks * block_size;
    const int grp = Hq / Hkv;
    const long groups = (long)B * Hkv * ((grp + 15) / 16);
    Kv8Plan p;
    p.per = groups >= 512 && most <= 1024 ? 1024 : groups * most >= 1536L * 768 ? 768 : groups * most >= 512L * 512 ? 512 : 256;
    p.per = std::max(p.per, (int)((most + 65534) / 65535 + 63) / 64 * 64);      // at most 65535 pieces: a dimension of the grid
    p.splits = (int)((most + p.per - 1) / p.per);
    return p;
}

template <int HD>
hipError_t launch_kv8(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* part, const int* table, const int* kv_len, int B,
                      int max_blocks, int Hq, const Kv8Cache& c) {
    const Kv8Plan p = plan_kv8(B, max_blocks, c.block_size, Hq, c.Hkv);
    const int lbs = c.block_size == 16 ? 4 : c.block_size == 32 ? 5 : 6, grp = Hq / c.Hkv;
    if (p.splits > 1 && !part) return hipErrorInvalidValue;
    kv8_attn_kernel<HD><<<dim3(c.Hkv * ((grp + 15) / 16), B, p.splits), NW8 * 64, 0, st>>>(
        qkv, c, table, kv_len, o, part, lbs, max_blocks, Hq, p.splits, p.per, 1.4426950408889634f / sqrtf((float)HD));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    if (p.splits > 16)
        kv8_combine_kernel<HD, 4><<<dim3(Hq, B), 256, 0, st>>>(part, kv_len, o, p.splits, p.per, max_blocks << lbs, Hq);
    else
        kv8_combine_kernel<HD, 1><<<dim3((Hq + 3) / 4, B), 256, 0, st>>>(part, kv_len, o, p.splits, p.per, max_blocks << lbs, Hq);
    return hipGetLastError();
}

}  // namespace

hipError_t spk_launch_kv8_append(hipStream_t st, const bf16_t* qkv, const int* slots, int T, int Hq, const Kv8Cache& c) {
    return c.hd == 128 ? launch_append<128>(st, qkv, slots, T, Hq, c) : c.hd == 64 ? launch_append<64>(st, qkv, slots, T, Hq, c)
                                                                                : hipErrorInvalidValue;
}

void spk_kv8_plan_host(int B, int max_blocks, int block_size, int Hq, int Hkv, int* out2) {
    const Kv8Plan p = plan_kv8(B, max_blocks, block_size, Hq, Hkv);
    out2[0] = p.splits; out2[1] = p.per;
}

size_t spk_kv8_scratch_bytes(int B, int max_blocks, int block_size, int Hq, int Hkv, int hd) {
    const Kv8Plan p = plan_kv8(B, max_blocks, block_size, Hq, Hkv);
    return p.splits == 1 ? 0 : (size_t)B * Hq * p.splits * (hd + 2) * 4;
}

hipError_t spk_launch_kv8_attention(hipStream_t st, const bf16_t* qkv, bf16_t* o, float* part, const int* table, const int* kv_len, int B,
                                    int max_blocks, int Hq, const Kv8Cache& c) {
    return c.hd == 128  ? launch_kv8<128>(st, qkv, o, part, table, kv_len, B, max_blocks, Hq, c)
           : c.hd == 64 ? launch_kv8<64>(st, qkv, o, part, table, kv_len, B, max_blocks, Hq, c)
                        : hipErrorInvalidValue;
}
