// C ABI of the operators over packed batches: argument checks in front of the launchers.
#include <limits.h>

#include <initializer_list>

#include "../../include/superpipe.h"
#include "../../include/superpipe_kernels.h"
#include "sp_kernels.h"

static int st(hipError_t e) {
    if (e == hipSuccess) return SP_OK;
    (void)hipGetLastError();
    return e == hipErrorInvalidValue ? SP_ERR_INVALID_ARG : SP_ERR_HIP;
}

static bool misaligned(int to, std::initializer_list<const void*> ptrs) {
    uintptr_t all = 0;
    for (const void* p : ptrs) all |= (uintptr_t)p;
    return (all & (uintptr_t)(to - 1)) != 0;
}

static bool any_null(std::initializer_list<const void*> ptrs) {
    for (const void* p : ptrs)
        if (!p) return true;
    return false;
}

constexpr int kMostPositions = 1 << 30;      // of a request, and rows of a packed batch: one and a stride of a grid, or a piece, fit an int

// The bytes of an array; NULL, or none, meets nothing.
struct Bytes {
    const void* p;
    size_t n;
    bool meets(const Bytes& o) const {
        const uintptr_t a = (uintptr_t)p, b = (uintptr_t)o.p;
        return p && o.p && n && o.n && a < b + o.n && b < a + n;
    }
};

// Work-groups run in any order: nothing that a call writes may lie over what it reads, or over something else that it writes.
static bool overlap(std::initializer_list<Bytes> written, std::initializer_list<Bytes> read) {
    for (const Bytes* w = written.begin(); w != written.end(); ++w) {
        for (const Bytes* v = written.begin(); v != w; ++v)
            if (w->meets(*v)) return true;
        for (const Bytes& r : read)
            if (w->meets(r)) return true;
    }
    return false;
}

static size_t ints(size_t n) { return n * 4; }
static size_t rows16(int T, int heads, int hd) { return (size_t)T * heads * hd * 2; }

static bool block_size_ok(int bs) { return bs == 16 || bs == 32 || bs == 64; }

extern "C" int spk_batch_plan(void* stream, const int32_t* lens, const int32_t* cached, const int32_t* free_blocks, int n_free,
                              int32_t* table, int max_blocks, int32_t* cu, int32_t* kv_len, int32_t* slots, int max_tokens,
                              int32_t* info, int n, int block_size) {
    if (any_null({lens, table, cu, kv_len, slots, info}) || (!free_blocks && n_free > 0)) return SP_ERR_INVALID_ARG;
    if (misaligned(4, {lens, cached, free_blocks, table, cu, kv_len, slots, info})) return SP_ERR_INVALID_ARG;
    if (n < 1 || n > kPackedMaxSeqs || n_free < 0 || max_tokens < 1 || max_tokens > kMostPositions || !block_size_ok(block_size) ||
        max_blocks < 1 || max_blocks > kMostPositions / block_size)
        return SP_ERR_INVALID_ARG;
    if (overlap({{table, ints((size_t)n * max_blocks)}, {cu, ints((size_t)n + 1)}, {kv_len, ints(n)}, {slots, ints(max_tokens)}, {info, ints(4)}},
                {{lens, ints(n)}, {cached, ints(n)}, {free_blocks, ints(n_free)}}))
        return SP_ERR_INVALID_ARG;
    return st(spk_launch_batch_plan((hipStream_t)stream, BatchPlanArgs{lens, cached, free_blocks, n_free, table, max_blocks, cu, kv_len, slots,
                                                                      max_tokens, info, n, block_size}));
}

// Everything but the pointers; slots of 32 rows are the most that any form launches per head.
static bool packed_ok(int n, int T, int Hq, int Hkv, int hd) {
    return n >= 1 && n <= kPackedMaxSeqs && T >= 1 && T <= kMostPositions && Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0 && Hq <= 16384 &&
           (hd == 64 || hd == 80 || hd == 128) && ((long)T / 32 + n) * Hq <= INT_MAX / 512;
}

extern "C" int spk_attention_packed(void* stream, const uint16_t* qkv, const int32_t* cu, uint16_t* o, float* lse, int n, int T,
                                    int Hq, int Hkv, int hd, int causal) {
    if (any_null({qkv, cu, o}) || misaligned(16, {qkv, o}) || misaligned(4, {cu, lse}) || !packed_ok(n, T, Hq, Hkv, hd))
        return SP_ERR_INVALID_ARG;
    if (overlap({{o, rows16(T, Hq, hd)}, {lse, ints((size_t)Hq * T)}}, {{qkv, rows16(T, Hq + 2 * Hkv, hd)}, {cu, ints((size_t)n + 1)}}))
        return SP_ERR_INVALID_ARG;
    return st(spk_launch_attention_packed((hipStream_t)stream, qkv, o, lse, PackedShape{cu, n, T, Hq, Hkv, hd, causal != 0}));
}

extern "C" size_t spk_attention_packed_bwd_scratch_bytes(int T, int Hq) {
    if (T < 1 || T > kMostPositions || Hq < 1) return 0;
    return ((size_t)T * Hq * 4 + 255) / 256 * 256;     // -rowsum(dO * O)
}

extern "C" int spk_attention_packed_bwd(void* stream, const uint16_t* qkv, const int32_t* cu, const uint16_t* o, const uint16_t* dO,
                                        const float* lse, void* scratch, uint16_t* dqkv, int n, int T, int Hq, int Hkv, int hd,
                                        int causal) {
    if (any_null({qkv, cu, o, dO, lse, scratch, dqkv}) || misaligned(16, {qkv, o, dO, scratch, dqkv}) || misaligned(4, {cu, lse}) ||
        !packed_ok(n, T, Hq, Hkv, hd))
        return SP_ERR_INVALID_ARG;
    if (overlap({{dqkv, rows16(T, Hq + 2 * Hkv, hd)}, {scratch, ints((size_t)Hq * T)}},
                {{qkv, rows16(T, Hq + 2 * Hkv, hd)}, {cu, ints((size_t)n + 1)}, {o, rows16(T, Hq, hd)}, {dO, rows16(T, Hq, hd)}, {lse, ints((size_t)Hq * T)}}))
        return SP_ERR_INVALID_ARG;
    return st(spk_launch_attention_packed_bwd((hipStream_t)stream, PackedBwdArgs{qkv, o, dO, lse, static_cast<float*>(scratch), dqkv},
                                              PackedShape{cu, n, T, Hq, Hkv, hd, causal != 0}));
}

static bool cache_ok(int blocks, int block_size, int Hq, int Hkv, int hd) {
    return block_size_ok(block_size) && blocks >= 1 && blocks <= INT_MAX / block_size && Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0 &&
           Hq <= 32767 && (hd == 64 || hd == 128);
}

static size_t codes(int blocks, int block_size, int Hkv, int hd) { return (size_t)blocks * block_size * Hkv * hd; }      // of keys or of values
static size_t scale_bytes(int blocks, int Hkv) { return (size_t)blocks * Hkv * 8; }

extern "C" int spk_kv8_append(void* stream, const uint16_t* qkv, const int32_t* slots, uint8_t* k8, uint8_t* v8, float* scales, int T,
                              int blocks, int block_size, int Hq, int Hkv, int hd) {
    if (any_null({qkv, slots, k8, v8, scales}) || misaligned(16, {qkv, k8, v8}) || misaligned(8, {scales}) || misaligned(4, {slots}))
        return SP_ERR_INVALID_ARG;
    if (T < 1 || T > kMostPositions || !cache_ok(blocks, block_size, Hq, Hkv, hd)) return SP_ERR_INVALID_ARG;
    const size_t half = codes(blocks, block_size, Hkv, hd);
    if (overlap({{k8, half}, {v8, half}, {scales, scale_bytes(blocks, Hkv)}}, {{qkv, rows16(T, Hq + 2 * Hkv, hd)}, {slots, ints(T)}}))
        return SP_ERR_INVALID_ARG;
    return st(spk_launch_kv8_append((hipStream_t)stream, qkv, slots, T, Hq, Kv8Cache{k8, v8, scales, blocks, block_size, Hkv, hd}));
}

static bool kv8_call_ok(int B, int max_blocks, int block_size, int Hq, int Hkv, int hd) {
    return B >= 1 && B <= 65535 && cache_ok(1, block_size, Hq, Hkv, hd) && max_blocks >= 1 && max_blocks <= kMostPositions / block_size;
}

extern "C" int spk_kv8_plan(int B, int max_blocks, int block_size, int Hq, int Hkv, int* out2) {
    if (!out2 || !kv8_call_ok(B, max_blocks, block_size, Hq, Hkv, 128)) return SP_ERR_INVALID_ARG;
    spk_kv8_plan_host(B, max_blocks, block_size, Hq, Hkv, out2);
    return SP_OK;
}

extern "C" size_t spk_kv8_attention_scratch_bytes(int B, int max_blocks, int block_size, int Hq, int Hkv, int hd) {
    if (!kv8_call_ok(B, max_blocks, block_size, Hq, Hkv, hd)) return 0;
    return spk_kv8_scratch_bytes(B, max_blocks, block_size, Hq, Hkv, hd);
}

extern "C" int spk_kv8_attention(void* stream, const uint16_t* qkv, const uint8_t* k8, const uint8_t* v8, const float* scales,
                                 const int32_t* table, const int32_t* kv_len, uint16_t* o, void* scratch, int B, int blocks,
                                 int block_size, int max_blocks, int Hq, int Hkv, int hd) {
    if (any_null({qkv, k8, v8, scales, table, kv_len, o}) || misaligned(16, {qkv, k8, v8, o, scratch}) || misaligned(8, {scales}) ||
        misaligned(4, {table, kv_len}))
        return SP_ERR_INVALID_ARG;
    if (!kv8_call_ok(B, max_blocks, block_size, Hq, Hkv, hd) || !cache_ok(blocks, block_size, Hq, Hkv, hd)) return SP_ERR_INVALID_ARG;
    const size_t need = spk_kv8_scratch_bytes(B, max_blocks, block_size, Hq, Hkv, hd), half = codes(blocks, block_size, Hkv, hd);
    if (!scratch && need) return SP_ERR_INVALID_ARG;
    if (overlap({{o, rows16(B, Hq, hd)}, {scratch, need}},
                {{qkv, rows16(B, Hq + 2 * Hkv, hd)}, {k8, half}, {v8, half}, {scales, scale_bytes(blocks, Hkv)},
                 {table, ints((size_t)B * max_blocks)}, {kv_len, ints(B)}}))
        return SP_ERR_INVALID_ARG;
    return st(spk_launch_kv8_attention((hipStream_t)stream, qkv, o, static_cast<float*>(scratch), table, kv_len, B, max_blocks, Hq,
                                       Kv8Cache{const_cast<uint8_t*>(k8), const_cast<uint8_t*>(v8), const_cast<float*>(scales), blocks,
                                                block_size, Hkv, hd}));
}
