// Block tables and slot maps of a batch of requests from their lengths (spk_batch_plan).
//
// Prefix sums over the requests, then one lookup per new token.  What bounds it is latency: a server's step writes
// some hundred kilobytes (4 bytes a row and a new block), and launches and dependent steps are what there is to save.  So it is one launch, without a
// hand-over between work-groups: every work-group computes the sums over all requests itself (n <= kPackedMaxSeqs lengths,
// which it reads through the L2), keeps them in LDS and then writes its own share of the tokens, of the requests and of
// the new table entries.  A block that a request gets by this call is read from the free list by whoever needs its
// number, never from the table, which another work-group may still be writing.
#include "sp_common.h"
#include "sp_kernels.h"

namespace {

constexpr int PLAN_THREADS = 512;
constexpr int PER_THREAD = kPackedMaxSeqs / PLAN_THREADS;
constexpr int TOKENS_PER_GROUP = PLAN_THREADS;

__device__ __forceinline__ long wave_scan(long v) {       // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    return v;
}

__global__ __launch_bounds__(PLAN_THREADS) void batch_plan_kernel(BatchPlanArgs g) {
    __shared__ int s_tok[kPackedMaxSeqs + 1], s_new[kPackedMaxSeqs + 1];     // first token / first new block of a request
    __shared__ long w_tok[PLAN_THREADS / 64], w_new[PLAN_THREADS / 64];
    __shared__ int w_max[PLAN_THREADS / 64], w_bad[PLAN_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int lbs = __builtin_ctz(g.block_size), bs = 1 << lbs, n = g.n;
    const long row = (long)g.max_blocks << lbs;
    // consecutive requests per thread
    long tok = 0, fresh = 0;
    int longest = 0, bad = 0;
    const int per = (n + PLAN_THREADS - 1) / PLAN_THREADS, r0 = tid * per;
    int len[PER_THREAD], need[PER_THREAD];
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) {
        len[i] = need[i] = 0;
        const int r = r0 + i;
        if (i < per && r < n) {
            const int L = g.lens[r], c = g.cached ? g.cached[r] : 0;
            bad |= (L < 0 || c < 0) ? 8 : (long)L + c > row ? 4 : 0;
            len[i] = max(L, 0);
            need[i] = (int)((((long)max(c, 0) + len[i] + bs - 1) >> lbs) - (((long)max(c, 0) + bs - 1) >> lbs));
            longest = max(longest, len[i]);
        }
        tok += len[i];
        fresh += need[i];
    }
    const long tok_in = wave_scan(tok), new_in = wave_scan(fresh);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        longest = max(longest, __shfl_xor(longest, o, 64));
        bad |= __shfl_xor(bad, o, 64);
    }
    if (lane == 63) { w_tok[w] = tok_in; w_new[w] = new_in; w_max[w] = longest; w_bad[w] = bad; }
    __syncthreads();
    long tok0 = tok_in - tok, new0 = new_in - fresh, tokens = 0, blocks = 0;
    longest = bad = 0;
#pragma unroll
    for (int k = 0; k < PLAN_THREADS / 64; ++k) {
        if (k < w) { tok0 += w_tok[k]; new0 += w_new[k]; }
        tokens += w_tok[k];
        blocks += w_new[k];
        longest = max(longest, w_max[k]);
        bad |= w_bad[k];
    }
    if (tokens > g.max_tokens) bad |= 1;
    if (blocks > g.n_free) bad |= 2;
    if (blockIdx.x == 0 && tid == 0) {
        g.info[0] = (int)min(tokens, 2147483647L);
        g.info[1] = (int)min(blocks, 2147483647L);
        g.info[2] = longest;
        g.info[3] = bad;
    }
    // what does not fit is not carried out: no new token, no new block
    if (!bad) {
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i)
            if (i < per && r0 + i < n) {
                s_tok[r0 + i] = (int)tok0;
                s_new[r0 + i] = (int)new0;
                tok0 += len[i];
                new0 += need[i];
            }
        if (tid == 0) { s_tok[n] = (int)tokens; s_new[n] = (int)blocks; }
    } else {
        for (int i = tid; i <= n; i += PLAN_THREADS) s_tok[i] = s_new[i] = 0;
        tokens = 0;
    }
    __syncthreads();
    const int first = blockIdx.x * PLAN_THREADS + tid, step = gridDim.x * PLAN_THREADS;
    for (int r = first; r <= n; r += step) {
        g.cu[r] = s_tok[r];
        if (r < n) g.kv_len[r] = (g.cached ? g.cached[r] : 0) + s_tok[r + 1] - s_tok[r];
    }
    // new table entries: entry i of all requests' new ones belongs to the last request whose first is <= i
    auto owner = [&](const int* start, int i) {
        int lo = 0, hi = n;              // start[lo] <= i < start[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= i) lo = mid; else hi = mid;
        }
        return lo;
    };
    const int all_new = s_new[n];
    for (int i = first; i < all_new; i += step) {
        const int r = owner(s_new, i), c = g.cached ? g.cached[r] : 0;
        g.table[(size_t)r * g.max_blocks + ((c + bs - 1) >> lbs) + i - s_new[r]] = g.free_blocks[i];
    }
    for (int t = first; t < g.max_tokens; t += step) {
        int slot = -1;
        if (t < tokens) {
            const int r = owner(s_tok, t), c = g.cached ? g.cached[r] : 0;
            const int pos = c + t - s_tok[r], held = (c + bs - 1) >> lbs, b = pos >> lbs;
            const int block = b < held ? g.table[(size_t)r * g.max_blocks + b] : g.free_blocks[s_new[r] + b - held];
            if ((unsigned)block < 1u << (31 - lbs)) slot = block * bs + (pos & (bs - 1));
        }
        g.slots[t] = slot;
    }
}

}  // namespace

hipError_t spk_launch_batch_plan(hipStream_t st, const BatchPlanArgs& g) {
    const int groups = std::max((g.max_tokens + TOKENS_PER_GROUP - 1) / TOKENS_PER_GROUP, 1);
    batch_plan_kernel<<<std::min(groups, 1024), PLAN_THREADS, 0, st>>>(g);
    return hipGetLastError();
}
