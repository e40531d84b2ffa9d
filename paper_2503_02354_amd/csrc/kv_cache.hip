// gfx950 kernels that keep the paged key/value cache of token-generating experts: a step's block tables and slot map, and the
// append of new rows.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

// ---- block tables and slot map -----------------------------------------------------------------------------------
// One launch.  Request r needs ceil((have + add) / block) - ceil(have / block) blocks; three running sums over the requests (blocks
// taken, tokens, blocks given back) say which of the ring's ids it takes, where its tokens stand and where its blocks go.  Every
// workgroup computes the sums of all requests for itself in LDS, where a token finds its request by bisection; the workgroups
// then share the tokens and the requests.  None waits for another: a token of a new block takes the block's id from the ring, not
// from the table that some other workgroup writes.
// What bounds it: latency (lengths in, one scan, slots out): 7.4 us for 192 requests with a token each, 8.5 us for 1500 requests and 86,000
// tokens, of which a launch with one load and one store takes 2.8.
constexpr int kPlanThreads = 256;
constexpr int kPlanInLds = 8192;              // requests whose lengths stay in LDS beside the sums (96 KiB); more ask memory again, per token
constexpr uint32_t kFreed = 0x80000000u;      // the entry counts blocks that a finished request gives back
constexpr uint32_t kTooLong = 0x40000000u;    // the request would outgrow its row of the table

// place `i` behind `head` in a ring of n entries; head < n
__device__ __forceinline__ uint32_t in_ring(uint32_t head, uint32_t i, uint32_t n)
{
    if (i >= n) i %= n;                       // only where more is given back than there is room for
    const uint32_t at = head + i;
    return at >= n ? at - n : at;
}

// inclusive sums over the workgroup of three values per thread; `part`: [3][kPlanThreads / 64]
__device__ __forceinline__ void scan3(uint32_t (&v)[3], uint32_t* part)
{
    const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const uint32_t u = __shfl_up(v[i], d, 64);
            if (lane >= d) v[i] += u;
        }
    if (lane == 63)
#pragma unroll
        for (int i = 0; i < 3; ++i) part[i * (kPlanThreads / 64) + wid] = v[i];
    __syncthreads();
    for (int i = 0; i < 3; ++i)
        for (int w = 0; w < wid; ++w) v[i] += part[i * (kPlanThreads / 64) + w];
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(int n, int shift, int n_blocks, int max_blocks, int token_cap,
                                                               const int32_t* __restrict__ have, const int32_t* __restrict__ add,
                                                               int32_t* __restrict__ ring, const int32_t* __restrict__ ring_state,
                                                               int32_t* __restrict__ table, int32_t* __restrict__ seq_len,
                                                               int32_t* __restrict__ q_off, int32_t* __restrict__ slot,
                                                               int32_t* __restrict__ position, int32_t* __restrict__ next_state)
{
    extern __shared__ uint32_t sums[];
    uint32_t* const tok = sums;               // [n + 1] new tokens of a request, then the sum over those before it
    uint32_t* const blk = sums + n + 1;       // [n] blocks taken (or kFreed | given back), then the sum over those before it
    uint32_t* const len = sums + 2 * n + 1;   // [n] cached tokens, where they fit
    const bool in_lds = n <= kPlanInLds;
    __shared__ uint32_t part[3 * (kPlanThreads / 64)];
    __shared__ int closed;
    const int tid = threadIdx.x;
    const uint32_t bs = 1u << shift, longest = (uint32_t)max_blocks << shift;
    if (tid == 0) closed = n;
    const int32_t head_in = ring_state[0], count_in = ring_state[1];
    const uint32_t count = (uint32_t)max(0, min(count_in, n_blocks));
    const uint32_t head = (uint32_t)head_in % (uint32_t)n_blocks;
    for (int r = tid; r < n; r += kPlanThreads) {
        const uint32_t h = min((uint32_t)max(have[r], 0), longest);
        const int32_t a = add[r];
        const uint32_t old_blocks = (h + bs - 1) >> shift;
        if (in_lds) len[r] = h;
        if (a < 0) {
            tok[r] = 0;
            blk[r] = kFreed | old_blocks;
        } else {
            const bool fits = (uint32_t)a <= longest - h;
            tok[r] = fits ? (uint32_t)a : 0u;
            blk[r] = fits ? ((h + (uint32_t)a + bs - 1) >> shift) - old_blocks : kTooLong;
        }
    }
    __syncthreads();
    // Sums past the request that closes the step may wrap and are not used; up to it they are exact (each term is below 2^31 and the
    // sum before it within the limits).
    const int per = (n + kPlanThreads - 1) / kPlanThreads | 1, begin = min(n, tid * per), end = min(n, begin + per);
    uint32_t own[3] = {0, 0, 0};              // an odd number of requests to a thread: LDS banks apart
    for (int r = begin; r < end; ++r) {
        const uint32_t b = blk[r];
        own[0] += b & kFreed ? 0u : b & ~kTooLong;
        own[1] += tok[r];
        own[2] += b & kFreed ? b & ~kFreed : 0u;
    }
    uint32_t at[3] = {own[0], own[1], own[2]};
    scan3(at, part);
#pragma unroll
    for (int i = 0; i < 3; ++i) at[i] -= own[i];
    int first_bad = n;
    for (int r = begin; r < end; ++r) {
        const uint32_t b = blk[r], t = tok[r];
        const bool freed = (b & kFreed) != 0;
        const uint32_t need = freed ? 0u : b & ~kTooLong;
        if (!freed && first_bad == n && ((b & kTooLong) || at[0] + need > count || at[1] + t > (uint32_t)token_cap)) first_bad = r;
        blk[r] = freed ? kFreed | at[2] : at[0];
        tok[r] = at[1];
        at[0] += need;
        at[1] += t;
        at[2] += freed ? b & ~kFreed : 0u;
    }
    if (first_bad < n) atomicMin(&closed, first_bad);
    __syncthreads();
    const int f = closed;                     // requests from here on do not grow
    // the thread whose stretch ends the requests has the sums over all of them
    __shared__ uint32_t freed_total, tokens_open, taken_open;
    if (begin < n && end == n) {
        freed_total = at[2];
        if (f == n) { tokens_open = at[1]; taken_open = at[0]; }
    }
    if (n == 0 && tid == 0) freed_total = tokens_open = taken_open = 0;
    if (f < n && tid == 0) { tokens_open = tok[f]; taken_open = blk[f]; }
    __syncthreads();
    const uint32_t tokens = tokens_open;
    if (tid == 0) tok[n] = tokens;
    __syncthreads();

    if (blockIdx.x == 0 && tid == 0) {
        next_state[0] = (int32_t)in_ring(head, taken_open, (uint32_t)n_blocks);
        next_state[1] = (int32_t)(count - taken_open + freed_total);
        next_state[2] = f;
        next_state[3] = (int32_t)tokens;
        q_off[n] = (int32_t)tokens;
    }
    auto cached = [&](int r) { return in_lds ? len[r] : min((uint32_t)max(have[r], 0), longest); };
    const int wave = (blockIdx.x * kPlanThreads + tid) >> 6, waves = gridDim.x * (kPlanThreads / 64), lane = tid & 63;
    for (int r = blockIdx.x * kPlanThreads + tid; r < n; r += gridDim.x * kPlanThreads) {
        // sums from f on may have wrapped into the flag: ask again
        const bool freed = r < f ? (blk[r] & kFreed) != 0 : add[r] < 0;
        seq_len[r] = freed ? 0 : (int32_t)(cached(r) + (r < f ? tok[r + 1] - tok[r] : 0u));
        q_off[r] = (int32_t)(r < f ? tok[r] : tokens);
    }
    for (int r = wave; r < n; r += waves) {   // blocks of finished requests to the ring's end
        if (!(blk[r] & kFreed) || add[r] >= 0) continue;
        const uint32_t blocks = (cached(r) + bs - 1) >> shift;
        const uint32_t to = count + (blk[r] & ~kFreed);
        for (uint32_t j = lane; j < blocks; j += 64) ring[in_ring(head, to + j, (uint32_t)n_blocks)] = table[(size_t)r * max_blocks + j];
    }
    for (uint32_t t = blockIdx.x * kPlanThreads + tid; t < (uint32_t)token_cap; t += gridDim.x * kPlanThreads) {      // a step past 2^31 stays above the cap
        if (t >= tokens) {
            slot[t] = -1;
            position[t] = -1;
            continue;
        }
        int lo = 0, hi = f;                   // the last request below f that starts at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (tok[mid] <= t) lo = mid;
            else hi = mid;
        }
        const uint32_t h = cached(lo), old_blocks = (h + bs - 1) >> shift;
        const uint32_t pos = h + t - tok[lo], page = pos >> shift;
        int32_t* const row = table + (size_t)lo * max_blocks;
        int32_t id;
        if (page < old_blocks) id = row[page];
        else {
            id = ring[in_ring(head, blk[lo] + (page - old_blocks), (uint32_t)n_blocks)];
            if ((pos & (bs - 1)) == 0) row[page] = id;        // a new block's first token
        }
        // an id outside the cache has no slot; its product could be one of another request's
        slot[t] = (uint32_t)id < (uint32_t)n_blocks ? (int32_t)(((uint32_t)id << shift) + (pos & (bs - 1))) : -1;
        position[t] = (int32_t)pos;
    }
}

// ---- append -------------------------------------------------------------------------------------------------------
// A copy of rows to scattered places; a thread moves 16 bytes of a key and the same of a value.  What bounds it: HBM, or the
// launch itself where there are few tokens: 8000 tokens of 8 heads of 128 (65.6 MB) 11.4 us, 5.7 TB/s, which is what a copy of that size
// reaches; 48 tokens 2.8 us.
__global__ __launch_bounds__(256) void kv_append_kernel(KvCache c, int n_tokens, const uint16_t* __restrict__ k, int64_t k_ts, int64_t k_hs,
                                                        const uint16_t* __restrict__ v, int64_t v_ts, int64_t v_hs,
                                                        const int32_t* __restrict__ slot)
{
    const int per_head = c.head_dim >> 3, per_token = per_head * c.kv_heads;
    const int tokens = max(1, 256 / per_token), sub = threadIdx.x / per_token;        // tokens of a workgroup
    for (long long t = (long long)blockIdx.x * tokens + sub; t < n_tokens && sub < tokens; t += (long long)gridDim.x * tokens) {
        const int32_t s = slot[t];
        const int32_t block = s >> c.block_shift, row = s & ((1 << c.block_shift) - 1);
        if (s < 0 || block >= c.n_blocks) continue;
        const int64_t base = block * c.block_stride + row * c.token_stride;
        for (int i = threadIdx.x - sub * per_token; i < per_token; i += 256) {
            const int head = i / per_head, ch = (i - head * per_head) * 8;
            const uint4 a = *(const uint4*)(k + t * k_ts + head * k_hs + ch), b = *(const uint4*)(v + t * v_ts + head * v_hs + ch);
            *(uint4*)(c.k + base + head * c.head_stride + ch) = a;
            *(uint4*)(c.v + base + head * c.head_stride + ch) = b;
        }
    }
}

}  // namespace

hipError_t kv_plan(int32_t n, int32_t block_shift, int32_t n_blocks, int32_t max_blocks, int32_t token_cap, const int32_t* have,
                   const int32_t* add, int32_t* ring, const int32_t* ring_state, int32_t* table, int32_t* seq_len, int32_t* q_off,
                   int32_t* slot, int32_t* position, int32_t* next_state, hipStream_t stream)
{
    const size_t lds = ((n <= kPlanInLds ? 3 : 2) * (size_t)n + 1) * 4;
    static const hipError_t configured = hipFuncSetAttribute((const void*)kv_plan_kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                             (int)((2 * (size_t)kPlanMaxRequests + 1) * 4));
    if (configured != hipSuccess) return configured;
    // A thread for every token while scans are short: 1500 requests with 86,000 tokens 8.4 us, 11.9 with four tokens to a thread; many requests one
    // workgroup per compute unit: 8000 with 240,000 tokens 23.5 us, 38 with two; 4000 with 200,000 15.1 and 13.8.
    const int by_tokens = (int)(((long long)token_cap + kPlanThreads - 1) / kPlanThreads), by_requests = (n + kPlanThreads - 1) / kPlanThreads;
    const int grid = std::max(1, std::min(n <= 4096 ? 512 : 256, std::max(by_tokens, by_requests)));
    hipLaunchKernelGGL(kv_plan_kernel, dim3(grid), dim3(kPlanThreads), lds, stream, n, block_shift, n_blocks, max_blocks, token_cap, have, add, ring,
                       ring_state, table, seq_len, q_off, slot, position, next_state);
    return hipGetLastError();
}

hipError_t kv_append(const KvCache& c, int32_t n_tokens, const uint16_t* k, int64_t k_ts, int64_t k_hs, const uint16_t* v, int64_t v_ts,
                     int64_t v_hs, const int32_t* slot, hipStream_t stream)
{
    const int per_token = c.kv_heads * (c.head_dim / 8), tokens = std::max(1, 256 / per_token);
    const long long blocks = ((long long)n_tokens + tokens - 1) / tokens;
    hipLaunchKernelGGL(kv_append_kernel, dim3((unsigned)std::min<long long>(blocks, 1 << 20)), dim3(256), 0, stream, c, n_tokens, k, k_ts, k_hs, v,
                       v_ts, v_hs, slot);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
