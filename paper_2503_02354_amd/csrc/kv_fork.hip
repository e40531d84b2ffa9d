// gfx950 kernels that reorder the paged key/value cache of requests searched with beams: block tables of rows that continue others, and
// the copies of blocks that are not full.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// What a request's rows were and become; in LDS.
struct Family {
    int parent[kBeamMax];                     // row of the request that row i continues; -1: none
    int blocks[kBeamMax], tail[kBeamMax];     // of the old rows: blocks, and tokens of the last one if it is not full
    int last[kBeamMax];                       // the old rows' last block where it is not full and lies in the cache, else -1
    int place[kBeamMax];                      // row i's copy among the request's, or -1
    uint32_t lives;                           // old rows that are continued
    int copies, most;                         // copies, most blocks of a row that is dropped
};
struct Counts { int32_t copies, freed; };     // of a request; the workspace holds them

__device__ __forceinline__ int length_of(const KvFork& f, int64_t row) { return max(0, min(f.seq_len[row], f.max_blocks << f.block_shift)); }

// by all threads of the workgroup
__device__ __forceinline__ void read_family(Family& o, const KvFork& f, int r)
{
    const int tid = threadIdx.x;
    const int64_t row0 = (int64_t)r * f.beams;
    if (tid < f.beams) {
        const int p = f.parent[row0 + tid], len = length_of(f, row0 + tid), size = 1 << f.block_shift;
        o.parent[tid] = p >= row0 && p < row0 + f.beams ? (int)(p - row0) : -1;
        const int blocks = (len + size - 1) >> f.block_shift, tail = len & (size - 1);
        o.blocks[tid] = blocks;
        o.tail[tid] = tail;
        const int id = tail ? f.table[(row0 + tid) * f.max_blocks + blocks - 1] : -1;
        o.last[tid] = (uint32_t)id < (uint32_t)f.n_blocks ? id : -1;
    }
    __syncthreads();
    if (tid == 0) {
        uint32_t lives = 0;
        int copies = 0, most = 0;
        for (int i = 0; i < f.beams; ++i) {
            const int p = o.parent[i];
            o.place[i] = p >= 0 && (lives >> p & 1) && o.last[p] >= 0 ? copies++ : -1;
            if (p >= 0) lives |= 1u << p;
        }
        for (int i = 0; i < f.beams; ++i)
            if (!(lives >> i & 1)) most = max(most, o.blocks[i]);
        o.lives = lives;
        o.copies = copies;
        o.most = most;
    }
    __syncthreads();
}
// the old rows whose block at place j is free: nobody continues the row, no row that is continued holds it, and none before it is dropped with it
__device__ __forceinline__ uint32_t freed_at(const Family& o, const KvFork& f, const int32_t* table, int j)
{
    uint32_t freed = 0;
    for (int d = 0; d < f.beams; ++d) {
        if ((o.lives >> d & 1) || j >= o.blocks[d]) continue;
        const int id = table[(int64_t)d * f.max_blocks + j];
        bool held = (uint32_t)id >= (uint32_t)f.n_blocks;
        for (int s = 0; s < f.beams && !held; ++s)
            if (j < o.blocks[s] && ((o.lives >> s & 1) || s < d)) held = table[(int64_t)s * f.max_blocks + j] == id;
        freed |= held ? 0u : 1u << d;
    }
    return freed;
}

__global__ __launch_bounds__(kThreads) void kv_fork_count_kernel(KvFork f, Counts* counts)
{
    __shared__ Family o;
    __shared__ int part[kWaves];
    const int tid = threadIdx.x, r = blockIdx.x;
    read_family(o, f, r);
    const int32_t* const table = f.table + (int64_t)r * f.beams * f.max_blocks;
    int freed = 0;
    for (int j = tid; j < o.most; j += kThreads) freed += __popc(freed_at(o, f, table, j));
    for (int d = 32; d > 0; d >>= 1) freed += __shfl_xor(freed, d, 64);
    if ((tid & 63) == 0) part[tid >> 6] = freed;
    __syncthreads();
    if (tid == 0) {
        freed = 0;
        for (int w = 0; w < kWaves; ++w) freed += part[w];
        counts[r] = {o.copies, freed};
    }
}

__device__ __forceinline__ int ring_at(uint32_t head, long long i, int n) { return (int)((head + (unsigned long long)i) % (uint32_t)n); }

// the sum over the workgroup of two values per thread
__device__ __forceinline__ void sum2(long long (&v)[2], long long (*part)[2])
{
    for (int d = 32; d > 0; d >>= 1)
        for (int e = 0; e < 2; ++e) v[e] += __shfl_xor(v[e], d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        for (int e = 0; e < 2; ++e) part[threadIdx.x >> 6][e] = v[e];
    __syncthreads();
    for (int e = 0; e < 2; ++e) {
        v[e] = 0;
        for (int w = 0; w < kWaves; ++w) v[e] += part[w][e];
    }
}

// A workgroup per request, and one more for the state.
__global__ __launch_bounds__(kThreads) void kv_fork_kernel(KvFork f, const Counts* counts)
{
    __shared__ Family o;
    __shared__ long long part[kWaves][2];
    __shared__ int own[kBeamMax], wave_sum[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, r = blockIdx.x;
    const long long count = max(0, min(f.ring_state[1], f.n_blocks));
    const uint32_t head = (uint32_t)f.ring_state[0] % (uint32_t)f.n_blocks;
    if (r == f.n_requests) {
        // the requests in order, until one needs more than is left
        if (tid == 0) {
            long long taken = 0, given = 0, copies = 0;
            int i = 0;
            for (; i < f.n_requests; ++i) {
                const Counts c = counts[i];
                if (taken + max(0, c.copies - c.freed) > count) break;
                taken += max(0, c.copies - c.freed);
                given += max(0, c.freed - c.copies);
                copies += c.copies;
            }
            f.next_state[0] = ring_at(head, taken, f.n_blocks);
            f.next_state[1] = (int32_t)(count - taken + given);
            f.next_state[2] = i;
            f.next_state[3] = (int32_t)copies;
        }
        return;
    }
    read_family(o, f, r);
    const Counts mine = counts[r];
    long long before[2] = {0, 0};             // taken from the ring, and given to it, by the requests before this one
    for (int i = tid; i < r; i += kThreads) {
        const Counts c = counts[i];
        before[0] += max(0, c.copies - c.freed);
        before[1] += max(0, c.freed - c.copies);
    }
    sum2(before, part);
    const bool open = before[0] + max(0, mine.copies - mine.freed) <= count;
    const int64_t row0 = (int64_t)r * f.beams;
    const int32_t* const table = f.table + row0 * f.max_blocks;
    if (open) {                               // blocks that are free, in order
        int carry = 0;
        for (int j0 = 0; j0 < o.most; j0 += kThreads) {
            uint32_t freed = j0 + tid < o.most ? freed_at(o, f, table, j0 + tid) : 0u;
            int sum = __popc(freed);
            const int v = sum;
            for (int d = 1; d < 64; d <<= 1) {
                const int u = __shfl_up(sum, d, 64);
                if (lane >= d) sum += u;
            }
            __syncthreads();
            if (lane == 63) wave_sum[wid] = sum;
            __syncthreads();
            int at = carry + sum - v;
            for (int w = 0; w < kWaves; ++w) {
                if (w < wid) at += wave_sum[w];
                carry += wave_sum[w];
            }
            for (; freed; freed &= freed - 1, ++at) {
                const int id = table[(int64_t)__builtin_ctz(freed) * f.max_blocks + j0 + tid];
                if (at < mine.copies) own[at] = id;
                else f.ring[ring_at(head, count + before[1] + (at - mine.copies), f.n_blocks)] = id;
            }
        }
    }
    __syncthreads();
    for (int i = 0; i < f.beams; ++i) {
        const int p = open ? o.parent[i] : i, place = open ? o.place[i] : -1;
        const int blocks = p >= 0 ? o.blocks[p] : 0;
        int id = -1;                          // of the row's own last block
        if (place >= 0) id = place < mine.freed ? own[place] : f.ring[ring_at(head, before[0] + (place - mine.freed), f.n_blocks)];
        for (int j = tid; j < blocks; j += kThreads) f.next_table[(row0 + i) * f.max_blocks + j] = place >= 0 && j == blocks - 1 ? id : table[(int64_t)p * f.max_blocks + j];
        if (tid == 0) {
            f.next_len[row0 + i] = p >= 0 ? length_of(f, row0 + p) : 0;
            f.copy[2 * (row0 + i)] = place >= 0 ? o.last[p] : -1;
            f.copy[2 * (row0 + i) + 1] = place >= 0 ? id : -1;
        }
    }
}

// A workgroup per row and layer.
__global__ __launch_bounds__(kThreads) void kv_copy_kernel(KvCaches caches, const int32_t* __restrict__ copy, const int32_t* __restrict__ seq_len)
{
    const KvCache& c = caches.c[blockIdx.y];
    const int i = blockIdx.x, from = copy[2 * i], to = copy[2 * i + 1];
    if ((uint32_t)from >= (uint32_t)c.n_blocks || (uint32_t)to >= (uint32_t)c.n_blocks) return;
    const int size = 1 << c.block_shift, tail = seq_len[i] & (size - 1), rows = tail ? tail : size;
    const int per_head = c.head_dim >> 3, per_row = per_head * c.kv_heads;
    for (int u = threadIdx.x; u < rows * per_row; u += kThreads) {
        const int row = u / per_row, rest = u - row * per_row, head = rest / per_head, ch = (rest - head * per_head) * 8;
        const int64_t at = row * c.token_stride + head * c.head_stride + ch;
        const uint4 a = *(const uint4*)(c.k + from * c.block_stride + at), b = *(const uint4*)(c.v + from * c.block_stride + at);
        *(uint4*)(c.k + to * c.block_stride + at) = a;
        *(uint4*)(c.v + to * c.block_stride + at) = b;
    }
}

}  // namespace

int64_t kv_fork_workspace(int32_t n_requests, int32_t) { return (int64_t)n_requests * (int64_t)sizeof(Counts); }

hipError_t kv_fork(const KvFork& f, void* workspace, hipStream_t stream)
{
    if (f.n_requests > 0) {
        hipLaunchKernelGGL(kv_fork_count_kernel, dim3((unsigned)f.n_requests), dim3(kThreads), 0, stream, f, (Counts*)workspace);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kv_fork_kernel, dim3((unsigned)f.n_requests + 1), dim3(kThreads), 0, stream, f, (const Counts*)workspace);
    return hipGetLastError();
}

hipError_t kv_copy(int32_t n_caches, const KvCaches& caches, int32_t n, const int32_t* copy, const int32_t* seq_len, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)n, (unsigned)n_caches), dim3(kThreads), 0, stream, caches, copy, seq_len);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
