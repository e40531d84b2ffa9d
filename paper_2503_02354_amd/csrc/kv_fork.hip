// gfx950 kernels that reorder the paged key/value cache of requests searched with beams: block tables of rows that continue others, and
// the copies of blocks that are not full.
// A request takes ids from the ring, or gives some back, behind those of all requests before it.  So one launch counts them for every request, and the next
// one sums up the counts before its own; one request does without the first.  Both are bound by latency: 24 requests of eight beams and up to 106 blocks 4.7
// and 7.3 us, 8 requests of 32 beams 11.7 and 18.5, one of four beams 5.1.
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
    int blocks[kBeamMax], length[kBeamMax];   // of the old rows: blocks, tokens
    int last[kBeamMax];                       // the old rows' last block where it is not full and lies in the cache, else -1
    int place[kBeamMax];                      // row i's copy among the request's, or -1
    int taken[kBeamMax];                      // blocks that row i takes over as they are
    uint32_t lives;                           // old rows that are continued
    int copies, most, longest;                // copies, most blocks of a row that is dropped, and of any row
};
struct Counts { int32_t copies, freed; };     // of a request; the workspace holds them

__device__ __forceinline__ int length_of(const KvFork& f, int64_t row) { return max(0, min(f.seq_len[row], f.max_blocks << f.block_shift)); }

// A barrier that LDS is ready behind; stores to memory need not have ended.
__device__ __forceinline__ void lds_barrier()
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
#endif
}
// f over a wavefront's lanes up to each, by register operations; lane 63 has all.  0 changes nothing to f.
template <class F> __device__ __forceinline__ int wave_scan(int v, F f)
{
#if defined(__HIP_DEVICE_COMPILE__)
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));      // one lane up, two, four, eight in a row of 16
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));      // a row's last lane to the next row, the second row's to the last two
    v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));
#endif
    return v;
}
__device__ __forceinline__ int wave_sums(int v) { return wave_scan(v, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int wave_max(int v) { return __builtin_amdgcn_readlane(wave_scan(v, [](int a, int b) { return max(a, b); }), 63); }
__device__ __forceinline__ uint32_t wave_or(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane(wave_scan((int)v, [](int a, int b) { return a | b; }), 63); }

// A thread's column of the old rows' tables: their blocks at one place, in LDS, a group of rows on their way together; of any value behind a row's blocks.
// ROWS: room for that many, kGroup or kBeamMax; 24 requests of eight beams with room for eight 22.3 us, for 32 23.2.  (Loops over groups and rows are left as they are:
// small launches like these are bound by latency, that of their instructions' first use among it.)
constexpr int kGroup = 8;
static_assert(kBeamMax % (2 * kGroup) == 0, "whole groups");
template <int ROWS> struct Columns {
    static constexpr int kTogether = ROWS < 2 * kGroup ? ROWS : 2 * kGroup;
    int32_t id[ROWS][kThreads];
};
template <int ROWS> __device__ __forceinline__ void read_column(Columns<ROWS>& ids, const KvFork& f, const int32_t* table, int j)
{
    constexpr int T = Columns<ROWS>::kTogether;
    const bool there = j < f.max_blocks;
    const int32_t* const from = table + (there ? j : 0);
#pragma nounroll
    for (int w0 = 0; w0 < f.beams; w0 += T) {
        int32_t v[T];
#pragma unroll
        for (int w = 0; w < T; ++w) v[w] = from[(int64_t)min(w0 + w, f.beams - 1) * f.max_blocks];
#pragma unroll
        for (int w = 0; w < T; ++w) ids.id[w0 + w][threadIdx.x] = v[w];
    }
}

// By all threads of the workgroup; a row to a lane of its first wavefront.  `ids` holds the first kThreads columns, whose loads share a round trip with
// the rows' own.
template <int ROWS> __device__ __forceinline__ void read_family(Family& o, Columns<ROWS>& ids, const KvFork& f, int r)
{
    const int lane = threadIdx.x;
    const int64_t row0 = (int64_t)r * f.beams;
    const int32_t* const table = f.table + row0 * f.max_blocks;
    const bool is = lane < f.beams;
    const int given = is ? f.parent[row0 + lane] : -1, len = is ? length_of(f, row0 + lane) : 0, size = 1 << f.block_shift;
    read_column(ids, f, table, threadIdx.x);
    __syncthreads();
    if (lane < 64) {
        const int p = given >= row0 && given < row0 + f.beams ? (int)(given - row0) : -1, blocks = (len + size - 1) >> f.block_shift;
        int id = -1;
        if (len & (size - 1)) id = blocks <= kThreads ? ids.id[lane][blocks - 1] : table[(int64_t)lane * f.max_blocks + blocks - 1];
        const int last = (uint32_t)id < (uint32_t)f.n_blocks ? id : -1;
        const uint32_t lives = wave_or(p >= 0 ? 1u << p : 0u);
        const int longest = wave_max(blocks), most = wave_max(lane < kBeamMax && (lives >> lane & 1) ? 0 : blocks);
        bool first = true;
#pragma nounroll
        for (int w = 0; w < f.beams; ++w) first &= (w >= lane) | (__builtin_amdgcn_readlane(p, w) != p);
        const int parents_last = __shfl(last, max(p, 0), 64);
        const bool copied = is && p >= 0 && !first && parents_last >= 0;
        const unsigned long long copies = __ballot(copied);
        const int parents_blocks = __shfl(blocks, max(p, 0), 64);
        if (lane < kBeamMax) {                // what is no row has no blocks
            o.taken[lane] = p < 0 ? 0 : parents_blocks - (copied ? 1 : 0);
            o.parent[lane] = p;
            o.blocks[lane] = blocks;
            o.length[lane] = len;
            o.last[lane] = last;
            o.place[lane] = copied ? __popcll(copies & ((1ull << lane) - 1)) : -1;
        }
        if (lane == 0) {
            o.lives = lives;
            o.copies = __popcll(copies);
            o.most = most;
            o.longest = longest;
        }
    }
    __syncthreads();
}
// Looking for free blocks is what these launches compute most, of rows by rows in every column; threads that have no column share those of others (24
// requests of eight beams 23.4 -> 22.3 us, 8 of 32 57 -> 43).
struct Share {
    int column, part, parts;                  // of `parts` threads with this column, the part-th
    uint32_t rows;                            // that it looks at
};
__device__ __forceinline__ Share share_of(int columns)
{
    const int parts = columns <= kThreads / 4 ? 4 : columns <= kThreads / 2 ? 2 : 1, part = (int)threadIdx.x / (kThreads / parts);
    return {(int)threadIdx.x % (kThreads / parts), part, parts, (parts == 4 ? 0x11111111u : parts == 2 ? 0x55555555u : ~0u) << part};
}
// Those of a share's rows whose block at place j, in `column`, is free: nobody continues the row, no row that is continued holds it, and none before it
// is dropped with it.
template <int ROWS> __device__ __forceinline__ uint32_t freed_in(const Columns<ROWS>& ids, const Family& o, const KvFork& f, int j, int column, uint32_t rows)
{
    constexpr int T = Columns<ROWS>::kTogether;
    uint32_t there = 0, freed = 0;
#pragma nounroll
    for (int s0 = 0; s0 < f.beams; s0 += T)
#pragma unroll
        for (int s = 0; s < T; ++s) there |= (j < o.blocks[s0 + s] ? 1u << s : 0u) << s0;
#pragma nounroll
    for (uint32_t dropped = there & ~o.lives & rows; dropped; dropped &= dropped - 1) {
        const int d = __builtin_ctz(dropped), id = ids.id[d][column];
        uint32_t same = 0;                    // rows that are not there have any bits
#pragma nounroll
        for (int s0 = 0; s0 < f.beams; s0 += T) {
            uint32_t some = 0;
#pragma unroll
            for (int s = 0; s < T; ++s) some |= ids.id[s0 + s][column] == id ? 1u << s : 0u;
            same |= some << s0;
        }
        freed |= (((uint32_t)id < (uint32_t)f.n_blocks) & !(same & there & (o.lives | ((1u << d) - 1)))) ? 1u << d : 0u;
    }
    return freed;
}

// what a request copies and frees; by all threads of the workgroup
template <int ROWS> __device__ __forceinline__ Counts count_request(Columns<ROWS>& ids, const Family& o, const KvFork& f, const int32_t* table, int* part)
{
    const int tid = threadIdx.x;
    const Share share = share_of(o.most);
    int freed = 0;
#pragma nounroll
    for (int j = share.column; j < o.most; j += kThreads) {
        if (j >= kThreads) read_column(ids, f, table, j);
        freed += __popc(freed_in(ids, o, f, j, share.column, share.rows));
    }
    freed = wave_sums(freed);
    if ((tid & 63) == 63) part[tid >> 6] = freed;
    __syncthreads();
    freed = 0;
    for (int w = 0; w < kWaves; ++w) freed += part[w];
    return {o.copies, freed};
}

template <int ROWS> __global__ __launch_bounds__(kThreads) void kv_fork_count_kernel(KvFork f, Counts* counts)
{
    __shared__ Family o;
    __shared__ Columns<ROWS> ids;
    __shared__ int part[kWaves];
    read_family(o, ids, f, blockIdx.x);
    const Counts c = count_request(ids, o, f, f.table + (int64_t)blockIdx.x * f.beams * f.max_blocks, part);
    if (threadIdx.x == 0) counts[blockIdx.x] = c;
}

// place `at` behind head in a ring of n entries; it passes n only where the state is none of a ring
__device__ __forceinline__ int ring_at(uint32_t head, uint32_t at, uint32_t n)
{
    if (at >= n) at %= n;
    at += head;
    return (int)(at >= n ? at - n : at);
}
__device__ __forceinline__ int taken_by(const Counts& c) { return max(0, c.copies - c.freed); }
__device__ __forceinline__ int given_by(const Counts& c) { return max(0, c.freed - c.copies); }

// The sums over the workgroup of three values per thread.  A request takes 31 ids at most, and gives what it holds: in a pool all of them fit 32 bits.
__device__ __forceinline__ void sum3(uint32_t (&v)[3], uint32_t (*part)[3])
{
#pragma unroll
    for (int e = 0; e < 3; ++e) v[e] = (uint32_t)wave_sums((int)v[e]);
    __syncthreads();
    if ((threadIdx.x & 63) == 63)
#pragma unroll
        for (int e = 0; e < 3; ++e) part[threadIdx.x >> 6][e] = v[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 3; ++e) {
        v[e] = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v[e] += part[w][e];
    }
}

// The first request that needs more than `count` ids with those before it; by all threads of the workgroup.
__device__ __forceinline__ int first_closed(const Counts* counts, int n, uint32_t count, uint32_t (*part)[3])
{
    __shared__ int closed;
    const int tid = threadIdx.x, wid = tid >> 6;
    if (tid == 0) closed = n;
    uint32_t carry = 0;
#pragma nounroll
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        uint32_t sum = (uint32_t)wave_sums(i0 + tid < n ? taken_by(counts[i0 + tid]) : 0);
        __syncthreads();
        if ((tid & 63) == 63) part[wid][0] = sum;
        __syncthreads();
        sum += carry;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wid) sum += part[w][0];
            carry += part[w][0];
        }
        if (i0 + tid < n && sum > count) atomicMin(&closed, i0 + tid);
    }
    __syncthreads();
    return closed;
}

// A workgroup per request, and one more for the state; with one request its counts are taken here (counts: null), and there is one workgroup.
template <int ROWS> __global__ __launch_bounds__(kThreads) void kv_fork_kernel(KvFork f, const Counts* counts)
{
    __shared__ Family o;
    __shared__ Columns<ROWS> ids;
    __shared__ uint32_t part[kWaves][3];
    __shared__ int own[kBeamMax], wave_sum[kWaves];
    __shared__ uint32_t some[kThreads];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, r = blockIdx.x;
    const uint32_t count = (uint32_t)max(0, min(f.ring_state[1], f.n_blocks));
    const uint32_t head = (uint32_t)f.ring_state[0] % (uint32_t)f.n_blocks;
    if (r == f.n_requests) {
        const int closed = first_closed(counts, f.n_requests, count, part);
        uint32_t sums[3] = {0, 0, 0};         // taken, given, copies
#pragma nounroll
        for (int i = tid; i < closed; i += kThreads) {
            const Counts c = counts[i];
            sums[0] += taken_by(c), sums[1] += given_by(c), sums[2] += c.copies;
        }
        sum3(sums, part);
        if (tid == 0) {
            f.next_state[0] = ring_at(head, sums[0], f.n_blocks);
            f.next_state[1] = (int32_t)(count - sums[0] + sums[1]);
            f.next_state[2] = closed;
            f.next_state[3] = (int32_t)sums[2];
        }
        return;
    }
    Counts mine{0, 0};
    uint32_t before[3] = {0, 0, 0};           // taken from the ring, and given to it, by the requests before this one
    if (counts) {
        mine = counts[r];
#pragma nounroll
        for (int i = tid; i < r; i += kThreads) {
            const Counts c = counts[i];
            before[0] += taken_by(c), before[1] += given_by(c);
        }
    }
    read_family(o, ids, f, r);
    const int64_t row0 = (int64_t)r * f.beams;
    const int32_t* const table = f.table + row0 * f.max_blocks;
    if (!counts) mine = count_request(ids, o, f, table, wave_sum);
    else if (r > 0) sum3(before, part);
    const bool open = before[0] + taken_by(mine) <= count;
    // ids that this request takes from the ring, should it
    const int ring_id = tid < taken_by(mine) && open ? f.ring[ring_at(head, before[0] + tid, f.n_blocks)] : -1;
    if (!counts && tid == 0) {
        f.next_state[0] = ring_at(head, open ? taken_by(mine) : 0, f.n_blocks);
        f.next_state[1] = (int32_t)(count + (open ? given_by(mine) - taken_by(mine) : 0));
        f.next_state[2] = open;
        f.next_state[3] = open ? mine.copies : 0;
    }
    // a column to a thread: what is free of it, in order, and what the new rows take over
    const Share share = share_of(o.most);
    int carry = 0;
#pragma nounroll
    for (int j0 = 0; j0 < o.longest; j0 += kThreads) {
        const int j = j0 + tid;
        if (j0 > 0 || (!counts && o.most > kThreads)) read_column(ids, f, table, j);       // the first are there, but where later ones were counted
        if (open && j0 < o.most) {
            uint32_t freed = freed_in(ids, o, f, j0 + share.column, share.column, share.rows);
            if (share.parts > 1) {            // one of a column's threads has them all
                some[tid] = freed;
                lds_barrier();
                freed = 0;
                if (share.part == 0)
                    for (int i = tid; i < kThreads; i += kThreads / share.parts) freed |= some[i];
            }
            const int v = __popc(freed), sum = wave_sums(v);
            lds_barrier();
            if (lane == 63) wave_sum[wid] = sum;
            lds_barrier();
            int at = carry + sum - v;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const int u = wave_sum[w];
                at += w < wid ? u : 0;
                carry += u;
            }
#pragma nounroll
            for (; freed; freed &= freed - 1, ++at) {
                const int id = ids.id[__builtin_ctz(freed)][tid];
                if (at < mine.copies) own[at] = id;
                else f.ring[ring_at(head, count + before[1] + (at - mine.copies), f.n_blocks)] = id;
            }
        }
#pragma unroll 4
        for (int i = 0; i < f.beams; ++i) {
            const int p = open ? o.parent[i] : i, blocks = open ? o.taken[i] : o.blocks[i];
            if (j < blocks) f.next_table[(row0 + i) * f.max_blocks + j] = ids.id[p][tid];
        }
    }
    if (open && tid < taken_by(mine)) own[mine.freed + tid] = ring_id;
    lds_barrier();
    if (tid < f.beams) {
        const int p = open ? o.parent[tid] : tid, place = open ? o.place[tid] : -1;
        const int id = place >= 0 ? own[place] : -1;          // the row's own last block
        if (place >= 0) f.next_table[(row0 + tid) * f.max_blocks + o.blocks[p] - 1] = id;
        f.next_len[row0 + tid] = p >= 0 ? o.length[p] : 0;
        *(int2*)(f.copy + 2 * (row0 + tid)) = make_int2(place >= 0 ? o.last[p] : -1, place >= 0 ? id : -1);
    }
}

// A workgroup per row and layer; what bounds it is memory, so a thread has several pieces on their way at once: 24 requests of eight beams, 6 layers of 8
// heads of 128 (38 MB read and written), 10.3 to 11 us; three copies in 12 small layers 3.4 us, latency.
constexpr int kPieces = 4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__global__ __launch_bounds__(kThreads) void kv_copy_kernel(KvCaches caches, const int32_t* __restrict__ copy, const int32_t* __restrict__ seq_len)
{
    const KvCache& c = caches.c[blockIdx.y];
    const int i = blockIdx.x, length = seq_len[i], from_id = copy[2 * i], to_id = copy[2 * i + 1];
    if ((uint32_t)from_id >= (uint32_t)c.n_blocks || (uint32_t)to_id >= (uint32_t)c.n_blocks) return;
    const int size = 1 << c.block_shift, tail = length & (size - 1), rows = tail ? tail : size;
    const int per_head = c.head_dim >> 3, per_row = per_head * c.kv_heads, n = rows * per_row;
    const int64_t block = c.block_stride, token = c.token_stride, head_step = c.head_stride;
    const uint16_t *const k_from = c.k + from_id * block, *const v_from = c.v + from_id * block;
    uint16_t *const k_to = c.k + to_id * block, *const v_to = c.v + to_id * block;
    auto place = [&](int u) {
        const int row = u / per_row, rest = u - row * per_row, head = rest / per_head;
        return row * token + head * head_step + (rest - head * per_head) * 8;
    };
    for (int u0 = threadIdx.x; u0 < n; u0 += kPieces * kThreads) {
        u32x4 a[kPieces], b[kPieces];
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int64_t at = place(min(u0 + p * kThreads, n - 1));
            a[p] = *(const u32x4*)(k_from + at);
            b[p] = *(const u32x4*)(v_from + at);
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            if (u0 + p * kThreads >= n) break;
            const int64_t at = place(u0 + p * kThreads);
            *(u32x4*)(k_to + at) = a[p];
            *(u32x4*)(v_to + at) = b[p];
        }
    }
}

}  // namespace

int64_t kv_fork_workspace(int32_t n_requests, int32_t) { return (int64_t)n_requests * (int64_t)sizeof(Counts); }

template <int ROWS> static hipError_t launch_fork(const KvFork& f, Counts* counts, hipStream_t stream)
{
    if (f.n_requests == 1) {
        hipLaunchKernelGGL(kv_fork_kernel<ROWS>, dim3(1), dim3(kThreads), 0, stream, f, (const Counts*)nullptr);
        return hipGetLastError();
    }
    if (f.n_requests > 0) {
        hipLaunchKernelGGL(kv_fork_count_kernel<ROWS>, dim3((unsigned)f.n_requests), dim3(kThreads), 0, stream, f, counts);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kv_fork_kernel<ROWS>, dim3((unsigned)f.n_requests + 1), dim3(kThreads), 0, stream, f, (const Counts*)counts);
    return hipGetLastError();
}

hipError_t kv_fork(const KvFork& f, void* workspace, hipStream_t stream)
{
    return f.beams <= kGroup ? launch_fork<kGroup>(f, (Counts*)workspace, stream) : launch_fork<kBeamMax>(f, (Counts*)workspace, stream);
}

hipError_t kv_copy(int32_t n_caches, const KvCaches& caches, int32_t n, const int32_t* copy, const int32_t* seq_len, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)n, (unsigned)n_caches), dim3(kThreads), 0, stream, caches, copy, seq_len);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
