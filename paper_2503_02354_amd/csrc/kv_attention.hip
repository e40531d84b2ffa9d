// gfx950 kernels for attention over the paged key/value cache of token-generating experts (bf16).
//
// A request with m new tokens and `heads / kv_heads` = G query heads to a cache head has m G query rows per cache head that look at
// the same keys and values.  Scores are computed transposed, S^T = K Q^T, so that a lane holds ONE query row (column l % 32) and of a
// block of 32 keys the keys 8 (v / 4) + 4 (l / 32) + v % 4: the running maximum and sum of a row live in lanes l and l ^ 32, and the
// exponentials, rounded to bf16, are the second operand of O^T = V^T P^T as they lie.  V^T comes from the transposing LDS read.
//   m' = max(m, max s)    l' = l 2^(m - m') + sum 2^(s - m')    o' = o 2^(m - m') + sum 2^(s - m') v        (s in units of ln 2)
// All three are fp32; only 2^(s - m') is rounded to bf16, for the matrix cores.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attention_tiles.h"
#include "kernels.h"

namespace coe {
namespace k {

namespace {

constexpr int kKeys = 32;                 // keys of a tile
constexpr int kFewRows = 32;              // query rows of a request and cache head that the kernel for few rows takes
constexpr int kFewWaves = 4;
constexpr int kFewGroups = 512;           // its workgroups: two per compute unit
static_assert(kFewGroups <= kMostParts, "a part of every stretch at most");

// A request's new tokens and the cached tokens [begin, end) that at least one of them sees.
struct Span {
    int m, rows, first_pos, begin, end;   // new tokens taken, query rows per cache head, position of the first new token
    __device__ __forceinline__ int first_tile() const { return begin / kKeys; }
    __device__ __forceinline__ int tiles() const { return rows == 0 ? 0 : max(1, (end + kKeys - 1) / kKeys - begin / kKeys); }
};
__device__ __forceinline__ Span make_span(int m, int first_pos, int group, int window)
{
    Span s;
    s.m = m;
    s.rows = m * group;
    s.first_pos = first_pos;
    s.end = max(0, first_pos + m);
    s.begin = window > 0 ? min(s.end, max(0, max(0, first_pos) - window + 1)) : 0;      // of the largest window too
    return s;
}
__device__ __forceinline__ Span span_of(const KvAttention& a, int r, int group, int table_tokens)
{
    const int q0 = max(0, min(a.q_off[r], a.n_tokens)), q1 = max(q0, min(a.q_off[r + 1], a.n_tokens));
    const int len = max(0, min(a.seq_len[r], table_tokens)), m_all = q1 - q0;
    return make_span(min(m_all, a.max_new), len - m_all, group, a.window);
}

// Four channels of query row `row` of a request and cache head, from the unnormalised output (divided by `grow`) relative to maximum mx.
__device__ __forceinline__ void finish_row(const KvCache& c, const KvAttention& a, int q0, int kvh, int row, int ch, float mx, float sum, float4 acc, float grow = 1.f)
{
    const int group = a.heads / c.kv_heads, token = row / group, head = kvh * group + (row - token * group);
    const bool empty = is_empty(mx, sum);
    if (empty) acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const float inv = empty ? 0.f : grow / sum;
    if (ch < c.head_dim)
        *(uint2*)(a.out + (int64_t)(q0 + token) * a.out_token_stride + (int64_t)head * a.out_head_stride + ch) =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    if (a.lse && ch == 0) a.lse[(int64_t)(q0 + token) * a.heads + head] = empty ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

#if defined(__HIP_DEVICE_COMPILE__)
// Where a key may be hidden from some rows, 0 * inf would reach them through the matrix core.  Which of the 32 keys of a tile at LDS
// address `tile` have a value that is not finite:
template <int D> __device__ __forceinline__ uint32_t odd_keys(uint32_t tile)
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));            // rarely needed: its addresses are not worth registers outside
    uint32_t odd = 0;
#pragma unroll
    for (int ch = 0; ch < D / 16; ++ch) {
        const u32x4 w = *(const __attribute__((address_space(3))) u32x4*)(tile + v_slot<D>(lane & 31, 2 * ch + (lane >> 5)));
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= ((w[e] & 0x7F80u) == 0x7F80u) | ((w[e] & 0x7F800000u) == 0x7F800000u);
    }
    const unsigned long long b = __ballot(odd);
    return (uint32_t)b | (uint32_t)(b >> 32);
}
// Their rows are added to the query rows that see them (`sees(key)` says for this lane's row) by themselves,
template <int D, class Sees>
__device__ __forceinline__ void add_odd_values(f32x16 (&acc)[D / 32], uint32_t tile, uint32_t odd, const u32x4 (&p)[2], Sees sees)
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int half = lane >> 5;
#pragma nounroll
    for (; odd; odd &= odd - 1) {
        const int key = __builtin_ctz(odd), d = (key >> 3 & 1) * 2 + (key >> 1 & 1);         // dword of p[key / 16] that holds it, in lanes of half key / 4 % 2
        const uint32_t lo = d == 0 ? p[0][0] : d == 1 ? p[0][1] : d == 2 ? p[0][2] : p[0][3], hi = d == 0 ? p[1][0] : d == 1 ? p[1][1] : d == 2 ? p[1][2] : p[1][3];
        const uint32_t word = __shfl(key < 16 ? lo : hi, (lane & 31) + 32 * (key >> 2 & 1), 64);
        const float q = __uint_as_float(key & 1 ? word & 0xFFFF0000u : word << 16);
        const bool mine = sees(key);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) {     // four channels of this lane's
                const uint2 w = *(const __attribute__((address_space(3))) uint2*)(tile + v_slot<D>(key, 4 * db + g) + 8 * half);
                const float v[4] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u)};
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[db][4 * g + e] = mine ? acc[db][4 * g + e] + q * v[e] : acc[db][4 * g + e];
            }
    }
}
// and taken out of the operands: what is left of 16 keys' pairs of values (dwords)
__device__ __forceinline__ u32x4 even_only(uint32_t odd, int t2, int half)
{
    u32x4 keep;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const uint32_t at = odd >> (16 * t2 + 8 * (e >> 2) + 4 * half + (e & 3));
        keep[e >> 1] = (at & 1 ? 0u : 0x0000FFFFu) | (at & 2 ? 0u : 0xFFFF0000u);
    }
    return keep;
}
#endif

// ---- few query rows (single tokens): at most 32 per request and cache head ------------------------------------------------
// The work is the list of all 32-key tiles, (request, cache head, tile) in that order; every workgroup takes an equal stretch of
// it, so that lengths of any mix fill the chip evenly.  A stretch may begin and end inside a history (a "part"): such parts go to the
// workspace as (maximum, sum, unnormalised output) and kv_attention_join_kernel adds them up; a history inside one stretch is
// finished here.  Inside a stretch the four wavefronts take tiles in turn, each for itself: keys go from memory straight into
// registers (they are the first operand as they lie), values through registers into LDS of the wavefront's own, and the next tile's
// are on their way while this one is multiplied.
// What bounds it: HBM, keys and values once.  96 requests of 50 to 5000 tokens, 32 heads on 8 of 128 channels: 1.006 GB in 213 to 220 us, 4.7 TB/s
// (a copy of 2 GiB: 4.9); 3 of 90,000 to 131,000 tokens, 32 heads on 4: 0.72 GB in 136 to 141 us, 5.2 TB/s.  Joining the parts takes 6 to 7 us.
// Two workgroups per compute unit are all that 250 registers a lane allow, and they suffice: LDS and matrix cores stand idle.
struct FewHeader {                        // at the workspace's start, for the joining kernel
    unsigned long long per;               // tiles of a stretch
    unsigned long long base[1];           // [n_requests + 1] tiles before request r, of one cache head
};
__host__ __device__ constexpr int64_t few_header_bytes(int n_requests) { return (16 + 8 * (int64_t)(n_requests + 1) + 255) / 256 * 256; }
// a part: maxima and sums [2][32], then the output [32][D]
template <int D> constexpr int kPartFloats = 2 * kFewRows + kFewRows * D;

template <int D> constexpr int kMergeRow = D + 4;          // floats between the rows of a wavefront's output in LDS
template <int D, int WAVES = kFewWaves> constexpr size_t kFewLds = (size_t)WAVES * kFewRows * kMergeRow<D> * 4;

#if defined(__HIP_DEVICE_COMPILE__)
// Query rows [row0, row0 + rows), at most 32, at positions low to high, of a request and cache head over the 32-key tiles [tile_begin, tile_stop), by WAVES wavefronts:
// write(row - row0, channel, maximum, sum, four channels of the unnormalised output) gets the result, relative to the row's maximum.
template <int D, bool PAD, int WAVES, class Write>
__device__ __forceinline__ void few_rows(const KvCache& c, const KvAttention& a, const Span& s, int r, int kvh, int row0, int rows, int low, int high, int tile_begin, int tile_stop, char* lds,
                                         float (*stat)[WAVES][kFewRows], Write write)
{
    constexpr int kSteps = D / 16, kBlocks = D / 32;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int group = a.heads / c.kv_heads, q0 = max(0, min(a.q_off[r], a.n_tokens));
    const int chunks = c.head_dim >> 3, last_step = (chunks - 1 - half) >> 1;       // this lane's last 16 bytes of a row; -1: none (8 channels)
    const float scale2 = a.scale * 1.44269504088896340736f;
    char* const v_lds = lds + wid * (kKeys * kRow<D> * 2);
    const uint32_t v_tile = lds_address(v_lds), v_read = v_tile + value_base<D>(lane);

    // this lane's query row
    const int row = row0 + l32, token = row / group, head = kvh * group + (row - token * group);
    const bool row_ok = l32 < rows;
    const int pos = s.first_pos + token, from = a.window > 0 ? pos - a.window : -1;       // sees keys from < j <= pos
    bf16x8 qf[kSteps];
    {
        const uint16_t* qp = a.q + (int64_t)(q0 + (row_ok ? token : 0)) * a.q_token_stride + (int64_t)(row_ok ? head : 0) * a.q_head_stride + half * 8;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            u32x4 w = {0, 0, 0, 0};
            if (row_ok && (!PAD || 2 * ks + half < chunks)) w = *(const u32x4*)(qp + ks * 16);
            qf[ks] = __builtin_bit_cast(bf16x8, w);
        }
    }
    float m = -INFINITY, l = 0.f;
    f32x16 o[kBlocks];
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[db][x] = 0.f;

    const int32_t* const ids = a.table + (size_t)r * a.max_blocks;
    const int64_t lane_at = kvh * c.head_stride + (PAD && last_step < 0 ? 0 : half * 8);
    const uint16_t *const k_base = c.k + lane_at, *const v_base = c.v + lane_at;
    auto id_of = [&](int tile) {      // block of this lane's key of a tile; -1: reads as zeros
        const int key = tile * kKeys + l32;
        int id = -1;
        if (key >= s.begin && key < s.end) id = ids[key >> c.block_shift];
        return (uint32_t)id < (uint32_t)c.n_blocks ? id : -1;
    };
    auto offset_of = [&](int tile, int id) {
        const int key = tile * kKeys + l32;
        return id < 0 ? (int64_t)0 : id * c.block_stride + (key & ((1 << c.block_shift) - 1)) * c.token_stride;
    };
    auto fetch = [&](const uint16_t* p, u32x4 (&w)[kSteps]) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) w[ks] = *(const u32x4*)(p + (PAD ? max(0, min(ks, last_step)) : ks) * 16);
    };
    u32x4 kw[kSteps], vw[kSteps];
    int tile = tile_begin + wid;
    int id = -1, id_next = -1;
    if (tile < tile_stop) {
        id = id_of(tile);
        const int64_t at = offset_of(tile, id);
        fetch(k_base + at, kw);
        fetch(v_base + at, vw);
        if (tile + WAVES < tile_stop) id_next = id_of(tile + WAVES);
    }
    for (; tile < tile_stop; tile += WAVES) {
        const bool more = tile + WAVES < tile_stop;
        if (__any(id < 0)) {          // rows outside the history, blocks outside the cache
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) {
                kw[ks] = id < 0 ? u32x4{0, 0, 0, 0} : kw[ks];
                vw[ks] = id < 0 ? u32x4{0, 0, 0, 0} : vw[ks];
            }
        }
        if (PAD)                      // what was read in the place of channels that are not there; the values' have results of their own
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) kw[ks] = ks <= last_step ? kw[ks] : u32x4{0, 0, 0, 0};
        f32x16 sc;
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kw[ks]), qf[ks], sc, 0, 0, 0);
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) *(u32x4*)(v_lds + v_slot<D>(l32, 2 * ks + half)) = vw[ks];
        if (more) {
            id = id_next;
            const int64_t at = offset_of(tile + WAVES, id);
            fetch(k_base + at, kw);
            fetch(v_base + at, vw);
            if (tile + 2 * WAVES < tile_stop) id_next = id_of(tile + 2 * WAVES);
        }
        const int key0 = tile * kKeys;
        const bool masked = key0 + kKeys - 1 > low || key0 < s.begin || (a.window > 0 && key0 <= high - a.window);
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            sc[x] *= scale2;
            const int key = key0 + 8 * (x >> 2) + 4 * half + (x & 3);
            if (masked) sc[x] = row_ok && key <= pos && key > from && key >= 0 ? sc[x] : -INFINITY;
            top = fmaxf(top, sc[x]);
        }
        top = max_halves(top);
        const float m_new = fmaxf(m, top);
        if (__any(m_new > m)) {
            const float shrink = m_new == m ? 1.f : exp2_fast(m - m_new);
            l *= shrink;
#pragma unroll
            for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                for (int x = 0; x < 16; ++x) o[db][x] *= shrink;
            m = m_new;
        }
        const float m_use = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            sc[x] = exp2_fast(sc[x] - m_use);
            l += sc[x];
        }
        u32x4 pw[2];
#pragma unroll
        for (int x = 0; x < 16; x += 2) pw[x >> 3][(x >> 1) & 3] = pack_bf16(sc[x], sc[x + 1]);
        if (masked && s.m > 1) {
            const uint32_t odd = odd_keys<D>(v_tile);
            if (odd) {                    // the tile is this wavefront's own: their rows are made zeros
                add_odd_values<D>(o, v_tile, odd, pw, [&](int j) { return row_ok && key0 + j <= pos && key0 + j > from; });
                if (odd >> l32 & 1)
                    for (int ch = half; ch < kRow<D> / 8; ch += 2) *(__attribute__((address_space(3))) u32x4*)(v_tile + v_slot<D>(l32, ch)) = u32x4{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) {
            u32x4 v[kBlocks];
            read_values<D>(v, v_read, t2);
            add_values<D>(o, v, pw[t2]);
        }
    }
    l = sum_halves(l);

    // the wavefronts' results
    __syncthreads();
    float* const mine = (float*)lds + wid * kFewRows * kMergeRow<D> + l32 * kMergeRow<D>;
    if (row_ok) {
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(float4*)(mine + db * 32 + g * 8 + half * 4) = make_float4(o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]);
    }
    if (half == 0) {
        stat[0][wid][l32] = m;
        stat[1][wid][l32] = l;
    }
    __syncthreads();
    for (int i = tid; i < rows * (D / 4); i += 64 * WAVES) {
        const int rw = i / (D / 4), ch = (i - rw * (D / 4)) * 4;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) mx = fmaxf(mx, stat[0][w][rw]);
        float sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float mw = stat[0][w][rw];
            const float f = mw == mx ? 1.f : exp2_fast(mw - mx);
            const float4 v = *(const float4*)((const float*)lds + (w * kFewRows + rw) * kMergeRow<D> + ch);
            sum += f * stat[1][w][rw];
            acc.x += f * v.x, acc.y += f * v.y, acc.z += f * v.z, acc.w += f * v.w;
        }
        write(rw, ch, mx, sum, acc);
    }
}
#endif

template <int D, bool PAD>
__global__ __launch_bounds__(64 * kFewWaves, 2) void kv_attention_few_kernel(KvCache c, KvAttention a, char* workspace)
{
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(4096))) char lds[];
    __shared__ float stat[2][kFewWaves][kFewRows];
    __shared__ unsigned long long part_sum[kFewWaves];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = a.heads / c.kv_heads, table_tokens = a.max_blocks << c.block_shift, n = a.n_requests;

    // tiles before every request
    unsigned long long* const base = (unsigned long long*)lds;
    unsigned long long carry = 0;
    for (int r0 = 0; r0 < n; r0 += 64 * kFewWaves) {
        unsigned long long v = 0;
        if (r0 + tid < n) {
            const Span s = span_of(a, r0 + tid, group, table_tokens);
            v = (unsigned long long)s.tiles();
        }
        unsigned long long sum = v;
        for (int d = 1; d < 64; d <<= 1) {
            const unsigned long long u = __shfl_up(sum, d, 64);
            if (lane >= d) sum += u;
        }
        if (lane == 63) part_sum[wid] = sum;
        __syncthreads();
        unsigned long long before = carry;
        for (int w = 0; w < kFewWaves; ++w) {
            if (w < wid) before += part_sum[w];
            carry += part_sum[w];
        }
        if (r0 + tid < n) base[r0 + tid] = before + sum - v;
        __syncthreads();
    }
    if (tid == 0) base[n] = carry;
    __syncthreads();
    const unsigned long long total = carry * (unsigned)c.kv_heads;
    const unsigned long long share = (total + gridDim.x - 1) / gridDim.x, per = max(4ull, (share + 3) / 4 * 4);
    if (blockIdx.x == 0) {
        FewHeader* h = (FewHeader*)workspace;
        for (int r = tid; r <= n; r += 64 * kFewWaves) h->base[r] = base[r];
        if (tid == 0) h->per = per;
    }
    unsigned long long now = blockIdx.x * per;
    const unsigned long long stop = min(total, now + per);
    if (now >= stop) return;
    int r = 0;
    for (int hi = n; hi - r > 1;) {       // the last request that begins at or before `now`
        const int mid = (r + hi) >> 1;
        if (base[mid] * (unsigned)c.kv_heads <= now) r = mid;
        else hi = mid;
    }
    r = __builtin_amdgcn_readfirstlane(r);
    unsigned long long into = now - base[r] * (unsigned)c.kv_heads;       // tiles of this request that others did
    __syncthreads();

    const unsigned long long start = now;

    while (now < stop && r < n) {
        Span s = span_of(a, r, group, table_tokens);
        const int tiles = s.tiles();
        if (into >= (unsigned long long)tiles * (unsigned)c.kv_heads) {
            into = 0;
            ++r;
            continue;
        }
        const int kvh = (int)(into / (unsigned)tiles), t_begin = (int)(into - (unsigned long long)kvh * (unsigned)tiles);
        const int t_end = (int)min((unsigned long long)tiles, t_begin + (stop - now)), first = s.first_tile();
        const int q0 = max(0, min(a.q_off[r], a.n_tokens));

        const bool whole = t_begin == 0 && t_end == tiles;
        float* const part = (float*)(workspace + few_header_bytes(n)) + ((size_t)blockIdx.x * 2 + (now != start)) * kPartFloats<D>;
        few_rows<D, PAD, kFewWaves>(c, a, s, r, kvh, 0, s.rows, s.first_pos, s.first_pos + s.m - 1, first + t_begin, first + t_end, lds, stat, [&](int rw, int ch, float mx, float sum, float4 acc) __attribute__((always_inline)) {
            if (whole) finish_row(c, a, q0, kvh, rw, ch, mx, sum, acc);
            else {
                *(float4*)(part + 2 * kFewRows + rw * D + ch) = acc;
                if (ch == 0) {
                    part[rw] = mx;
                    part[kFewRows + rw] = sum;
                }
            }
        });
        __syncthreads();
        now += (unsigned)(t_end - t_begin);
        into += (unsigned)(t_end - t_begin);
    }
#endif
}

// Where histories are short and rows are few: a workgroup per request, cache head and 32 query rows (those that see most first), one launch,
// and no parts to join.  What bounds it: latency, tiles in turn; one token behind 612, 12 heads of 64 channels, 9.3 us.
template <int D, bool PAD, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 8 / WAVES) void kv_attention_short_kernel(KvCache c, KvAttention a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(4096))) char lds[];
    __shared__ float stat[2][WAVES][kFewRows];
    const int r = blockIdx.x / c.kv_heads, kvh = blockIdx.x - r * c.kv_heads, row0 = (int)(gridDim.y - 1 - blockIdx.y) * kFewRows, group = a.heads / c.kv_heads;
    const Span s = span_of(a, r, group, a.max_blocks << c.block_shift);
    if (row0 >= s.rows) return;
    const int q0 = max(0, min(a.q_off[r], a.n_tokens)), rows = min(kFewRows, s.rows - row0);
    const int low = s.first_pos + (row0 == 0 ? 0 : row0 / group), high = s.first_pos + (row0 + rows == s.rows ? s.m : (row0 + rows - 1) / group + 1) - 1;
    const int begin = a.window > 0 ? max(0, max(0, low) - a.window + 1) : 0, end = max(0, high + 1);
    few_rows<D, PAD, WAVES>(c, a, s, r, kvh, row0, rows, low, high, begin / kKeys, (end + kKeys - 1) / kKeys, lds, stat,
                            [&](int rw, int ch, float mx, float sum, float4 acc) __attribute__((always_inline)) { finish_row(c, a, q0, kvh, row0 + rw, ch, mx, sum, acc); });
#endif
}

// Adds up the parts of a history that several workgroups shared: a workgroup per request, cache head and kJoinRows query rows
// (blockIdx.y).  Several threads share the parts of a row's four channels, since a long history has many; each leaves its sum
// relative to its own maximum, and the first adds those up in their order.  What bounds it: round trips to memory, so every thread fetches
// four parts at a time: three histories of 131,000 tokens, a hundred parts and more to each, 6.5 us (9.2 with two at a time, 8.3 with 1024
// threads, which cost 96 requests 18.5 instead of 6.9).
constexpr int kJoinRows = 1, kAhead = 4;
template <int D>
__global__ __launch_bounds__(256) void kv_attention_join_kernel(KvCache c, KvAttention a, const char* workspace)
{
    constexpr int kColumns = kJoinRows * D / 4, kSplit = 256 / kColumns;
    __shared__ float4 sums[256];
    __shared__ float2 stats[256];
    const FewHeader* const h = (const FewHeader*)workspace;
    const int r = blockIdx.x / c.kv_heads, kvh = blockIdx.x - r * c.kv_heads, group = a.heads / c.kv_heads;
    const unsigned long long first = h->base[r], tiles = h->base[r + 1] - first, per = h->per;
    const int rows = span_of(a, r, group, a.max_blocks << c.block_shift).rows, q0 = max(0, min(a.q_off[r], a.n_tokens));      // on their way together
    if (tiles == 0) return;
    const unsigned long long begin = first * (unsigned)c.kv_heads + (unsigned)kvh * tiles, end = begin + tiles;
    const unsigned long long w0 = begin / per, w1 = (end - 1) / per;
    if (w0 == w1) return;
    const int column = threadIdx.x % kColumns, share = threadIdx.x / kColumns;
    const int rw = blockIdx.y * kJoinRows + column / (D / 4), ch = column % (D / 4) * 4;
    if (blockIdx.y * kJoinRows >= rows) return;
    // a stretch's first history leaves the first part, its last one the second
    const float* const parts = (const float*)(workspace + few_header_bytes(a.n_requests));
    auto part_of = [&](unsigned long long w) { return parts + (w * 2 + (begin > w * per)) * kPartFloats<D>; };
    float mx = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (rw < rows && share < kSplit)
        for (unsigned long long w = w0 + share; w <= w1; w += kAhead * kSplit) {
            float mw[kAhead], lw[kAhead];
            float4 v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {            // on their way together
                const float* const p = part_of(min(w + i * kSplit, w1));
                mw[i] = p[rw];
                lw[i] = p[kFewRows + rw];
                v[i] = *(const float4*)(p + 2 * kFewRows + rw * D + ch);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (w + i * kSplit > w1) continue;
                const float m_new = fmaxf(mx, mw[i]), keep = weight_of_part(mx, m_new), f = weight_of_part(mw[i], m_new);
                sum = sum * keep + f * lw[i];
                const float g = f * kJoinRoom;
                acc.x = acc.x * keep + g * v[i].x, acc.y = acc.y * keep + g * v[i].y, acc.z = acc.z * keep + g * v[i].z, acc.w = acc.w * keep + g * v[i].w;
                mx = m_new;
            }
        }
    sums[threadIdx.x] = acc;
    stats[threadIdx.x] = make_float2(mx, sum);
    __syncthreads();
    if (share > 0 || rw >= rows) return;
    for (int i = 1; i < kSplit; ++i) mx = fmaxf(mx, stats[i * kColumns + column].x);
    sum = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < kSplit; ++i) {
        const float2 st = stats[i * kColumns + column];
        const float f = weight_of_part(st.x, mx);
        const float4 v = sums[i * kColumns + column];
        sum += f * st.y;
        acc.x += f * v.x, acc.y += f * v.y, acc.z += f * v.z, acc.w += f * v.w;
    }
    finish_row(c, a, q0, kvh, rw, ch, mx, sum, acc, 1.f / kJoinRoom);
}

// ---- many query rows (chunks of prompts, single tokens among them): steps with more than 32 per request and cache head that are not short ----
// Units of work are tiles of 128 query rows (32 to a wavefront) of a request and cache head, with all the 64-key tiles that one of
// them sees.  A scheduling launch lists them, longest first, so that the last workgroups to start are short ones; where there are too
// few units to fill the chip it cuts long ones into parts over the keys, which kv_attention_join_units_kernel adds up.  Block b
// takes cache head b % kv_heads, so that with eight of them (or four, or two) the units of one head meet in the same second-level caches.
// K tiles go from memory into two LDS buffers by DMA, V tiles into three, in turn; a wavefront reads every key and value of a tile for
// its 32 rows.  What bounds it: matrix and vector instructions, at the clock that the power leaves (1.85 GHz): two prompts of some 8,000
// tokens behind 1000 and 2000, 32 heads on 8 of 128 channels, 1.28 TFLOP in 1.24 to 1.39 ms, 0.92 to 1.03 PFLOP/s from card to card, where a matrix product of
// 8192 x 8192 x 8192 reaches 1.16 to 1.19; a matrix instruction takes 1 KiB of LDS reads, without bank conflicts.  Wavefronts of 64 rows would halve
// those and do not fit the registers (4.8 ms).
constexpr int kManyRows = 128, kManyKeys = 64, kManyWaves = 4;
constexpr int kManyGroups = 512;          // two workgroups per compute unit

struct Unit {
    int32_t request, first_row;           // request; first query row of the tile
    int32_t tile, tiles;                  // 64-key tiles
    int32_t part;                         // -1, or the part of the workspace that takes the result (times kv_heads)
    int32_t q0, m, first_pos;             // the request's first new token, how many, and its position
};
struct Joined {
    int32_t first_row, part, parts, q0;
    int32_t rows, pad[3];                 // of the request
};
struct ManyHeader { int32_t units, joined, pad[62]; };

// where the workspace's pieces begin
struct ManyLayout {
    int64_t most_units, most_joined, header, units, joined, parts, end;
};
__host__ __device__ inline ManyLayout many_layout(int32_t n_requests, int32_t n_tokens, int32_t heads, int32_t kv_heads, int32_t dim)
{
    ManyLayout l;
    const int64_t rows = (int64_t)n_tokens * (heads / kv_heads), cuts = (kManyGroups + kv_heads - 1) / kv_heads;
    l.most_units = rows / kManyRows + n_requests + cuts;
    l.most_joined = cuts;
    l.header = 0;
    l.units = sizeof(ManyHeader);
    l.joined = l.units + round256(l.most_units * (int64_t)sizeof(Unit));
    l.parts = l.joined + round256(l.most_joined * (int64_t)sizeof(Joined));
    l.end = l.parts + 2 * cuts * kv_heads * (int64_t)(2 * kManyRows + kManyRows * dim) * 4;
    return l;
}

// 64-key tiles that the query rows [row, row + 128) of a request see
__device__ __forceinline__ void tiles_of(const Span& s, int window, int group, int row, int& first, int& count)
{
    const int last = min(s.rows, row + kManyRows) - 1;
    const int end = max(0, s.first_pos + last / group + 1), begin = window > 0 ? min(end, max(0, max(0, s.first_pos + row / group) - window + 1)) : 0;
    first = begin / kManyKeys;
    count = max(1, (end + kManyKeys - 1) / kManyKeys - first);
}

// One workgroup: latency.  6.7 us for 40 requests.
constexpr int kSchedThreads = 1024, kSchedBins = 2048, kSchedInLds = 4096;
__global__ __launch_bounds__(kSchedThreads) void kv_attention_schedule_kernel(KvCache c, KvAttention a, char* workspace, ManyLayout at)
{
    extern __shared__ int32_t first_segment[];            // [n_requests + 1] row tiles before request r
    __shared__ unsigned long long wave_sum[kSchedThreads / 64];
    __shared__ int32_t bins[kSchedBins];
    __shared__ int32_t n_parts, n_joined;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = a.n_requests;
    const int group = a.heads / c.kv_heads, table_tokens = a.max_blocks << c.block_shift;
    int32_t *const news = first_segment + n + 1, *const firsts = news + n, *const q0s = firsts + n;        // of the requests, where they fit
    const bool in_lds = n <= kSchedInLds;
    auto sum_before = [&](uint32_t v, unsigned long long& all) {          // 64 of them are below 2^32
        uint32_t sum = v;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t u = __shfl_up(sum, d, 64);
            if (lane >= d) sum += u;
        }
        __syncthreads();
        if (lane == 63) wave_sum[wid] = sum;
        __syncthreads();
        unsigned long long before = sum - v;
        all = 0;
#pragma unroll
        for (int w = 0; w < kSchedThreads / 64; ++w) {
            const unsigned long long u = wave_sum[w];
            before += w < wid ? u : 0;
            all += u;
        }
        return before;
    };
    unsigned long long segments = 0;
    for (int r0 = 0; r0 < n; r0 += kSchedThreads) {
        int v = 0;
        if (r0 + tid < n) {
            const Span s = span_of(a, r0 + tid, group, table_tokens);
            v = (s.rows + kManyRows - 1) / kManyRows;     // below 2^24
            if (in_lds) {
                news[r0 + tid] = s.m;
                firsts[r0 + tid] = s.first_pos;
                q0s[r0 + tid] = max(0, min(a.q_off[r0 + tid], a.n_tokens));
            }
        }
        unsigned long long all;
        const unsigned long long before = segments + sum_before((uint32_t)v, all);
        if (r0 + tid < n) first_segment[r0 + tid] = (int32_t)min(before, (unsigned long long)at.most_units);
        segments += all;
    }
    const int count = (int)min(segments, (unsigned long long)at.most_units);      // the sum of the requests' rows is at most n_tokens * group
    if (tid == 0) first_segment[n] = count;
    for (int i = tid; i < kSchedBins; i += kSchedThreads) bins[i] = 0;
    if (tid == 0) n_parts = n_joined = 0;
    __syncthreads();
    struct Segment { int r, row, first, tiles, q0; Span s; };
    auto find = [&](int i) {
        Segment g;
        int r = 0;
        for (int hi = n; hi - r > 1;) {
            const int mid = (r + hi) >> 1;
            if (first_segment[mid] <= i) r = mid;
            else hi = mid;
        }
        g.r = r;
        g.s = in_lds ? make_span(news[r], firsts[r], group, a.window) : span_of(a, r, group, table_tokens);
        g.q0 = in_lds ? q0s[r] : max(0, min(a.q_off[r], a.n_tokens));
        g.row = (i - first_segment[r]) * kManyRows;
        tiles_of(g.s, a.window, group, g.row, g.first, g.tiles);
        return g;
    };
    const Segment own = tid < count ? find(tid) : Segment{};             // the only one in most steps
    auto segment = [&](int i) { return i == tid ? own : find(i); };
    unsigned long long mine = 0;
    for (int i = tid; i < count; i += kSchedThreads) mine += (unsigned)segment(i).tiles;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) mine += __shfl_xor(mine, d, 64);
    if (lane == 0) wave_sum[wid] = mine;      // read by all before the barrier that ends the segments' sums
    __syncthreads();
    unsigned long long total = 0;
#pragma unroll
    for (int w = 0; w < kSchedThreads / 64; ++w) total += wave_sum[w];
    // no part is shorter than 8 tiles, or than what fills the chip once
    const int most = (int)max(8ull, (total * (unsigned)c.kv_heads + kManyGroups - 1) / kManyGroups);
    // longest first: by length, the longer halves of the range in coarser steps
    int scale = 0;
    while ((most >> scale) >= kSchedBins) ++scale;
    auto bin_of = [&](int tiles) { return kSchedBins - 1 - min(kSchedBins - 1, tiles >> scale); };
    for (int i = tid; i < count; i += kSchedThreads) {
        const int tiles = segment(i).tiles, parts = (tiles + most - 1) / most, each = (tiles + parts - 1) / parts;
        atomicAdd(&bins[bin_of(each)], parts);
    }
    __syncthreads();
    {                                         // exclusive sums of the bins
        constexpr int kPer = kSchedBins / kSchedThreads;
        int own[kPer], sum = 0;
        for (int j = 0; j < kPer; ++j) {
            own[j] = bins[tid * kPer + j];
            sum += own[j];
        }
        unsigned long long all;
        int before = (int)sum_before((uint32_t)sum, all);
        for (int j = 0; j < kPer; ++j) {
            bins[tid * kPer + j] = before;
            before += own[j];
        }
        if (tid == 0) ((ManyHeader*)(workspace + at.header))->units = (int32_t)min(all, (unsigned long long)at.most_units);
    }
    __syncthreads();
    Unit* const units = (Unit*)(workspace + at.units);
    Joined* const joined = (Joined*)(workspace + at.joined);
    for (int i = tid; i < count; i += kSchedThreads) {
        const Segment g = segment(i);
        const int tiles = g.tiles, parts = (tiles + most - 1) / most, each = (tiles + parts - 1) / parts, q0 = g.q0;
        const int to = atomicAdd(&bins[bin_of(each)], parts);
        int part = -1;
        if (parts > 1) {
            part = atomicAdd(&n_parts, parts);
            const int j = atomicAdd(&n_joined, 1);
            if (j < at.most_joined) joined[j] = {g.row, part, parts, q0, g.s.rows, {0, 0, 0}};
        }
        for (int p = 0; p < parts; ++p) {
            const int t0 = p * each, t1 = min(tiles, t0 + each);
            if (to + p < at.most_units) units[to + p] = {g.r, g.row, g.first + t0, max(0, t1 - t0), part < 0 ? -1 : part + p, q0, g.s.m, g.s.first_pos};
        }
    }
    __syncthreads();
    if (tid == 0) ((ManyHeader*)(workspace + at.header))->joined = min(n_joined, (int)at.most_joined);
}

typedef const __attribute__((address_space(4))) int32_t constant_int;

template <int D> constexpr int kManyTile = kManyKeys * kRow<D> * 2;  // bytes of a K (or V) tile

template <int D>
__global__ __launch_bounds__(64 * kManyWaves, 2) void kv_attention_many_kernel(KvCache c, KvAttention a, char* workspace, ManyLayout layout)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int DH = kRow<D>, kSteps = D / 16, kBlocks = D / 32, kTile = kManyTile<D>;
    constexpr int kRowsPerLoad = 1024 / (DH * 2), kLoads = kManyKeys / kRowsPerLoad / kManyWaves;     // of K, and the same of V
    extern __shared__ __attribute__((aligned(4096))) char lds[];          // two buffers of K tiles, three of V
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int kvh = blockIdx.x % c.kv_heads, index = blockIdx.x / c.kv_heads;
    // one round trip for the number of units and the unit, whose place is there in any case
    const int units = ((const ManyHeader*)(workspace + layout.header))->units;
    const int4 *const up = (const int4*)((const Unit*)(workspace + layout.units) + index), u0 = up[0], u1 = up[1];
    if (index >= units) return;
    const int r = __builtin_amdgcn_readfirstlane(u0.x), row0 = __builtin_amdgcn_readfirstlane(u0.y);
    const int tile0 = __builtin_amdgcn_readfirstlane(u0.z), tiles = __builtin_amdgcn_readfirstlane(u0.w), part = __builtin_amdgcn_readfirstlane(u1.x);
    const int group = a.heads / c.kv_heads, q0 = __builtin_amdgcn_readfirstlane(u1.y);
    const Span s = make_span(__builtin_amdgcn_readfirstlane(u1.z), __builtin_amdgcn_readfirstlane(u1.w), group, a.window);
    const int chunks = c.head_dim >> 3;

    // this lane's query row; a negative scale moves to the queries
    const int row = row0 + wid * 32 + l32, token = row / group, head = kvh * group + (row - token * group);
    const bool row_ok = row < s.rows;
    const int pos = s.first_pos + token, from = a.window > 0 ? pos - a.window : -1;
    // positions of this wavefront's first and last row
    const int low = __builtin_amdgcn_readfirstlane(s.first_pos + (row0 + wid * 32) / group);
    const int high = __builtin_amdgcn_readfirstlane(s.first_pos + (min(s.rows, row0 + wid * 32 + 32) - 1) / group);
    const bool works = row0 + wid * 32 < s.rows;
    u32x4 q_raw[kSteps];
    {                                         // all on their way before one is looked at; what is no row or channel becomes zeros then
        const uint16_t* const qp = a.q + (int64_t)(q0 + (row_ok ? token : 0)) * a.q_token_stride + (int64_t)(row_ok ? head : 0) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) q_raw[ks] = *(const u32x4*)(qp + (2 * ks + half < chunks ? ks * 16 + half * 8 : 0));
    }
    bf16x8 qf[kSteps];
    const float scale2 = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 1.4e-45f);          // a mask of -inf stays one with a scale of 0

    // Lane i of a load fills slot i % (DH / 8) of row i / (DH / 8) of its rows, and fetches the chunk that belongs there.
    const int ld_row = lane / (DH / 8), ld_slot = lane % (DH / 8);
    const uint32_t row_bytes = (uint32_t)c.token_stride * 2u;
    constant_int* const ids = (constant_int*)(uint64_t)(a.table + (size_t)r * a.max_blocks);
    const uint64_t head_bytes = (uint64_t)kvh * (uint64_t)c.head_stride * 2u;
    const int block_mask = (1 << c.block_shift) - 1;
    uint32_t lane_at[kLoads];                 // offset from this wavefront's first row of a tile, all of them in one block
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int chunk = (int)(v_slot<D>((wid * kLoads + j) * kRowsPerLoad + ld_row, ld_slot) / 16) & (DH / 8 - 1);        // the order is its own inverse
        lane_at[j] = chunk < chunks ? (uint32_t)(j * kRowsPerLoad + ld_row) * row_bytes + (uint32_t)chunk * 16u : kOutOfRange;
    }
    const int wave_row = wid * kLoads * kRowsPerLoad;
    auto id_at = [&](int key) { return ids[max(0, min(key, s.end - 1)) >> c.block_shift]; };
    auto block_of = [&](int id, int key) {    // byte offset of a row in the cache
        return (uint64_t)id * (uint64_t)c.block_stride * 2u + head_bytes + (uint64_t)(key & block_mask) * row_bytes;
    };
    // K of tile t goes to buffer t % 2, V to buffer t % 3: while tile t is worked on, K and V of t + 1 are there or on their way.  The block id
    // of this wavefront's sixteen rows is on its way before the tile's turn.
    int next_id = 0;
    auto fetch_id = [&](int t) __attribute__((always_inline)) { next_id = id_at((tile0 + t) * kManyKeys + wave_row); };
    auto load = [&](int t) __attribute__((always_inline)) {
        char *const k_to = lds + t % 2 * kTile + wave_row * (DH * 2), *const v_to = lds + (2 + t % 3) * kTile + wave_row * (DH * 2);
        const int key0 = (tile0 + t) * kManyKeys, first = key0 + wave_row;
        // two prompts of 4000 tokens: blocks of 16 and 64 rows, which are loaded here, 494 us, blocks of 8 rows 556
        if (key0 >= s.begin && key0 + kManyKeys <= s.end && block_mask >= 15 && (uint32_t)next_id < (uint32_t)c.n_blocks) {
            const uint64_t block = block_of(next_id, first);
            const __amdgpu_buffer_rsrc_t k_rsrc = __builtin_amdgcn_make_buffer_rsrc((char*)c.k + block, 0, 0x7FFFFFFF, 0x00020000);
            const __amdgpu_buffer_rsrc_t v_rsrc = __builtin_amdgcn_make_buffer_rsrc((char*)c.v + block, 0, 0x7FFFFFFF, 0x00020000);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (lds_void*)(k_to + j * 1024), 16, lane_at[j], 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (lds_void*)(v_to + j * 1024), 16, lane_at[j], 0, 0, 0);
            }
            return;
        }
        // the history's first or last tile, blocks of eight rows, blocks outside the cache
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int key = first + j * kRowsPerLoad, id = id_at(key);
            const bool known = (uint32_t)id < (uint32_t)c.n_blocks, inside = key + ld_row < s.end && key + ld_row >= s.begin;
            const uint32_t at = inside && lane_at[j] != kOutOfRange ? lane_at[j] - (uint32_t)(j * kRowsPerLoad) * row_bytes : kOutOfRange;
            const uint64_t block = block_of(known ? id : 0, key);
            const int size = known ? 0x7FFFFFFF : 0;
            const __amdgpu_buffer_rsrc_t k_rsrc = __builtin_amdgcn_make_buffer_rsrc((char*)c.k + block, 0, size, 0x00020000);
            const __amdgpu_buffer_rsrc_t v_rsrc = __builtin_amdgcn_make_buffer_rsrc((char*)c.v + block, 0, size, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (lds_void*)(k_to + j * 1024), 16, at, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (lds_void*)(v_to + j * 1024), 16, at, 0, 0, 0);
        }
    };
    // operand addresses inside a tile; 16 channels further is a bit of the chunks' order
    const uint32_t lds0 = lds_address(lds), k_base = v_slot<D>(l32, half), v_base = value_base<D>(lane);
    uint32_t k_read[kSteps], v_read[kBlocks][2];                          // of the tile that is read next
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) k_read[ks] = lds0 + (k_base ^ (ks * 32));
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int i = 0; i < 2; ++i) v_read[db][i] = lds0 + 2 * kTile + (v_base ^ (db * 64 + i * (32 + 16 * DH)));

    float m = -INFINITY, l = 0.f;
    f32x16 o[kBlocks], sc, next;
    u32x4 v0[kBlocks], v1[kBlocks];           // values of the half that is worked on
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[db][x] = 0.f;

    // Half a tile at a time: scores of the next half (matrix cores) are computed beside the exponentials of this one (vector unit), and the
    // next half's maximum beside this one's values.
    auto read_keys = [&](u32x4 (&k)[kSteps], int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) k[ks] = *(const __attribute__((address_space(3))) u32x4*)(k_read[ks] + kb * 32 * DH * 2);
    };
    auto read_half = [&](u32x4 (&v)[kBlocks], int kb, int t2) __attribute__((always_inline)) {
#pragma unroll
        for (int db = 0; db < kBlocks; ++db) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v_read[db][0] + (kb * 32 + t2 * 16) * DH * 2));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v_read[db][1] + (kb * 32 + t2 * 16) * DH * 2));
            v[db] = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
    auto scores = [&](f32x16& to, const u32x4 (&k)[kSteps]) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 16; ++x) to[x] = 0.f;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[ks]), qf[ks], to, 0, 0, 0);
    };
    auto is_masked = [&](int t, int kb) {
        const int key0 = (tile0 + t) * kManyKeys + kb * 32;
        return key0 + 31 > low || (a.window > 0 && key0 <= high - a.window);
    };
    auto mask = [&](f32x16& v, int t, int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const int key = (tile0 + t) * kManyKeys + kb * 32 + 8 * (x >> 2) + 4 * half + (x & 3);
            if (!(row_ok && key <= pos && key > from)) v[x] = -INFINITY;
        }
    };
    auto highest = [&](const f32x16& v) __attribute__((always_inline)) {
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 16; ++x) top = fmaxf(top, v[x]);
        top = max_halves(top);
        return top == -INFINITY ? top : top * scale2;         // scale2 >= 0 keeps the order; 0 times -inf would not be a mask any more
    };
    auto raise = [&](float top) __attribute__((always_inline)) {
        const float m_new = fmaxf(m, top), shrink = m_new == m ? 1.f : exp2_fast(m - m_new);
        l *= shrink;
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int x = 0; x < 16; ++x) o[db][x] *= shrink;
        m = m_new;
    };
    // The exponentials of a half, packed; returns this lane's sum.
    auto weigh = [&](const f32x16& v, u32x4 (&pw)[2]) __attribute__((always_inline)) {
        const float m_use = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int x = 0; x < 16; x += 2) {
            const float p0 = exp2_fast(__builtin_fmaf(v[x], scale2, -m_use)), p1 = exp2_fast(__builtin_fmaf(v[x + 1], scale2, -m_use));
            sum += p0 + p1;
            pw[x >> 3][(x >> 1) & 3] = pack_bf16(p0, p1);
        }
        return sum;
    };
    // the half (t, kb), whose scores are in `cur`; the next half's, (tn, kn), go to `to` (of no use behind the last one, and not used)
    auto half_step = [&](f32x16& cur, f32x16& to, int t, int kb, int tn, int kn) __attribute__((always_inline)) {
        const bool masked = is_masked(t, kb);
        // Scores are multiplied between the exponentials of the half before; operands come while the first of those are taken, or earlier.
        u32x4 k[kSteps], pw[2];
        read_keys(k, kn);
        if (kn == 1) {
            const uint32_t on = t % 2 ? -kTile : kTile;
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) k_read[ks] += on;
        }
        if (kb == 1) {
            read_half(v0, kb, 0);
            read_half(v1, kb, 1);
            const uint32_t on = t % 3 == 2 ? -2 * kTile : kTile;
#pragma unroll
            for (int db = 0; db < kBlocks; ++db) v_read[db][0] += on, v_read[db][1] += on;
        }
        __builtin_amdgcn_sched_barrier(0);
        // The reference is a row's first maximum, and moves only when the row's sum so far, this half's with it, passes 2^16 in a lane (of two): floats of
        // any size are equally exact, and looking for the maximum of every half costs a quarter of the vector instructions.  It moves to this half's maximum, or
        // by 2^8 where many keys of little more than the reference's weight made the sum (beyond scores of 2^26, which are 8 and more apart, equal ones may
        // grow to more).
        float sum = weigh(cur, pw);
        scores(to, k);
        asm volatile("" : "+v"(pw[0]), "+v"(pw[1]));
        __builtin_amdgcn_sched_group_barrier(0x402, 20, 0);
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x402, 6, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        const bool left = !(l + sum <= 0x1p16f) || m == -INFINITY;
        if (__any(left)) {                    // of this row, in either half of the wavefront: what other rows need does not change its bits
            const bool moves = left | (__shfl_xor((int)left, 32, 64) != 0);
            const float top = fmaxf(highest(cur), m + 8.f);
            raise(moves ? top : -INFINITY);
            sum = weigh(cur, pw);
        }
        l += sum;
        if (masked) {
            const uint32_t vt = lds0 + (2 + t % 3) * kTile + kb * 32 * DH * 2, odd = odd_keys<D>(vt);
            if (odd) {
                const int key0 = (tile0 + t) * kManyKeys + kb * 32;
                add_odd_values<D>(o, vt, odd, pw, [&](int j) { return row_ok && key0 + j <= pos && key0 + j > from; });
                const u32x4 keep0 = even_only(odd, 0, half), keep1 = even_only(odd, 1, half);
#pragma unroll
                for (int db = 0; db < kBlocks; ++db) {
                    v0[db] &= keep0;
                    v1[db] &= keep1;
                }
            }
        }
        add_values<D>(o, v0, pw[0]);
        add_values<D>(o, v1, pw[1]);
        if (kb == 1) {                        // the next tile's first values; then what would hold them up: they wait for every load that is on its way
            read_half(v0, 0, 0);
            read_half(v1, 0, 1);
            __builtin_amdgcn_sched_barrier(0);
            if (t + 2 < tiles) load(t + 2);
        }
        if (is_masked(tn, kn)) mask(to, tn, kn);
    };

    if (tiles > 0) {
        fetch_id(0);
        load(0);
        fetch_id(1);
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, row_ok && 2 * ks + half < chunks ? q_raw[ks] ^ flip : u32x4{0, 0, 0, 0});
        __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8));
        __builtin_amdgcn_s_barrier();
        if (works) {
            read_half(v0, 0, 0);
            read_half(v1, 0, 1);
        }
        if (tiles > 1) load(1);
        fetch_id(2);
        if (works) {
            u32x4 k[kSteps];
            read_keys(k, 0);
            scores(sc, k);
            if (is_masked(0, 0)) mask(sc, 0, 0);
        }
    }
    for (int t = 0; t < tiles; ++t) {
        if (works) half_step(sc, next, t, 0, t, 1);
        // the next tile has landed, and everybody is through with this one's K and the last one's V
        __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8));
        __builtin_amdgcn_s_barrier();
        if (works) half_step(next, sc, t, 1, t + 1, 0);
        else if (t + 2 < tiles) load(t + 2);
        fetch_id(t + 3);
    }
    l = sum_halves(l);
    if (!row_ok) return;
    if (part < 0) {
        const bool empty = is_empty(m, l);
        const float inv = empty ? 0.f : 1.f / l;
        if (empty)
#pragma unroll
            for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                for (int x = 0; x < 16; ++x) o[db][x] = 0.f;
        uint16_t* const to = a.out + (int64_t)(q0 + token) * a.out_token_stride + (int64_t)head * a.out_head_stride + half * 4;
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (db * 32 + g * 8 < c.head_dim)
                    *(uint2*)(to + db * 32 + g * 8) = make_uint2(pack_bf16(o[db][4 * g] * inv, o[db][4 * g + 1] * inv), pack_bf16(o[db][4 * g + 2] * inv, o[db][4 * g + 3] * inv));
        if (a.lse && half == 0) a.lse[(int64_t)(q0 + token) * a.heads + head] = empty ? -INFINITY : (m + log2f(l)) * kLn2;
    } else {
        float* const to = (float*)(workspace + layout.parts) + ((size_t)part * c.kv_heads + kvh) * (2 * kManyRows + kManyRows * D);
        const int rw = wid * 32 + l32;
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(float4*)(to + 2 * kManyRows + rw * D + db * 32 + g * 8 + half * 4) = make_float4(o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]);
        if (half == 0) {
            to[rw] = m;
            to[kManyRows + rw] = l;
        }
    }
#endif
}

// Adds up the parts of a unit that was cut; blockIdx.y: 16 of its rows.  Latency: 8.3 us with 25 cut units of 8 heads, 4.7 without any.  The last
// workgroup of a unit doing it instead costs more: what makes parts visible on all of the chip, a release of the second-level cache, slowed
// the units down from 88 to 183 us.
constexpr int kUnitRows = 16;
template <int D> constexpr int kUnitThreads = kUnitRows * D / 4;          // four channels of a row each
template <int D>
__global__ __launch_bounds__(kUnitThreads<D>) void kv_attention_join_units_kernel(KvCache c, KvAttention a, const char* workspace, ManyLayout layout)
{
    const int kvh = blockIdx.x % c.kv_heads, index = blockIdx.x / c.kv_heads;
    const int n_joined = ((const ManyHeader*)(workspace + layout.header))->joined;
    const Joined u = ((const Joined*)(workspace + layout.joined))[index];         // its place is there in any case
    if (index >= n_joined) return;
    const size_t stride = (size_t)c.kv_heads * (2 * kManyRows + kManyRows * D);
    const float* const parts = (const float*)(workspace + layout.parts) + ((size_t)u.part * c.kv_heads + kvh) * (2 * kManyRows + kManyRows * D);
    const int rw = blockIdx.y * kUnitRows + (int)threadIdx.x / (D / 4), ch = (int)threadIdx.x % (D / 4) * 4, row = u.first_row + rw;
    if (row >= u.rows) return;
    float mx = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < u.parts; p += kAhead) {
        float mp[kAhead], lp[kAhead];
        float4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {                // on their way together
            const float* const from = parts + min(p + i, u.parts - 1) * stride;
            mp[i] = from[rw];
            lp[i] = from[kManyRows + rw];
            v[i] = *(const float4*)(from + 2 * kManyRows + rw * D + ch);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (p + i >= u.parts) continue;
            const float m_new = fmaxf(mx, mp[i]), keep = weight_of_part(mx, m_new), f = weight_of_part(mp[i], m_new);
            sum = sum * keep + f * lp[i];
            const float g = f * kJoinRoom;
            acc.x = acc.x * keep + g * v[i].x, acc.y = acc.y * keep + g * v[i].y, acc.z = acc.z * keep + g * v[i].z, acc.w = acc.w * keep + g * v[i].w;
            mx = m_new;
        }
    }
    finish_row(c, a, u.q0, kvh, row, ch, mx, sum, acc, 1.f / kJoinRoom);
}

// channels that the kernels compute with: the next multiple of 32
int padded_dim(int32_t head_dim) { return (head_dim + 31) / 32 * 32; }
int64_t few_bytes(int32_t n_requests, int dim)
{
    return few_header_bytes(n_requests) + (int64_t)kFewGroups * 2 * (2 * kFewRows + kFewRows * dim) * 4;
}
// Rows that one wavefront's tile holds go to the kernel that reads every key once.  8 cache heads of 128, us, few / many: 4 requests of 3000 tokens with 8 rows
// 25 / 30, with 32 rows 29 / 35; 32 requests 94 / 99 and 108 / 104; 64 of 1500 tokens 97 / 89 to 98 and 121 / 94.
bool is_few(int32_t max_new, int32_t heads, int32_t kv_heads) { return (int64_t)max_new * (heads / kv_heads) <= kFewRows; }

// Whether a workgroup of its own for every history is faster than equal stretches and a join: where the block tables, all that is known
// here of the lengths, hold few tokens.  Single tokens in replayed graphs, us, stretches / whole histories, tables as long as their histories.  At
// the limits: one request, 12 heads of 64 channels, 640 tokens 9.6 / 8.6, 8 cache heads of 128, 320 tokens 13.2 / 9.3; 16 requests, 12 x 64, 1536
// tokens 25.1 / 17.5, 8 x 128, 768 tokens 20.3 / 19.4; 200 requests 188 / 186 and 137 / 138.  Past them the whole histories' gain shrinks, then turns: one
// request, 12 x 64, 832 tokens 11.8 / 10.3, 1024 tokens 9.8 / 11.6, 8 x 128, 432 tokens 13.3 / 11.7, 528 tokens 10.9 / 12.6; 16 requests, 12 x 64, 2064 tokens
// 28.9 / 21.2, 8 x 128, 1024 tokens 21.5 / 23.4; 200 requests, 12 x 64, 2064 tokens 236 / 244, 8 x 128, 1024 tokens 173 / 180.
// Chunks, us, units and a join / a workgroup for 32 rows of each: one prompt of 500 tokens, 12 heads of 64, 25.5 / 12.6, 32 on 8 of 128 29.5 / 21.2, of 1000 tokens
// 28 / 20 and 40 / 52; 8 prompts of 128, 32 on 8 of 128 23.3 / 21.1, of 256 30.7 / 45.9; 64 tokens behind 900, 32 on 8 of 128, 34 / 24;
// 40 prompts of 64, 32 on 8 of 128 (2560 workgroups) 35 / 42.
int64_t row_blocks(const KvAttention& a, const KvCache& c) { return ((int64_t)a.max_new * (a.heads / c.kv_heads) + kFewRows - 1) / kFewRows; }
bool is_short(const KvAttention& a, const KvCache& c)
{
    const int64_t blocks = row_blocks(a, c), groups = (int64_t)a.n_requests * c.kv_heads * blocks, longest = ((int64_t)a.max_blocks << c.block_shift) * padded_dim(c.head_dim);
    if (blocks == 1) return longest <= (groups >= 128 ? 98304 : 40960);
    return groups <= 2048 && longest <= 131072 && groups * longest <= 52ll << 20;
}

template <int D, bool PAD, int WAVES> hipError_t launch_short(const KvCache& c, const KvAttention& a, hipStream_t stream)
{
    constexpr size_t kLds = kFewLds<D, WAVES>;
    static const hipError_t configured =
        hipFuncSetAttribute((const void*)kv_attention_short_kernel<D, PAD, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    if (configured != hipSuccess) return configured;
    hipLaunchKernelGGL((kv_attention_short_kernel<D, PAD, WAVES>), dim3((unsigned)a.n_requests * c.kv_heads, (unsigned)row_blocks(a, c)), dim3(64 * WAVES), kLds, stream, c, a);
    return hipGetLastError();
}

template <int D, bool PAD> hipError_t launch_few(const KvCache& c, const KvAttention& a, char* workspace, hipStream_t stream)
{
    const size_t lds = std::max(kFewLds<D>, ((size_t)a.n_requests + 1) * 8);
    static const hipError_t configured =
        hipFuncSetAttribute((const void*)kv_attention_few_kernel<D, PAD>, hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024);
    if (configured != hipSuccess) return configured;
    hipLaunchKernelGGL((kv_attention_few_kernel<D, PAD>), dim3(kFewGroups), dim3(64 * kFewWaves), lds, stream, c, a, workspace);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int most_rows = a.max_new * (a.heads / c.kv_heads);
    hipLaunchKernelGGL(kv_attention_join_kernel<D>, dim3((unsigned)a.n_requests * c.kv_heads, (most_rows + kJoinRows - 1) / kJoinRows), dim3(256), 0,
                       stream, c, a, workspace);
    return hipGetLastError();
}

template <int D> hipError_t launch_many(const KvCache& c, const KvAttention& a, char* workspace, hipStream_t stream)
{
    constexpr int kLds = 5 * kManyTile<D>;
    static const hipError_t configured[2] = {
        hipFuncSetAttribute((const void*)kv_attention_many_kernel<D>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds),
        hipFuncSetAttribute((const void*)kv_attention_schedule_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (kPlanMaxRequests + 1) * 4)};
    static_assert(4 * kSchedInLds <= kPlanMaxRequests, "lengths beside the sums");
    if (configured[0] != hipSuccess || configured[1] != hipSuccess) return configured[0] != hipSuccess ? configured[0] : configured[1];
    const ManyLayout at = many_layout(a.n_requests, a.n_tokens, a.heads, c.kv_heads, D);
    if (at.most_units * c.kv_heads > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const size_t sched_lds = ((a.n_requests <= kSchedInLds ? 4 : 1) * (size_t)a.n_requests + 1) * 4;
    hipLaunchKernelGGL(kv_attention_schedule_kernel, dim3(1), dim3(kSchedThreads), sched_lds, stream, c, a, workspace, at);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(kv_attention_many_kernel<D>, dim3((unsigned)(at.most_units * c.kv_heads)), dim3(64 * kManyWaves), kLds, stream, c, a, workspace, at);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(kv_attention_join_units_kernel<D>, dim3((unsigned)(at.most_joined * c.kv_heads), kManyRows / kUnitRows), dim3(kUnitThreads<D>), 0, stream, c, a, workspace, at);
    return hipGetLastError();
}

template <int D> hipError_t launch(const KvCache& c, const KvAttention& a, char* workspace, hipStream_t stream)
{
    if (is_short(a, c)) {                     // eight wavefronts while there is a compute unit for every workgroup: one request, 624 tokens, 12 x 64: 11.6 -> 9.2 us
        const bool wide = (int64_t)a.n_requests * c.kv_heads * row_blocks(a, c) <= kFewGroups / 2;
        if (c.head_dim == D) return wide ? launch_short<D, false, 8>(c, a, stream) : launch_short<D, false, kFewWaves>(c, a, stream);
        return wide ? launch_short<D, true, 8>(c, a, stream) : launch_short<D, true, kFewWaves>(c, a, stream);
    }
    if (!is_few(a.max_new, a.heads, c.kv_heads)) return launch_many<D>(c, a, workspace, stream);
    return c.head_dim == D ? launch_few<D, false>(c, a, workspace, stream) : launch_few<D, true>(c, a, workspace, stream);
}

}  // namespace

int64_t kv_attention_workspace(int32_t n_requests, int32_t n_tokens, int32_t max_new, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    if (is_few(std::min(max_new, n_tokens), heads, kv_heads)) return few_bytes(n_requests, padded_dim(head_dim));
    return many_layout(n_requests, n_tokens, heads, kv_heads, padded_dim(head_dim)).end;
}

hipError_t kv_attention(const KvCache& c, const KvAttention& a, void* workspace, hipStream_t stream)
{
    switch (padded_dim(c.head_dim)) {
    case 32: return launch<32>(c, a, (char*)workspace, stream);
    case 64: return launch<64>(c, a, (char*)workspace, stream);
    case 96: return launch<96>(c, a, (char*)workspace, stream);
    default: return launch<128>(c, a, (char*)workspace, stream);
    }
}

}  // namespace k
}  // namespace coe
