// gfx950 kernels for attention of a decoder's tokens over an encoder's states (bf16).
//
// A source with m queries and `heads / kv_heads` = G query heads to a head of the states has m G query rows per head that all look at all
// of its rows (beams of one request are queries of one source).  Scores are computed transposed, S^T = K Q^T, so that a lane holds ONE query
// row (column l % 32) and of a block of 32 keys the keys 8 (v / 4) + 4 (l / 32) + v % 4: the running maximum and sum of a row live in lanes l and
// l ^ 32, and the exponentials, rounded to bf16, are the second operand of O^T = V^T P^T as they lie.  V^T comes from the transposing
// LDS read.
//   m' = max(m, max s)    l' = l 2^(m - m') + sum 2^(s - m')    o' = o 2^(m - m') + sum 2^(s - m') v        (s in units of ln 2)
// All three are fp32; only 2^(s - m') is rounded to bf16, for the matrix cores.  A row that is hidden is hidden from every query: its key and
// value are read as zeros and its scores replaced by -inf, so that none of its bits meets a product.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attention_tiles.h"
#include "kernels.h"

namespace coe {
namespace k {

namespace {

constexpr int kKeys = 32;                 // keys of a tile of the kernels for few rows
constexpr int kFewRows = 32;              // query rows of a source and head that they take at a time
constexpr int kFewWaves = 4;
// workgroups: two, three or four per compute unit, as many as registers allow
template <int D> constexpr int kFewGroups = D <= 32 ? 1024 : D <= 64 ? 768 : 512;
constexpr int kMostFewGroups = 1024;
static_assert(kMostFewGroups <= kMostParts, "a part of every stretch at most");

// A source's queries and rows, within the arrays.
struct Source {
    int q0, m, first, keys;
    __device__ __forceinline__ int tiles() const { return m == 0 ? 0 : max(1, (int)(((unsigned)keys + kKeys - 1) / kKeys)); }
};
__device__ __forceinline__ Source source_of(const States& st, const CrossAttention& a, int s)
{
    const int begin = a.q_off[s * a.beams], end = a.q_off[(s + 1) * a.beams], first = a.first[s], length = a.length[s];   // on their way together
    Source o;
    const int q1 = max(0, min(end, a.n_tokens));
    o.q0 = max(0, min(begin, a.n_tokens));
    o.m = min(max(q1 - o.q0, 0), a.max_new);
    const bool there = first >= 0 && first < st.n_rows;
    o.first = there ? first : 0;
    o.keys = there ? max(0, min(min(length, a.max_rows), st.n_rows - first)) : 0;
    return o;
}

// Four channels of query row `row` of a source and head, from the unnormalised output (divided by `grow`) relative to maximum mx.
__device__ __forceinline__ void finish_row(const States& st, const CrossAttention& a, int q0, int kvh, int row, int ch, float mx, float sum, float4 acc, float grow = 1.f)
{
    const int group = a.heads / st.kv_heads, token = row / group, head = kvh * group + (row - token * group);
    const bool empty = is_empty(mx, sum);
    if (empty) acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const float inv = empty ? 0.f : grow / sum;
    if (ch < st.head_dim)
        *(uint2*)(a.out + (int64_t)(q0 + token) * a.out_token_stride + (int64_t)head * a.out_head_stride + ch) =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    if (a.lse && ch == 0) a.lse[(int64_t)(q0 + token) * a.heads + head] = empty ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

// ---- few query rows (beams' single tokens): at most 32 per source and head ---------------------------------------------------
// The work is the list of all 32-key tiles, (source, head, tile) in that order; every workgroup takes an equal stretch of it, so that
// lengths of any mix fill the chip evenly.  A stretch may begin and end inside a source (a "part"): such parts go to the workspace as
// (maximum, sum, unnormalised output) and cross_attention_join_kernel adds them up; a source inside one stretch is finished here.  Inside a
// stretch the four wavefronts take tiles in turn, each for itself: keys go from memory straight into registers (they are the first
// operand as they lie), values through registers into LDS of the wavefront's own, and the next tile's are on their way while this one is multiplied.
// What bounds it is memory: three sources of 20,000 to 60,000 rows, 32 query heads on 8 of 128 (516 MB), take 102 us where the rate of a large copy
// would take 106; matrix cores are busy 7 % of that.
struct FewHeader {                        // at the workspace's start, for the joining kernel
    unsigned long long per;               // tiles of a stretch
    unsigned long long base[1];           // [n_sources + 1] tiles before source s, of one head
};
__host__ __device__ constexpr int64_t few_header_bytes(int n_sources) { return round256(16 + 8 * (int64_t)(n_sources + 1)); }
// a part: maxima and sums [2][32], then the output [32][D]
template <int D> constexpr int kPartFloats = 2 * kFewRows + kFewRows * D;

template <int D> constexpr int kMergeRow = D + 4;          // floats between the rows of a wavefront's output in LDS
template <int D, int WAVES = kFewWaves> constexpr size_t kFewLds = (size_t)WAVES * kFewRows * kMergeRow<D> * 4;

#if defined(__HIP_DEVICE_COMPILE__)
// Query rows [row0, row0 + rows), at most 32, of a source and head over its 32-key tiles [tile_begin, tile_stop), by WAVES wavefronts:
// write(row - row0, channel, maximum, sum, four channels of the unnormalised output) gets the result, relative to the row's maximum.
template <int D, bool PAD, int WAVES, class Write>
__device__ __forceinline__ void few_rows(const States& st, const CrossAttention& a, const Source& o, int kvh, int row0, int rows, int tile_begin, int tile_stop, char* lds,
                                         float (*stat)[WAVES][kFewRows], Write write)
{
    constexpr int kSteps = D / 16, kBlocks = D / 32;
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int group = a.heads / st.kv_heads;
    const int chunks = st.head_dim >> 3, last_step = (chunks - 1 - half) >> 1;      // this lane's last 16 bytes of a row; -1: none (8 channels)
    const float scale2 = a.scale * 1.44269504088896340736f;
    char* const v_lds = lds + wid * (kKeys * kRow<D> * 2);
    const uint32_t v_tile = lds_address(v_lds), v_read = v_tile + value_base<D>(lane);
    tile_stop = min(tile_stop, (int)(((unsigned)o.keys + kKeys - 1) / kKeys));      // a source without rows has a tile in the list, and nothing in it

    const int row = row0 + l32, token = row / group, head = kvh * group + (row - token * group);      // this lane's query row
    const bool row_ok = l32 < rows;
    const uint16_t *const k_base = st.k + (int64_t)o.first * st.k_row_stride + kvh * st.k_head_stride + (PAD && last_step < 0 ? 0 : half * 8);
    const uint16_t *const v_base = st.v + (int64_t)o.first * st.v_row_stride + kvh * st.v_head_stride + (PAD && last_step < 0 ? 0 : half * 8);
    const uint8_t* const seen = st.seen ? st.seen + o.first : nullptr;
    auto there_at = [&](int tile) {           // whether this lane's key of a tile is there and not hidden
        const int key = tile * kKeys + l32;
        return key < o.keys && (!seen || seen[key] != 0);
    };
    // a row that is not there is read in another's place: the source's first
    auto fetch = [&](const uint16_t* p, u32x4 (&w)[kSteps]) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) w[ks] = *(const u32x4*)(p + (PAD ? max(0, min(ks, last_step)) : ks) * 16);
    };
    u32x4 kw[kSteps], vw[kSteps];
    int tile = tile_begin + wid;
    bool there = false, there_next = false;
    if (tile < tile_stop) {
        there = there_at(tile);
        const int64_t key = there ? tile * kKeys + l32 : 0;
        fetch(k_base + key * st.k_row_stride, kw);
        fetch(v_base + key * st.v_row_stride, vw);
        if (tile + WAVES < tile_stop) there_next = there_at(tile + WAVES);
    }
    bf16x8 qf[kSteps];
    {
        const uint16_t* qp = a.q + (int64_t)(o.q0 + (row_ok ? token : 0)) * a.q_token_stride + (int64_t)(row_ok ? head : 0) * a.q_head_stride + half * 8;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            u32x4 w = {0, 0, 0, 0};
            if (row_ok && (!PAD || 2 * ks + half < chunks)) w = *(const u32x4*)(qp + ks * 16);
            qf[ks] = __builtin_bit_cast(bf16x8, w);
        }
    }
    float m = -INFINITY, l = 0.f;
    f32x16 acc[kBlocks];
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[db][x] = 0.f;
    for (; tile < tile_stop; tile += WAVES) {
        const bool more = tile + WAVES < tile_stop;
        const uint32_t shown = (uint32_t)__ballot(there);             // lanes l and l + 32 hold the same key
        if (shown != 0xFFFFFFFFu) {
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) {
                kw[ks] = there ? kw[ks] : u32x4{0, 0, 0, 0};
                vw[ks] = there ? vw[ks] : u32x4{0, 0, 0, 0};
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
            there = there_next;
            const int64_t key = there ? (tile + WAVES) * kKeys + l32 : 0;
            fetch(k_base + key * st.k_row_stride, kw);
            fetch(v_base + key * st.v_row_stride, vw);
            if (tile + 2 * WAVES < tile_stop) there_next = there_at(tile + 2 * WAVES);
        }
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            sc[x] *= scale2;
            if (shown != 0xFFFFFFFFu) sc[x] = (shown >> (4 * half)) >> (8 * (x >> 2) + (x & 3)) & 1 ? sc[x] : -INFINITY;
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
                for (int x = 0; x < 16; ++x) acc[db][x] *= shrink;
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
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) {
            u32x4 v[kBlocks];
            read_values<D>(v, v_read, t2);
            add_values<D>(acc, v, pw[t2]);
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
                *(float4*)(mine + db * 32 + g * 8 + half * 4) = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
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
        float4 all = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float mw = stat[0][w][rw];
            const float f = mw == mx ? 1.f : exp2_fast(mw - mx);
            const float4 v = *(const float4*)((const float*)lds + (w * kFewRows + rw) * kMergeRow<D> + ch);
            sum += f * stat[1][w][rw];
            all.x += f * v.x, all.y += f * v.y, all.z += f * v.z, all.w += f * v.w;
        }
        write(rw, ch, mx, sum, all);
    }
}
#endif

template <int D, bool PAD>
__global__ __launch_bounds__(64 * kFewWaves, 2) void cross_attention_few_kernel(States st, CrossAttention a, char* workspace)
{
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(4096))) char lds[];
    __shared__ float stat[2][kFewWaves][kFewRows];
    __shared__ unsigned long long part_sum[kFewWaves];
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6), n = a.n_sources, group = a.heads / st.kv_heads;

    // tiles before every source
    unsigned long long* const base = (unsigned long long*)lds;
    unsigned long long carry = 0;
    for (int s0 = 0; s0 < n; s0 += 64 * kFewWaves) {
        const unsigned long long v = s0 + tid < n ? (unsigned long long)source_of(st, a, s0 + tid).tiles() : 0ull;
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
        if (s0 + tid < n) base[s0 + tid] = before + sum - v;
        __syncthreads();
    }
    if (tid == 0) base[n] = carry;
    __syncthreads();
    const unsigned long long total = carry * (unsigned)st.kv_heads;
    const unsigned long long share = (total + gridDim.x - 1) / gridDim.x, per = max(4ull, (share + 3) / 4 * 4);
    if (blockIdx.x == 0) {
        FewHeader* h = (FewHeader*)workspace;
        for (int s = tid; s <= n; s += 64 * kFewWaves) h->base[s] = base[s];
        if (tid == 0) h->per = per;
    }
    const unsigned index = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
    unsigned long long now = index * per;
    const unsigned long long stop = min(total, now + per);
    if (now >= stop) return;
    int s = 0;
    for (int hi = n; hi - s > 1;) {       // the last source that begins at or before `now`
        const int mid = (s + hi) >> 1;
        if (base[mid] * (unsigned)st.kv_heads <= now) s = mid;
        else hi = mid;
    }
    s = __builtin_amdgcn_readfirstlane(s);
    unsigned long long into = now - base[s] * (unsigned)st.kv_heads;       // tiles of this source that others did
    __syncthreads();

    const unsigned long long start = now;
    while (now < stop && s < n) {
        const Source o = source_of(st, a, s);
        const int tiles = o.tiles();
        if (into >= (unsigned long long)tiles * (unsigned)st.kv_heads) {
            into = 0;
            ++s;
            continue;
        }
        const int kvh = (int)(into / (unsigned)tiles), t_begin = (int)(into - (unsigned long long)kvh * (unsigned)tiles);
        const int t_end = (int)min((unsigned long long)tiles, t_begin + (stop - now));
        const bool whole = t_begin == 0 && t_end == tiles;
        float* const part = (float*)(workspace + few_header_bytes(n)) + ((size_t)index * 2 + (now != start)) * kPartFloats<D>;
        few_rows<D, PAD, kFewWaves>(st, a, o, kvh, 0, o.m * group, t_begin, t_end, lds, stat, [&](int rw, int ch, float mx, float sum, float4 acc) __attribute__((always_inline)) {
            if (whole) finish_row(st, a, o.q0, kvh, rw, ch, mx, sum, acc);
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

// Where sources are short, or many: a workgroup per source, head and 32 query rows, one launch, and no parts to join.  All heads of a source go to one
// of the chip's eight dies, to which workgroups are dealt in turn: their rows' bytes lie side by side.  ORDERED: the longest sources first (every
// workgroup ranks them all, at most kRanked), so that those which start last are short, and that every die gets its share; each second round of
// workgroups (one to a compute unit) the other way round, so that every unit gets long and short ones.  Bound by memory, or by a
// chain of round trips where there is little of it: 64 sources of 60 to 1500 rows with five beams, 16 heads of 64 (209 MB), 38 us where they have just been
// read and 51 where not (the rate of a copy: 43); one source of 197 rows, four beams, 12 heads, 6.0 us in a graph.
constexpr int kRanked = 256;
template <int D, bool PAD, int WAVES, bool ORDERED>
__global__ __launch_bounds__(64 * WAVES, 2) void cross_attention_whole_kernel(States st, CrossAttention a, int dies, int per_round)
{
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(4096))) char lds[];
    __shared__ float stat[2][WAVES][kFewRows];
    const int turn = blockIdx.x / dies, s = turn / st.kv_heads * dies + blockIdx.x % dies, kvh = turn % st.kv_heads, row0 = (int)blockIdx.y * kFewRows, group = a.heads / st.kv_heads;
    if (s >= a.n_sources) return;
    Source o;
    if (ORDERED) {
        int* const keys = (int*)lds;          // [kRanked]: lengths and, among equal ones, places
        int4* const chosen = (int4*)(keys + kRanked);
        const int tid = threadIdx.x, n = a.n_sources, chunk = s / per_round, place = chunk & 1 ? min(chunk * per_round + per_round, n) - 1 - (s - chunk * per_round) : s;
        if (tid < n) o = source_of(st, a, tid);
        const int key = tid < n ? o.keys << 8 | (kRanked - 1 - tid) : -1;          // is_whole() has at most 8192 rows
        keys[tid] = key;
        __syncthreads();
        int before = 0;
#pragma unroll 4
        for (int i = 0; i < n; i += 4) {      // without a branch, so that many reads are on their way
            const int4 four = *(const int4*)(keys + i);
            before += (four.x > key) + (four.y > key) + (four.z > key) + (four.w > key);
        }
        if (tid < n && before == place) *chosen = make_int4(o.q0, o.m, o.first, o.keys);
        __syncthreads();
        const int4 v = *chosen;
        o = {__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z), __builtin_amdgcn_readfirstlane(v.w)};
        __syncthreads();
    } else o = source_of(st, a, s);
    const int all = o.m * group;
    if (row0 >= all) return;
    few_rows<D, PAD, WAVES>(st, a, o, kvh, row0, min(kFewRows, all - row0), 0, o.tiles(), lds, stat,
                            [&](int rw, int ch, float mx, float sum, float4 acc) __attribute__((always_inline)) { finish_row(st, a, o.q0, kvh, row0 + rw, ch, mx, sum, acc); });
#endif
}

// the sum of two parts' weights and outputs; an output's parts are taken times kJoinRoom
__device__ __forceinline__ void add_part(float& mx, float& sum, float4& acc, float m_part, float l_part, float4 v)
{
    const float m_new = fmaxf(mx, m_part), keep = weight_of_part(mx, m_new), f = weight_of_part(m_part, m_new), g = f * kJoinRoom;
    sum = sum * keep + f * l_part;
    acc.x = acc.x * keep + g * v.x, acc.y = acc.y * keep + g * v.y, acc.z = acc.z * keep + g * v.z, acc.w = acc.w * keep + g * v.w;
    mx = m_new;
}

// Adds up the parts of a source that several workgroups shared: a workgroup per source, head and query row (blockIdx.y).  Several threads share
// the parts of a row's four channels, since a long source has many; each leaves its sum relative to its own maximum, and the first adds
// those up in their order.  Round trips to memory bound it, so every thread fetches four parts at a time: 5.2 us for the
// three long sources.
constexpr int kAhead = 4;
template <int D>
__global__ __launch_bounds__(256) void cross_attention_join_kernel(States st, CrossAttention a, const char* workspace)
{
    constexpr int kColumns = D / 4, kSplit = 256 / kColumns;
    __shared__ float4 sums[256];
    __shared__ float2 stats[256];
    const FewHeader* const h = (const FewHeader*)workspace;
    const int s = blockIdx.x / st.kv_heads, kvh = blockIdx.x - s * st.kv_heads, group = a.heads / st.kv_heads;
    const unsigned long long first = h->base[s], tiles = h->base[s + 1] - first, per = h->per;
    const Source o = source_of(st, a, s);     // on their way together
    if (tiles == 0) return;
    const unsigned long long begin = first * (unsigned)st.kv_heads + (unsigned)kvh * tiles, end = begin + tiles;
    const unsigned long long w0 = begin / per, w1 = (end - 1) / per;
    const int rw = blockIdx.y, ch = (int)threadIdx.x % kColumns * 4, share = threadIdx.x / kColumns;
    if (w0 == w1 || rw >= o.m * group) return;
    // a stretch's first source leaves the first part, its last one the second
    const float* const parts = (const float*)(workspace + few_header_bytes(a.n_sources));
    auto part_of = [&](unsigned long long w) { return parts + (w * 2 + (begin > w * per)) * kPartFloats<D>; };
    float mx = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (share < kSplit)
        for (unsigned long long w = w0 + share; w <= w1; w += kAhead * kSplit) {
            float mw[kAhead], lw[kAhead];
            float4 v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const float* const p = part_of(min(w + i * kSplit, w1));
                mw[i] = p[rw];
                lw[i] = p[kFewRows + rw];
                v[i] = *(const float4*)(p + 2 * kFewRows + rw * D + ch);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (w + i * kSplit <= w1) add_part(mx, sum, acc, mw[i], lw[i], v[i]);
        }
    sums[threadIdx.x] = acc;
    stats[threadIdx.x] = make_float2(mx, sum);
    __syncthreads();
    if (share > 0) return;
    for (int i = 1; i < kSplit; ++i) mx = fmaxf(mx, stats[i * kColumns + threadIdx.x].x);
    sum = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < kSplit; ++i) {
        const float2 part = stats[i * kColumns + threadIdx.x];
        const float f = weight_of_part(part.x, mx);
        const float4 v = sums[i * kColumns + threadIdx.x];
        sum += f * part.y;
        acc.x += f * v.x, acc.y += f * v.y, acc.z += f * v.z, acc.w += f * v.w;
    }
    finish_row(st, a, o.q0, kvh, rw, ch, mx, sum, acc, 1.f / kJoinRoom);
}

// ---- many query rows (prompts, answers that are scored): more than 32 per source and head --------------------------------------------
// Units of work are tiles of 128 query rows (32 to a wavefront) of a source and head, with all its 64-key tiles, the longest first, so that the last
// workgroups to start are short ones.  Every workgroup finds its own where there are few sources; else a scheduling launch lists them, which also cuts
// long ones into parts over the keys where there are too few to fill the chip; cross_attention_join_units_kernel adds those up.  Block b takes head b % kv_heads, so that with eight of them
// (or four, or two) the units of one head meet in the same second-level caches.  K tiles go from memory into two LDS buffers by DMA, V
// tiles into three, in turn; a wavefront reads every key and value of a tile for its 32 rows.
// Bound by the matrix cores and the vector unit, which takes the exponentials: a 32 x 32 x 16 product hides about 20 of its 32 cycles of vector instructions,
// and beside each lie some 36 cycles of them with 64 channels, 18 with 128.  Four sources of 3500 to 7000 rows with 2901 to 4900 tokens each, 32 heads on 8 of 128:
// 1,420 to 1,620 us by card, 0.94 to 1.07 PFLOP/s, clocks of 1.66 to 1.75 GHz among them; 16 of 4000 rows with 2000 tokens, 24 heads of 64, 0.88 to 0.91; 20 of 200 to 2100 with 30 to 900, 0.67,
// units of 18 tiles, whose beginnings and ends (first loads, a first maximum, stores) count.
constexpr int kManyRows = 128, kManyKeys = 64, kManyWaves = 4;
constexpr int kManyGroups = 512;          // two workgroups per compute unit; a unit has no more parts
static_assert(kManyGroups <= kMostParts, "joins have room for all of them");
constexpr int kListed = 64;               // sources that a workgroup looks at for its unit: one to a lane

struct Unit {
    int32_t first_row, tile, tiles, part;      // first query row; 64-key tiles; -1, or the part of the workspace that takes the result (times kv_heads)
    int32_t q0, m, first, keys;                // of the source
};
struct Joined {
    int32_t first_row, part, parts, q0;
    int32_t rows, pad[3];                      // query rows of the source
};
struct ManyHeader { int32_t units, joined, pad[62]; };

// where the workspace's pieces begin
struct ManyLayout {
    int64_t most_units, most_joined, units, joined, parts, end;
};
__host__ __device__ inline ManyLayout many_layout(int32_t n_sources, int32_t n_tokens, int32_t heads, int32_t kv_heads, int32_t dim)
{
    ManyLayout l;
    const int64_t rows = (int64_t)n_tokens * (heads / kv_heads), cuts = (kManyGroups + kv_heads - 1) / kv_heads;
    l.most_units = rows / kManyRows + n_sources + cuts;
    l.most_joined = cuts;
    l.units = sizeof(ManyHeader);
    l.joined = l.units + round256(l.most_units * (int64_t)sizeof(Unit));
    l.parts = l.joined + round256(l.most_joined * (int64_t)sizeof(Joined));
    l.end = l.parts + 2 * cuts * kv_heads * (int64_t)(2 * kManyRows + kManyRows * dim) * 4;
    return l;
}

// One workgroup, bound by latency: 6.2 us for one source, 7.7 for 90.  Row tiles of a source are of one length, its number of 64-key tiles.
constexpr int kSchedThreads = 1024, kSchedBins = 2048, kSchedInLds = 4096;
__global__ __launch_bounds__(kSchedThreads) void cross_attention_schedule_kernel(States st, CrossAttention a, char* workspace, ManyLayout at)
{
    extern __shared__ int32_t first_segment[];            // [n_sources + 1] row tiles before source s
    __shared__ unsigned long long wave_sum[kSchedThreads / 64];
    __shared__ int32_t bins[kSchedBins];
    __shared__ int32_t n_parts, n_joined;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = a.n_sources, group = a.heads / st.kv_heads;
    int4* const sources = (int4*)(first_segment + ((n + 1 + 3) & ~3));    // where they fit
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
    auto tiles_of = [&](int keys) { return max(1, (int)(((unsigned)keys + kManyKeys - 1) / kManyKeys)); };
    for (int i = tid; i < kSchedBins; i += kSchedThreads) bins[i] = 0;
    if (tid == 0) n_parts = n_joined = 0;
    unsigned long long segments = 0, mine = 0;
    for (int s0 = 0; s0 < n; s0 += kSchedThreads) {
        int v = 0;
        if (s0 + tid < n) {
            const Source o = source_of(st, a, s0 + tid);
            v = (int)(((unsigned)(o.m * group) + kManyRows - 1) / kManyRows);         // below 2^24
            mine += (unsigned long long)v * (unsigned)tiles_of(o.keys);
            if (in_lds) sources[s0 + tid] = make_int4(o.q0, o.m, o.first, o.keys);
        }
        unsigned long long all;
        const unsigned long long before = segments + sum_before((uint32_t)v, all);
        if (s0 + tid < n) first_segment[s0 + tid] = (int32_t)min(before, (unsigned long long)at.most_units);
        segments += all;
    }
    const int count = (int)min(segments, (unsigned long long)at.most_units);      // the sum of the sources' rows is at most n_tokens * group
    if (tid == 0) first_segment[n] = count;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) mine += __shfl_xor(mine, d, 64);
    __syncthreads();
    if (lane == 0) wave_sum[wid] = mine;
    __syncthreads();
    unsigned long long total = 0;
#pragma unroll
    for (int w = 0; w < kSchedThreads / 64; ++w) total += wave_sum[w];
    struct Segment { Source o; int row, tiles; };
    auto find = [&](int i) {
        Segment g;
        int s = 0;
        for (int hi = n; hi - s > 1;) {
            const int mid = (s + hi) >> 1;
            if (first_segment[mid] <= i) s = mid;
            else hi = mid;
        }
        if (in_lds) {
            const int4 o = sources[s];
            g.o = {o.x, o.y, o.z, o.w};
        } else g.o = source_of(st, a, s);
        g.row = (i - first_segment[s]) * kManyRows;
        g.tiles = tiles_of(g.o.keys);
        return g;
    };
    const Segment own = tid < count ? find(tid) : Segment{};             // the only one in most calls
    auto segment = [&](int i) { return i == tid ? own : find(i); };
    // No part is shorter than 8 tiles, or than twice a workgroup's share: at one share 8 sources of 200 tokens and 600 rows, 32 heads on 8 of 128, took 61 us
    // instead of 41, one and a half or twice make no difference.
    const int most = (int)min(1ull << 30, max(8ull, (2 * total * (unsigned)st.kv_heads + kManyGroups - 1) / kManyGroups));
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
        int own_bins[kPer], sum = 0;
        for (int j = 0; j < kPer; ++j) {
            own_bins[j] = bins[tid * kPer + j];
            sum += own_bins[j];
        }
        unsigned long long all;
        int before = (int)sum_before((uint32_t)sum, all);
        for (int j = 0; j < kPer; ++j) {
            bins[tid * kPer + j] = before;
            before += own_bins[j];
        }
        if (tid == 0) ((ManyHeader*)workspace)->units = (int32_t)min(all, (unsigned long long)at.most_units);
    }
    __syncthreads();
    Unit* const units = (Unit*)(workspace + at.units);
    Joined* const joined = (Joined*)(workspace + at.joined);
    for (int i = tid; i < count; i += kSchedThreads) {
        const Segment g = segment(i);
        const int tiles = g.tiles, parts = (tiles + most - 1) / most, each = (tiles + parts - 1) / parts;
        const int to = atomicAdd(&bins[bin_of(each)], parts);
        int part = -1;
        if (parts > 1) {
            part = atomicAdd(&n_parts, parts);
            const int j = atomicAdd(&n_joined, 1);
            if (j < at.most_joined) joined[j] = {g.row, part, parts, g.o.q0, g.o.m * group, {0, 0, 0}};
        }
        for (int p = 0; p < parts; ++p) {
            const int t0 = p * each, t1 = min(tiles, t0 + each);
            if (to + p < at.most_units) units[to + p] = {g.row, t0, max(0, t1 - t0), part < 0 ? -1 : part + p, g.o.q0, g.o.m, g.o.first, g.o.keys};
        }
    }
    __syncthreads();
    if (tid == 0) ((ManyHeader*)workspace)->joined = min(n_joined, (int)at.most_joined);
}

template <int D> constexpr int kManyTile = kManyKeys * kRow<D> * 2;  // bytes of a K (or V) tile

template <int D>
__global__ __launch_bounds__(64 * kManyWaves, 2) void cross_attention_many_kernel(States st, CrossAttention a, char* workspace, ManyLayout layout, bool listed)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int DH = kRow<D>, kSteps = D / 16, kBlocks = D / 32, kTile = kManyTile<D>;
    constexpr int kRowsPerLoad = 1024 / (DH * 2), kLoads = kManyKeys / kRowsPerLoad / kManyWaves;     // of K, and the same of V
    extern __shared__ __attribute__((aligned(4096))) char lds[];          // two buffers of K tiles, three of V
    const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int kvh = blockIdx.x % st.kv_heads, index = blockIdx.x / st.kv_heads;
    const int group = a.heads / st.kv_heads;
    int row0, tile0 = 0, part = -1, q0, rows, first, keys, tiles;
    if (listed) {                             // a source to a lane; the unit is one of the source that `index` falls to
        const int n = a.n_sources, s = min(lane, n - 1);
        const Source o = source_of(st, a, s);
        const int length = (int)(((unsigned)o.keys + kManyKeys - 1) / kManyKeys), order = length << 6 | (63 - lane);         // unequal, below 2^31
        const int segments = lane < n ? (int)(((unsigned)(o.m * group) + kManyRows - 1) / kManyRows) : 0;
        int before = 0;
        for (int i = 0; i < n; ++i) before += __builtin_amdgcn_readlane(order, i) > order ? __builtin_amdgcn_readlane(segments, i) : 0;
        const unsigned long long owner = __ballot(index >= before && index < before + segments);
        if (!owner) return;
        const int from = __builtin_ctzll(owner);
        row0 = (index - __builtin_amdgcn_readlane(before, from)) * kManyRows;
        q0 = __builtin_amdgcn_readlane(o.q0, from), rows = __builtin_amdgcn_readlane(o.m, from) * group;
        first = __builtin_amdgcn_readlane(o.first, from), keys = __builtin_amdgcn_readlane(o.keys, from), tiles = __builtin_amdgcn_readlane(length, from);
    } else {
        // one round trip for the number of units and the unit, whose place is there in any case
        const int units = ((const ManyHeader*)workspace)->units;
        const int4 *const up = (const int4*)((const Unit*)(workspace + layout.units) + index), u0 = up[0], u1 = up[1];
        if (index >= units) return;
        row0 = __builtin_amdgcn_readfirstlane(u0.x), tile0 = __builtin_amdgcn_readfirstlane(u0.y), part = __builtin_amdgcn_readfirstlane(u0.w);
        q0 = __builtin_amdgcn_readfirstlane(u1.x), rows = __builtin_amdgcn_readfirstlane(u1.y) * group;
        first = __builtin_amdgcn_readfirstlane(u1.z), keys = __builtin_amdgcn_readfirstlane(u1.w);
        tiles = keys == 0 ? 0 : __builtin_amdgcn_readfirstlane(u0.z);
    }
    const int chunks = st.head_dim >> 3;

    // this lane's query row; a negative scale moves to the queries
    const int row = row0 + wid * 32 + l32, token = row / group, head = kvh * group + (row - token * group);
    const bool row_ok = row < rows;
    const bool works = row0 + wid * 32 < rows;
    u32x4 q_raw[kSteps];
    {                                         // all on their way before one is looked at; what is no row or channel becomes zeros then
        const uint16_t* const qp = a.q + (int64_t)(q0 + (row_ok ? token : 0)) * a.q_token_stride + (int64_t)(row_ok ? head : 0) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) q_raw[ks] = *(const u32x4*)(qp + (2 * ks + half < chunks ? ks * 16 + half * 8 : 0));
    }
    bf16x8 qf[kSteps];
    const float scale2 = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 1.4e-45f);          // a mask of -inf stays one with a scale of 0

    // Lane i of a load fills slot i % (DH / 8) of row i / (DH / 8) of its rows, and fetches the chunk that belongs there.
    const int ld_row = lane / (DH / 8), ld_slot = lane % (DH / 8), wave_row = wid * kLoads * kRowsPerLoad;
    uint32_t k_at[kLoads], v_at[kLoads];      // offsets from the tile's first row
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int r = wave_row + j * kRowsPerLoad + ld_row, chunk = (int)(v_slot<D>(r, ld_slot) / 16) & (DH / 8 - 1);        // the order is its own inverse
        k_at[j] = chunk < chunks ? (uint32_t)r * (uint32_t)st.k_row_stride * 2u + (uint32_t)chunk * 16u : kOutOfRange;
        v_at[j] = chunk < chunks ? (uint32_t)r * (uint32_t)st.v_row_stride * 2u + (uint32_t)chunk * 16u : kOutOfRange;
    }
    const char* const k_head = (const char*)(st.k + (int64_t)first * st.k_row_stride + kvh * st.k_head_stride);
    const char* const v_head = (const char*)(st.v + (int64_t)first * st.v_row_stride + kvh * st.v_head_stride);
    const uint8_t* const seen = st.seen ? st.seen + first : nullptr;
    // Which keys of a tile are there and not hidden; a byte to a lane, on its way before the tile's turn.
    auto fetch_seen = [&](int t) {
        int byte = 1;
        if (seen) byte = seen[max(0, min((tile0 + t) * kManyKeys + lane, keys - 1))];
        return byte;
    };
    auto shown_of = [&](int t, int byte) {
        asm volatile("" : "+v"(byte));        // not looked at before its turn
        return __ballot((tile0 + t) * kManyKeys + lane < keys && t < tiles && byte != 0);
    };
    unsigned long long shown[3];              // of tiles t, t + 1 and t + 2, in turn
    // K of tile t goes to buffer t % 2, V to buffer t % 3: while tile t is worked on, K and V of t + 1 are there or on their way.
    auto load = [&](int t, unsigned long long there) __attribute__((always_inline)) {
        char *const k_to = lds + t % 2 * kTile + wave_row * (DH * 2), *const v_to = lds + (2 + t % 3) * kTile + wave_row * (DH * 2);
        const int64_t key0 = (int64_t)(tile0 + t) * kManyKeys;
        const __amdgpu_buffer_rsrc_t k_rsrc = __builtin_amdgcn_make_buffer_rsrc((char*)k_head + key0 * st.k_row_stride * 2, 0, 0x7FFFFFFF, 0x00020000);
        const __amdgpu_buffer_rsrc_t v_rsrc = __builtin_amdgcn_make_buffer_rsrc((char*)v_head + key0 * st.v_row_stride * 2, 0, 0x7FFFFFFF, 0x00020000);
        if (there == ~0ull) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (lds_void*)(k_to + j * 1024), 16, k_at[j], 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (lds_void*)(v_to + j * 1024), 16, v_at[j], 0, 0, 0);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {    // zeros for rows that are not there or hidden
            const bool is = there >> (wave_row + j * kRowsPerLoad + ld_row) & 1;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (lds_void*)(k_to + j * 1024), 16, is ? k_at[j] : kOutOfRange, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (lds_void*)(v_to + j * 1024), 16, is ? v_at[j] : kOutOfRange, 0, 0, 0);
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
    f32x16 acc[kBlocks], sc, next;
    u32x4 v0[kBlocks], v1[kBlocks];           // values of the half that is worked on
#pragma unroll
    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[db][x] = 0.f;

    // Half a tile at a time: scores of the next half (matrix cores) are computed beside the exponentials of this one (vector unit).
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
    auto mask = [&](f32x16& v, unsigned long long there, int kb) __attribute__((always_inline)) {
        const uint32_t bits = (uint32_t)(there >> (32 * kb));
        if (bits == 0xFFFFFFFFu) return;
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (!((bits >> (4 * half)) >> (8 * (x >> 2) + (x & 3)) & 1)) v[x] = -INFINITY;
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
            for (int x = 0; x < 16; ++x) acc[db][x] *= shrink;
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
    // the half kb of tile t, whose scores are in `cur`; the next half's, kn of the tile whose keys `there_next` shows, go to `to` (of no use behind the
    // last one, and not used)
    auto half_step = [&](f32x16& cur, f32x16& to, int t, int kb, int kn, unsigned long long there_next) __attribute__((always_inline)) {
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
        add_values<D>(acc, v0, pw[0]);
        add_values<D>(acc, v1, pw[1]);
        if (kb == 1) {                        // the next tile's first values; then what would hold them up: they wait for every load that is on its way
            read_half(v0, 0, 0);
            read_half(v1, 0, 1);
            __builtin_amdgcn_sched_barrier(0);
            if (t + 2 < tiles) load(t + 2, shown[2]);
        }
        mask(to, there_next, kn);
    };

    if (tiles > 0) {
        const int s0 = fetch_seen(0), s1 = fetch_seen(1), s2 = fetch_seen(2);
        shown[0] = shown_of(0, s0);
        load(0, shown[0]);
        shown[1] = shown_of(1, s1);
        if (tiles > 1) load(1, shown[1]);
        shown[2] = shown_of(2, s2);
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, row_ok && 2 * ks + half < chunks ? q_raw[ks] ^ flip : u32x4{0, 0, 0, 0});
        __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8));
        __builtin_amdgcn_s_barrier();
        if (works) {
            read_half(v0, 0, 0);
            read_half(v1, 0, 1);
            u32x4 k[kSteps];
            read_keys(k, 0);
            scores(sc, k);
            mask(sc, shown[0], 0);
            m = highest(sc);                  // what the first half would move the reference to
        }
    }
    for (int t = 0; t < tiles; ++t) {
        const int ahead = fetch_seen(t + 3);
        if (works) half_step(sc, next, t, 0, 1, shown[0]);
        // the next tile has landed, and everybody is through with this one's K and the last one's V
        __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8));
        __builtin_amdgcn_s_barrier();
        if (works) half_step(next, sc, t, 1, 0, shown[1]);
        else if (t + 2 < tiles) load(t + 2, shown[2]);
        shown[0] = shown[1];
        shown[1] = shown[2];
        shown[2] = shown_of(t + 3, ahead);
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
                for (int x = 0; x < 16; ++x) acc[db][x] = 0.f;
        uint16_t* const to = a.out + (int64_t)(q0 + token) * a.out_token_stride + (int64_t)head * a.out_head_stride + half * 4;
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (db * 32 + g * 8 < st.head_dim)
                    *(uint2*)(to + db * 32 + g * 8) = make_uint2(pack_bf16(acc[db][4 * g] * inv, acc[db][4 * g + 1] * inv), pack_bf16(acc[db][4 * g + 2] * inv, acc[db][4 * g + 3] * inv));
        if (a.lse && half == 0) a.lse[(int64_t)(q0 + token) * a.heads + head] = empty ? -INFINITY : (m + log2f(l)) * kLn2;
    } else {
        float* const to = (float*)(workspace + layout.parts) + ((size_t)part * st.kv_heads + kvh) * (2 * kManyRows + kManyRows * D);
        const int rw = wid * 32 + l32;
#pragma unroll
        for (int db = 0; db < kBlocks; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(float4*)(to + 2 * kManyRows + rw * D + db * 32 + g * 8 + half * 4) = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
        if (half == 0) {
            to[rw] = m;
            to[kManyRows + rw] = l;
        }
    }
#endif
}

// Adds up the parts of a unit that was cut; blockIdx.y: 16 of its rows.  Latency: 5.1 us where nothing is to be joined, 5.8 for ten parts of 16 units.
constexpr int kUnitRows = 16;
template <int D> constexpr int kUnitThreads = kUnitRows * D / 4;          // four channels of a row each
template <int D>
__global__ __launch_bounds__(kUnitThreads<D>) void cross_attention_join_units_kernel(States st, CrossAttention a, const char* workspace, ManyLayout layout)
{
    const int kvh = blockIdx.x % st.kv_heads, index = blockIdx.x / st.kv_heads;
    const int n_joined = ((const ManyHeader*)workspace)->joined;
    const Joined u = ((const Joined*)(workspace + layout.joined))[index];         // its place is there in any case
    if (index >= n_joined) return;
    const size_t stride = (size_t)st.kv_heads * (2 * kManyRows + kManyRows * D);
    const float* const parts = (const float*)(workspace + layout.parts) + ((size_t)u.part * st.kv_heads + kvh) * (2 * kManyRows + kManyRows * D);
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
        for (int i = 0; i < kAhead; ++i)
            if (p + i < u.parts) add_part(mx, sum, acc, mp[i], lp[i], v[i]);
    }
    finish_row(st, a, u.q0, kvh, row, ch, mx, sum, acc, 1.f / kJoinRoom);
}

// channels that the kernels compute with: the next multiple of 32
int padded_dim(int32_t head_dim) { return (head_dim + 31) / 32 * 32; }

struct Sizes {                            // what the choice of a kernel goes by
    int64_t n_sources, max_new, max_rows, heads, kv_heads, dim;
    int64_t rows() const { return max_new * (heads / kv_heads); }
    int64_t row_blocks() const { return (rows() + kFewRows - 1) / kFewRows; }
    int64_t groups() const { return n_sources * kv_heads * row_blocks(); }
};
bool is_few(const Sizes& z) { return z.rows() <= kFewRows; }
// Whether a workgroup of its own for every source and head is faster than equal stretches and a join, by the longest source and the number of
// workgroups.  Single tokens of four beams in a graph, whole / stretches, us, sources of equal lengths, then of lengths from one up: 16 heads of 64, 1 source
// 1000 rows 11.0 / 13.5, 2000 17.9 / 15.6; 4 sources 2000 19.0 / 19.7 and 18.9 / 16.0; 8 sources 2000 19.3 / 23.7 and 18.9 / 20.4, 4000 50.5 / 41.2 and
// 32.5 / 23.9; 16 sources 2000 32.4 / 43.1 and 19.5 / 25.0, 4000 60.1 / 68.8 and 50.5 / 45.2; 32 sources 2000 62.4 / 69.5 and 36.3 / 54.6, 4000 123 / 121 and
// 67 / 79; 64 sources 2000 118 / 118 and 67 / 101, 4000 237 / 230 and 129 / 152.  8 heads of 128: 8 sources 500 rows 12.9 / 15.0, 1000 20.0 / 16.1; 16 sources
// 1000 20.3 / 21.2 and 19.7 / 24.3, 2000 50.4 / 38.9; 32 sources 1000 33.1 / 37.8 and 21.0 / 42.2, 4000 113 / 117 and 96 / 70; 64 sources 1000 63.7 / 62.6 and
// 36.9 / 53.6, 2000 117 / 115 and 67 / 87, 4000 from one up 122 / 118.
// Chunks of tokens, a workgroup for 32 rows of each / units, listed or scheduled, 16 heads of 64: one source 40 tokens 1000 rows 11.6 / 17.5, 4000 33.0 / 22.9,
// 300 tokens 1000 rows 12.1 / 19.4, 1000 tokens (512 workgroups) 500 rows 13.4 / 13.1; 4 sources 100 tokens 2000 rows 20.6 / 25.9, 4000 34.1 / 33.1; 300 tokens
// (640) 200 rows 11.3 / 9.8, 1000 28.0 / 20.8; 16 sources 300 tokens 1000 rows 103 / 38.  32 heads on 8 of 128: one source 100 tokens 1000 rows 20.1 / 26.1, 2000
// 33.5 / 29.2; 300 tokens (304) 500 rows 21.9 / 17.4.  Above kListed sources units are scheduled, which costs more: 70 sources of 33 tokens (980) 200 rows of 64
// 18.3 / 19.5, 500 rows 26.2 / 23.9.
bool is_whole(const Sizes& z)
{
    const int64_t longest = z.max_rows * z.dim, groups = z.groups();
    if (z.row_blocks() == 1) return longest <= (groups > 256 ? 262144 : groups >= 128 ? 163840 : 81920);
    if (groups <= 256) return longest <= 163840;
    return z.n_sources > kListed && groups <= 1536 && groups * longest <= 16ll << 20;
}

// units of a call, at most
int64_t most_units(const Sizes& z, int64_t n_tokens)
{
    return std::min(z.n_sources * ((z.rows() + kManyRows - 1) / kManyRows), n_tokens * (z.heads / z.kv_heads) / kManyRows + z.n_sources);
}
// Whether units are listed by their own workgroups and none is cut: where the scheduling launch and the join, which cost 7 to 10 us, would not shorten the longest
// by more than 12 tiles (by what the states' rows say of their mean length).  Listed / scheduled, us, 16 heads of 64: 4 sources 300 tokens 500 rows 14.1 /
// 21.4, 2000 rows (192 units of 32 tiles) 34.7 / 38.9, 4000 60 / 56; one source 1000 tokens 2000 rows (128 of 32) 34.8 / 33.0; 32 sources 20 to 500 tokens on 200 to
// 3000 rows 105 / 108.  32 heads on 8 of 128: one source 300 tokens 1000 rows (80 of 16) 27 / 31, 2000 47 / 39; 8 sources 1000 tokens 4000 rows 265 / 273.
bool is_listed(const Sizes& z, int64_t n_tokens, int64_t n_rows)
{
    if (z.n_sources > kListed) return false;
    auto tiles = [](int64_t rows) { return (rows + kManyKeys - 1) / kManyKeys; };
    const int64_t share = most_units(z, n_tokens) * z.kv_heads * tiles(std::min(z.max_rows, n_rows / std::max<int64_t>(z.n_sources, 1))) / kManyGroups;
    return tiles(z.max_rows) - std::max<int64_t>(8, 2 * share) <= 12;
}

template <int D, bool PAD, int WAVES, bool ORDERED> hipError_t launch_whole(const Sizes& z, const States& st, const CrossAttention& a, hipStream_t stream)
{
    constexpr size_t kLds = kFewLds<D, WAVES>;
    static_assert(!ORDERED || (kLds >= (kRanked + 4) * 4 && 64 * WAVES == kRanked), "a source to a thread");
    static const hipError_t configured =
        hipFuncSetAttribute((const void*)cross_attention_whole_kernel<D, PAD, WAVES, ORDERED>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    if (configured != hipSuccess) return configured;
    // 100 sources of 200 to 600 rows, 16 heads of 64, 46.3 us with dies and 49.3 without, 64 sources the same, 16 of 500 rows 10.9 and 10.4
    const int dies = a.n_sources >= 64 ? 8 : 1;
    hipLaunchKernelGGL((cross_attention_whole_kernel<D, PAD, WAVES, ORDERED>), dim3((unsigned)((a.n_sources + dies - 1) / dies * dies * st.kv_heads), (unsigned)z.row_blocks()),
                       dim3(64 * WAVES), kLds, stream, st, a, dies, (int)std::max<int64_t>(1, 256 / st.kv_heads));
    return hipGetLastError();
}

template <int D, bool PAD> hipError_t launch_few(const Sizes& z, const States& st, const CrossAttention& a, char* workspace, hipStream_t stream)
{
    const size_t lds = std::max(kFewLds<D>, ((size_t)a.n_sources + 1) * 8);
    static const hipError_t configured = hipFuncSetAttribute((const void*)cross_attention_few_kernel<D, PAD>, hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024);
    if (configured != hipSuccess) return configured;
    hipLaunchKernelGGL((cross_attention_few_kernel<D, PAD>), dim3(kFewGroups<D>), dim3(64 * kFewWaves), lds, stream, st, a, workspace);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(cross_attention_join_kernel<D>, dim3((unsigned)(a.n_sources * st.kv_heads), (unsigned)z.rows()), dim3(256), 0, stream, st, a, workspace);
    return hipGetLastError();
}

template <int D> hipError_t launch_many(const Sizes& z, const States& st, const CrossAttention& a, char* workspace, hipStream_t stream)
{
    constexpr int kLds = 5 * kManyTile<D>;
    constexpr size_t kSchedLds = std::max((size_t)(kPlanMaxRequests + 4) * 4, (size_t)(kSchedInLds + 4) * 4 + kSchedInLds * 16);
    static const hipError_t configured[2] = {
        hipFuncSetAttribute((const void*)cross_attention_many_kernel<D>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds),
        hipFuncSetAttribute((const void*)cross_attention_schedule_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kSchedLds)};
    if (configured[0] != hipSuccess || configured[1] != hipSuccess) return configured[0] != hipSuccess ? configured[0] : configured[1];
    const ManyLayout at = many_layout(a.n_sources, a.n_tokens, a.heads, st.kv_heads, D);
    if (is_listed(z, a.n_tokens, st.n_rows)) {
        hipLaunchKernelGGL(cross_attention_many_kernel<D>, dim3((unsigned)(most_units(z, a.n_tokens) * st.kv_heads)), dim3(64 * kManyWaves), kLds, stream, st, a, workspace, at, true);
        return hipGetLastError();
    }
    const size_t sched_lds = ((size_t)a.n_sources + 4) * 4 + (a.n_sources <= kSchedInLds ? (size_t)a.n_sources * 16 : 0);
    hipLaunchKernelGGL(cross_attention_schedule_kernel, dim3(1), dim3(kSchedThreads), sched_lds, stream, st, a, workspace, at);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(cross_attention_many_kernel<D>, dim3((unsigned)(at.most_units * st.kv_heads)), dim3(64 * kManyWaves), kLds, stream, st, a, workspace, at, false);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(cross_attention_join_units_kernel<D>, dim3((unsigned)(at.most_joined * st.kv_heads), kManyRows / kUnitRows), dim3(kUnitThreads<D>), 0, stream, st, a, workspace, at);
    return hipGetLastError();
}

template <int D> hipError_t launch(const Sizes& z, const States& st, const CrossAttention& a, char* workspace, hipStream_t stream)
{
    const bool exact = st.head_dim == D;
    if (is_whole(z)) {
        // Eight wavefronts while there is a compute unit for every workgroup, where a row has little to read: one source, 8 heads of 32, 1000 rows 7.6 us with
        // eight, 8.7 with four, 2000 10.9 and 13.4; 16 heads of 64, 500 rows 8.9 and 8.3, 8 of 128, 640 rows 14.3 and 13.4.
        if constexpr (D == 32)
            if (z.groups() <= 256) return exact ? launch_whole<D, false, 8, false>(z, st, a, stream) : launch_whole<D, true, 8, false>(z, st, a, stream);
        // Ranked / as they come, us, 16 heads of 64 and four beams: 24 sources of 60 to 1500 rows 18.7 / 24.9, 64 53.1 / 62.0, 64 of 197 16.6 / 15.0, 80 of 1 to
        // 600 28.1 / 29.7, 100 of 60 to 1500 73 / 88, 125 of 1 to 600 43.1 / 39.6 (every workgroup ranks them all), 150 of 500 to 1000 99 / 98.  Sizes do not tell
        // equal lengths, which are ranked for nothing: 64 of 197 is what that costs.
        const int64_t groups = z.groups(), longest = z.max_rows * z.dim;
        if (z.n_sources <= kRanked && groups > 256 && (groups <= 1024 || (groups <= 2048 && longest >= 49152)))
            return exact ? launch_whole<D, false, kFewWaves, true>(z, st, a, stream) : launch_whole<D, true, kFewWaves, true>(z, st, a, stream);
        return exact ? launch_whole<D, false, kFewWaves, false>(z, st, a, stream) : launch_whole<D, true, kFewWaves, false>(z, st, a, stream);
    }
    if (!is_few(z)) return launch_many<D>(z, st, a, workspace, stream);
    return exact ? launch_few<D, false>(z, st, a, workspace, stream) : launch_few<D, true>(z, st, a, workspace, stream);
}

}  // namespace

int64_t cross_attention_workspace(int32_t n_sources, int32_t n_tokens, int32_t max_new, int32_t max_rows, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    const int dim = padded_dim(head_dim);
    const Sizes z{n_sources, max_new, max_rows, heads, kv_heads, dim};
    if (is_whole(z)) return 0;
    if (!is_few(z) && is_listed(z, n_tokens, 0)) return 0;      // and so with any number of rows
    if (is_few(z)) return few_header_bytes(n_sources) + (int64_t)kMostFewGroups * 2 * (2 * kFewRows + kFewRows * dim) * 4;
    return many_layout(n_sources, n_tokens, heads, kv_heads, dim).end;
}

hipError_t cross_attention(const States& st, const CrossAttention& a, void* workspace, hipStream_t stream)
{
    const Sizes z{a.n_sources, a.max_new, a.max_rows, a.heads, st.kv_heads, padded_dim(st.head_dim)};
    switch (z.dim) {
    case 32: return launch<32>(z, st, a, (char*)workspace, stream);
    case 64: return launch<64>(z, st, a, (char*)workspace, stream);
    case 96: return launch<96>(z, st, a, (char*)workspace, stream);
    default: return launch<128>(z, st, a, (char*)workspace, stream);
    }
}

}  // namespace k
}  // namespace coe
