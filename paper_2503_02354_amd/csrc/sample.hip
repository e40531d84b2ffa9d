// gfx950 kernels that draw a token from every row of logits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

// Order of a row: descending logits, equal ones by ascending index.  The logit as an unsigned key that grows with it (-0 and +0 the
// same; NaN counts as -inf), so that "comes before" is a comparison of integers.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
__device__ __forceinline__ unsigned long long order_of(float x, uint32_t i) { return (unsigned long long)key_of(x) << 32 | (uint32_t)~i; }

__device__ __forceinline__ float number(float x) { return x == x ? x : -INFINITY; }
__device__ __forceinline__ float logit(const float* row, int i) { return number(row[i]); }
__device__ __forceinline__ float logit(const uint16_t* row, int i) { return number(__uint_as_float((uint32_t)row[i] << 16)); }

// 16 bytes of logits
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kWidth = 4;
    static __device__ __forceinline__ float at(const uint4& w, int e) { return __uint_as_float(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w); }
};
template <> struct Vec<uint16_t> {
    static constexpr int kWidth = 8;
    static __device__ __forceinline__ float at(const uint4& w, int e)
    {
        const uint32_t d = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
        return __uint_as_float(e & 1 ? d & 0xFFFF0000u : d << 16);
    }
};

__device__ __forceinline__ float exp2_fast(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(v);         // one instruction; weights below 2^-126 are 0
#else
    return v;
#endif
}

typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));      // of any fp32 row

struct Best { float score; uint32_t index; };
constexpr uint32_t kNone = 0xFFFFFFFFu;
__device__ __forceinline__ bool better_than(float score, uint32_t index, Best a) { return (score > a.score) | ((score == a.score) & (index < a.index)); }
__device__ __forceinline__ Best better(Best a, Best b) { return better_than(b.score, b.index, a) ? b : a; }

// Of a wavefront's part of a row: the largest logit and where, the winner of the race (score relative to 2^at), the sum of the weights
// relative to 2^at.  odd: the sum is no number; tiny: a random number below 2^-40.
struct Record {
    Best top, won;
    float at, sum;
    uint32_t odd, tiny;
};

constexpr int kMostCandidates = 4096, kMostBorder = 1024, kPairs = 256, kBins = 512;
template <int THREADS> struct Shared {
    static constexpr int kWaves = THREADS / 64;
    // a wavefront's part of a reduction; two sets in turn, so that one barrier is enough
    Best best[2][kWaves];
    float2 sums[2][kWaves];
    Record record[kWaves];
    uint32_t hist[kBins];
    uint32_t pick, before_pick;
    uint32_t n_candidates, n_border;
    alignas(16) unsigned long long candidate[kMostCandidates];
    alignas(16) unsigned long long border[kMostBorder + 4];
    float weight[kPairs], score[kPairs];      // of a short list, in order
    uint32_t index[kPairs];
};

__device__ __forceinline__ Best wave_best(Best v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = better(v, Best{__shfl_xor(v.score, d, 64), (uint32_t)__shfl_xor((int)v.index, d, 64)});
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}
// `set` counts a thread's reductions.
template <int THREADS> __device__ __forceinline__ Best block_best(Best v, Shared<THREADS>& sh, int& set)
{
    Best* const part = sh.best[set++ & 1];
    v = wave_best(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < Shared<THREADS>::kWaves; ++w) v = better(v, part[w]);
    return v;
}
template <int THREADS> __device__ __forceinline__ float2 block_sums(float2 v, Shared<THREADS>& sh, int& set)
{
    float2* const part = sh.sums[set++ & 1];
    v = make_float2(wave_sum(v.x), wave_sum(v.y));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < Shared<THREADS>::kWaves; ++w) v.x += part[w].x, v.y += part[w].y;
    return v;
}
template <int THREADS> __device__ __forceinline__ float block_sum(float v, Shared<THREADS>& sh, int& set)
{
    return block_sums(make_float2(v, 0.f), sh, set).x;
}

// Sums whose terms are whole numbers do not depend on their order.
template <int THREADS> __device__ __forceinline__ unsigned long long block_count(unsigned long long v, Shared<THREADS>& sh, int& set)
{
    unsigned long long* const part = (unsigned long long*)sh.sums[set++ & 1];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < Shared<THREADS>::kWaves; ++w) v += part[w];
    return v;
}

// The row in batches, this thread's share: f(x[], n, first index) for n logits as they are (NaN too), W at a time from 16 bytes (in_batch
// has their indices); n = 1 at the row's ends, whose alignment may be any.  A thread's indices ascend.
template <int THREADS, typename T, class F> __device__ __forceinline__ void batches(const T* row, int vocab, F f)
{
    constexpr int W = Vec<T>::kWidth, kAhead = 16 / W;
    const int tid = threadIdx.x;
    const int lead = min(vocab, (int)((-(uintptr_t)row & 15) / sizeof(T))), vecs = (vocab - lead) / W, tail = lead + vecs * W;
    const uint4* const body = (const uint4*)(row + lead);
    float x[16];
    if (tid < lead) {
        x[0] = logit(row, tid);
        f(x, std::integral_constant<int, 1>(), (uint32_t)tid);
    }
    int v = tid;
    uint4 next[kAhead];
    if (v + (kAhead - 1) * THREADS < vecs)
#pragma unroll
        for (int j = 0; j < kAhead; ++j) next[j] = body[v + j * THREADS];
    for (; v + (kAhead - 1) * THREADS < vecs; v += kAhead * THREADS) {
        uint4 w[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) w[j] = next[j];
        if (v + (2 * kAhead - 1) * THREADS < vecs)
#pragma unroll
            for (int j = 0; j < kAhead; ++j) next[j] = body[v + (kAhead + j) * THREADS];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int e = 0; e < W; ++e) x[j * W + e] = Vec<T>::at(w[j], e);
        f(x, std::integral_constant<int, 16>(), (uint32_t)(lead + v * W));
    }
    for (; v < vecs; v += THREADS) {
        const uint4 w = body[v];
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = Vec<T>::at(w, e);
        f(x, std::integral_constant<int, W>(), (uint32_t)(lead + v * W));
    }
    if (tid < vocab - tail) {
        x[0] = logit(row, tail + tid);
        f(x, std::integral_constant<int, 1>(), (uint32_t)(tail + tid));
    }
}
// index of element e of a batch that begins at i
template <int THREADS, typename T> __device__ __forceinline__ uint32_t in_batch(uint32_t i, int e)
{
    constexpr int W = Vec<T>::kWidth;
    return i + (uint32_t)(e / W * THREADS * W + e % W);
}
// f(x, index) for every logit
template <int THREADS, typename T, class F> __device__ __forceinline__ void each(const T* row, int vocab, F f)
{
    batches<THREADS>(row, vocab, [&](const float (&x)[16], auto n, uint32_t i) {
#pragma unroll
        for (int e = 0; e < n; ++e) f(x[e], in_batch<THREADS, T>(i, e));
    });
}

// The beginning of the order: tokens with a logit above x, and those of logit x with an index below `end`.
struct Front {
    float x;
    uint32_t end;
    __device__ __forceinline__ bool holds(float v, uint32_t i) const { return (v > x) | ((v == x) & (i < end)); }
};

// What a row's weights are relative to, and in which unit.
struct Scale {
    float top, per2;                          // largest logit; 1 / T in units of ln 2
    float reference;                          // top per2, rounded
    bool far;                                 // the row is no common one: near_weight may not be asked
    // log2 of the weight: 0 for the largest itself, be it infinite, and -inf for others then
    __device__ __forceinline__ float rel2(float x) const { return (x == top ? 0.f : x - top) * per2; }
    __device__ __forceinline__ float weight(float x) const { return exp2_fast(rel2(x)); }
    // the same but for a factor near 1 that all tokens of the row share
    __device__ __forceinline__ float near_weight(float x) const { return exp2_fast(__builtin_fmaf(x, per2, -reference)); }
};

constexpr float kTiny = 0x1p-40f;
// This thread's winner of the race among the tokens of a front: the largest log2(w) - log2 E.
template <int THREADS, typename T>
__device__ __attribute__((noinline)) Best winner_by_logs(const T* row, const float* noise, int vocab, uint32_t top_index, Front front, float least, Scale scale)
{
    Best win{-INFINITY, kNone};
    each<THREADS>(row, vocab, [&](float x, uint32_t i) {
        if (!front.holds(x, i) | (x == -INFINITY)) return;
        const float z = scale.rel2(x), score = z - log2f(noise[i]);
        if (((z >= least) | (i == top_index)) & (score > -INFINITY)) win = better(win, Best{score, i});
    });
    return win;
}

// The same by cross products of w and E; the logarithms are taken of a thread's winner only.  near: fp32 holds the products (no random
// number is below 2^-40; a winner below 2^-40 says that it may not).
template <int THREADS, typename T>
__device__ __forceinline__ Best winner(const T* row, const float* noise, int vocab, uint32_t top_index, Front front, float least, Scale scale, bool& near)
{
    uint32_t index = kNone;
    float win_w = 0.f, win_q = 1.f, smallest = 1.f;
    batches<THREADS>(row, vocab, [&](const float (&x)[16], auto n, uint32_t i) {
        float high = x[0];
#pragma unroll
        for (int e = 1; e < n; ++e) high = fmaxf(high, x[e]);
        if (!(high >= front.x)) return;
        float q[16];
        if constexpr (n == 1) q[0] = noise[i];
        else {
#pragma unroll
            for (int e = 0; e < n; e += 4) {
                const f32x4 v = *(const f32x4*)(noise + in_batch<THREADS, T>(i, e));
                q[e] = v[0], q[e + 1] = v[1], q[e + 2] = v[2], q[e + 3] = v[3];
            }
        }
#pragma unroll
        for (int e = 0; e < n; ++e) {
            const uint32_t at = in_batch<THREADS, T>(i, e);
            const float z = (x[e] - scale.top) * scale.per2, w = exp2_fast(z);
            smallest = fminf(smallest, q[e]);
            const bool wins = front.holds(x[e], at) & ((z >= least) | (at == top_index)) & (q[e] >= 0.f) & (w * win_q > win_w * q[e]);
            win_w = wins ? w : win_w;
            win_q = wins ? q[e] : win_q;
            index = wins ? at : index;
        }
    });
    near = !(smallest < kTiny);
    return Best{index == kNone ? -INFINITY : log2f(win_w) - log2f(win_q), index};
}

// Whether a thread whose winner `at` is not kept hides another token of the front that beats `best`: its share of the row is looked
// through.  Every thread takes a part of the share.
template <int THREADS, typename T>
__device__ __forceinline__ bool hides(const T* row, const float* noise, int vocab, int at, uint32_t top_index, Front front, float least, Scale scale, Best best)
{
    constexpr int W = Vec<T>::kWidth;
    const int lead = min(vocab, (int)((-(uintptr_t)row & 15) / sizeof(T))), vecs = (vocab - lead) / W, tail = lead + vecs * W;
    const int owner = at < lead ? at : at >= tail ? at - tail : (at - lead) / W % THREADS;
    const int own_vecs = vecs > owner ? (vecs - owner + THREADS - 1) / THREADS : 0;
    bool hidden = false;
    for (int k = threadIdx.x; k < own_vecs * W + 2; k += blockDim.x) {
        const uint32_t place = k < own_vecs * W ? lead + (owner + k / W * THREADS) * W + k % W : k == own_vecs * W ? (owner < lead ? owner : vocab) : (uint32_t)tail + owner;
        if (place >= (uint32_t)vocab) continue;
        const int i = (int)place;
        const float x = logit(row, i), z = scale.rel2(x), score = z - log2f(noise[i]);
        hidden = hidden || (front.holds(x, (uint32_t)i) && (z >= least || i == (int)top_index) && better_than(score, (uint32_t)i, best));
    }
    return hidden;
}

__device__ __forceinline__ float least_of(float min_p) { return min_p > 0.f ? log2f(min_p) : -INFINITY; }

// The weights of the tokens before two tokens of the order.  For a batch that lies before (behind) a token by index, the bound itself counts
// equal logits in (out).
template <int THREADS, typename T, class Weight>
__device__ __forceinline__ float2 masses_before(const T* row, int vocab, const Front (&ahead)[2], Weight weight)
{
    constexpr uint32_t kReach = (16 / Vec<T>::kWidth - 1) * THREADS * Vec<T>::kWidth + Vec<T>::kWidth;      // of a batch
    // the next lower number: to be above it is to reach the bound
    const float with[2] = {nextafterf(ahead[0].x, -INFINITY), nextafterf(ahead[1].x, -INFINITY)};
    float before[2] = {0.f, 0.f};
    const float lowest = fminf(ahead[0].x, ahead[1].x);
    batches<THREADS>(row, vocab, [&](const float (&x)[16], auto n, uint32_t i) {
        float high = x[0];
#pragma unroll
        for (int e = 1; e < n; ++e) high = fmaxf(high, x[e]);
        if (!(high >= lowest)) return;
        float above[2];
        bool clear = true;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            above[j] = i + kReach <= ahead[j].end ? with[j] : ahead[j].x;
            clear &= (i + kReach <= ahead[j].end) | (i >= ahead[j].end);
        }
        if (clear) {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float w = weight(x[e]);
#pragma unroll
                for (int j = 0; j < 2; ++j) before[j] += x[e] > above[j] ? w : 0.f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float w = weight(x[e]);
#pragma unroll
                for (int j = 0; j < 2; ++j) before[j] += ahead[j].holds(x[e], in_batch<THREADS, T>(i, e)) ? w : 0.f;
            }
        }
    });
    return make_float2(before[0], before[1]);
}

// The race decided by what the filters say.  It needs no sorted row: its winner among a front that holds all kept tokens is the drawn
// token if it is kept itself, and whether it is takes one sum over the tokens before it.  If it is not, no token from its place on
// is kept either, and the race is for the others.  The sums of the two best threads' winners are taken in one pass, since a row
// whose winner falls to the nucleus would keep the launch waiting for another two.
// `first` and `mine` (this thread's) are the winners of a race that has been run; without an index: none has.  mass: near_weights' of
// a row that is not far, else weights'.
template <int THREADS, typename T>
__device__ uint32_t race(const T* row, const float* noise, int vocab, uint32_t top_index, Front front, float top_p, float mass, float min_p, Scale scale, Best first,
                         Best mine, Shared<THREADS>& sh, int& set)
{
    // what lies before the second token is the first one's weight: a nucleus of one
    if (top_p < 1.f && !((scale.far ? 1.f : scale.near_weight(scale.top)) < top_p * mass)) return top_index;
    const float least = least_of(min_p);
    bool by_logs = !(scale.top < INFINITY);
    for (;;) {                                // the front shrinks with every round that goes on
        Best c[2] = {first, Best{-INFINITY, kNone}};
        if (!by_logs) {
            if (first.index == kNone) {
                bool near;
                mine = winner<THREADS>(row, noise, vocab, top_index, front, least, scale, near);
                by_logs = __syncthreads_or(!near);
                c[0] = block_best(mine, sh, set);
                by_logs |= !(c[0].score > -40.f);
            }
            if (!by_logs && top_p < 1.f && c[0].index != top_index) {
                if (mine.index == c[0].index) mine = Best{-INFINITY, kNone};
                c[1] = block_best(mine, sh, set);
            }
        }
        first.index = kNone;
        if (by_logs) c[0] = block_best(winner_by_logs<THREADS>(row, noise, vocab, top_index, front, least, scale), sh, set);
        if (c[0].index == kNone) return top_index;
        if (!(top_p < 1.f) || c[0].index == top_index) return c[0].index;

        const Front ahead[2] = {Front{logit(row, c[0].index), c[0].index}, c[1].index == kNone ? Front{INFINITY, 0} : Front{logit(row, c[1].index), c[1].index}};
        const float2 before = scale.far ? masses_before<THREADS>(row, vocab, ahead, [&](float x) { return scale.weight(x); })
                                        : masses_before<THREADS>(row, vocab, ahead, [&](float x) { return scale.near_weight(x); });
        const float2 masses = block_sums(before, sh, set);
        if (masses.x < top_p * mass) return c[0].index;
        if (front.holds(ahead[0].x, ahead[0].end)) front = ahead[0];
        if (c[1].index == kNone) continue;
        if (c[1].index == top_index || masses.y < top_p * mass) {
            if (!__syncthreads_or(hides<THREADS>(row, noise, vocab, (int)c[0].index, top_index, front, least, scale, c[1]))) return c[1].index;
        } else if (front.holds(ahead[1].x, ahead[1].end))
            front = ahead[1];
    }
}

// The front of the first top_k tokens, byte by byte from the top of the order as one number, key first, then index.  What bounds it: eight passes
// over the row, with LDS atomics.  96 rows of 128,000 fp32 with a top_k from 2049 on 242 to 273 us, where a list of 2000 takes 54.7.
template <int THREADS, typename T> __device__ Front front_of(const T* row, int vocab, uint32_t left, Shared<THREADS>& sh)
{
    const int tid = threadIdx.x;
    unsigned long long last = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int b = tid; b < 256; b += THREADS) sh.hist[b] = 0;
        __syncthreads();
        each<THREADS>(row, vocab, [&](float x, uint32_t i) {
            const unsigned long long o = order_of(number(x), i);
            if (shift == 56 || (o >> (shift + 8)) == (last >> (shift + 8))) atomicAdd(&sh.hist[(o >> shift) & 255], 1u);
        });
        __syncthreads();
        if (tid == 0) {
            int b = 255;
            uint32_t above = 0;
            while (above + sh.hist[b] < left) above += sh.hist[b--];
            sh.pick = (uint32_t)b;
            sh.hist[b] = left - above;
        }
        __syncthreads();
        last |= (unsigned long long)sh.pick << shift;
        left = sh.hist[sh.pick];
        __syncthreads();
    }
    return {logit_of((uint32_t)(last >> 32)), ~(uint32_t)last + 1};
}

// A small top_k from a short list.  Every thread has met the largest logits of parts of its share; with at least top_k of all these
// at or above a bound, so are the first top_k tokens.  One pass collects what reaches the bound (little more than top_k tokens),
// and the filters are decided on that.  The bound is the edge of a bin of the distances from the largest logit, 64 bins to an octave
// of 1 + distance.
constexpr uint32_t kOne = 0x3F800000u, kBinShift = 17;
__device__ __forceinline__ uint32_t bin_of(float x, Scale scale) { return min(kBins - 1u, (__float_as_uint(1.f - scale.rel2(x)) - kOne) >> kBinShift); }
// the bin that holds the top_k-th of those counted (the last one if there are fewer), and how many lie in those before it
template <int THREADS> __device__ __forceinline__ void pick_bin(uint32_t top_k, Shared<THREADS>& sh)
{
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid == 0) sh.pick = kBins - 1;
    __syncthreads();
    if (tid < 64) {                           // lane l holds bins 8 l .. 8 l + 7
        constexpr int kPer = kBins / 64;
        uint32_t h[kPer], sum = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) sum += h[j] = sh.hist[kPer * lane + j];
        uint32_t before = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t u = __shfl_up(before, d, 64);
            if (lane >= d) before += u;
        }
        before -= sum;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (before < top_k && before + h[j] >= top_k) {
                sh.pick = (uint32_t)(kPer * lane + j);
                sh.before_pick = before;
            }
            before += h[j];
        }
    }
    __syncthreads();
}
template <int THREADS, typename T>
__device__ __forceinline__ uint32_t collect(const T* row, int vocab, const float (&own_max)[4], uint32_t top_k, Scale scale, Shared<THREADS>& sh)
{
    const int tid = threadIdx.x;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (own_max[j] > -INFINITY) atomicAdd(&sh.hist[bin_of(own_max[j], scale)], 1u);
    if (tid == 0) sh.n_candidates = sh.n_border = 0;
    pick_bin(top_k, sh);
    // the bin's far edge as a logit, a little further out than any rounding of the distances reaches
    const uint32_t bin = sh.pick;
    const float far = (__uint_as_float(kOne + ((bin + 1) << kBinShift)) * 1.00001f - 1.f) / scale.per2;
    const float least = bin == kBins - 1 || !(scale.top < INFINITY) ? -INFINITY : scale.top - far * 1.00001f - fabsf(scale.top) * 1e-6f;
    for (int b = tid; b < kBins; b += THREADS) sh.hist[b] = 0;          // for the list's own bins
    batches<THREADS>(row, vocab, [&](const float (&x)[16], auto n, uint32_t i) {
        float high = x[0];
#pragma unroll
        for (int e = 1; e < n; ++e) high = fmaxf(high, x[e]);
        if (!(high >= least)) return;
#pragma unroll
        for (int e = 0; e < n; ++e)
            if (x[e] >= least && x[e] > -INFINITY) {
                const uint32_t at = atomicAdd(&sh.n_candidates, 1u);
                if (at < kMostCandidates) sh.candidate[at] = order_of(x[e], in_batch<THREADS, T>(i, e));
            }
    });
    __syncthreads();
    return sh.n_candidates;
}
// The token of a list of n tokens that holds the first top_k, n <= kPairs; wavefront 0 has it.  The list is put in order by comparing
// all pairs, so that the order which atomics gave it has no say in anything, and one wavefront goes through it.
template <int THREADS>
__device__ uint32_t from_short_list(uint32_t n, const float* noise, uint32_t top_k, float top_p, float min_p, Scale scale, Shared<THREADS>& sh)
{
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    if (tid < 3) sh.candidate[n + tid] = 0;
    __syncthreads();
    if (tid < n) {
        const unsigned long long o = sh.candidate[tid];
        uint32_t rank = 0;
        for (uint32_t j = 0; j < n; j += 4) {             // the places up to the next multiple of four hold zeros
            const ulonglong2 a = *(const ulonglong2*)&sh.candidate[j], b = *(const ulonglong2*)&sh.candidate[j + 2];
            rank += (a.x > o) + (a.y > o) + (b.x > o) + (b.y > o);
        }
        if (rank < top_k) {
            const float z = scale.rel2(logit_of((uint32_t)(o >> 32)));
            sh.weight[rank] = exp2_fast(z);
            sh.score[rank] = z - log2f(noise[~(uint32_t)o]);
            sh.index[rank] = ~(uint32_t)o;
        }
    }
    __syncthreads();
    const uint32_t kept = min(n, top_k);
    // the sums in the order of the ranks, 64 of them at a time; the whole sum first
    if (wid > 0) return 0;
    float mass = 0.f;
    if (top_p < 1.f) {
        for (uint32_t rank = lane; rank < kept; rank += 64) mass += sh.weight[rank];
        mass = wave_sum(mass);
    }
    Best win{-INFINITY, kNone};
    float ahead = 0.f;
    for (uint32_t base = 0; base < kept; base += 64) {
        const uint32_t rank = base + lane;
        const float w = rank < kept ? sh.weight[rank] : 0.f;
        float sum = w;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const float u = __shfl_up(sum, d, 64);
            if (lane >= d) sum += u;
        }
        const float shifted = __shfl_up(sum, 1, 64), before = ahead + (lane == 0 ? 0.f : shifted);
        if (rank < kept && (rank == 0 || ((!(top_p < 1.f) || before < top_p * mass) && (!(min_p > 0.f) || w >= min_p)))) {
            const float score = sh.score[rank];
            if (score > -INFINITY) win = better(win, Best{score, sh.index[rank]});
        }
        ahead += __shfl(sum, 63, 64);
    }
    win = wave_best(win);
    return win.index == kNone ? sh.index[0] : win.index;
}
// The same of a longer one, all wavefronts; kNone where too many equal tokens lie across the cut.  Nothing depends on the list's order:
// tokens are compared as (logit, index), and masses are sums of whole numbers, weights in units of 2^-40.  The race goes as for whole
// rows, but a round costs two reductions only.  96 rows of 128,000 fp32, us by pairs / in rounds: 27.4 / 32.8 with a top_k of 50 and a
// nucleus (lists of 80), 37 / 32 with one of 400 (450); 58.7 sorted / 38.8 with one of 1000.
template <int THREADS>
__device__ uint32_t from_list(uint32_t n, const float* noise, uint32_t top_index, uint32_t top_k, float top_p, float min_p, Scale scale, Shared<THREADS>& sh, int& set)
{
    const int tid = threadIdx.x;
    constexpr int kEach = kMostCandidates / THREADS;
    unsigned long long o[kEach];              // 0: none
#pragma unroll
    for (int j = 0; j < kEach; ++j) o[j] = tid + j * THREADS < n ? sh.candidate[tid + j * THREADS] : 0;
    auto logit_in = [](unsigned long long v) { return logit_of((uint32_t)(v >> 32)); };
    if (n > top_k) {                          // the cut: all before one bin, and of that bin the first
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (o[j]) atomicAdd(&sh.hist[bin_of(logit_in(o[j]), scale)], 1u);
        __syncthreads();
        pick_bin(top_k, sh);
        const uint32_t pick = sh.pick, need = top_k - sh.before_pick;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (!o[j]) continue;
            const uint32_t bin = bin_of(logit_in(o[j]), scale);
            if (bin == pick) {
                const uint32_t at = atomicAdd(&sh.n_border, 1u);
                if (at < kMostBorder) sh.border[at] = o[j];
            } else if (bin > pick)
                o[j] = 0;
        }
        __syncthreads();
        const uint32_t border = sh.n_border;
        if (border > kMostBorder) return kNone;
        if (border > need) {
            if (tid < 3) sh.border[border + tid] = 0;
            __syncthreads();
            const unsigned long long low = need;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if (!o[j] || bin_of(logit_in(o[j]), scale) != pick) continue;
                uint32_t rank = 0;
                for (uint32_t i = 0; i < border; i += 4) {            // the places up to the next multiple of four hold zeros
                    const ulonglong2 a = *(const ulonglong2*)&sh.border[i], b = *(const ulonglong2*)&sh.border[i + 2];
                    rank += (a.x > o[j]) + (a.y > o[j]) + (b.x > o[j]) + (b.y > o[j]);
                }
                if (rank >= low) o[j] = 0;
            }
        }
    }
    float score[kEach];
    unsigned long long weight[kEach], mass = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        score[j] = -INFINITY;
        weight[j] = 0;
        if (!o[j]) continue;
        const uint32_t index = ~(uint32_t)o[j];
        const float z = scale.rel2(logit_in(o[j])), w = exp2_fast(z);
        weight[j] = (unsigned long long)(w * 0x1p40f);
        if (!(min_p > 0.f) || w >= min_p || index == top_index) score[j] = z - log2f(noise[index]);
        mass += weight[j];
    }
    const bool nucleus = top_p < 1.f;
    const double limit = nucleus ? (double)top_p * (double)block_count(mass, sh, set) : 0.;
    for (;;) {                                // every round takes the winner and what is behind it out
        Best win{-INFINITY, kNone};
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (score[j] > -INFINITY) win = better(win, Best{score[j], ~(uint32_t)o[j]});
        const Best mine = win;
        win = block_best(win, sh, set);
        if (win.index == kNone) return top_index;
        if (!nucleus || win.index == top_index) return win.index;
        if (mine.index == win.index)
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (~(uint32_t)o[j] == win.index && o[j]) sh.candidate[0] = o[j];
        __syncthreads();
        const unsigned long long at = sh.candidate[0];
        unsigned long long before = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            before += o[j] > at ? weight[j] : 0;
            if (o[j] <= at) score[j] = -INFINITY;
        }
        if ((double)block_count(before, sh, set) < limit) return win.index;
    }
}

// A thread's share of a row: its largest logit and where, the sum of its weights relative to 2^at, the largest logits of four parts of
// it, and with RACE the winner among all its tokens (score relative to 2^at) and its smallest random number.
// Weights are x unit - at in one rounding, whatever number `at` is.  It follows the largest logit so far, but not below -2^20: masks of
// the type's lowest value weigh nothing then, and what a rounding of `at` leaves of the largest weight stays near 1.
constexpr float kFar = 1048576.f;
struct Share {
    Best top, won;
    float at, sum, smallest, part_max[4];
};
template <int THREADS, bool RACE, typename T> __device__ __forceinline__ Share first_pass(const T* row, const float* noise, int vocab, float unit)
{
    Best top{-INFINITY, kNone};
    float part_max[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    float at = -kFar, sum = 0.f;              // a share with nothing in it does not raise its wavefront's reference
    uint32_t index = kNone;
    float win_w = 0.f, win_q = 1.f, smallest = 1.f;
    batches<THREADS>(row, vocab, [&](const float (&x)[16], auto n, uint32_t i) {
        float q[16];
        if constexpr (RACE) {
            if constexpr (n == 1) q[0] = noise[i];
            else {
#pragma unroll
                for (int e = 0; e < n; e += 4) {
                    const f32x4 v = *(const f32x4*)(noise + in_batch<THREADS, T>(i, e));
                    q[e] = v[0], q[e + 1] = v[1], q[e + 2] = v[2], q[e + 3] = v[3];
                }
            }
        }
        float high[4];
#pragma unroll
        for (int e = 0; e < n; ++e) high[e / 4] = e % 4 ? fmaxf(high[e / 4], x[e]) : x[e];
        constexpr int kParts = (n + 3) / 4;
        if constexpr (!RACE) {
#pragma unroll
            for (int j = 0; j < kParts; ++j) part_max[j] = fmaxf(part_max[j], high[j]);
        }
#pragma unroll
        for (int j = 1; j < kParts; ++j) high[0] = fmaxf(high[0], high[j]);
        if (high[0] > top.score) {
            uint32_t where = 0;
#pragma unroll
            for (int e = n - 1; e >= 0; --e) where = x[e] == high[0] ? in_batch<THREADS, T>(i, e) : where;
            const float now = fmaxf(high[0] * unit, -kFar), keep = exp2_fast(at - now);
            sum = top.index == kNone ? 0.f : sum * keep;
            if constexpr (RACE) win_w = top.index == kNone ? 0.f : win_w * keep;
            at = now;
            top = Best{high[0], where};
        }
#pragma unroll
        for (int e = 0; e < n; ++e) {
            const float w = exp2_fast(__builtin_fmaf(x[e], unit, -at));
            sum += w;
            if constexpr (RACE) {
                smallest = fminf(smallest, q[e]);
                const bool wins = (q[e] >= 0.f) & (w * win_q > win_w * q[e]);
                win_w = wins ? w : win_w;
                win_q = wins ? q[e] : win_q;
                index = wins ? in_batch<THREADS, T>(i, e) : index;
            }
        }
    });
    return Share{top, Best{index == kNone ? -INFINITY : log2f(win_w) - log2f(win_q), index}, at, sum, smallest, {part_max[0], part_max[1], part_max[2], part_max[3]}};
}

// A workgroup per row.  What bounds it: a row's passes, one after the other, at what one compute unit takes from memory, and vector
// instructions where there are rows for all of them.  One row of 50,001 fp32 logits with top_k 40 and a nucleus 14.6 us;
// 96 rows of 128,000 with mixed filters 28.4 us (93 MB from memory, 3.3 TB/s from 96 of 256 compute units); 600 rows of 32,003 bf16 with a nucleus
// of 0.92 48.8 us (145 MB, 3.0 TB/s), where one pass without noise takes 13.5 and with it 26.  A row shared by several
// workgroups, its passes as launches, is no faster: 23.9 and 39.9 us for the first two (14.8 and 38.4 then).
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void sample_kernel(Sampling s)
{
    __shared__ Shared<THREADS> sh;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, vocab = s.vocab;
    int set = 0;
    const size_t r = blockIdx.x;
    for (int b = tid; b < kBins; b += THREADS) sh.hist[b] = 0;
    const T* const row = (const T*)s.logits + r * s.logits_stride;
    const float* const noise = s.noise ? s.noise + r * s.noise_stride : nullptr;
    const float temperature = s.temperature ? s.temperature[r] : 1.f;
    const bool greedy = !(temperature > 0.f) || !noise;
    const float unit = fminf(fmaxf(1.44269504088896340736f / (temperature > 0.f ? temperature : 1.f), 1.4e-45f), 3.402823466e38f);      // neither 0 nor inf for any temperature
    const int32_t top_k = s.top_k ? s.top_k[r] : 0;
    const float top_p = s.top_p ? s.top_p[r] : 1.f, min_p = s.min_p ? s.min_p[r] : 0.f;
    const bool cut = top_k > 0 && top_k < vocab;

    // One pass: the largest logit and where it is, and the sum of the weights relative to it, which is scaled down whenever a thread
    // meets a larger one.  Where all tokens are in the race, for all that is known yet, it is run beside that on the same weights.
    const bool at_once = !greedy && !cut && !(min_p > 0.f);
    Share own = at_once ? first_pass<THREADS, true>(row, noise, vocab, unit) : first_pass<THREADS, false>(row, noise, vocab, unit);
    Best top, first{-INFINITY, kNone};
    float all, mass = 0.f, reference;         // sums of weights and of near_weights
    bool far, near = true;
    {
#pragma clang fp contract(off)                // the reference is the rounded product in every use
        // one barrier for all of it; what is relative to something is brought to a common reference on the way
        Record part{wave_best(own.top), first, own.at, 0.f, (uint32_t)__any(!(own.sum < INFINITY)), (uint32_t)__any(own.smallest < kTiny)};
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) part.at = fmaxf(part.at, __shfl_xor(part.at, d, 64));
        part.sum = wave_sum(own.top.index == kNone ? 0.f : own.sum * exp2_fast(own.at - part.at));
        if (at_once) {
            own.won.score += own.at - part.at;
            part.won = wave_best(own.won);
        }
        if (lane == 0) sh.record[wid] = part;
        __syncthreads();
        top = sh.record[0].top;
#pragma unroll
        for (int w = 1; w < Shared<THREADS>::kWaves; ++w) top = better(top, sh.record[w].top);
        reference = top.score * unit;
        const float factor = __builtin_fmaf(top.score, unit, -reference);     // log2 of the largest logit's near_weight
        far = !(fabsf(reference) < kFar);
#pragma unroll
        for (int w = 0; w < Shared<THREADS>::kWaves; ++w) {
            const Record v = sh.record[w];
            mass += v.sum * exp2_fast(v.at - reference);
            far |= v.odd != 0;
            near &= v.tiny == 0;
            if (at_once) first = better(first, Best{v.won.score + (v.at - reference) - factor, v.won.index});
        }
        own.won.score += part.at - reference - factor;
        all = mass * exp2_fast(-factor);
    }
    if (far || !near || !(first.score > -40.f)) first.index = kNone;
    if (far) {
        // NaN among the logits, infinite ones, numbers too large for that, or none at all
        top = Best{-INFINITY, kNone};
        each<THREADS>(row, vocab, [&](float raw, uint32_t i) {
            const float x = number(raw);
            if (x > top.score) top = Best{x, i};
        });
        own.part_max[0] = top.score;
        own.part_max[1] = own.part_max[2] = own.part_max[3] = -INFINITY;
        top = block_best(top, sh, set);
        const Scale scale{top.score, unit, 0.f, true};
        all = 0.f;
        each<THREADS>(row, vocab, [&](float raw, uint32_t) { all += number(raw) > -INFINITY ? scale.weight(raw) : 0.f; });
        all = mass = block_sum(all, sh, set);
    }
    if (top.index == kNone) {
        if (tid == 0) {
            s.token[r] = -1;
            if (s.logprob) s.logprob[r] = -INFINITY;
        }
        return;
    }
    const Scale scale{top.score, unit, reference, far};

    uint32_t token = top.index;
    if (!greedy) {
        token = kNone;
        if (cut && top_k <= 2 * THREADS) {
            // more tokens may reach the bound, because many are equal or because the bins do not reach as far
            const uint32_t n = collect(row, vocab, own.part_max, (uint32_t)top_k, scale, sh);
            if (n <= kPairs) token = from_short_list(n, noise, (uint32_t)top_k, top_p, min_p, scale, sh);
            else if (n <= kMostCandidates) token = from_list(n, noise, top.index, (uint32_t)top_k, top_p, min_p, scale, sh, set);
        }
        if (token == kNone) {
            Front last{-INFINITY, kNone};
            if (cut) {
                last = front_of(row, vocab, (uint32_t)top_k, sh);
                mass = 0.f;
                each<THREADS>(row, vocab, [&](float x, uint32_t i) {
                    const float w = far ? scale.weight(x) : scale.near_weight(x);
                    mass += (last.holds(x, i) & (x > -INFINITY)) ? w : 0.f;
                });
                mass = block_sum(mass, sh, set);
            }
            if (top_p < 1.f) {
                // Tokens lighter than (1 - top_p) mass / vocab weigh less than what the nucleus leaves out, all together: none of them is in
                // it.  A quarter of that, so that no rounding matters.
                const float least = top.score + log2f(0.25f * (1.f - fmaxf(top_p, 0.f)) * mass / (float)vocab) / unit;
                if (least > last.x) last = Front{least, kNone};
            }
            token = race(row, noise, vocab, top.index, last, top_p, mass, min_p, scale, first, own.won, sh, set);
        }
    }
    if (tid == 0) {
        s.token[r] = (int32_t)token;
        if (s.logprob) s.logprob[r] = (scale.rel2(logit(row, token)) - log2f(all)) * 0.69314718055994530942f;
    }
}

template <int THREADS> void launch(int dtype, int32_t n_rows, const Sampling& s, hipStream_t stream)
{
    if (dtype == 0) hipLaunchKernelGGL((sample_kernel<float, THREADS>), dim3(n_rows), dim3(THREADS), 0, stream, s);
    else hipLaunchKernelGGL((sample_kernel<uint16_t, THREADS>), dim3(n_rows), dim3(THREADS), 0, stream, s);
}

}  // namespace

int64_t sample_workspace(int32_t, int32_t) { return 0; }

hipError_t sample_tokens(int dtype, int32_t n_rows, const Sampling& s, void*, hipStream_t stream)
{
    // While every row has a compute unit of its own, 1024 threads: 96 rows of 128,000 fp32, us with 1024 / 512 threads, 28.1 / 31.5, 256 rows 41.3 /
    // 40.4; 300 rows of 32,000 30.9 / 20.6.
    if (n_rows <= 256) launch<1024>(dtype, n_rows, s, stream);
    else launch<512>(dtype, n_rows, s, stream);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
