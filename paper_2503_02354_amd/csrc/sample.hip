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

__device__ __forceinline__ float number(float x) { return fmaxf(x, -INFINITY); }        // NaN becomes -inf
__device__ __forceinline__ float logit(const float* row, int i) { return number(row[i]); }
__device__ __forceinline__ float logit(const uint16_t* row, int i) { return number(__uint_as_float((uint32_t)row[i] << 16)); }

// 16 bytes of logits
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kWidth = 4;
    static __device__ __forceinline__ float at(const uint4& w, int e) { return number(__uint_as_float(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w)); }
};
template <> struct Vec<uint16_t> {
    static constexpr int kWidth = 8;
    static __device__ __forceinline__ float at(const uint4& w, int e)
    {
        const uint32_t d = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
        return number(__uint_as_float(e & 1 ? d & 0xFFFF0000u : d << 16));
    }
};

struct Best { float score; uint32_t index; };
constexpr uint32_t kNone = 0xFFFFFFFFu;
__device__ __forceinline__ Best better(Best a, Best b) { return b.score > a.score || (b.score == a.score && b.index < a.index) ? b : a; }

// A row and the workgroup's shared memory; every method is called by all threads.
constexpr int kMostCandidates = 2048, kMostTopK = 512, kSorted = 1024;
template <int THREADS> struct Shared {
    static constexpr int kWaves = THREADS / 64;
    Best best[kWaves];
    float sums[kWaves];
    float sum_pair[kWaves];
    uint32_t hist[256];
    uint32_t pick[2];
    uint32_t n_candidates;
    unsigned long long candidate[kMostCandidates];
    float weight[kSorted];
    uint32_t index[kSorted];
};

template <int THREADS> __device__ __forceinline__ Best block_best(Best v, Shared<THREADS>& sh)
{
    for (int d = 32; d > 0; d >>= 1) v = better(v, Best{__shfl_xor(v.score, d, 64), (uint32_t)__shfl_xor((int)v.index, d, 64)});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh.best[0];
    for (int w = 1; w < Shared<THREADS>::kWaves; ++w) v = better(v, sh.best[w]);
    return v;
}
template <int THREADS> __device__ __forceinline__ float block_sum(float v, Shared<THREADS>& sh)
{
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.sums[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < Shared<THREADS>::kWaves; ++w) v += sh.sums[w];
    return v;
}

// The row in pieces of up to 16 bytes, this thread's share: f(x[], n, first index), n = W for whole vectors and 1 at the row's ends,
// whose alignment may be any.
template <int THREADS, typename T, class F> __device__ __forceinline__ void pieces(const T* row, int vocab, F f)
{
    constexpr int W = Vec<T>::kWidth, kAhead = 16 / W;
    const int tid = threadIdx.x;
    const int lead = min(vocab, (int)((-(uintptr_t)row & 15) / sizeof(T))), vecs = (vocab - lead) / W, tail = lead + vecs * W;
    const uint4* const body = (const uint4*)(row + lead);
    float x[W];
    if (tid < lead) {
        x[0] = logit(row, tid);
        f(x, std::integral_constant<int, 1>(), (uint32_t)tid);
    }
    int v = tid;
    for (; v + (kAhead - 1) * THREADS < vecs; v += kAhead * THREADS) {
        uint4 w[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) w[j] = body[v + j * THREADS];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
#pragma unroll
            for (int e = 0; e < W; ++e) x[e] = Vec<T>::at(w[j], e);
            f(x, std::integral_constant<int, W>(), (uint32_t)(lead + (v + j * THREADS) * W));
        }
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
// f(x, index) for every logit
template <int THREADS, typename T, class F> __device__ __forceinline__ void each(const T* row, int vocab, F f)
{
    pieces<THREADS>(row, vocab, [&](const float (&x)[Vec<T>::kWidth], auto n, uint32_t i) {
#pragma unroll
        for (int e = 0; e < n; ++e) f(x[e], i + e);
    });
}

// The beginning of the order: tokens with a logit above x, and those of logit x with an index below `end`.
struct Front {
    float x;
    uint32_t end;
    __device__ __forceinline__ bool holds(float v, uint32_t i) const { return v > x || (v == x && i < end); }
};

// What a row's weights are relative to, and in which unit.
struct Scale {
    float top, per2;                          // largest logit; 1 / T in units of ln 2
    // log2 of the weight: 0 for the largest itself, whatever it is
    __device__ __forceinline__ float rel2(float x) const
    {
        const float d = x - top;
        return x == top ? 0.f : d == -INFINITY ? d : d * per2;
    }
    __device__ __forceinline__ float weight(float x) const { return __builtin_exp2f(rel2(x)); }
};

// The race among the tokens of a front, decided by what the filters say.  The race (largest (x - max) / T - ln E) needs no sorted row:
// its winner among a set of tokens that holds all kept ones is the drawn token if it is kept itself, and whether it is takes one
// sum over the tokens before it.  If it is not, no token from its place on is kept either, and the race is run again among those
// before it.
template <int THREADS, typename T>
__device__ uint32_t race(const T* row, const float* noise, int vocab, uint32_t top_index, Front last, float top_p, float mass, float min_p, Scale scale,
                         Shared<THREADS>& sh)
{
    const float least = min_p > 0.f ? log2f(min_p) : -INFINITY;
    for (;;) {                                // the front shrinks with every round that goes on
        Best win{-INFINITY, kNone};
        pieces<THREADS>(row, vocab, [&](const float (&x)[Vec<T>::kWidth], auto n, uint32_t i) {
            bool any = false;
#pragma unroll
            for (int e = 0; e < n; ++e) any |= x[e] >= last.x;
            if (!any) return;
            float q[Vec<T>::kWidth];
#pragma unroll
            for (int e = 0; e < n; ++e) q[e] = noise[i + e];
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float z = scale.rel2(x[e]), score = z - log2f(q[e]);
                const bool in = last.holds(x[e], i + e) && x[e] > -INFINITY && (z >= least || i + e == top_index) && score > -INFINITY;
                if (in) win = better(win, Best{score, i + e});
            }
        });
        win = block_best(win, sh);
        if (win.index == kNone) return top_index;
        if (!(top_p < 1.f) || win.index == top_index) return win.index;
        const Front ahead{logit(row, win.index), win.index};
        float before = 0.f;
        each<THREADS>(row, vocab, [&](float x, uint32_t i) { before += ahead.holds(x, i) ? scale.weight(x) : 0.f; });
        before = block_sum(before, sh);
        if (before < top_p * mass) return win.index;
        last = ahead;
    }
}

// The front of the first top_k tokens, byte by byte from the top of the order as one number, key first, then index.
template <int THREADS, typename T> __device__ Front front_of(const T* row, int vocab, uint32_t left, Shared<THREADS>& sh)
{
    const int tid = threadIdx.x;
    unsigned long long last = 0;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int b = tid; b < 256; b += THREADS) sh.hist[b] = 0;
        __syncthreads();
        each<THREADS>(row, vocab, [&](float x, uint32_t i) {
            const unsigned long long o = order_of(x, i);
            if (shift == 56 || (o >> (shift + 8)) == (last >> (shift + 8))) atomicAdd(&sh.hist[(o >> shift) & 255], 1u);
        });
        __syncthreads();
        if (tid == 0) {
            int b = 255;
            uint32_t above = 0;
            while (above + sh.hist[b] < left) above += sh.hist[b--];
            sh.pick[0] = (uint32_t)b;
            sh.pick[1] = left - above;
        }
        __syncthreads();
        last |= (unsigned long long)sh.pick[0] << shift;
        left = sh.pick[1];
        __syncthreads();
    }
    return {logit_of((uint32_t)(last >> 32)), ~(uint32_t)last + 1};
}

// Top_k up to 512 from a short list.  With at least top_k of the threads' largest logits at or above a bound, so are the first top_k
// tokens: one pass collects what reaches the bound (little more than top_k tokens of 1024 threads), which then is ranked by
// comparing all pairs, and the filters are decided on it.  Returns kNone where the list does not hold (more than 2048 tokens reach
// the bound, because many are equal).
template <int THREADS, typename T>
__device__ uint32_t from_list(const T* row, const float* noise, int vocab, float own_max, uint32_t top_k, float top_p, float min_p, Scale scale, Shared<THREADS>& sh)
{
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    // the bound: two bytes of the top_k-th largest of the threads' maxima
    const uint32_t own_key = key_of(own_max);
    uint32_t bound = 0, left = top_k;
    for (int shift = 24; shift >= 16; shift -= 8) {
        for (int b = tid; b < 256; b += THREADS) sh.hist[b] = 0;
        __syncthreads();
        if (shift == 24 || own_key >> 24 == bound >> 24) atomicAdd(&sh.hist[(own_key >> shift) & 255], 1u);
        __syncthreads();
        if (wid == 0) {                       // lane l holds bins 255 - 4 l .. 252 - 4 l
            uint32_t h[4], sum = 0;
            for (int j = 0; j < 4; ++j) sum += h[j] = sh.hist[255 - 4 * lane - j];
            uint32_t before = sum;
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t u = __shfl_up(before, d, 64);
                if (lane >= d) before += u;
            }
            before -= sum;
            for (int j = 0; j < 4; ++j) {
                if (before < left && before + h[j] >= left) {
                    sh.pick[0] = (uint32_t)(255 - 4 * lane - j);
                    sh.pick[1] = left - before;
                }
                before += h[j];
            }
        }
        __syncthreads();
        bound |= sh.pick[0] << shift;
        left = sh.pick[1];
    }
    if (tid == 0) sh.n_candidates = 0;
    __syncthreads();
    const float least = logit_of(bound);      // -inf where the bound's bits are no number's: everything
    each<THREADS>(row, vocab, [&](float x, uint32_t i) {
        if ((x >= least || !(least == least)) && x > -INFINITY) {
            const uint32_t at = atomicAdd(&sh.n_candidates, 1u);
            if (at < kMostCandidates) sh.candidate[at] = order_of(x, i);
        }
    });
    __syncthreads();
    const uint32_t n = sh.n_candidates;
    if (n > kMostCandidates) return kNone;
    // rank of every candidate; the list's own order, which atomics made, has no say in anything below
    for (uint32_t c = tid; c < n; c += THREADS) {
        const unsigned long long o = sh.candidate[c];
        uint32_t rank = 0;
        for (uint32_t j = 0; j < n; ++j) rank += sh.candidate[j] > o;
        if (rank < top_k) {
            sh.weight[rank] = scale.rel2(logit_of((uint32_t)(o >> 32)));
            sh.index[rank] = ~(uint32_t)o;
        }
    }
    __syncthreads();
    const uint32_t kept = min(n, top_k);
    float before = 0.f, mass = 0.f, z[(kMostTopK + THREADS - 1) / THREADS], w[(kMostTopK + THREADS - 1) / THREADS];
    Best win{-INFINITY, kNone};
    // one token per thread and round; sums in the order of the ranks
    constexpr int kRounds = (kMostTopK + THREADS - 1) / THREADS;
    float at[kRounds];
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
        const uint32_t rank = round * THREADS + tid;
        z[round] = rank < kept ? sh.weight[rank] : -INFINITY;
        w[round] = __builtin_exp2f(z[round]);
        float sum = w[round];
        for (int d = 1; d < 64; d <<= 1) {
            const float u = __shfl_up(sum, d, 64);
            if (lane >= d) sum += u;
        }
        float* const part = round & 1 ? sh.sum_pair : sh.sums;
        if (lane == 63) part[wid] = sum;
        __syncthreads();
        before = mass;
        for (int v = 0; v < Shared<THREADS>::kWaves; ++v) {
            if (v < wid) before += part[v];
            mass += part[v];
        }
        const float shifted = __shfl_up(sum, 1, 64);      // the sum before this lane, without taking its own off again
        at[round] = before + (lane == 0 ? 0.f : shifted);
        __syncthreads();
    }
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
        const uint32_t rank = round * THREADS + tid;
        if (rank < kept && (rank == 0 || ((!(top_p < 1.f) || at[round] < top_p * mass) && (!(min_p > 0.f) || w[round] >= min_p)))) {
            const uint32_t i = sh.index[rank];
            const float score = z[round] - log2f(noise[i]);
            if (score > -INFINITY) win = better(win, Best{score, i});
        }
    }
    win = block_best(win, sh);
    return win.index == kNone ? sh.index[0] : win.index;
}

// A workgroup per row.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, 8) void sample_kernel(Sampling s)
{
    __shared__ Shared<THREADS> sh;
    const int tid = threadIdx.x, vocab = s.vocab;
    const size_t r = blockIdx.x;
    const T* const row = (const T*)s.logits + r * s.logits_stride;
    const float* const noise = s.noise ? s.noise + r * s.noise_stride : nullptr;
    const float temperature = s.temperature ? s.temperature[r] : 1.f;
    const bool greedy = !(temperature > 0.f) || !noise;
    const float div = temperature > 0.f ? temperature : 1.f;
    const int32_t top_k = s.top_k ? s.top_k[r] : 0;
    const float top_p = s.top_p ? s.top_p[r] : 1.f, min_p = s.min_p ? s.min_p[r] : 0.f;

    // One pass: the largest logit and where it is, and the sum of the weights relative to it, which is scaled down whenever a thread
    // meets a larger one.
    constexpr float kLowest = -3.402823466e38f;
    const float unit = 1.44269504088896340736f / div;
    float most = kLowest, sum = 0.f;
    Best top{-INFINITY, kNone};
    pieces<THREADS>(row, vocab, [&](const float (&x)[Vec<T>::kWidth], auto n, uint32_t i) {
        float high = x[0];
#pragma unroll
        for (int e = 1; e < n; ++e) high = fmaxf(high, x[e]);
        if (high > top.score) {
            uint32_t at = 0;
#pragma unroll
            for (int e = n - 1; e >= 0; --e) at = x[e] == high ? e : at;
            top = Best{high, i + at};
            sum *= __builtin_exp2f((most - high) * unit);
            most = fmaxf(high, kLowest);
        }
#pragma unroll
        for (int e = 0; e < n; ++e) sum += __builtin_exp2f((x[e] - most) * unit);
    });
    const float own_max = top.score;
    top = block_best(top, sh);
    if (top.index == kNone) {
        if (tid == 0) {
            s.token[r] = -1;
            if (s.logprob) s.logprob[r] = -INFINITY;
        }
        return;
    }
    const Scale scale{top.score, unit};
    float all;
    if (top.score < INFINITY && unit > 0.f && unit < INFINITY) all = block_sum(own_max == -INFINITY ? 0.f : sum * scale.weight(most), sh);
    else {                                    // infinite logits or temperatures: the weights are 0 and 1
        all = 0.f;
        each<THREADS>(row, vocab, [&](float x, uint32_t) { all += x > -INFINITY ? scale.weight(x) : 0.f; });
        all = block_sum(all, sh);
    }

    uint32_t token = top.index;
    if (!greedy) {
        const bool cut = top_k > 0 && top_k < vocab;
        token = kNone;
        if (cut && top_k <= min(kMostTopK, THREADS / 2)) token = from_list(row, noise, vocab, own_max, (uint32_t)top_k, top_p, min_p, scale, sh);
        if (token == kNone) {
            Front last{-INFINITY, kNone};
            float mass = all;
            if (cut) {
                last = front_of(row, vocab, (uint32_t)top_k, sh);
                mass = 0.f;
                each<THREADS>(row, vocab, [&](float x, uint32_t i) { mass += last.holds(x, i) && x > -INFINITY ? scale.weight(x) : 0.f; });
                mass = block_sum(mass, sh);
            }
            if (top_p < 1.f) {
                // Tokens lighter than (1 - top_p) mass / vocab weigh less than what the nucleus leaves out, all together: none of them is in
                // it.  A quarter of that, so that no rounding matters.
                const float least = top.score + log2f(0.25f * (1.f - fmaxf(top_p, 0.f)) * mass / (float)vocab) / unit;
                if (least > last.x) last = Front{least, kNone};
            }
            token = race(row, noise, vocab, top.index, last, top_p, mass, min_p, scale, sh);
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
    if (n_rows <= 256) launch<1024>(dtype, n_rows, s, stream);
    else launch<512>(dtype, n_rows, s, stream);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
