// gfx950 kernel that draws a token from every row of logits.
#include <hip/hip_runtime.h>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// Order of a row: descending logits, equal ones by ascending index.  The logit as an unsigned key that grows with it (-0 and +0 the
// same; NaN counts as -inf), so that "comes before" is a comparison of integers.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <typename T> __device__ __forceinline__ float logit(const T* row, int i);
template <> __device__ __forceinline__ float logit<float>(const float* row, int i)
{
    const float x = row[i];
    return x == x ? x : -INFINITY;
}
template <> __device__ __forceinline__ float logit<uint16_t>(const uint16_t* row, int i)
{
    const float x = __uint_as_float((uint32_t)row[i] << 16);
    return x == x ? x : -INFINITY;
}

struct Best { float score; uint32_t index; };
__device__ __forceinline__ Best better(Best a, Best b) { return b.score > a.score || (b.score == a.score && b.index < a.index) ? b : a; }

__device__ __forceinline__ Best block_best(Best v, Best* part)
{
    for (int d = 32; d > 0; d >>= 1) v = better(v, Best{__shfl_xor(v.score, d, 64), (uint32_t)__shfl_xor((int)v.index, d, 64)});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kWaves; ++w) v = better(v, part[w]);
    return v;
}
__device__ __forceinline__ float block_sum(float v, float* part)
{
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < kWaves; ++w) v += part[w];
    return v;
}

// A workgroup per row.  The race (largest (x - max) / T - ln E) needs no sorted row: its winner among a set of tokens that holds all
// kept ones is the drawn token if it is kept itself, and whether it is takes one sum over the tokens before it.  If it is not, no
// token from its place on is kept either, and the race is run again among those before it.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(Sampling s)
{
    __shared__ Best best[kWaves];
    __shared__ float sums[kWaves];
    __shared__ uint32_t hist[256];
    __shared__ uint32_t pick[2];
    const int tid = threadIdx.x, vocab = s.vocab;
    const size_t r = blockIdx.x;
    const T* const row = (const T*)s.logits + r * s.logits_stride;
    const float* const noise = s.noise ? s.noise + r * s.noise_stride : nullptr;

    Best top{-INFINITY, 0xFFFFFFFFu};
    for (int i = tid; i < vocab; i += kThreads) {
        const float x = logit(row, i);
        if (x > -INFINITY) top = better(top, Best{x, (uint32_t)i});
    }
    top = block_best(top, best);
    if (top.index == 0xFFFFFFFFu) {
        if (tid == 0) {
            s.token[r] = -1;
            if (s.logprob) s.logprob[r] = -INFINITY;
        }
        return;
    }
    const float temperature = s.temperature ? s.temperature[r] : 1.f;
    const bool greedy = !(temperature > 0.f) || !noise;
    const float div = temperature > 0.f ? temperature : 1.f;
    // distance of a logit from the largest one, in units of the temperature: 0 for the largest itself, whatever it is
    auto rel = [&](float x) {
        const float d = x - top.score;
        return x == top.score ? 0.f : d == -INFINITY ? d : d / div;
    };
    float all = 0.f;
    for (int i = tid; i < vocab; i += kThreads) {
        const float x = logit(row, i);
        all += x > -INFINITY ? expf(rel(x)) : 0.f;
    }
    all = block_sum(all, sums);

    uint32_t token = top.index;
    if (!greedy) {
        const int32_t top_k = s.top_k ? s.top_k[r] : 0;
        const float top_p = s.top_p ? s.top_p[r] : 1.f, min_p = s.min_p ? s.min_p[r] : 0.f;
        // the last token of the first top_k: its key, and its index among equals, byte by byte from the top
        unsigned long long last = 0;          // order as one number: key, then the complement of the index; the smallest that is kept
        float mass = all;
        if (top_k > 0 && top_k < vocab) {
            uint32_t left = (uint32_t)top_k;
            for (int shift = 56; shift >= 0; shift -= 8) {
                if (tid < 256) hist[tid] = 0;
                __syncthreads();
                for (int i = tid; i < vocab; i += kThreads) {
                    const unsigned long long o = (unsigned long long)key_of(logit(row, i)) << 32 | (uint32_t)~i;
                    if (shift == 56 || (o >> (shift + 8)) == (last >> (shift + 8))) atomicAdd(&hist[(o >> shift) & 255], 1u);
                }
                __syncthreads();
                if (tid == 0) {
                    int b = 255;
                    uint32_t above = 0;
                    while (above + hist[b] < left) above += hist[b--];
                    pick[0] = (uint32_t)b;
                    pick[1] = left - above;
                }
                __syncthreads();
                last |= (unsigned long long)pick[0] << shift;
                left = pick[1];
                __syncthreads();
            }
            float part = 0.f;
            for (int i = tid; i < vocab; i += kThreads) {
                const float x = logit(row, i);
                const unsigned long long o = (unsigned long long)key_of(x) << 32 | (uint32_t)~i;
                part += o >= last && x > -INFINITY ? expf(rel(x)) : 0.f;
            }
            mass = block_sum(part, sums);
        }
        const unsigned long long first = (unsigned long long)key_of(top.score) << 32 | (uint32_t)~top.index;
        for (;;) {                            // `last` grows with every round that goes on
            Best win{-INFINITY, 0xFFFFFFFFu};
            for (int i = tid; i < vocab; i += kThreads) {
                const float x = logit(row, i);
                const unsigned long long o = (unsigned long long)key_of(x) << 32 | (uint32_t)~i;
                if (o < last || x == -INFINITY) continue;
                const float z = rel(x);
                if (o != first && !(min_p <= 0.f) && !(expf(z) >= min_p)) continue;
                const float score = z - logf(noise[i]);
                if (score > -INFINITY) win = better(win, Best{score, (uint32_t)i});
            }
            win = block_best(win, best);
            if (win.index == 0xFFFFFFFFu) break;
            token = win.index;
            if (!(top_p < 1.f)) break;
            const unsigned long long o_win = (unsigned long long)key_of(logit(row, win.index)) << 32 | (uint32_t)~win.index;
            if (o_win == first) break;
            float before = 0.f;
            for (int i = tid; i < vocab; i += kThreads) {
                const float x = logit(row, i);
                const unsigned long long o = (unsigned long long)key_of(x) << 32 | (uint32_t)~i;
                before += o > o_win && x > -INFINITY ? expf(rel(x)) : 0.f;
            }
            before = block_sum(before, sums);
            if (before < top_p * mass) break;
            last = o_win + 1;
            token = top.index;
        }
    }
    if (tid == 0) {
        s.token[r] = (int32_t)token;
        if (s.logprob) s.logprob[r] = rel(logit(row, token)) - logf(all);
    }
}

}  // namespace

int64_t sample_workspace(int32_t, int32_t) { return 0; }

hipError_t sample_tokens(int dtype, int32_t n_rows, const Sampling& s, void*, hipStream_t stream)
{
    if (dtype == 0) hipLaunchKernelGGL(sample_kernel<float>, dim3(n_rows), dim3(kThreads), 0, stream, s);
    else hipLaunchKernelGGL(sample_kernel<uint16_t>, dim3(n_rows), dim3(kThreads), 0, stream, s);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
