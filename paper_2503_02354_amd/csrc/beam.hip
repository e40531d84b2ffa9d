// gfx950 kernels for the selection of a beam search: the best continuations of a request's beams.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float logit_at(const float* x, int64_t i) { return x[i]; }
__device__ __forceinline__ float logit_at(const uint16_t* x, int64_t i) { return __uint_as_float((uint32_t)x[i] << 16); }
__device__ __forceinline__ float known(float x) { return x == x ? x : -INFINITY; }     // NaN weighs nothing

struct Candidate {
    double score;
    int row, token;                           // row < 0: none
    float x;
};
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b)         // a is taken before b
{
    if (b.row < 0 || a.row < 0) return a.row >= 0;
    if (a.score != b.score && a.row != b.row) return a.score > b.score;
    if (a.row != b.row) return a.row < b.row;
    return a.x != b.x ? a.x > b.x : a.token < b.token;
}

// A workgroup per request: the rows' maxima and sums, then the best candidate behind the last one, picks times.
template <typename T>
__global__ __launch_bounds__(kThreads) void beam_plain_kernel(BeamSelection s)
{
    __shared__ double part[kThreads];
    __shared__ float top[kThreads];
    __shared__ Candidate best[kThreads];
    __shared__ float row_max[kBeamMax];
    __shared__ double row_log[kBeamMax];
    const int tid = threadIdx.x, r = blockIdx.x;
    for (int b = 0; b < s.beams; ++b) {
        const int64_t row = (int64_t)r * s.beams + b;
        const float so_far = s.score[row];
        if (!(so_far > -INFINITY) || (s.ended && s.ended[row])) continue;
        const T* const x = (const T*)s.logits + row * s.logits_stride;
        float m = -INFINITY;
        for (int i = tid; i < s.vocab; i += kThreads) m = fmaxf(m, known(logit_at(x, i)));
        top[tid] = m;
        __syncthreads();
        for (int d = kThreads / 2; d > 0; d >>= 1) {
            if (tid < d) top[tid] = fmaxf(top[tid], top[tid + d]);
            __syncthreads();
        }
        m = top[0];
        double sum = 0;
        for (int i = tid; i < s.vocab; i += kThreads) {
            const float v = known(logit_at(x, i));
            if (v > -INFINITY) sum += v == m ? 1. : exp((double)v - m);
        }
        part[tid] = sum;
        __syncthreads();
        for (int d = kThreads / 2; d > 0; d >>= 1) {
            if (tid < d) part[tid] += part[tid + d];
            __syncthreads();
        }
        if (tid == 0) {
            row_max[b] = m;
            row_log[b] = log(part[0]);
        }
        __syncthreads();
    }
    Candidate last{INFINITY, -1, -1, 0.f};
    bool any = true;
    for (int p = 0; p < s.picks; ++p) {
        Candidate mine{0, -1, -1, 0.f};
        for (int b = 0; b < s.beams && any; ++b) {
            const int64_t row = (int64_t)r * s.beams + b;
            const float so_far = s.score[row];
            if (!(so_far > -INFINITY)) continue;
            auto offer = [&](double score, int token, float v) {
                const Candidate c{score, (int)row, token, v};
                if ((last.row < 0 || before(last, c)) && before(c, mine)) mine = c;
            };
            if (s.ended && s.ended[row]) {
                if (tid == 0) offer(so_far, s.end_token, 0.f);
                continue;
            }
            const T* const x = (const T*)s.logits + row * s.logits_stride;
            for (int i = tid; i < s.vocab; i += kThreads) {
                const float v = known(logit_at(x, i));
                if (v > -INFINITY && (v == row_max[b] || row_max[b] < INFINITY)) offer(so_far + ((v == row_max[b] ? 0. : (double)v - row_max[b]) - row_log[b]), i, v);
            }
        }
        best[tid] = mine;
        __syncthreads();
        for (int d = kThreads / 2; d > 0; d >>= 1) {
            if (tid < d && before(best[tid + d], best[tid])) best[tid] = best[tid + d];
            __syncthreads();
        }
        last = best[0];
        any = last.row >= 0;
        __syncthreads();
        if (tid == 0) {
            const int64_t at = (int64_t)r * s.picks + p;
            s.next_score[at] = any ? (float)last.score : -INFINITY;
            s.next_row[at] = any ? last.row : -1;
            s.next_token[at] = any ? last.token : -1;
            if (s.next_ended) s.next_ended[at] = any && ((s.ended && s.ended[last.row]) || last.token == s.end_token);
        }
    }
}

}  // namespace

int64_t beam_workspace(int32_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t beam_select(int dtype, const BeamSelection& s, void*, hipStream_t stream)
{
    if (dtype == 0) hipLaunchKernelGGL(beam_plain_kernel<float>, dim3((unsigned)s.n_requests), dim3(kThreads), 0, stream, s);
    else hipLaunchKernelGGL(beam_plain_kernel<uint16_t>, dim3((unsigned)s.n_requests), dim3(kThreads), 0, stream, s);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
