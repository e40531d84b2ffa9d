// gfx950 kernels for attention of a decoder's tokens over an encoder's states (bf16).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

constexpr float kLn2 = 0.69314718055994530942f;

// A source's queries and rows, within the arrays.
struct Source {
    int q0, m, first, rows;
};
__device__ __forceinline__ Source source_of(const States& st, const CrossAttention& a, int s)
{
    Source o;
    const int q1 = max(0, min(a.q_off[(s + 1) * a.beams], a.n_tokens));
    o.q0 = max(0, min(a.q_off[s * a.beams], a.n_tokens));
    o.m = min(max(q1 - o.q0, 0), a.max_new);
    o.first = a.first[s];
    o.rows = o.first < 0 ? 0 : max(0, min(min(a.length[s], a.max_rows), st.n_rows - min(o.first, st.n_rows)));
    return o;
}

// A wavefront per query and head; 64 rows at a time: a lane's score, then two channels of the output to a lane.
__global__ __launch_bounds__(64) void cross_attention_plain_kernel(States st, CrossAttention a)
{
    __shared__ float query[128], weight[64];
    const int lane = threadIdx.x, s = blockIdx.y, head = blockIdx.z, kvh = head / (a.heads / st.kv_heads), dim = st.head_dim;
    const Source o = source_of(st, a, s);
    for (int i = blockIdx.x; i < o.m; i += gridDim.x) {
        const int64_t token = o.q0 + i;
        __syncthreads();
        for (int ch = lane; ch < dim; ch += 64) query[ch] = __uint_as_float((uint32_t)a.q[token * a.q_token_stride + head * a.q_head_stride + ch] << 16);
        __syncthreads();
        float mx = -INFINITY, sum = 0.f, acc[2] = {0.f, 0.f};
        for (int j0 = 0; j0 < o.rows; j0 += 64) {
            const int j = j0 + lane;
            const int64_t row = o.first + (int64_t)j;
            const bool there = j < o.rows && (!st.seen || st.seen[row] != 0);
            float score = -INFINITY;
            if (there) {
                const uint16_t* const kp = st.k + row * st.k_row_stride + kvh * st.k_head_stride;
                score = 0.f;
                for (int ch = 0; ch < dim; ++ch) score += query[ch] * __uint_as_float((uint32_t)kp[ch] << 16);
                score *= a.scale;
            }
            float top = score;
            for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
            const float m_new = fmaxf(mx, top), shrink = m_new == mx ? 1.f : expf(mx - m_new), m_use = m_new == -INFINITY ? 0.f : m_new;
            float w = there ? expf(score - m_use) : 0.f;
            weight[lane] = w;
            for (int d = 32; d > 0; d >>= 1) w += __shfl_xor(w, d, 64);
            sum = sum * shrink + w;
            mx = m_new;
            const unsigned long long seen = __ballot(there);
            __syncthreads();
            for (int e = 0; e < 2; ++e) {
                const int ch = lane + 64 * e;
                acc[e] *= shrink;
                if (ch < dim)
                    for (unsigned long long b = seen; b; b &= b - 1) {
                        const int jj = __builtin_ctzll(b);
                        acc[e] += weight[jj] * __uint_as_float((uint32_t)st.v[(o.first + (int64_t)j0 + jj) * st.v_row_stride + kvh * st.v_head_stride + ch] << 16);
                    }
            }
            __syncthreads();
        }
        const bool empty = mx == -INFINITY && sum == 0.f;
        for (int e = 0; e < 2; ++e) {
            const int ch = lane + 64 * e;
            const __bf16 b = (__bf16)(empty ? 0.f : acc[e] / sum);
            if (ch < dim) a.out[token * a.out_token_stride + head * a.out_head_stride + ch] = __builtin_bit_cast(uint16_t, b);
        }
        if (a.lse && lane == 0) a.lse[token * a.heads + head] = empty ? -INFINITY : mx + log2f(sum) * kLn2;
    }
}

}  // namespace

int64_t cross_attention_workspace(int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t cross_attention(const States& st, const CrossAttention& a, void*, hipStream_t stream)
{
    hipLaunchKernelGGL(cross_attention_plain_kernel, dim3((unsigned)std::min(a.max_new, 4096), (unsigned)a.n_sources, (unsigned)a.heads), dim3(64), 0, stream, st, a);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
