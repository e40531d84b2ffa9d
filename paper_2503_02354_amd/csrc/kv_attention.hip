// gfx950 kernels for attention over the paged key/value cache of token-generating experts (bf16).
#include <hip/hip_runtime.h>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint16_t to_bf16(float v)
{
    f32x2 f = {v, 0.f};
    return (uint16_t)__builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));   // round to nearest even
}

// One wavefront per query row: 64 keys at a time, a lane scores one of them; then a lane sums two channels over the 64 values.
__global__ __launch_bounds__(64) void kv_attention_rows_kernel(KvCache c, KvAttention a)
{
    __shared__ float q[128], p[64];
    __shared__ int32_t blocks[64];
    const int t = blockIdx.x / a.heads, head = blockIdx.x - t * a.heads, lane = threadIdx.x;
    int lo = 0, hi = a.n_requests;
    if (a.q_off[0] > t || a.q_off[hi] <= t) return;       // a row of no request
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_off[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int r = lo, bs = 1 << c.block_shift, dim = c.head_dim;
    const int len = max(0, min(a.seq_len[r], a.max_blocks << c.block_shift));
    const int pos = len - (a.q_off[r + 1] - t);
    const int begin = a.window > 0 ? max(0, pos - a.window + 1) : 0, end = pos + 1;
    for (int d = lane; d < dim; d += 64) q[d] = __uint_as_float((uint32_t)a.q[t * a.q_token_stride + head * a.q_head_stride + d] << 16);
    __syncthreads();
    const int64_t head_at = (head / (a.heads / c.kv_heads)) * c.head_stride;
    float m = -INFINITY, sum = 0.f, o[2] = {0.f, 0.f};
    for (int j0 = begin; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        float s = -INFINITY;
        int32_t block = -1;
        if (j < end) {
            block = a.table[(size_t)r * a.max_blocks + (j >> c.block_shift)];
            if (block < 0 || block >= c.n_blocks) block = -1;
            s = 0.f;
            if (block >= 0) {
                const uint16_t* row = c.k + block * c.block_stride + (j & (bs - 1)) * c.token_stride + head_at;
                for (int d = 0; d < dim; d += 8) {
                    const uint4 w = *(const uint4*)(row + d);
                    s += q[d] * bf16_lo(w.x) + q[d + 1] * bf16_hi(w.x) + q[d + 2] * bf16_lo(w.y) + q[d + 3] * bf16_hi(w.y) +
                         q[d + 4] * bf16_lo(w.z) + q[d + 5] * bf16_hi(w.z) + q[d + 6] * bf16_lo(w.w) + q[d + 7] * bf16_hi(w.w);
                }
            }
            s *= a.scale;
        }
        blocks[lane] = block;
        float top = s;
        for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
        const float m_new = fmaxf(m, top), shrink = m == m_new ? 1.f : expf(m - m_new);
        const float e = j < end ? expf(s - m_new) : 0.f;
        float part = e;
        for (int d = 32; d > 0; d >>= 1) part += __shfl_xor(part, d, 64);
        sum = sum * shrink + part;
        m = m_new;
        p[lane] = __uint_as_float((uint32_t)to_bf16(e) << 16);
        __syncthreads();
        o[0] *= shrink;
        o[1] *= shrink;
        const int n = min(64, end - j0);
        for (int i = 0; i < n; ++i) {
            if (blocks[i] < 0) continue;
            const uint16_t* row = c.v + blocks[i] * c.block_stride + ((j0 + i) & (bs - 1)) * c.token_stride + head_at;
            for (int d = lane, x = 0; d < dim; d += 64, ++x) o[x] += p[i] * __uint_as_float((uint32_t)row[d] << 16);
        }
        __syncthreads();
    }
    const float inv = end > begin ? 1.f / sum : 0.f;
    for (int d = lane, x = 0; d < dim; d += 64, ++x)
        a.out[t * a.out_token_stride + head * a.out_head_stride + d] = end > begin ? to_bf16(o[x] * inv) : 0;
    if (a.lse && lane == 0) a.lse[(int64_t)t * a.heads + head] = end > begin ? m + logf(sum) : -INFINITY;
}

}  // namespace

int64_t kv_attention_workspace(int32_t, int32_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t kv_attention(const KvCache& c, const KvAttention& a, void*, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_attention_rows_kernel, dim3((unsigned)(a.n_tokens * a.heads)), dim3(64), 0, stream, c, a);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
