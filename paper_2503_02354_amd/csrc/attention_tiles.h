// What the attention kernels of token-generating experts share: operand types, lane exchanges, the layout of value tiles in LDS and the
// arithmetic of softmax parts.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace coe {
namespace k {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));   // round to nearest even
}
// the larger (the sum) of a value and that of lane ^ 32
[[maybe_unused]] __device__ __forceinline__ float max_halves(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
#endif
    return v;
}
[[maybe_unused]] __device__ __forceinline__ float sum_halves(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(h[0]) + __uint_as_float(h[1]);
#endif
    return v;
}
[[maybe_unused]] __device__ __forceinline__ float exp2_fast(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(v);
#else
    return v;
#endif
}

// Nothing above -inf among a row's scores.  A maximum passes NaN by, a sum does not: where the scores are NaN and none is above -inf, the
// maximum is -inf too, but the sum is NaN.
__device__ __forceinline__ bool is_empty(float mx, float sum) { return mx == -INFINITY && sum == 0.f; }

// What a part relative to 2^from weighs relative to 2^to, the larger: 1 where both are -inf (or inf), so that a NaN in a part stays.
[[maybe_unused]] __device__ __forceinline__ float weight_of_part(float from, float to) { return from == to ? 1.f : exp2f(from - to); }

// Room for values of 2^110: the weights that meet in a sum of fp32 add up to 2^17, so that they and the values stay below 2^128.  A part's
// own do: the few-rows kernels' are 1 at most (and their stretches hold 2^17 keys of a history or source at most, unless a step has 2^26 cached tokens x cache
// heads, or rows x heads of states), the many-rows kernels move their reference.  Joining adds up kMostParts parts at most: their outputs are
// taken times 1 / kMostParts, so that all of them together are no more than one, and the result back.
[[maybe_unused]] constexpr int kMostParts = 1024;
[[maybe_unused]] constexpr float kJoinRoom = 1.f / kMostParts;

// Where 16-byte chunk c of row r of a V tile lies: chunks in an order that spreads both the writes (sixteen rows of
// one chunk) and the transposing reads (four rows of four chunks) over all LDS banks.
template <int D> constexpr int kRow = D <= 64 ? 64 : 128;     // channels that a row of D channels takes in LDS
template <int D> __device__ __forceinline__ uint32_t v_slot(int r, int c)
{
    constexpr int DH = kRow<D>;
    const int f = DH == 128 ? (r & 3) * 4 + ((r >> 2) & 3) : ((r >> 1) & 1) * 4 + ((r >> 2) & 3);
    return (uint32_t)(r * DH * 2 + ((c ^ f) & (DH / 8 - 1)) * 16);
}

#if defined(__HIP_DEVICE_COMPILE__)
// The addresses of a V tile's reads differ from one lane's base by bits that the order of the chunks flips: 32 channels further, and eight
// rows further.  The tile begins at a multiple of 4 KiB.
template <int D> __device__ __forceinline__ uint32_t value_base(int lane)
{
    return v_slot<D>(4 * (lane >> 5) + ((lane >> 2) & 3), ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8;
}
// V^T of 16 keys for channels 32 db .. : `base` is the LDS address of the tile's 32 (or 16) rows + value_base
template <int D> __device__ __forceinline__ u32x4 values(uint32_t base, int db, int t2)
{
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((base ^ (db * 64)) + t2 * 32 * kRow<D>));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((base ^ (db * 64 + 32 + 16 * kRow<D>)) + t2 * 32 * kRow<D>));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// V^T of 16 keys, all channels
template <int D> __device__ __forceinline__ void read_values(u32x4 (&v)[D / 32], uint32_t base, int t2)
{
#pragma unroll
    for (int db = 0; db < D / 32; ++db) v[db] = values<D>(base, db, t2);
}
// acc += V^T P^T for 16 keys
template <int D> __device__ __forceinline__ void add_values(f32x16 (&acc)[D / 32], const u32x4 (&v)[D / 32], u32x4 p)
{
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[db]), __builtin_bit_cast(bf16x8, p), acc[db], 0, 0, 0);
}
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }
#endif

__host__ __device__ constexpr int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }
typedef __attribute__((address_space(3))) void lds_void;
[[maybe_unused]] constexpr uint32_t kOutOfRange = 0x80000000u;   // buffer offset beyond any block: loads return zeros

}  // namespace
}  // namespace k
}  // namespace coe
