// gfx950 kernels for the selection of a beam search: the best continuations of a request's beams.
//
// A row's candidates come in the order of their logits, and what they are short of the score, ln sum exp x, is one number for all of them.  So
// one pass over a row finds both that sum and its best logits, and the rows of a request meet afterwards with a few candidates each:
//   score(row, v) = score[row] + (x_v - lse)      lse = (log2 S - c) / L      S = sum 2^(x L + c)      c = -m L, rounded      m = max x
// L is log2 e as fp32 has it, 1.3e-8 (relative) off, which puts that times the row's entropy on lse: below 2e-7, and the same to a tenth of that for rows as
// alike as a request's.  x L + c is rounded once, in the multiply-add.  Candidates of different rows may be as near to each other as their
// logits' last bits, so scores are fp64, and so are S (from fp32 sums of a lane's terms relative to the lane's largest, whose errors are
// independent) and its logarithm.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace coe {
namespace k {

namespace {

// 16 bytes of logits of any alignment: which lane sums which tokens goes by the index alone, so that equal rows have equal sums
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kWidth = 4;
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ float at(const type& w, int e) { return __uint_as_float(w[e]); }
};
template <> struct Vec<uint16_t> {
    static constexpr int kWidth = 8;
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ float one(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
    static __device__ __forceinline__ float at(const type& w, int e) { return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16); }
};

// A candidate of a row as an integer that grows in the row's order: the logit (-0 and +0 the same), then the complement of the index.  0: none.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

__device__ __forceinline__ float exp2_fast(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_exp2f(v);
#else
    return v;
#endif
}
constexpr float kLog2e = 1.44269504088896340736f;
// c = -m L; 0 where there is no m.  Beyond kHuge its rounding is no longer small beside 1, and sums are relative to e^m.
constexpr float kHuge = 0x1p16f;
__device__ __forceinline__ bool is_huge(float m) { return fabsf(m) > kHuge; }
__device__ __forceinline__ float offset_of(float m) { return m == -INFINITY ? 0.f : -(m * kLog2e); }
// what a sum relative to the maximum `from` weighs in one relative to `to`, the larger
__device__ __forceinline__ double weight_of(float from, float to)
{
    if (from == to) return 1.;
    if (from == -INFINITY) return 0.;
    const double c = offset_of(from), L = kLog2e;
    if (!is_huge(to) && !is_huge(from)) return exp2((double)offset_of(to) - c);
    // by way of e^m
    return exp2(((double)from - (double)to) * 1.44269504088896340736 - (is_huge(from) ? 0. : from * L + c) + (is_huge(to) ? 0. : to * L + (double)offset_of(to)));
}
// the largest of three; a signalling NaN among them makes it NaN (fmaxf would quiet every operand first, an instruction each)
__device__ __forceinline__ float max3(float a, float b, float c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
#else
    return a + b + c;
#endif
}
__device__ __forceinline__ int count_of(bool b) { return __popcll(__ballot(b)); }
// LDS that the lanes of a wavefront write for each other
__device__ __forceinline__ void wave_sync()
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#endif
}

// the largest of a wavefront's values, in every lane's hands; six register operations
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false));        // one lane up, two, four, eight in a row of 16
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false));        // a row's last lane to the next row, the second row's to the last two
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false));
    v = (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
#endif
    return v;
}
__device__ __forceinline__ uint32_t wave_min(uint32_t v) { return ~wave_max(~v); }

// ---- rows ---------------------------------------------------------------------------------------------------------
// A workgroup takes a part of a row, its wavefronts steps of 1024 logits in turn.  A lane keeps its largest logit and its sum of weights
// relative to it.  A wavefront keeps a list, in LDS, of all that it has seen above a threshold, which `picks` logits of the part are known to reach: a
// quarter of them in every wavefront (each says what its quarter reaches after its first step, its second, its fourth, ...; the lowest of the four holds), or
// all of them in its own list.  A list that grows all the same is cut back to at most kSlack more than picks.  Indices ascend from step to step, so an
// equal logit that comes later in the same wavefront is never wanted, but in another it may be.
// What bounds it is waiting for memory, half of a wavefront's time: 512 rows of 128,000 in bf16 (131 MB) 35.8 us, 3.7 TB/s; where a seventh of them has no pass (113 MB) 34.6,
// 3.3 TB/s, since their compute units have fewer wavefronts than others then.  Four rows of 50,001 fp32 7.0 us, of which a step's round trip, the threshold and the lists at
// the end are most.
// Finite masks cost a second pass: a lane that begins with nothing above -88.7 scales its sum, 0, by more than fp32 holds, and so does one whose maximum stays
// beyond kHuge; both say NaN, and the part is read again with SAFE.  The same call with nine logits in ten masked, at random, by -88 or -inf 40 us, by -90 to -3e38 76 to 77;
// four rows 12.0 and 16.3.  And a step of one value is a list of 1024 equal logits, to be cut: the last nine tenths of every row -50 143 us, -1e4 281, -inf 36.
constexpr int kWaves = 4, kThreads = 64 * kWaves, kPerLane = 16, kStep = 64 * kPerLane, kSlack = 32, kGrow = 64;
constexpr int kList = kBeamPicksMax + kGrow + kStep;
static_assert(kBeamPicksMax + kGrow <= 128 && kWaves * 128 <= kList, "two keys of a list to a lane, all lists in the place of one");
// The workspace: [rows][parts] of these, then a request's lists of keys across each other: all parts' best, all parts' second, ...; an odd number of keys from
// one to the next, so that no thread of those that share them out meets a list twice before all others have.
__host__ __device__ constexpr int pitch_of(int beams, int parts) { return beams * parts | 1; }
struct RowPart {
    double sum;
    float top;
    int32_t pad;
};
constexpr uint32_t kLeast = 0x00800000u;      // key of the lowest finite logit: -inf is no candidate
// the largest logit below those of key `low` (> kLeast - 1)
__device__ __forceinline__ float below(uint32_t low) { return logit_of(low - (low == 0x80000000u ? 2 : 1)); }

// A key that at least `picks` of a wavefront's keys (N to a lane) reach, and at most `enough` more unless they are equal.  That many reach lo, and
// none passes hi.
template <int N> __device__ __forceinline__ uint32_t reached(const uint32_t (&key)[N], int picks, int enough, uint32_t lo, uint32_t hi)
{
    auto count = [&](uint32_t t) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) c += count_of(key[i] >= t);
        return c;
    };
    int c = count(lo);
#pragma nounroll
    while (c > picks + enough && lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        const int now = count(mid);
        if (now >= picks) lo = mid, c = now;
        else hi = mid - 1;
    }
    return lo;
}

// Cuts a list of n keys to the largest, at least `picks` and at most kSlack more: those from a threshold on, which is a logit where that does it, else a
// key.  `low` is the least of its logits that may be there; returns the list's new length, and in `low` what the rest lies at or above.
__device__ int cut_list(unsigned long long* list, int n, int picks, uint32_t& low)
{
    const int lane = threadIdx.x & 63;
    wave_sync();
    auto count = [&](auto holds) {
        int c = 0;
#pragma nounroll
        for (int i = 0; i < n; i += 64) c += count_of(i + lane < n && holds(list[i + lane]));
        return c;
    };
    uint32_t lo = low, hi = 0;                // enough of them are at or above lo; above hi there are none
#pragma nounroll
    for (int i = lane; i < n; i += 64) hi = max(hi, (uint32_t)(list[i] >> 32));
    hi = wave_max(hi);
    int at_lo = n;
#pragma nounroll
    while (at_lo > picks + kSlack && lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        const int c = count([&](unsigned long long k) { return (uint32_t)(k >> 32) >= mid; });
        if (c >= picks) lo = mid, at_lo = c;
        else hi = mid - 1;
    }
    uint32_t index = 0;                       // of logits equal to lo, those from here on (complements of indices)
    if (at_lo > picks + kSlack) {
        const int above = count([&](unsigned long long k) { return (uint32_t)(k >> 32) > lo; });
        uint32_t top = 0xFFFFFFFFu;
#pragma nounroll
        while (at_lo > picks + kSlack && index < top) {
            const uint32_t mid = index + (top - index) / 2 + 1;
            const int c = above + count([&](unsigned long long k) { return (uint32_t)(k >> 32) == lo && (uint32_t)k >= mid; });
            if (c >= picks) index = mid, at_lo = c;
            else top = mid - 1;
        }
    }
    const unsigned long long from = (unsigned long long)lo << 32 | index;
    int kept = 0;
#pragma nounroll
    for (int i = 0; i < n; i += 64) {
        const unsigned long long k = i + lane < n ? list[i + lane] : 0;
        const bool keep = i + lane < n && k >= from;
        const unsigned long long b = __ballot(keep);
        wave_sync();
        if (keep) list[kept + __popcll(b & ((1ull << lane) - 1))] = k;
        wave_sync();
        kept += __popcll(b);
    }
    low = lo;
    return kept;
}

// One wavefront's share of a part of a row, its 16-byte pieces [begin, end); all of the workgroup's wavefronts call this together.  SAFE: NaN counts as
// -inf, and equal infinities weigh 1; without it they, and maxima beyond kHuge, make the sum NaN.  quarter: [kWaves] what every wavefront's quarter of the picks reaches, 0 for
// not yet.
template <typename T, bool SAFE, bool STREAM>
__device__ __forceinline__ void scan_row(const T* row, int vocab, int begin, int end, int wid, int picks, unsigned long long* list, volatile uint32_t* quarter, int& n, float& top, double& sum)
{
    typedef typename Vec<T>::type Piece;
    constexpr int W = Vec<T>::kWidth, kPieces = kPerLane / W, kStride = kWaves * kPieces * 64;
    const int lane = threadIdx.x & 63, whole = min(end, vocab / W);       // pieces without the row's end in them
    const int share = (picks + kWaves - 1) / kWaves;
    float m = -INFINITY, s = 0.f;
    constexpr int kDepth = kPieces <= 2 ? 2 : 1;          // steps ahead: 64 bytes of a lane
    Piece next[kDepth][kPieces];
    auto fetch = [&](Piece (&to)[kPieces], long long at) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const long long piece = at + j * 64 + lane;
            if (piece < whole) {
                if constexpr (STREAM) to[j] = __builtin_nontemporal_load((const Piece*)(row + piece * W));
                else to[j] = *(const Piece*)(row + piece * W);
            }
        }
    };
    auto unpack = [&](float (&x)[kPerLane], const Piece (&from)[kPieces], long long at) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int e = 0; e < W; ++e) x[j * W + e] = Vec<T>::at(from[j], e);
        if (at + kPieces * 64 > whole)        // the part's last step, in one wavefront or none
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const long long piece = at + j * 64 + lane;
                if (piece < whole) continue;
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const long long i = piece * W + e;
                    x[j * W + e] = piece < end && i < vocab ? Vec<T>::one(row + i) : -INFINITY;
                }
            }
        if (SAFE)
#pragma unroll
            for (int e = 0; e < kPerLane; ++e) x[e] = x[e] == x[e] ? x[e] : -INFINITY;
    };
    auto most_of = [&](const float (&x)[kPerLane], float (&four)[kPerLane / 4]) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < kPerLane / 4; ++g) four[g] = max3(max3(x[4 * g], x[4 * g + 1], x[4 * g + 2]), x[4 * g + 3], x[4 * g + 3]);
        return max3(max3(four[0], four[1], four[2]), four[3], four[3]);
    };
    auto weigh = [&](const float (&x)[kPerLane], float most) __attribute__((always_inline)) {
        const float m_new = max3(m, most, m), c = offset_of(m_new);
        float part[4] = {0.f, 0.f, 0.f, 0.f};
        if (SAFE) {
            s = m == m_new ? s : s * exp2_fast((m - m_new) * kLog2e);
#pragma unroll
            for (int e = 0; e < kPerLane; ++e) part[e & 3] += x[e] == -INFINITY ? 0.f : x[e] == m_new ? 1.f : exp2_fast((x[e] - m_new) * kLog2e);
        } else {
            s = m == m_new ? s : s * exp2_fast(c - offset_of(m));
#pragma unroll
            for (int e = 0; e < kPerLane; ++e) part[e & 3] += exp2_fast(__builtin_fmaf(x[e], kLog2e, c));
        }
        s += (part[0] + part[1]) + (part[2] + part[3]);
        m = m_new;
    };
    n = 0;
    uint32_t low = kLeast;                    // what the list's logits lie at or above
    float threshold = -INFINITY;              // what is wanted lies above
    auto put = [&](const float (&x)[kPerLane], const float (&four)[kPerLane / 4], long long at) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < kPerLane / 4; ++g)
            if (__any(four[g] > threshold))
#pragma unroll
                for (int e = 4 * g; e < 4 * g + 4; ++e) {
                    const bool take = x[e] > threshold;
                    const unsigned long long b = __ballot(take);
                    if (b) {
                        const uint32_t i = (uint32_t)((at + e / W * 64 + lane) * W + e % W);
                        if (take) list[n + __popcll(b & ((1ull << lane) - 1))] = (unsigned long long)key_of(x[e]) << 32 | (uint32_t)~i;
                        n += __popcll(b);
                    }
                }
        if (n > picks + kGrow) {
            n = cut_list(list, n, picks, low);
            threshold = fmaxf(threshold, logit_of(low));
        }
    };
    // what a quarter of the picks reaches in this wavefront's list
    auto tell = [&]() __attribute__((always_inline)) {
        wave_sync();
        uint32_t key[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) key[i] = i * 64 + lane < n ? (uint32_t)(list[i * 64 + lane] >> 32) : 0u;
        const uint32_t least = wave_min(min(key[0] - 1, key[1] - 1)) + 1;     // of those that are there
        const uint32_t mine = reached(key, share, share / 2, least, wave_max(max(key[0], key[1])));
        if (lane == 0 && mine > quarter[wid]) quarter[wid] = mine;
    };
    auto all_reach = [&]() { return min(min(quarter[0], quarter[1]), min(quarter[2], quarter[3])); };

    long long at = begin + (long long)wid * kPieces * 64;
#pragma unroll
    for (int d = 0; d < kDepth; ++d) fetch(next[d], at + d * kStride);
    int step = 0;
    auto go = [&](Piece (&from)[kPieces]) __attribute__((always_inline)) {
        float x[kPerLane];
        unpack(x, from, at);
        fetch(from, at + kDepth * kStride);
        float four[kPerLane / 4];
        const float most = most_of(x, four);
        if (step == 0) {                      // the lanes' maxima stand for the first step
            const uint32_t key[1] = {most > -INFINITY ? key_of(most) : 0u};
            const uint32_t least = wave_min(key[0] - 1) + 1, high = wave_max(key[0]);       // of those that are there, `some`
            const int some = count_of(key[0] != 0);
            const uint32_t mine = some >= share ? reached(key, share, share / 2, least, high) : 0u;
            if (lane == 0) quarter[wid] = mine;
            weigh(x, most);
            __syncthreads();
            if (all_reach() == 0 && some >= picks) threshold = below(reached(key, picks, picks, least, high));
        } else weigh(x, most);
        const uint32_t q = all_reach();
        if (q) threshold = fmaxf(threshold, below(q));
        if (__any(most > threshold)) put(x, four, at);
        if (step > 0 && (step & (step + 1)) == 0 && n >= share) tell();
        at += kStride;
        ++step;
    };
    if (at >= end) __syncthreads();
#pragma nounroll
    while (at < end) {
        go(next[0]);
        if (kDepth > 1 && at < end) go(next[kDepth - 1]);
    }
    // the lanes' sums
    if (SAFE && m > -INFINITY && !is_huge(m)) s *= exp2_fast(__builtin_fmaf(m, kLog2e, offset_of(m)));      // they were relative to e^m
    float wave_top = m;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) wave_top = fmaxf(wave_top, __shfl_xor(wave_top, d, 64));
    double v = (double)s * weight_of(m, wave_top);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    top = wave_top;
    sum = __any(s != s || (!SAFE && m > -INFINITY && is_huge(m))) ? __longlong_as_double(0x7FF8000000000000ll) : v;
    wave_sync();
}

__device__ __forceinline__ bool is_there(const BeamSelection& s, int64_t row) { return s.score[row] > -INFINITY; }

template <typename T, bool STREAM>
__global__ __launch_bounds__(kThreads, 4) void beam_rows_kernel(BeamSelection s, int parts, RowPart* stats, unsigned long long* lists)
{
    constexpr int W = Vec<T>::kWidth;
    __shared__ unsigned long long list[kWaves][kList];
    __shared__ int lengths[kWaves];
    __shared__ float tops[kWaves];
    __shared__ double sums[kWaves];
    __shared__ uint32_t quarter[kWaves];
    const int tid = threadIdx.x, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = blockIdx.x / parts;
    const int part = blockIdx.x - (int)row * parts;
    if (!is_there(s, row) || (s.ended && s.ended[row])) return;
    const T* const x = (const T*)s.logits + row * s.logits_stride;
    const int pieces = (int)(((long long)s.vocab + W - 1) / W), each = (int)(((long long)pieces + parts - 1) / parts);
    const int begin = (int)min((long long)pieces, (long long)part * each), end = (int)min((long long)pieces, (long long)begin + each);
    int n;
    float top;
    double sum;
    if (tid < kWaves) quarter[tid] = 0;
    __syncthreads();
    scan_row<T, false, STREAM>(x, s.vocab, begin, end, wid, s.picks, list[wid], quarter, n, top, sum);
    if (__syncthreads_or(sum != sum)) {       // a quarter that counted NaN or signs of them holds for nobody
        if (tid < kWaves) quarter[tid] = 0;
        __syncthreads();
        scan_row<T, true, STREAM>(x, s.vocab, begin, end, wid, s.picks, list[wid], quarter, n, top, sum);
    }
    // the wavefronts' lists without what the quarters pass, behind each other; then a key to a thread: its place is the number of larger ones
    const int lane = tid & 63;
    const uint32_t q = min(min(quarter[0], quarter[1]), min(quarter[2], quarter[3]));
    int mine = 0;
#pragma nounroll
    for (int i = 0; i < n; i += 64) {
        const unsigned long long k = i + lane < n ? list[wid][i + lane] : 0;
        const bool keep = k != 0 && (uint32_t)(k >> 32) >= q;
        const unsigned long long b = __ballot(keep);
        wave_sync();
        if (keep) list[wid][mine + __popcll(b & ((1ull << lane) - 1))] = k;
        wave_sync();
        mine += __popcll(b);
    }
    if (lane == 0) {
        lengths[wid] = mine;
        tops[wid] = top;
        sums[wid] = sum;
    }
    __syncthreads();
    int all = 0, ahead = 0;
    for (int w = 0; w < kWaves; ++w) {
        ahead += w < wid ? lengths[w] : 0;
        all += lengths[w];
    }
    unsigned long long own[2];                // a list is at most picks + kGrow long
#pragma unroll
    for (int i = 0; i < 2; ++i) own[i] = i * 64 + lane < mine ? list[wid][i * 64 + lane] : 0;
    __syncthreads();
    unsigned long long* const joined = &list[0][0];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (own[i]) joined[ahead + i * 64 + lane] = own[i];
    __syncthreads();
    const int64_t request = row / s.beams;
    const int pitch = pitch_of(s.beams, parts);
    unsigned long long* const out = lists + request * pitch * s.picks + (blockIdx.x - request * s.beams * parts);
    if (tid == kThreads - 1) {
        float t = tops[0];
        for (int w = 1; w < kWaves; ++w) t = fmaxf(t, tops[w]);
        double v = 0;
#pragma nounroll
        for (int w = 0; w < kWaves; ++w) v += sums[w] * weight_of(tops[w], t);
        stats[blockIdx.x] = {v, t, 0};
    }
    for (int i = tid; i < all; i += kThreads) {
        const unsigned long long key = joined[i];
        int place = 0;
#pragma unroll 4
        for (int j = 0; j < all; ++j) place += joined[j] > key;
        if (place < s.picks) out[(int64_t)place * pitch] = key;
    }
    for (int i = all + tid; i < s.picks; i += kThreads) out[(int64_t)i * pitch] = 0;
}

// ---- requests -----------------------------------------------------------------------------------------------------
// A workgroup per request: the rows' sums, then the best of all lists.  From a score on that enough of the threads' best reach, candidates are listed and
// counted against each other.  Where that is too many, since few lists have the best of all, the score is searched for among all candidates; where those that
// are equal are too many still (rows of one value), they are found one after the other, at 6 us each.
// Bound by latency, that of its instructions' first use among it, so its loops are left as they are: 5.9 us for one request of four beams, 7.0 for 64 of eight,
// 10 to 12 for 2048 keys.
constexpr int kMeet = 512, kKeys = 2048;      // candidates that are listed; a request's keys, which are kept in LDS
static_assert(kBeamMax * kBeamPicksMax <= kKeys, "one part of a row at least");
constexpr int kHeld = (kKeys + kBeamPicksMax + kThreads - 1) / kThreads * kThreads;       // with one of every pitch that is none
struct Candidate {
    unsigned long long score;                 // fp64 as an integer that grows with it; 0: none
    unsigned long long key;                   // of the row
    int32_t row;                              // of the request
};
__device__ __forceinline__ unsigned long long order_of(double v)
{
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.);
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double score_of(unsigned long long o) { return __longlong_as_double((long long)(o >> 63 ? o & ~(1ull << 63) : ~o)); }
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b)
{
    if (a.score != b.score) return a.score > b.score;     // equal ones are rare
    return a.row != b.row ? a.row < b.row : a.key > b.key;
}
// done: the row has ended
__device__ __forceinline__ void write_pick(const BeamSelection& s, int r, int place, const Candidate& c, bool done)
{
    const int64_t at = (int64_t)r * s.picks + place, row = (int64_t)r * s.beams + c.row;
    const int token = c.score == 0 ? -1 : done ? s.end_token : (int)~(uint32_t)c.key;
    s.next_score[at] = c.score ? (float)score_of(c.score) : -INFINITY;
    s.next_row[at] = c.score ? (int)row : -1;
    s.next_token[at] = token;
    if (s.next_ended) s.next_ended[at] = c.score != 0 && (done || token == s.end_token);
}

__global__ __launch_bounds__(kThreads) void beam_meet_kernel(BeamSelection s, int parts, const RowPart* __restrict__ stats, const unsigned long long* __restrict__ lists)
{
    constexpr int kLanes = kThreads / kBeamMax;           // that share a row's parts
    __shared__ float row_top[kBeamMax];
    __shared__ double row_log[kBeamMax], row_score[kBeamMax];
    __shared__ int row_state[kBeamMax];       // 0: not there, 1: candidates, 2: ended
    __shared__ __attribute__((aligned(16))) uint32_t best[kThreads];
    __shared__ unsigned long long held[kHeld], scores[kHeld];
    __shared__ unsigned long long met_score[kMeet], met_key[kMeet];
    __shared__ int met_row[kMeet];
    __shared__ Candidate found[kThreads];
    __shared__ int n_met;
    const int tid = threadIdx.x, lane = tid & 63, r = blockIdx.x;
    const size_t first = (size_t)r * s.beams;
    const int segments = s.beams * parts, pitch = pitch_of(s.beams, parts), n = pitch * s.picks;
    const unsigned long long* const keys = lists + (size_t)r * n;
    {
        const int b = tid / kLanes, sub = tid % kLanes;
        RowPart v{0, -INFINITY, 0};
        float so_far = -INFINITY;
        int ended = 0;
        if (b < s.beams) {                    // a row's parts are of any bits where it has none; all on their way together
            v = stats[(first + b) * parts + min(sub, parts - 1)];
            so_far = s.score[first + b];
            if (s.ended) ended = s.ended[first + b];
        }
        {
            constexpr int kFirst = 4;         // of a thread, more where there are more
            unsigned long long k[kHeld / kThreads];
#pragma unroll
            for (int c = 0; c < kFirst; ++c) k[c] = keys[min(tid + c * kThreads, n - 1)];
            if (n > kFirst * kThreads)
#pragma unroll
                for (int c = kFirst; c < kHeld / kThreads; ++c) k[c] = keys[min(tid + c * kThreads, n - 1)];
#pragma unroll
            for (int c = 0; c < kFirst; ++c) held[tid + c * kThreads] = k[c];
            if (n > kFirst * kThreads)
#pragma unroll
                for (int c = kFirst; c < kHeld / kThreads; ++c) held[tid + c * kThreads] = k[c];
        }
        const int state = !(so_far > -INFINITY) ? 0 : ended ? 2 : 1, mine = state == 1 && sub < parts;
        float top = mine ? v.top : -INFINITY;
        double sum = 0;
        const int rounds = state == 1 ? (parts + kLanes - 1) / kLanes : 0;
#pragma nounroll
        for (int p = 1; p < rounds; ++p)
            if (p * kLanes + sub < parts) top = fmaxf(top, stats[(first + b) * parts + p * kLanes + sub].top);
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
#pragma nounroll
        for (int p = 0; p < rounds; ++p) {
            if (p * kLanes + sub >= parts) break;
            if (p > 0) v = stats[(first + b) * parts + p * kLanes + sub];
            sum += v.sum * weight_of(v.top, top);
        }
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d, 64);
        if (sub == 0 && b < s.beams) {
            // a candidate's logit less this: lse, or what is on top of a huge maximum
            row_top[b] = top;
            row_log[b] = is_huge(top) ? log(sum) : (log2(sum) - (double)offset_of(top)) / (double)kLog2e;
            row_score[b] = so_far;
            row_state[b] = state;
        }
    }
    if (tid == 0) n_met = 0;
    __syncthreads();
    // f(candidate) for all of this thread's, and the row itself where it has ended.  known: not the first time
    const float per_part = 1.f / (float)parts;
    auto each = [&](auto known, auto f) __attribute__((always_inline)) {
        if (tid < s.beams && row_state[tid] == 2) f(Candidate{order_of(row_score[tid]), 0, tid});
        int segment = tid % pitch;
        const int step = kThreads % pitch;
#pragma nounroll
        for (int i = tid; i < n; i += kThreads) {
            const bool is = segment < segments;
            const int b = is ? (int)(((float)segment + 0.5f) * per_part) : 0;         // segment / parts: both are below 2^12
            segment += step;
            if (segment >= pitch) segment -= pitch;
            const unsigned long long key = held[i];
            unsigned long long score = 0;
            if (known) score = scores[i];
            else {
                const float x = logit_of((uint32_t)(key >> 32)), top = row_top[b];
                const double of = is_huge(top) ? x == top ? 0. : (double)x - (double)top : (double)x;
                if (is & (row_state[b] == 1) & (key != 0) & ((x == top) | (top < INFINITY))) score = order_of(row_score[b] + (of - row_log[b]));
                scores[i] = score;
            }
            if (score) f(Candidate{score, key, b});
        }
    };
    unsigned long long mine = 0;
    each(std::false_type(), [&](const Candidate& c) { mine = max(mine, c.score); });
    best[tid] = (uint32_t)(mine >> 32);
    __syncthreads();
    uint32_t low;
    {
        const uint4 four = *(const uint4*)(best + 4 * lane);
        const uint32_t key[4] = {four.x, four.y, four.z, four.w};
        const uint32_t most = max(max(key[0], key[1]), max(key[2], key[3]));
        low = max(reached(key, s.picks, 24, wave_min(most), wave_max(most)), 1u);             // no score's upper half is 0
    }
    auto list = [&]() __attribute__((always_inline)) {
        each(std::true_type(), [&](const Candidate& c) {
            if ((uint32_t)(c.score >> 32) < low) return;
            const int at = atomicAdd(&n_met, 1);
            if (at < kMeet) met_score[at] = c.score, met_key[at] = c.key, met_row[at] = c.row;
        });
        __syncthreads();
        return n_met;
    };
    int all = list();
    if (all > kMeet) {                        // one list has most of the best: a threshold that all candidates are counted against
        uint32_t high = 0;
        for (int i = 0; i < kThreads; ++i) high = max(high, best[i]);
#pragma nounroll
        while (all > kMeet && low < high) {
            const uint32_t mid = low + (high - low) / 2 + 1;
            int more = 0;
            each(std::true_type(), [&](const Candidate& c) { more += (uint32_t)(c.score >> 32) >= mid; });
            __syncthreads();
            if (tid == 0) n_met = 0;
            __syncthreads();
            if (more) atomicAdd(&n_met, more);
            __syncthreads();
            const int now = n_met;
            if (now >= s.picks) low = mid, all = now;
            else high = mid - 1;
        }
        __syncthreads();
        if (tid == 0) n_met = 0;
        __syncthreads();
        all = list();
    }
    if (all <= kMeet) {
        for (int i = tid; i < max(all, s.picks); i += kThreads) {
            Candidate c{0, 0, 0};
            int place = i;
            if (i < all) {
                c = {met_score[i], met_key[i], met_row[i]};
                place = 0;
#pragma unroll 4
                for (int j = 0; j < all; ++j) {           // before(), without a branch
                    const unsigned long long v = met_score[j], k = met_key[j];
                    const int w = met_row[j];
                    place += (v > c.score) | ((v == c.score) & ((w < c.row) | ((w == c.row) & (k > c.key))));
                }
            }
            if (place < s.picks) write_pick(s, r, place, c, row_state[c.row] == 2);
        }
        return;
    }
    Candidate last{~0ull, ~0ull, -1};
    for (int p = 0; p < s.picks; ++p) {
        Candidate c{0, 0, 0};
        each(std::true_type(), [&](const Candidate& v) {
            if (before(last, v) && before(v, c)) c = v;
        });
        __syncthreads();
        found[tid] = c;
        __syncthreads();
        for (int d = kThreads / 2; d > 0; d >>= 1) {
            if (tid < d && before(found[tid + d], found[tid])) found[tid] = found[tid + d];
            __syncthreads();
        }
        last = found[0];
        if (tid == 0) write_pick(s, r, p, last, row_state[last.row] == 2);
    }
}

// Parts of a row: as many as fill the chip (three workgroups to a compute unit), of 4096 logits or more, while the launch that merges them keeps its
// keys.  512 rows of 128,000 in bf16, 16 picks, 512 / 768 / 1024 / 2048 workgroups 54.9 / 45.0 / 45.0 / 52.6 us; 400 rows, 8 picks 41 / 41 / 47 / 49.
int row_parts(int64_t rows, int32_t beams, int32_t picks, int32_t vocab)
{
    const int64_t fill = (768 + rows - 1) / std::max<int64_t>(rows, 1), length = ((int64_t)vocab + 4095) / 4096, held = kKeys / ((int64_t)beams * picks);
    return (int)std::max<int64_t>(1, std::min(std::min(fill, length), held));
}

}  // namespace

int64_t beam_workspace(int32_t n_requests, int32_t beams, int32_t picks, int32_t vocab)
{
    const int64_t rows = (int64_t)n_requests * beams;
    const int parts = row_parts(rows, beams, picks, vocab);
    return rows * parts * (int64_t)sizeof(RowPart) + (int64_t)n_requests * pitch_of(beams, parts) * picks * 8;
}

hipError_t beam_select(int dtype, const BeamSelection& s, void* workspace, hipStream_t stream)
{
    const int64_t rows = (int64_t)s.n_requests * s.beams;
    const int parts = row_parts(rows, s.beams, s.picks, s.vocab);
    RowPart* const stats = (RowPart*)workspace;
    unsigned long long* const lists = (unsigned long long*)(stats + rows * parts);
    // Logits that would fill the second-level caches pass by them: 512 rows of 128,000 in bf16 44.5 -> 42.2 us, of 64,000 in fp32 38.3 -> 35.0, 64 rows 22.6 ->
    // 21.8; 32 rows, 8 MB, 37.7 -> 39.8 with 32 picks.
    const bool stream_by = rows * s.vocab * (dtype == 0 ? 4 : 2) >= 12ll << 20;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * parts)), dim3(kThreads), 0, stream, s, parts, stats, lists); };
    if (dtype == 0) stream_by ? launch(beam_rows_kernel<float, true>) : launch(beam_rows_kernel<float, false>);
    else stream_by ? launch(beam_rows_kernel<uint16_t, true>) : launch(beam_rows_kernel<uint16_t, false>);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(beam_meet_kernel, dim3((unsigned)s.n_requests), dim3(kThreads), 0, stream, s, parts, stats, lists);
    return hipGetLastError();
}

}  // namespace k
}  // namespace coe
