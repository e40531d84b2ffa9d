// C entry points of the calls for token-generating experts: argument checks, nothing else.
#include <cstdarg>
#include <cstdio>

#include "../../include/coe.h"
#include "kernels.h"

namespace {

int fail(int code, const char* format, ...)
{
    char text[256];
    va_list args;
    va_start(args, format);
    vsnprintf(text, sizeof(text), format, args);
    va_end(args);
    return coe::context_free_error(code, text);
}

int launched(const char* call, hipError_t e)
{
    if (e == hipSuccess) return COE_OK;
    return fail(e == hipErrorInvalidValue ? COE_EINVAL : COE_EDEVICE, "%s: %s", call, hipGetErrorString(e));
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// log2 of a block size that is supported, else -1
int block_shift(int32_t block_size)
{
    for (int s = 3; s <= 10; ++s)
        if (block_size == 1 << s) return s;
    return -1;
}

int check_cache(const char* call, const coe_kv_cache* c, coe::k::KvCache* out)
{
    if (!c || !c->k || !c->v) return fail(COE_EINVAL, "%s: null cache", call);
    if (c->dtype != COE_DT_BF16) return fail(COE_EINVAL, "%s: the cache's dtype must be COE_DT_BF16", call);
    const int shift = block_shift(c->block_size);
    if (shift < 0) return fail(COE_EINVAL, "%s: block_size %d is not a power of two in 8..1024", call, c->block_size);
    if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8)
        return fail(COE_EINVAL, "%s: head_dim %d is not a multiple of 8 in 8..128", call, c->head_dim);
    if (c->kv_heads <= 0 || c->kv_heads > 65535) return fail(COE_EINVAL, "%s: kv_heads %d", call, c->kv_heads);
    if (c->n_blocks <= 0 || (long long)c->n_blocks * c->block_size > 0x7FFFFFFFll)
        return fail(COE_EINVAL, "%s: n_blocks * block_size must be in 1..2^31 - 1", call);
    if (!aligned16(c->k) || !aligned16(c->v)) return fail(COE_EINVAL, "%s: k and v must be 16-byte aligned", call);
    if (c->block_stride < 0 || c->token_stride < 0 || c->head_stride < 0 || c->block_stride % 8 || c->token_stride % 8 || c->head_stride % 8)
        return fail(COE_EINVAL, "%s: cache strides must be multiples of 8 elements, not negative", call);
    if (c->token_stride > 0x7FFFFFFFll / 2 / c->block_size - 256)
        return fail(COE_EINVAL, "%s: the rows of a block must lie within 2^31 bytes", call);
    // a stride that makes two rows share bytes cannot be told from a wrong one
    if (c->token_stride < c->head_dim || (c->kv_heads > 1 && c->head_stride < c->head_dim) || (c->n_blocks > 1 && c->block_stride < c->head_dim))
        return fail(COE_EINVAL, "%s: a cache stride is smaller than head_dim", call);
    *out = {(uint16_t*)c->k, (uint16_t*)c->v, c->block_stride, c->token_stride, c->head_stride, c->n_blocks, shift, c->kv_heads, c->head_dim};
    return COE_OK;
}

bool row_strides_ok(int64_t token_stride, int64_t head_stride)
{
    return token_stride >= 0 && head_stride >= 0 && token_stride % 8 == 0 && head_stride % 8 == 0;
}

// kernels round rows up to whole tiles, and look a few tiles ahead, in 32 bits
constexpr long long kMostRows = (1ll << 31) - 4096;

}  // namespace

extern "C" {

static_assert(COE_KV_MAX_REQUESTS == coe::k::kPlanMaxRequests, "header and kernel agree on the limit");

int coe_kv_plan(int32_t n_requests, int32_t block_size, int32_t n_blocks, int32_t max_blocks, int32_t token_cap, const int32_t* have,
                const int32_t* add, int32_t* ring, const int32_t* ring_state, int32_t* table, int32_t* seq_len, int32_t* q_off,
                int32_t* slot, int32_t* position, int32_t* next_state, void* stream)
{
    const char* const call = "coe_kv_plan";
    if (n_requests < 0 || n_requests > COE_KV_MAX_REQUESTS) return fail(COE_EINVAL, "%s: n_requests %d outside 0..%d", call, n_requests, COE_KV_MAX_REQUESTS);
    const int shift = block_shift(block_size);
    if (shift < 0) return fail(COE_EINVAL, "%s: block_size %d is not a power of two in 8..1024", call, block_size);
    if (n_blocks <= 0 || (long long)n_blocks * block_size > 0x7FFFFFFFll) return fail(COE_EINVAL, "%s: n_blocks * block_size must be in 1..2^31 - 1", call);
    if (max_blocks <= 0 || (long long)max_blocks * block_size > 0x7FFFFFFFll) return fail(COE_EINVAL, "%s: max_blocks * block_size must be in 1..2^31 - 1", call);
    if (token_cap < 0) return fail(COE_EINVAL, "%s: negative token_cap", call);
    if (!ring || !ring_state || !q_off || !next_state || (n_requests > 0 && (!have || !add || !table || !seq_len)) || (token_cap > 0 && (!slot || !position)))
        return fail(COE_EINVAL, "%s: null argument", call);
    if (seq_len == have || seq_len == add || next_state == ring_state) return fail(COE_EINVAL, "%s: outputs must not alias inputs", call);
    return launched(call, coe::k::kv_plan(n_requests, shift, n_blocks, max_blocks, token_cap, have, add, ring, ring_state, table, seq_len, q_off,
                                          slot, position, next_state, (hipStream_t)stream));
}

int coe_kv_append(const coe_kv_cache* cache, int32_t n_tokens, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                  int64_t v_token_stride, int64_t v_head_stride, const int32_t* slot, void* stream)
{
    const char* const call = "coe_kv_append";
    coe::k::KvCache c;
    if (int rc = check_cache(call, cache, &c)) return rc;
    if (n_tokens < 0) return fail(COE_EINVAL, "%s: negative n_tokens", call);
    if (n_tokens == 0) return COE_OK;
    if (!k || !v || !slot) return fail(COE_EINVAL, "%s: null argument", call);
    if (!aligned16(k) || !aligned16(v) || !row_strides_ok(k_token_stride, k_head_stride) || !row_strides_ok(v_token_stride, v_head_stride))
        return fail(COE_EINVAL, "%s: rows must be 16-byte aligned, strides multiples of 8 elements", call);
    return launched(call, coe::k::kv_append(c, n_tokens, (const uint16_t*)k, k_token_stride, k_head_stride, (const uint16_t*)v, v_token_stride,
                                            v_head_stride, slot, (hipStream_t)stream));
}

int64_t coe_kv_attention_workspace(int32_t n_requests, int32_t n_tokens, int32_t max_new, int32_t heads, int32_t kv_heads, int32_t head_dim)
{
    if (n_requests < 0 || n_requests > COE_KV_MAX_REQUESTS || n_tokens < 0 || max_new < 0 || kv_heads <= 0 || kv_heads > 65535 || heads <= 0 ||
        heads % kv_heads || heads > 65535 || head_dim < 8 || head_dim > 128 || head_dim % 8)
        return fail(COE_EINVAL, "coe_kv_attention_workspace: bad size");
    return coe::k::kv_attention_workspace(n_requests, n_tokens, max_new, heads, kv_heads, head_dim);
}

int coe_kv_attention(const coe_kv_cache* cache, int32_t n_requests, int32_t n_tokens, int32_t max_new, int32_t heads, int32_t window,
                     float scale, const void* q, int64_t q_token_stride, int64_t q_head_stride, const int32_t* q_off, const int32_t* seq_len,
                     const int32_t* table, int32_t max_blocks, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                     void* workspace, int64_t workspace_bytes, void* stream)
{
    const char* const call = "coe_kv_attention";
    coe::k::KvCache c;
    if (int rc = check_cache(call, cache, &c)) return rc;
    if (n_requests < 0 || n_requests > COE_KV_MAX_REQUESTS || n_tokens < 0 || max_new < 0 || window < 0)
        return fail(COE_EINVAL, "%s: a size is negative or n_requests exceeds %d", call, COE_KV_MAX_REQUESTS);
    if (heads <= 0 || heads > 65535 || heads % c.kv_heads) return fail(COE_EINVAL, "%s: heads %d is not a multiple of kv_heads %d", call, heads, c.kv_heads);
    // the kernels round positions and rows up to whole tiles, and look a few tiles ahead, in 32 bits
    constexpr long long kMost = (1ll << 31) - 4096;
    if (max_blocks <= 0 || (long long)max_blocks * cache->block_size > kMost)
        return fail(COE_EINVAL, "%s: max_blocks * block_size must be in 1..2^31 - 4096", call);
    if ((long long)n_tokens * heads > kMost || (long long)n_requests * c.kv_heads > 0x7FFFFFFFll)
        return fail(COE_EINVAL, "%s: n_tokens * heads must be at most 2^31 - 4096", call);
    if (!(scale == scale) || scale - scale != 0.f) return fail(COE_EINVAL, "%s: scale must be finite", call);
    if (n_requests == 0 || n_tokens == 0 || max_new == 0) return COE_OK;
    if (!q || !q_off || !seq_len || !table || !out) return fail(COE_EINVAL, "%s: null argument", call);
    if (!aligned16(q) || !aligned16(out) || !row_strides_ok(q_token_stride, q_head_stride) || !row_strides_ok(out_token_stride, out_head_stride))
        return fail(COE_EINVAL, "%s: rows must be 16-byte aligned, strides multiples of 8 elements", call);
    if ((n_tokens > 1 && out_token_stride < c.head_dim) || (heads > 1 && out_head_stride < c.head_dim))
        return fail(COE_EINVAL, "%s: an output stride is smaller than head_dim", call);
    const int64_t need = coe::k::kv_attention_workspace(n_requests, n_tokens, max_new, heads, c.kv_heads, c.head_dim);
    if (workspace_bytes < need) return fail(COE_ERANGE, "%s: workspace of %lld bytes, %lld needed", call, (long long)workspace_bytes, (long long)need);
    if (need > 0 && (!workspace || !aligned16(workspace))) return fail(COE_EINVAL, "%s: workspace must be 16-byte aligned", call);
    const coe::k::KvAttention a{n_requests, n_tokens, max_new < n_tokens ? max_new : n_tokens, heads, window, max_blocks, scale, (const uint16_t*)q,
                                q_token_stride, q_head_stride, q_off, seq_len, table, (uint16_t*)out, out_token_stride, out_head_stride, lse};
    return launched(call, coe::k::kv_attention(c, a, workspace, (hipStream_t)stream));
}

int64_t coe_sample_workspace(int32_t n_rows, int32_t vocab)
{
    if (n_rows < 0 || vocab <= 0) return fail(COE_EINVAL, "coe_sample_workspace: bad size");
    return coe::k::sample_workspace(n_rows, vocab);
}

int coe_sample_tokens(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits, int64_t logits_stride, const float* temperature,
                      const int32_t* top_k, const float* top_p, const float* min_p, const float* noise, int64_t noise_stride, int32_t* token,
                      float* logprob, void* workspace, int64_t workspace_bytes, void* stream)
{
    const char* const call = "coe_sample_tokens";
    if (n_rows < 0 || vocab <= 0) return fail(COE_EINVAL, "%s: n_rows %d, vocab %d", call, n_rows, vocab);
    if (dtype != COE_DT_F32 && dtype != COE_DT_BF16) return fail(COE_EINVAL, "%s: unknown dtype %d", call, dtype);
    if (n_rows == 0) return COE_OK;
    if (!logits || !token) return fail(COE_EINVAL, "%s: null argument", call);
    if (!noise && !temperature) return fail(COE_EINVAL, "%s: noise may be null only where a temperature says that rows are greedy", call);
    if (((uintptr_t)logits & (dtype == COE_DT_F32 ? 3 : 1)) || ((uintptr_t)noise & 3)) return fail(COE_EINVAL, "%s: misaligned logits or noise", call);
    if (n_rows > 1 && (logits_stride < vocab || (noise && noise_stride < vocab))) return fail(COE_EINVAL, "%s: a row stride is smaller than vocab", call);
    const int64_t need = coe::k::sample_workspace(n_rows, vocab);
    if (workspace_bytes < need) return fail(COE_ERANGE, "%s: workspace of %lld bytes, %lld needed", call, (long long)workspace_bytes, (long long)need);
    if (need > 0 && (!workspace || !aligned16(workspace))) return fail(COE_EINVAL, "%s: workspace must be 16-byte aligned", call);
    const coe::k::Sampling s{logits, logits_stride, noise_stride, temperature, top_p, min_p, noise, top_k, token, logprob, vocab};
    return launched(call, coe::k::sample_tokens(dtype, n_rows, s, workspace, (hipStream_t)stream));
}

int coe_kv_append_rotated(const coe_kv_cache* cache, int32_t n_tokens, int32_t heads, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                          void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                          const void* v, int64_t v_token_stride, int64_t v_head_stride, const int32_t* slot, const int32_t* position,
                          const float* frequency, int32_t rotated, int32_t pairing, void* stream)
{
    const char* const call = "coe_kv_append_rotated";
    coe::k::KvCache c;
    if (int rc = check_cache(call, cache, &c)) return rc;
    if (n_tokens < 0) return fail(COE_EINVAL, "%s: negative n_tokens", call);
    if (heads < 0 || heads > 65535) return fail(COE_EINVAL, "%s: heads %d outside 0..65535", call, heads);
    if (rotated < 2 || rotated > c.head_dim || rotated % 2) return fail(COE_EINVAL, "%s: rotated %d is not an even number in 2..head_dim", call, rotated);
    if (pairing != COE_PAIR_HALVES && pairing != COE_PAIR_NEIGHBOURS) return fail(COE_EINVAL, "%s: unknown pairing %d", call, pairing);
    if (n_tokens == 0) return COE_OK;
    if (!k || !v || !slot || !position || !frequency || (heads > 0 && (!q || !q_out))) return fail(COE_EINVAL, "%s: null argument", call);
    if (!aligned16(k) || !aligned16(v) || !row_strides_ok(k_token_stride, k_head_stride) || !row_strides_ok(v_token_stride, v_head_stride) ||
        (heads > 0 && (!aligned16(q) || !aligned16(q_out) || !row_strides_ok(q_token_stride, q_head_stride) || !row_strides_ok(q_out_token_stride, q_out_head_stride))))
        return fail(COE_EINVAL, "%s: rows must be 16-byte aligned, strides multiples of 8 elements", call);
    if (heads > 0 && ((n_tokens > 1 && q_out_token_stride < c.head_dim) || (heads > 1 && q_out_head_stride < c.head_dim)))
        return fail(COE_EINVAL, "%s: an output stride is smaller than head_dim", call);
    if (heads > 0 && q == q_out && ((n_tokens > 1 && q_token_stride != q_out_token_stride) || (heads > 1 && q_head_stride != q_out_head_stride)))
        return fail(COE_EINVAL, "%s: in place, q and q_out need the same strides", call);
    const coe::k::Rotation r{(const uint16_t*)q, q_token_stride, q_head_stride, (uint16_t*)q_out, q_out_token_stride, q_out_head_stride, (const uint16_t*)k,
                             k_token_stride, k_head_stride, (const uint16_t*)v, v_token_stride, v_head_stride, slot, position, frequency, n_tokens, heads,
                             rotated, pairing};
    return launched(call, coe::k::kv_append_rotated(c, r, (hipStream_t)stream));
}

// a launch of a workgroup to 128 query rows of a head, and one more to a source and head, holds fewer than 2^32 threads
constexpr long long kMostCrossRows = 1ll << 30, kMostCrossHeads = 1ll << 22;
int64_t coe_cross_attention_workspace(int32_t n_sources, int32_t n_tokens, int32_t max_new, int32_t max_rows, int32_t heads, int32_t kv_heads,
                                      int32_t head_dim)
{
    if (n_sources < 0 || n_sources > COE_KV_MAX_REQUESTS || n_tokens < 0 || max_new < 0 || max_rows < 0 || max_rows > kMostRows || kv_heads <= 0 ||
        kv_heads > 65535 || heads <= 0 || heads % kv_heads || heads > 65535 || (long long)n_tokens * heads > kMostCrossRows ||
        (long long)n_sources * kv_heads > kMostCrossHeads || head_dim < 8 || head_dim > 128 || head_dim % 8)
        return fail(COE_EINVAL, "coe_cross_attention_workspace: bad size");
    return coe::k::cross_attention_workspace(n_sources, n_tokens, max_new < n_tokens ? max_new : n_tokens, max_rows, heads, kv_heads, head_dim);
}

int coe_cross_attention(const coe_states* states, int32_t n_sources, int32_t n_tokens, int32_t beams, int32_t max_new, int32_t max_rows, int32_t heads,
                        float scale, const void* q, int64_t q_token_stride, int64_t q_head_stride, const int32_t* q_off, const int32_t* first,
                        const int32_t* length, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace,
                        int64_t workspace_bytes, void* stream)
{
    const char* const call = "coe_cross_attention";
    if (!states) return fail(COE_EINVAL, "%s: null states", call);
    if (states->dtype != COE_DT_BF16) return fail(COE_EINVAL, "%s: the states' dtype must be COE_DT_BF16", call);
    if (states->n_rows < 0) return fail(COE_EINVAL, "%s: negative n_rows", call);
    if (states->head_dim < 8 || states->head_dim > 128 || states->head_dim % 8)
        return fail(COE_EINVAL, "%s: head_dim %d is not a multiple of 8 in 8..128", call, states->head_dim);
    if (states->kv_heads <= 0 || states->kv_heads > 65535) return fail(COE_EINVAL, "%s: kv_heads %d", call, states->kv_heads);
    const bool any = states->n_rows > 0;
    if (any && (!states->k || !states->v)) return fail(COE_EINVAL, "%s: null k or v", call);
    if (!aligned16(states->k) || !aligned16(states->v)) return fail(COE_EINVAL, "%s: k and v must be 16-byte aligned", call);
    if (!row_strides_ok(states->k_row_stride, states->k_head_stride) || !row_strides_ok(states->v_row_stride, states->v_head_stride))
        return fail(COE_EINVAL, "%s: strides of k and v must be multiples of 8 elements, not negative", call);
    // a tile of 64 rows is addressed in 31 bits
    constexpr int64_t kMostRowStride = 0x7FFFFFFFll / 2 / 64 - 256;
    if (states->k_row_stride > kMostRowStride || states->v_row_stride > kMostRowStride) return fail(COE_EINVAL, "%s: 64 rows must lie within 2^31 bytes", call);
    if (n_sources < 0 || beams <= 0 || n_tokens < 0 || max_new < 0 || max_rows < 0 || max_rows > kMostRows || (long long)n_sources * beams > COE_KV_MAX_REQUESTS)
        return fail(COE_EINVAL, "%s: a size is out of range (n_sources * beams: at most %d)", call, COE_KV_MAX_REQUESTS);
    if (heads <= 0 || heads > 65535 || heads % states->kv_heads) return fail(COE_EINVAL, "%s: heads %d is not a multiple of kv_heads %d", call, heads, states->kv_heads);
    if ((long long)n_tokens * heads > kMostCrossRows) return fail(COE_EINVAL, "%s: n_tokens * heads must be at most 2^30", call);
    if ((long long)n_sources * states->kv_heads > kMostCrossHeads) return fail(COE_EINVAL, "%s: n_sources * kv_heads must be at most 2^22", call);
    if (!(scale == scale) || scale - scale != 0.f) return fail(COE_EINVAL, "%s: scale must be finite", call);
    if (n_sources == 0 || n_tokens == 0 || max_new == 0) return COE_OK;
    if (!q || !q_off || !first || !length || !out) return fail(COE_EINVAL, "%s: null argument", call);
    if (!aligned16(q) || !aligned16(out) || !row_strides_ok(q_token_stride, q_head_stride) || !row_strides_ok(out_token_stride, out_head_stride))
        return fail(COE_EINVAL, "%s: rows must be 16-byte aligned, strides multiples of 8 elements", call);
    if ((n_tokens > 1 && out_token_stride < states->head_dim) || (heads > 1 && out_head_stride < states->head_dim))
        return fail(COE_EINVAL, "%s: an output stride is smaller than head_dim", call);
    const int32_t most = max_new < n_tokens ? max_new : n_tokens;
    const int64_t need = coe::k::cross_attention_workspace(n_sources, n_tokens, most, max_rows, heads, states->kv_heads, states->head_dim);
    if (workspace_bytes < need) return fail(COE_ERANGE, "%s: workspace of %lld bytes, %lld needed", call, (long long)workspace_bytes, (long long)need);
    if (need > 0 && (!workspace || !aligned16(workspace))) return fail(COE_EINVAL, "%s: workspace must be 16-byte aligned", call);
    const coe::k::States st{(const uint16_t*)states->k, (const uint16_t*)states->v, states->k_row_stride, states->k_head_stride, states->v_row_stride,
                            states->v_head_stride, states->seen, states->n_rows, states->kv_heads, states->head_dim};
    const coe::k::CrossAttention a{n_sources, n_tokens, beams, most, max_rows, heads, scale, (const uint16_t*)q, q_token_stride, q_head_stride, q_off, first,
                                   length, (uint16_t*)out, out_token_stride, out_head_stride, lse};
    return launched(call, coe::k::cross_attention(st, a, workspace, (hipStream_t)stream));
}

static_assert(COE_BEAM_MAX == coe::k::kBeamMax && COE_BEAM_PICKS_MAX == coe::k::kBeamPicksMax, "header and kernels agree on the limits");

int64_t coe_beam_workspace(int32_t n_requests, int32_t beams, int32_t picks, int32_t vocab)
{
    if (n_requests < 0 || beams <= 0 || beams > COE_BEAM_MAX || picks <= 0 || picks > COE_BEAM_PICKS_MAX || vocab <= 0 || (long long)n_requests * beams >= 1 << 23)
        return fail(COE_EINVAL, "coe_beam_workspace: bad size");
    return coe::k::beam_workspace(n_requests, beams, picks, vocab);
}

int coe_beam_select(int32_t n_requests, int32_t beams, int32_t picks, int32_t vocab, int32_t dtype, const void* logits, int64_t logits_stride,
                    const float* score, const int32_t* ended, int32_t end_token, float* next_score, int32_t* next_row, int32_t* next_token,
                    int32_t* next_ended, void* workspace, int64_t workspace_bytes, void* stream)
{
    const char* const call = "coe_beam_select";
    if (n_requests < 0 || vocab <= 0) return fail(COE_EINVAL, "%s: n_requests %d, vocab %d", call, n_requests, vocab);
    if (beams <= 0 || beams > COE_BEAM_MAX) return fail(COE_EINVAL, "%s: beams %d outside 1..%d", call, beams, COE_BEAM_MAX);
    if (picks <= 0 || picks > COE_BEAM_PICKS_MAX) return fail(COE_EINVAL, "%s: picks %d outside 1..%d", call, picks, COE_BEAM_PICKS_MAX);
    if ((long long)n_requests * beams >= 1 << 23) return fail(COE_EINVAL, "%s: n_requests * beams must be below 2^23", call);
    if (dtype != COE_DT_F32 && dtype != COE_DT_BF16) return fail(COE_EINVAL, "%s: unknown dtype %d", call, dtype);
    if (n_requests == 0) return COE_OK;
    if (!logits || !score || !next_score || !next_row || !next_token) return fail(COE_EINVAL, "%s: null argument", call);
    if ((uintptr_t)logits & (dtype == COE_DT_F32 ? 3 : 1)) return fail(COE_EINVAL, "%s: misaligned logits", call);
    if ((long long)n_requests * beams > 1 && logits_stride < vocab) return fail(COE_EINVAL, "%s: a row stride is smaller than vocab", call);
    if (next_score == score || (ended && next_ended == ended)) return fail(COE_EINVAL, "%s: outputs must not alias inputs", call);
    const int64_t need = coe::k::beam_workspace(n_requests, beams, picks, vocab);
    if (workspace_bytes < need) return fail(COE_ERANGE, "%s: workspace of %lld bytes, %lld needed", call, (long long)workspace_bytes, (long long)need);
    if (need > 0 && (!workspace || !aligned16(workspace))) return fail(COE_EINVAL, "%s: workspace must be 16-byte aligned", call);
    const coe::k::BeamSelection s{logits, logits_stride, score, ended, next_score, next_row, next_token, next_ended, n_requests, beams, picks, vocab, end_token};
    return launched(call, coe::k::beam_select(dtype, s, workspace, (hipStream_t)stream));
}

int64_t coe_kv_fork_workspace(int32_t n_requests, int32_t beams)
{
    if (n_requests < 0 || beams <= 0 || beams > COE_BEAM_MAX || (long long)n_requests * beams > COE_KV_MAX_REQUESTS)
        return fail(COE_EINVAL, "coe_kv_fork_workspace: bad size");
    return coe::k::kv_fork_workspace(n_requests, beams);
}

int coe_kv_fork(int32_t n_requests, int32_t beams, int32_t block_size, int32_t n_blocks, int32_t max_blocks, const int32_t* parent, const int32_t* seq_len,
                const int32_t* table, int32_t* ring, const int32_t* ring_state, int32_t* next_table, int32_t* next_len, int32_t* copy,
                int32_t* next_state, void* workspace, int64_t workspace_bytes, void* stream)
{
    const char* const call = "coe_kv_fork";
    if (beams <= 0 || beams > COE_BEAM_MAX) return fail(COE_EINVAL, "%s: beams %d outside 1..%d", call, beams, COE_BEAM_MAX);
    if (n_requests < 0 || (long long)n_requests * beams > COE_KV_MAX_REQUESTS)
        return fail(COE_EINVAL, "%s: n_requests %d, n_requests * beams outside 0..%d", call, n_requests, COE_KV_MAX_REQUESTS);
    const int shift = block_shift(block_size);
    if (shift < 0) return fail(COE_EINVAL, "%s: block_size %d is not a power of two in 8..1024", call, block_size);
    if (n_blocks <= 0 || (long long)n_blocks * block_size > 0x7FFFFFFFll) return fail(COE_EINVAL, "%s: n_blocks * block_size must be in 1..2^31 - 1", call);
    if (max_blocks <= 0 || (long long)max_blocks * block_size > 0x7FFFFFFFll) return fail(COE_EINVAL, "%s: max_blocks * block_size must be in 1..2^31 - 1", call);
    // a request's blocks are counted in 31 bits
    if ((long long)max_blocks * beams > 0x3FFFFFFFll) return fail(COE_EINVAL, "%s: max_blocks * beams must be below 2^30", call);
    if (!ring || !ring_state || !next_state || (n_requests > 0 && (!parent || !seq_len || !table || !next_table || !next_len || !copy)))
        return fail(COE_EINVAL, "%s: null argument", call);
    if ((uintptr_t)copy & 7) return fail(COE_EINVAL, "%s: copy must be 8-byte aligned", call);
    if (next_state == ring_state || (n_requests > 0 && (next_table == table || next_len == seq_len || next_len == parent))) return fail(COE_EINVAL, "%s: outputs must not alias inputs", call);
    const int64_t need = coe::k::kv_fork_workspace(n_requests, beams);
    if (workspace_bytes < need) return fail(COE_ERANGE, "%s: workspace of %lld bytes, %lld needed", call, (long long)workspace_bytes, (long long)need);
    if (need > 0 && (!workspace || !aligned16(workspace))) return fail(COE_EINVAL, "%s: workspace must be 16-byte aligned", call);
    const coe::k::KvFork f{n_requests, beams, shift, n_blocks, max_blocks, parent, seq_len, table, ring, ring_state, next_table, next_len, copy, next_state};
    return launched(call, coe::k::kv_fork(f, workspace, (hipStream_t)stream));
}

int coe_kv_copy(int32_t n_caches, const coe_kv_cache* caches, int32_t n, const int32_t* copy, const int32_t* seq_len, void* stream)
{
    const char* const call = "coe_kv_copy";
    if (n_caches < 0 || n < 0) return fail(COE_EINVAL, "%s: n_caches %d, n %d", call, n_caches, n);
    if (n > COE_KV_MAX_REQUESTS) return fail(COE_EINVAL, "%s: n %d exceeds %d", call, n, COE_KV_MAX_REQUESTS);
    if (n_caches > 0 && !caches) return fail(COE_EINVAL, "%s: null caches", call);
    coe::k::KvCache c;
    for (int32_t i = 0; i < n_caches; ++i) {  // all of them before the first launch
        if (int rc = check_cache(call, caches + i, &c)) return rc;
        if (caches[i].block_size != caches[0].block_size) return fail(COE_EINVAL, "%s: caches of different block_size", call);
    }
    if (n_caches == 0 || n == 0) return COE_OK;
    if (!copy || !seq_len) return fail(COE_EINVAL, "%s: null argument", call);
    if ((uintptr_t)copy & 7) return fail(COE_EINVAL, "%s: copy must be 8-byte aligned", call);
    for (int32_t at = 0; at < n_caches; at += coe::k::kCopyCaches) {
        coe::k::KvCaches some{};
        const int32_t count = n_caches - at < coe::k::kCopyCaches ? n_caches - at : coe::k::kCopyCaches;
        for (int32_t i = 0; i < count; ++i) check_cache(call, caches + at + i, &some.c[i]);
        if (int rc = launched(call, coe::k::kv_copy(count, some, n, copy, seq_len, (hipStream_t)stream))) return rc;
    }
    return COE_OK;
}

}  // extern "C"
