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

}  // extern "C"
