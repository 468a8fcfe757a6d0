// Entry points of the attention operators: checks of their arguments, and the plan of a call.
#include <climits>
#include <cmath>

#include "attention.h"
#include "shflbw.h"
#include "shflbw_internal.h"

namespace shflbw {
namespace {

bool head_dim_ok(int d) { return d == 64 || d == 96 || d == 128; }
bool page_ok(int p) { return p >= 32 && p <= 1024 && (p & (p - 1)) == 0; }
float softmax_scale(int head_dim) { return (float)(1.4426950408889634 / std::sqrt((double)head_dim)); }

int check_sizes(int pages, int page_tokens, int heads, int head_dim)
{
    if (!page_ok(page_tokens)) return fail(SHFLBW_ERR_BAD_SHAPE, "page_tokens must be a power of two from 32 to 1024");
    if (!head_dim_ok(head_dim)) return fail(SHFLBW_ERR_BAD_SHAPE, "head_dim must be 64, 96 or 128");
    if (heads < 1 || heads > 16384 || pages < 1) return fail(SHFLBW_ERR_BAD_SHAPE, "heads must be 1 to 16384, pages 1 or more");
    if (heads * (head_dim / 32) > 65535) return fail(SHFLBW_ERR_BAD_SHAPE, "more than 65535 blocks of 32 features in all heads");
    if ((int64_t)pages * page_tokens > INT_MAX) return fail(SHFLBW_ERR_BAD_SHAPE, "more than 2^31 - 1 slots");
    return SHFLBW_OK;
}

int check_sequences(const shflbw_kv_cache* c, const shflbw_kv_sequences* s)
{
    if (!s) return fail(SHFLBW_ERR_NULL_ARG, "sequences is NULL");
    if (s->batch < 0 || s->tokens < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "batch < 0 or tokens < 0");
    if (s->q_heads < 1 || s->q_heads % c->heads) return fail(SHFLBW_ERR_BAD_SHAPE, "q_heads must be a multiple of the cache's heads (%d)", c->heads);
    if (s->q_heads > 65535) return fail(SHFLBW_ERR_BAD_SHAPE, "more than 65535 query heads");
    if (s->window < 0 || s->sinks < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "window and sinks must be >= 0");
    if (s->max_queries < 1) return fail(SHFLBW_ERR_BAD_SHAPE, "max_queries < 1");
    if (s->max_length < 1 || s->max_length > (int64_t)s->table_pages * c->page_tokens)
        return fail(SHFLBW_ERR_BAD_SHAPE, "max_length must lie between 1 and the tokens of table_pages pages");
    if (s->table_pages < 1 || s->table_ld < s->table_pages) return fail(SHFLBW_ERR_BAD_SHAPE, "table_pages < 1 or table_ld < table_pages");
    if ((int64_t)s->table_pages * c->page_tokens > INT_MAX - 1024) return fail(SHFLBW_ERR_BAD_SHAPE, "more than 2^31 tokens in a sequence's pages");
    if (s->tokens > INT_MAX) return fail(SHFLBW_ERR_BAD_SHAPE, "more than 2^31 - 1 tokens");
    if (!s->starts && (s->tokens != s->batch || s->max_queries != 1))
        return fail(SHFLBW_ERR_BAD_SHAPE, "without starts every sequence has one query: tokens must be batch and max_queries 1");
    return SHFLBW_OK;
}

AttnPlan plan_of(const shflbw_kv_cache* c, const shflbw_kv_sequences* s)
{
    return plan_cache_attention(s->batch, c->heads, s->q_heads / c->heads, c->head_dim, s->tokens, s->max_queries, s->max_length,
                                s->window ? s->window : INT_MAX, s->sinks);
}

}  // namespace

int check_cache(const shflbw_kv_cache* c)
{
    if (!c || !c->data) return fail(SHFLBW_ERR_NULL_ARG, "cache or its data is NULL");
    const int rc = check_sizes(c->pages, c->page_tokens, c->heads, c->head_dim);
    if (rc < 0) return rc;
    if (c->dtype != SHFLBW_F16 && c->dtype != SHFLBW_BF16) return fail(SHFLBW_ERR_BAD_DTYPE, "dtype must be SHFLBW_F16 or SHFLBW_BF16");
    if (reinterpret_cast<uintptr_t>(c->data) % 128) return fail(SHFLBW_ERR_BAD_SHAPE, "the cache's data must be 128-byte aligned");
    return SHFLBW_OK;
}

}  // namespace shflbw

extern "C" {

size_t shflbw_kv_cache_bytes(int pages, int page_tokens, int heads, int head_dim)
{
    using namespace shflbw;
    if (check_sizes(pages, page_tokens, heads, head_dim) < 0) return 0;
    return (size_t)pages * (size_t)heads * (size_t)page_head_bytes(page_tokens, head_dim);
}

int64_t shflbw_kv_attention_workspace(const shflbw_kv_cache* cache, const shflbw_kv_sequences* sequences)
{
    using namespace shflbw;
    int rc = check_cache(cache);
    if (rc < 0 || (rc = check_sequences(cache, sequences)) < 0) return rc;
    return sequences->batch ? plan_of(cache, sequences).workspace : 0;
}

int shflbw_kv_attention(const shflbw_kv_cache* cache, const shflbw_kv_sequences* s, const void* q, int64_t ldq, void* out, int64_t ldo,
                        void* workspace, int64_t workspace_bytes, void* stream)
{
    using namespace shflbw;
    int rc = check_cache(cache);
    if (rc < 0 || (rc = check_sequences(cache, s)) < 0) return rc;
    if (s->batch == 0 || s->tokens == 0) return SHFLBW_OK;
    if (!q || !out || !s->table || !s->lengths) return fail(SHFLBW_ERR_NULL_ARG, "q, out, table and lengths must not be NULL");
    if (ldq < s->tokens || ldo < s->tokens) return fail(SHFLBW_ERR_BAD_SHAPE, "leading dimension too small");
    const AttnPlan plan = plan_of(cache, s);
    if (plan.workspace > workspace_bytes || (plan.workspace && !workspace))
        return fail(SHFLBW_ERR_NULL_ARG, "the call needs a workspace of %lld bytes", (long long)plan.workspace);
    if (plan.workspace && reinterpret_cast<uintptr_t>(workspace) % 16) return fail(SHFLBW_ERR_BAD_SHAPE, "the workspace must be 16-byte aligned");
    AttnArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.cache = static_cast<const char*>(cache->data);
    a.table = s->table;
    a.lengths = s->lengths;
    a.starts = s->starts;
    a.out = static_cast<uint16_t*>(out);
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.part_o + (int64_t)plan.splits * s->q_heads * s->tokens * cache->head_dim;
    a.ldq = ldq; a.ldo = ldo;
    a.table_ld = s->table_ld;
    a.tokens = s->tokens;
    a.table_width = s->table_pages;
    a.batch = s->batch;
    a.heads = cache->heads;
    a.group = s->q_heads / cache->heads;
    a.pages = cache->pages;
    a.page_shift = __builtin_ctz(cache->page_tokens);
    a.window = s->window ? s->window : INT_MAX;
    a.sinks = s->sinks;
    a.scale = softmax_scale(cache->head_dim);
    a.splits = plan.splits;
    a.split_tiles = plan.split_tiles;
    a.col_blocks = plan.col_blocks;
    return cache->dtype == SHFLBW_BF16 ? run_attention_bf16(a, plan, cache->head_dim, false, stream)
                                       : run_attention_f16(a, plan, cache->head_dim, false, stream);
}

int shflbw_window_attention(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, void* out, int64_t ldo,
                            int q_heads, int heads, int head_dim, int64_t tokens, const int32_t* starts, int sequences, int64_t max_tokens,
                            int window, int sinks, shflbw_dtype dtype, void* stream)
{
    using namespace shflbw;
    if (dtype != SHFLBW_F16 && dtype != SHFLBW_BF16) return fail(SHFLBW_ERR_BAD_DTYPE, "dtype must be SHFLBW_F16 or SHFLBW_BF16");
    if (!head_dim_ok(head_dim)) return fail(SHFLBW_ERR_BAD_SHAPE, "head_dim must be 64, 96 or 128");
    if (heads < 1 || q_heads < 1 || q_heads % heads) return fail(SHFLBW_ERR_BAD_SHAPE, "q_heads must be a multiple of heads");
    if (tokens < 0 || tokens > INT_MAX - 1024 || sequences < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "tokens must be 0 to 2^31 - 1025, sequences >= 0");
    if (!starts && sequences != 1) return fail(SHFLBW_ERR_BAD_SHAPE, "without starts there is one sequence");
    if (max_tokens < 0 || max_tokens > tokens) return fail(SHFLBW_ERR_BAD_SHAPE, "max_tokens must be 0 to tokens");
    if (window < 0 || sinks < 0) return fail(SHFLBW_ERR_BAD_SHAPE, "window and sinks must be >= 0");
    if (tokens == 0 || sequences == 0 || max_tokens == 0) return SHFLBW_OK;
    if (!q || !k || !v || !out) return fail(SHFLBW_ERR_NULL_ARG, "q, k, v and out must not be NULL");
    if (ldq < tokens || ldk < tokens || ldv < tokens || ldo < tokens) return fail(SHFLBW_ERR_BAD_SHAPE, "leading dimension too small");
    if (ldk >= ATTN_MAX_LD || ldv >= ATTN_MAX_LD) return fail(SHFLBW_ERR_BAD_SHAPE, "leading dimensions of k and v must be below 2^26");
    const AttnPlan plan = plan_prompt(sequences, heads, q_heads / heads, head_dim, max_tokens, window ? window : INT_MAX, sinks, tokens);
    AttnArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.out = static_cast<uint16_t*>(out);
    a.starts = starts;
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo;
    a.tokens = tokens;
    a.batch = sequences;
    a.heads = heads;
    a.group = q_heads / heads;
    a.window = window ? window : INT_MAX;
    a.sinks = sinks;
    a.scale = softmax_scale(head_dim);
    a.splits = plan.splits;
    a.split_tiles = plan.split_tiles;
    a.col_blocks = plan.col_blocks;
    return dtype == SHFLBW_BF16 ? run_attention_bf16(a, plan, head_dim, true, stream) : run_attention_f16(a, plan, head_dim, true, stream);
}

}  // extern "C"
