// C-ABI entry points of a serving step (tri_append, tri_attend, tri_attend_shared): host-side validation and dispatch.
#include <algorithm>
#include <cmath>

#include "tri_serve.h"

namespace tri {

static int elem_bytes(const tri_cache &c) { return c.dtype == TRI_BF16 ? 2 : 4; }

tri_status check_layer(const tri_model *m, const tri_cache *c, int32_t layer, const char *what)
{
    if (layer < 0 || layer >= m->n_layers) {
        set_error("%s: layer %d of %d", what, layer, m->n_layers);
        return TRI_ERR_INVALID_ARG;
    }
    if (c->n_blocks < 0) {
        set_error("%s: n_blocks %d", what, c->n_blocks);
        return TRI_ERR_INVALID_ARG;
    }
    if ((int64_t)c->n_seqs * m->n_kv_heads > 65535) {
        set_error("%s: n_seqs * n_kv_heads must be below 65536", what);
        return TRI_ERR_UNSUPPORTED;
    }
    return TRI_OK;
}

tri_status check_tokens(const tri_cache *c, const tri_tokens *t, const char *what)
{
    if (!t) {
        set_error("%s: tokens is NULL", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (t->n_tokens < 0 || (!t->start && t->n_tokens != c->n_seqs)) {
        set_error("%s: n_tokens %d (without start, one per sequence: %d)", what, t->n_tokens, c->n_seqs);
        return TRI_ERR_INVALID_ARG;
    }
    if (t->start && t->n_tokens > 0 && (t->max_tokens < 1 || t->max_tokens > t->n_tokens)) {
        set_error("%s: max_tokens %d is not in [1, n_tokens = %d]", what, t->max_tokens, t->n_tokens);
        return TRI_ERR_INVALID_ARG;
    }
    if (t->start && !t->pos && t->n_tokens > 0) {
        set_error("%s: pos required where start is given", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (t->rotated != 0 && t->rotated != 1) {
        set_error("%s: rotated must be 0 or 1", what);
        return TRI_ERR_INVALID_ARG;
    }
    return TRI_OK;
}

tri_status check_rows(const void *p, int64_t stride_token, int64_t stride_head, int eb, const char *what, const char *which)
{
    const int64_t a16 = 16 / eb;
    if (!p || ((uintptr_t)p & 15) || stride_token < 0 || stride_head < 0 || stride_token % a16 || stride_head % a16) {
        set_error("%s: %s must be 16-byte aligned, with strides that are and are not negative", what, which);
        return TRI_ERR_INVALID_ARG;
    }
    return TRI_OK;
}

int32_t most_tokens(const tri_tokens &t) { return t.start ? std::max(t.max_tokens, 1) : 1; }

namespace {

struct AttendPlan {
    AttendSplit own, prefix;
    int32_t parts;    // 0: no partial results
    int64_t groups;   // of the largest launch
    size_t o_bytes, ml_bytes, total;
};

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

AttendPlan attend_plan(const tri_model &m, const tri_cache *prefix, const tri_cache &c, const tri_tokens &t)
{
    AttendPlan p{};
    p.own = attend_split(m, c, most_tokens(t), t.n_tokens);
    if (prefix) p.prefix = attend_split(m, *prefix, std::max(t.n_tokens, 1), t.n_tokens);
    p.parts = p.own.n_split + p.prefix.n_split;
    if (p.parts == 1) p.parts = 0;
    const size_t rows = (size_t)t.n_tokens * m.n_q_heads;
    p.groups = std::max(p.own.groups + p.prefix.groups, p.parts ? join_groups((int64_t)rows, p.parts) : 0);   // (both caches may go in one launch)
    p.o_bytes = up256(p.parts * rows * kHeadDim * sizeof(float));
    p.ml_bytes = up256(p.parts * rows * sizeof(float2));
    p.total = p.o_bytes + p.ml_bytes;
    return p;
}

// What the workspace's size needs of the arguments: geometry and bounds, no pointers but the model's and tokens->start.
tri_status check_bounds(const tri_model *model, const tri_cache *prefix, const tri_cache *cache, const tri_tokens *tokens, const char *what)
{
    tri_status rc = check_model(model);
    if (rc != TRI_OK) return rc;
    if (!cache || cache->n_seqs < 1 || cache->max_seq_len < 0 || (prefix && (prefix->n_seqs < 1 || prefix->max_seq_len < 0))) {
        set_error("%s: caches with n_seqs >= 1 and max_seq_len >= 0 required", what);
        return TRI_ERR_INVALID_ARG;
    }
    if ((cache->dtype != TRI_F32 && cache->dtype != TRI_BF16) || (prefix && prefix->dtype != cache->dtype)) {
        set_error("%s: dtype %d, the prefix's %d", what, cache->dtype, prefix ? prefix->dtype : cache->dtype);
        return TRI_ERR_INVALID_ARG;
    }
    if ((rc = check_tokens(cache, tokens, what)) != TRI_OK) return rc;
    const int64_t rows = (int64_t)tokens->n_tokens * model->n_q_heads;
    for (const tri_cache *c : {cache, prefix})
        if (c && (int64_t)c->n_seqs * model->n_kv_heads > 65535) {
            set_error("%s: n_seqs * n_kv_heads must be below 65536", what);
            return TRI_ERR_UNSUPPORTED;
        }
    if (rows > 0x7fffffff) {
        set_error("%s: %lld rows of queries exceed what one call takes; split the batch", what, (long long)rows);
        return TRI_ERR_UNSUPPORTED;
    }
    const int64_t groups = attend_plan(*model, prefix, *cache, *tokens).groups;
    if (groups > kMostGroups) {
        set_error("%s: %lld workgroups exceed what one launch takes; split the batch", what, (long long)groups);
        return TRI_ERR_UNSUPPORTED;
    }
    return TRI_OK;
}

tri_status attend(const tri_model *model, const tri_cache *prefix, const int32_t *group, const tri_cache *cache, int32_t layer,
                  const tri_tokens *tokens, const tri_attention *at, void *ws, size_t ws_bytes, hipStream_t st, const char *what)
{
    tri_status rc = check_model(model);
    if (rc != TRI_OK) return rc;
    if ((rc = check_cache(model, cache, true, what)) != TRI_OK) return rc;
    if ((rc = check_layer(model, cache, layer, what)) != TRI_OK) return rc;
    if ((rc = check_bounds(model, prefix, cache, tokens, what)) != TRI_OK) return rc;
    if (prefix) {
        if ((rc = check_cache(model, prefix, true, what)) != TRI_OK) return rc;
        if ((rc = check_layer(model, prefix, layer, what)) != TRI_OK) return rc;
        if (!group && prefix->n_seqs != 1) {
            set_error("%s: without group there is one prefix (n_seqs 1, not %d)", what, prefix->n_seqs);
            return TRI_ERR_INVALID_ARG;
        }
    }
    if (!at || !(at->scale > 0.f) || !std::isfinite(at->scale) || (at->causal != 0 && at->causal != 1)) {
        set_error("%s: attention with a finite scale > 0 and causal 0 or 1 required", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (tokens->n_tokens == 0) return TRI_OK;
    const int eb = elem_bytes(*cache);
    if ((rc = check_rows(at->q, at->q_stride_token, at->q_stride_head, eb, what, "q")) != TRI_OK) return rc;
    if ((rc = check_rows(at->out, at->out_stride_token, at->out_stride_head, eb, what, "out")) != TRI_OK) return rc;
    if (at->out == at->q) {
        set_error("%s: out must not be q", what);
        return TRI_ERR_INVALID_ARG;
    }
    const AttendPlan plan = attend_plan(*model, prefix, *cache, *tokens);
    if (plan.total && (!ws || ((uintptr_t)ws & 255) || ws_bytes < plan.total)) {
        set_error("%s: workspace must be 256-byte aligned and hold %zu bytes (got %zu)", what, plan.total, ws_bytes);
        return TRI_ERR_WORKSPACE;
    }
    AttendArgs a{};
    a.turns = band_turns(model->rope_theta);
    a.start = tokens->start;
    a.pos = tokens->pos ? tokens->pos : cache->cur_pos;
    a.q = (const char *)at->q;
    a.out = (char *)at->out;
    a.q_stride_token = at->q_stride_token;
    a.q_stride_head = at->q_stride_head;
    a.out_stride_token = at->out_stride_token;
    a.out_stride_head = at->out_stride_head;
    a.part_o = plan.parts ? (float *)ws : nullptr;
    a.part_ml = plan.parts ? (float2 *)((char *)ws + plan.o_bytes) : nullptr;
    a.scale_log2 = (float)((double)at->scale * 1.44269504088896340736);
    a.n_steps_seqs = cache->n_seqs;
    a.layer = layer;
    a.n_tokens = tokens->n_tokens;
    a.group_size = model->n_q_heads / model->n_kv_heads;
    a.causal = at->causal;
    a.rotate_q = !tokens->rotated;
    a.half = model->pairs == TRI_PAIR_HALF;
    const AttendSource own{make_view(*model, *cache), nullptr, tokens->head_len, cache->n_blocks, 0, most_tokens(*tokens), plan.own.n_split, 0, plan.own.least_keys, plan.own.fill, plan.own.fill_keys,
                           most_tokens(*tokens) > 1};
    if (prefix) {
        a.src = AttendSource{make_view(*model, *prefix), group, nullptr, prefix->n_blocks, group ? 0 : 1, tokens->n_tokens, plan.prefix.n_split, plan.own.n_split,
                             plan.prefix.least_keys, plan.prefix.fill, plan.prefix.fill_keys, 0};
        a.other = own;
        rc = launch_attend_both(a, *prefix, *cache, st);
    } else {
        a.src = own;
        rc = launch_attend(a, *cache, st);
    }
    if (rc != TRI_OK) return rc;
    return plan.parts ? launch_join(a, plan.parts, model->n_q_heads, cache->dtype, st) : TRI_OK;
}

}  // namespace

}  // namespace tri

using namespace tri;

extern "C" {

tri_status tri_append(const tri_model *model, const tri_cache *cache, int32_t layer, const tri_tokens *tokens, const void *k_new,
                      const void *v_new, int64_t stride_token, int64_t stride_head, int32_t *new_seq_len, void *stream)
{
    tri_status rc = check_model(model);
    if (rc != TRI_OK) return rc;
    if ((rc = check_cache(model, cache, true, "tri_append")) != TRI_OK) return rc;
    if ((rc = check_layer(model, cache, layer, "tri_append")) != TRI_OK) return rc;
    if ((rc = check_tokens(cache, tokens, "tri_append")) != TRI_OK) return rc;
    if (tokens->rotated && !cache->k_rotated) {
        set_error("tri_append: rotated rows for a cache of pre-RoPE keys");
        return TRI_ERR_UNSUPPORTED;
    }
    if (new_seq_len && (new_seq_len == cache->seq_len || new_seq_len == tokens->head_len)) {
        set_error("tri_append: new_seq_len must not be the lengths that the call reads");
        return TRI_ERR_INVALID_ARG;
    }
    const int eb = elem_bytes(*cache);
    if (tokens->n_tokens > 0) {
        if ((rc = check_rows(k_new, stride_token, stride_head, eb, "tri_append", "k_new")) != TRI_OK) return rc;
        if ((rc = check_rows(v_new, stride_token, stride_head, eb, "tri_append", "v_new")) != TRI_OK) return rc;
    }
    if (append_threads((int64_t)tokens->n_tokens * model->n_kv_heads, cache->dtype) > kMostGroups * 256) {
        set_error("tri_append: %d tokens exceed what one call takes; split the batch", tokens->n_tokens);
        return TRI_ERR_UNSUPPORTED;
    }
    AppendArgs a{};
    a.cache = make_view(*model, *cache);
    a.rotate = cache->k_rotated && !tokens->rotated;
    if (a.rotate) a.turns = band_turns(model->rope_theta);
    a.start = tokens->start;
    a.pos = tokens->pos ? tokens->pos : cache->cur_pos;
    a.head_len = tokens->head_len;
    a.k_new = (const char *)k_new;
    a.v_new = (const char *)v_new;
    a.new_seq_len = new_seq_len;
    a.stride_token = stride_token;
    a.stride_head = stride_head;
    a.layer = layer;
    a.n_tokens = tokens->n_tokens;
    a.n_blocks = cache->n_blocks;
    a.half = model->pairs == TRI_PAIR_HALF;
    return launch_append(a, cache->dtype, (hipStream_t)stream);
}

size_t tri_attend_workspace_size(const tri_model *model, const tri_cache *prefix, const tri_cache *cache, const tri_tokens *tokens)
{
    if (check_bounds(model, prefix, cache, tokens, "tri_attend_workspace_size") != TRI_OK) return (size_t)-1;
    return attend_plan(*model, prefix, *cache, *tokens).total;
}

tri_status tri_attend(const tri_model *model, const tri_cache *cache, int32_t layer, const tri_tokens *tokens,
                      const tri_attention *attention, void *workspace, size_t ws_bytes, void *stream)
{
    return attend(model, nullptr, nullptr, cache, layer, tokens, attention, workspace, ws_bytes, (hipStream_t)stream, "tri_attend");
}

tri_status tri_attend_shared(const tri_model *model, const tri_cache *prefix, const int32_t *group, const tri_cache *cache,
                             int32_t layer, const tri_tokens *tokens, const tri_attention *attention, void *workspace,
                             size_t ws_bytes, void *stream)
{
    if (!prefix) {
        set_error("tri_attend_shared: prefix is NULL");
        return TRI_ERR_INVALID_ARG;
    }
    return attend(model, prefix, group, cache, layer, tokens, attention, workspace, ws_bytes, (hipStream_t)stream, "tri_attend_shared");
}

}  // extern "C"
