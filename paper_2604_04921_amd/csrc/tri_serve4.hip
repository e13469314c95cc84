// C-ABI entry points of caches held in 4 bits: host-side validation and dispatch.
#include <algorithm>
#include <cmath>

#include "tri_serve4.h"

namespace tri {

namespace {

// c4 completed: sequences and bounds are those of `like` where it is given (a destination's).
tri_status check_cache4(const tri_model *m, const tri_cache4 *x, const tri_cache *like, int32_t slots, const char *what)
{
    if (!x) {
        set_error("%s: the cache of 4 bits is NULL", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (x->c.dtype != TRI_FP4) {
        set_error("%s: dtype %d of a cache of 4 bits is not TRI_FP4", what, x->c.dtype);
        return TRI_ERR_INVALID_ARG;
    }
    tri_cache c = x->c;
    c.dtype = TRI_BF16;   // (the strides' alignment is said below)
    if (like) c.n_seqs = like->n_seqs, c.seq_len = like->seq_len, c.cur_pos = like->cur_pos, c.max_seq_len = slots;
    const tri_status rc = check_cache(m, &c, true, what);
    if (rc != TRI_OK) return rc;
    if (c.stride_slot % 32 || c.stride_head % 32 || c.stride_layer % 32 || c.stride_seq_or_block % 32) {
        set_error("%s: strides of a cache of 4 bits must be multiples of 32", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (!x->k_scale || !x->v_scale || ((uintptr_t)x->k_scale & 3) || ((uintptr_t)x->v_scale & 3)) {
        set_error("%s: k_scale and v_scale, 4-byte aligned, required", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (c.n_blocks < 0) {
        set_error("%s: n_blocks %d", what, c.n_blocks);
        return TRI_ERR_INVALID_ARG;
    }
    if (c.stride_slot >= (1 << 24)) {
        set_error("%s: slots of a cache of 4 bits must be less than 2^24 elements apart", what);
        return TRI_ERR_UNSUPPORTED;
    }
    if (c.k_rotated != 1) {
        set_error("%s: a cache of 4 bits holds post-RoPE keys (k_rotated 1)", what);
        return TRI_ERR_UNSUPPORTED;
    }
    return TRI_OK;
}

tri_status check_row_type(const tri_cache4 *x, const char *what)
{
    if (x->rows == TRI_F32 || x->rows == TRI_BF16) return TRI_OK;
    set_error("%s: rows of type %d", what, x->rows);
    return TRI_ERR_INVALID_ARG;
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct Plan {
    AttendSplit packed, own;
    int32_t parts;    // 0: no partial results
    int64_t groups;   // of the largest launch
    size_t o_bytes, total;
};

Plan plan_of(const tri_model &m, const tri_cache4 &x, const tri_cache *own, const tri_tokens &t)
{
    Plan p{};
    const int32_t most = own ? std::max(t.n_tokens, 1) : most_tokens(t);
    p.packed = attend4_split(m, x.c, most, t.n_tokens, x.rows);
    if (own) p.own = attend_split(m, *own, most_tokens(t), t.n_tokens);
    p.parts = p.packed.n_split + p.own.n_split;
    if (p.parts == 1) p.parts = 0;
    const size_t rows = (size_t)t.n_tokens * m.n_q_heads;
    p.groups = std::max({p.packed.groups, p.own.groups, p.parts ? join_groups((int64_t)rows, p.parts) : 0});
    p.o_bytes = up256(p.parts * rows * kHeadDim * sizeof(float));
    p.total = p.o_bytes + up256(p.parts * rows * sizeof(float2));
    return p;
}

// What the workspace's size needs of the arguments: geometry and bounds, no pointers but the model's and tokens->start.
tri_status check_bounds4(const tri_model *model, const tri_cache4 *x, const tri_cache *own, const tri_tokens *tokens, const char *what)
{
    tri_status rc = check_model(model);
    if (rc != TRI_OK) return rc;
    if (!x || x->c.n_seqs < 1 || x->c.max_seq_len < 0 || (own && (own->n_seqs < 1 || own->max_seq_len < 0))) {
        set_error("%s: caches with n_seqs >= 1 and max_seq_len >= 0 required", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (x->c.dtype != TRI_FP4 || (own && own->dtype != x->rows)) {
        set_error("%s: dtype %d of a cache of 4 bits, rows of type %d, the sequences' own of type %d", what, x->c.dtype, x->rows, own ? own->dtype : x->rows);
        return TRI_ERR_INVALID_ARG;
    }
    if (x->c.max_seq_len > 0x7fffffff - 4096) {   // (kernels look a few tiles of keys ahead)
        set_error("%s: max_seq_len of a cache of 4 bits must be at most 2^31 - 4097", what);
        return TRI_ERR_UNSUPPORTED;
    }
    if ((rc = check_row_type(x, what)) != TRI_OK) return rc;
    if ((rc = check_tokens(own ? own : &x->c, tokens, what)) != TRI_OK) return rc;
    for (const tri_cache *c : {&x->c, own})
        if (c && (int64_t)c->n_seqs * model->n_kv_heads > 65535) {
            set_error("%s: n_seqs * n_kv_heads must be below 65536", what);
            return TRI_ERR_UNSUPPORTED;
        }
    if ((int64_t)tokens->n_tokens * model->n_q_heads > 0x7fffffff) {
        set_error("%s: %lld rows of queries exceed what one call takes; split the batch", what, (long long)tokens->n_tokens * model->n_q_heads);
        return TRI_ERR_UNSUPPORTED;
    }
    const int64_t groups = plan_of(*model, *x, own, *tokens).groups;
    if (groups > kMostGroups) {
        set_error("%s: %lld workgroups exceed what one launch takes; split the batch", what, (long long)groups);
        return TRI_ERR_UNSUPPORTED;
    }
    return TRI_OK;
}

// own: the sequences' own caches, x being their prefixes'; or NULL
tri_status attend4(const tri_model *model, const tri_cache4 *x, const int32_t *group, const tri_cache *own, int32_t layer, const tri_tokens *tokens,
                   const tri_attention *at, void *ws, size_t ws_bytes, hipStream_t st, const char *what)
{
    tri_status rc = check_model(model);
    if (rc != TRI_OK) return rc;
    if ((rc = check_cache4(model, x, nullptr, 0, what)) != TRI_OK) return rc;
    if ((rc = check_layer(model, &x->c, layer, what)) != TRI_OK) return rc;
    if (own) {
        if ((rc = check_cache(model, own, true, what)) != TRI_OK) return rc;
        if ((rc = check_layer(model, own, layer, what)) != TRI_OK) return rc;
        if (!group && x->c.n_seqs != 1) {
            set_error("%s: without group there is one prefix (n_seqs 1, not %d)", what, x->c.n_seqs);
            return TRI_ERR_INVALID_ARG;
        }
    }
    if ((rc = check_bounds4(model, x, own, tokens, what)) != TRI_OK) return rc;
    if (!at || !(at->scale > 0.f) || !std::isfinite(at->scale) || (at->causal != 0 && at->causal != 1)) {
        set_error("%s: attention with a finite scale > 0 and causal 0 or 1 required", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (tokens->n_tokens == 0) return TRI_OK;
    const int eb = x->rows == TRI_BF16 ? 2 : 4;
    if ((rc = check_rows(at->q, at->q_stride_token, at->q_stride_head, eb, what, "q")) != TRI_OK) return rc;
    if ((rc = check_rows(at->out, at->out_stride_token, at->out_stride_head, eb, what, "out")) != TRI_OK) return rc;
    if (at->out == at->q) {
        set_error("%s: out must not be q", what);
        return TRI_ERR_INVALID_ARG;
    }
    const Plan plan = plan_of(*model, *x, own, *tokens);
    if (plan.total && (!ws || ((uintptr_t)ws & 255) || ws_bytes < plan.total)) {
        set_error("%s: workspace must be 256-byte aligned and hold %zu bytes (got %zu)", what, plan.total, ws_bytes);
        return TRI_ERR_WORKSPACE;
    }
    const tri_cache &steps = own ? *own : x->c;   // whose sequences the tokens are
    AttendArgs a{};
    a.k_scale = x->k_scale;
    a.v_scale = x->v_scale;
    a.turns = band_turns(model->rope_theta);
    a.start = tokens->start;
    a.pos = tokens->pos ? tokens->pos : steps.cur_pos;
    a.q = (const char *)at->q;
    a.out = (char *)at->out;
    a.q_stride_token = at->q_stride_token;
    a.q_stride_head = at->q_stride_head;
    a.out_stride_token = at->out_stride_token;
    a.out_stride_head = at->out_stride_head;
    a.part_o = plan.parts ? (float *)ws : nullptr;
    a.part_ml = plan.parts ? (float2 *)((char *)ws + plan.o_bytes) : nullptr;
    a.scale_log2 = (float)((double)at->scale * 1.44269504088896340736);
    a.n_steps_seqs = steps.n_seqs;
    a.layer = layer;
    a.n_tokens = tokens->n_tokens;
    a.group_size = model->n_q_heads / model->n_kv_heads;
    a.causal = at->causal;
    a.rotate_q = !tokens->rotated;
    a.half = model->pairs == TRI_PAIR_HALF;
    a.src = AttendSource{make_view(*model, x->c), own ? group : nullptr, own ? nullptr : tokens->head_len, x->c.n_blocks, own && !group ? 1 : 0, own ? tokens->n_tokens : most_tokens(*tokens),
                         plan.packed.n_split, 0, plan.packed.least_keys, plan.packed.fill, plan.packed.fill_keys, !own && most_tokens(*tokens) > 1};
    if ((rc = launch_attend4(a, x->rows, st)) != TRI_OK) return rc;
    if (own) {
        a.src = AttendSource{make_view(*model, *own), nullptr, tokens->head_len, own->n_blocks, 0, most_tokens(*tokens), plan.own.n_split, plan.packed.n_split, plan.own.least_keys, plan.own.fill,
                             plan.own.fill_keys, most_tokens(*tokens) > 1};
        if ((rc = launch_attend(a, *own, st)) != TRI_OK) return rc;
    }
    return plan.parts ? launch_join(a, plan.parts, model->n_q_heads, x->rows, st) : TRI_OK;
}

// The checks of tri_pack4 and tri_unpack4 (which of src and dst is in 4 bits being x), and their launch.
tri_status move(const tri_model *model, const tri_cache *src, const tri_cache *dst, const tri_cache4 *x, bool pack, int32_t budget, const int32_t *kept_idx, const int32_t *kept_cnt,
                int32_t *new_seq_len, hipStream_t st, const char *what)
{
    tri_status rc = check_model(model);
    if (rc != TRI_OK) return rc;
    if (budget < 1) {
        set_error("%s: budget %d", what, budget);
        return TRI_ERR_INVALID_ARG;
    }
    if ((rc = pack ? check_cache(model, src, true, what) : check_cache4(model, x, nullptr, 0, what)) != TRI_OK) return rc;
    if (!dst) {
        set_error("%s: dst is NULL", what);
        return TRI_ERR_INVALID_ARG;
    }
    const int32_t slots = std::min(budget, src->max_seq_len);
    tri_cache d = *dst;
    d.n_seqs = src->n_seqs, d.seq_len = src->seq_len, d.cur_pos = src->cur_pos, d.max_seq_len = slots;
    if ((rc = pack ? check_cache4(model, x, src, slots, what) : check_cache(model, &d, true, what)) != TRI_OK) return rc;
    if (dst->k == src->k || dst->v == src->v || dst->pos == src->pos) {
        set_error("%s: src and dst must not overlap", what);
        return TRI_ERR_INVALID_ARG;
    }
    if (src->n_blocks < 0 || dst->n_blocks < 0) {
        set_error("%s: n_blocks %d, %d", what, src->n_blocks, dst->n_blocks);
        return TRI_ERR_INVALID_ARG;
    }
    if (!pack && dst->k_rotated != 1) {
        set_error("%s: what is read back is post-RoPE (dst with k_rotated 1)", what);
        return TRI_ERR_UNSUPPORTED;
    }
    if (new_seq_len && (new_seq_len == src->seq_len || new_seq_len == kept_cnt)) {
        set_error("%s: new_seq_len must not be the lengths that the call reads", what);
        return TRI_ERR_INVALID_ARG;
    }
    Pack4Args a{};
    a.row_blocks = pack ? pack4_row_blocks(slots) : unpack4_row_blocks(slots);
    const int64_t groups = (int64_t)model->n_layers * src->n_seqs * model->n_kv_heads * a.row_blocks;
    if (groups > kMostGroups) {
        set_error("%s: %d layers of %d sequences of up to %d slots exceed what one call takes; split the batch", what, model->n_layers, src->n_seqs, slots);
        return TRI_ERR_UNSUPPORTED;
    }
    if (slots == 0 && !new_seq_len) return TRI_OK;
    a.src = make_view(*model, *src);
    a.dst = make_view(*model, d);
    a.kept_idx = kept_idx;
    a.kept_cnt = kept_cnt;
    a.new_seq_len = new_seq_len;
    a.k_scale = x->k_scale;
    a.v_scale = x->v_scale;
    a.budget = budget;
    a.slots = slots;
    a.src_blocks = src->n_blocks;
    a.dst_blocks = dst->n_blocks;
    if (!pack) return launch_unpack4(a, groups, dst->dtype, st);
    const bool turn = !src->k_rotated;
    if (turn) a.turns = band_turns(model->rope_theta);
    return launch_pack4(a, groups, src->dtype, turn, model->pairs == TRI_PAIR_HALF, st);
}

}  // namespace

}  // namespace tri

using namespace tri;

extern "C" {

tri_status tri_append4(const tri_model *model, const tri_cache4 *cache, int32_t layer, const tri_tokens *tokens, const void *k_new,
                       const void *v_new, int64_t stride_token, int64_t stride_head, int32_t *new_seq_len, void *stream)
{
    tri_status rc = check_model(model);
    if (rc != TRI_OK) return rc;
    if ((rc = check_cache4(model, cache, nullptr, 0, "tri_append4")) != TRI_OK) return rc;
    if ((rc = check_row_type(cache, "tri_append4")) != TRI_OK) return rc;
    const tri_cache &c = cache->c;
    if ((rc = check_layer(model, &c, layer, "tri_append4")) != TRI_OK) return rc;
    if ((rc = check_tokens(&c, tokens, "tri_append4")) != TRI_OK) return rc;
    if (new_seq_len && (new_seq_len == c.seq_len || new_seq_len == tokens->head_len)) {
        set_error("tri_append4: new_seq_len must not be the lengths that the call reads");
        return TRI_ERR_INVALID_ARG;
    }
    const int eb = cache->rows == TRI_BF16 ? 2 : 4;
    if (tokens->n_tokens > 0) {
        if ((rc = check_rows(k_new, stride_token, stride_head, eb, "tri_append4", "k_new")) != TRI_OK) return rc;
        if ((rc = check_rows(v_new, stride_token, stride_head, eb, "tri_append4", "v_new")) != TRI_OK) return rc;
    }
    if (append4_groups(tokens->n_tokens, model->n_kv_heads) > kMostGroups) {
        set_error("tri_append4: %d tokens exceed what one call takes; split the batch", tokens->n_tokens);
        return TRI_ERR_UNSUPPORTED;
    }
    Append4Args args{};
    AppendArgs &a = args.a;
    args.k_scale = cache->k_scale;
    args.v_scale = cache->v_scale;
    a.cache = make_view(*model, c);
    a.rotate = !tokens->rotated;
    if (a.rotate) a.turns = band_turns(model->rope_theta);
    a.start = tokens->start;
    a.pos = tokens->pos ? tokens->pos : c.cur_pos;
    a.head_len = tokens->head_len;
    a.k_new = (const char *)k_new;
    a.v_new = (const char *)v_new;
    a.new_seq_len = new_seq_len;
    a.stride_token = stride_token;
    a.stride_head = stride_head;
    a.layer = layer;
    a.n_tokens = tokens->n_tokens;
    a.n_blocks = c.n_blocks;
    a.half = model->pairs == TRI_PAIR_HALF;
    return launch_append4(args, cache->rows, (hipStream_t)stream);
}

tri_status tri_pack4(const tri_model *model, const tri_cache *src, const tri_cache4 *dst, int32_t budget, const int32_t *kept_idx,
                     const int32_t *kept_cnt, int32_t *new_seq_len, void *stream)
{
    return move(model, src, dst ? &dst->c : nullptr, dst, true, budget, kept_idx, kept_cnt, new_seq_len, (hipStream_t)stream, "tri_pack4");
}

tri_status tri_unpack4(const tri_model *model, const tri_cache4 *src, const tri_cache *dst, int32_t budget, const int32_t *kept_idx,
                       const int32_t *kept_cnt, int32_t *new_seq_len, void *stream)
{
    return move(model, src ? &src->c : nullptr, dst, src, false, budget, kept_idx, kept_cnt, new_seq_len, (hipStream_t)stream, "tri_unpack4");
}

size_t tri_attend4_workspace_size(const tri_model *model, const tri_cache4 *cache, const tri_cache *own, const tri_tokens *tokens)
{
    if (check_bounds4(model, cache, own, tokens, "tri_attend4_workspace_size") != TRI_OK) return (size_t)-1;
    return plan_of(*model, *cache, own, *tokens).total;
}

tri_status tri_attend4(const tri_model *model, const tri_cache4 *cache, int32_t layer, const tri_tokens *tokens,
                       const tri_attention *attention, void *workspace, size_t ws_bytes, void *stream)
{
    return attend4(model, cache, nullptr, nullptr, layer, tokens, attention, workspace, ws_bytes, (hipStream_t)stream, "tri_attend4");
}

tri_status tri_attend4_shared(const tri_model *model, const tri_cache4 *prefix, const int32_t *group, const tri_cache *cache,
                              int32_t layer, const tri_tokens *tokens, const tri_attention *attention, void *workspace,
                              size_t ws_bytes, void *stream)
{
    if (!cache) {
        set_error("tri_attend4_shared: cache is NULL");
        return TRI_ERR_INVALID_ARG;
    }
    return attend4(model, prefix, group, cache, layer, tokens, attention, workspace, ws_bytes, (hipStream_t)stream, "tri_attend4_shared");
}

}  // extern "C"
