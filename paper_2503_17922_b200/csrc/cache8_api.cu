// Host side of the norms with rotary positions, the 8-bit cache and drafted tokens: validation and kernel choice.
#include "cache_common.cuh"

using namespace wkv;

namespace {

int check_norm(const wkv_head_norm *n)
{
    if (n->struct_size != sizeof(wkv_head_norm)) {
        set_error_detail("norm: struct_size %u != %zu", n->struct_size, sizeof(wkv_head_norm));
        return WKV_ERR_SHAPE;
    }
    if (!(n->eps >= 0.f) || !isfinite(n->eps) || !isfinite(n->offset) || n->reserved != 0) {
        set_error_detail("norm: eps %g (finite, >= 0), offset %g (finite) or reserved word not 0", n->eps, n->offset);
        return WKV_ERR_SHAPE;
    }
    return WKV_OK;
}
// `tokens`: positions of one axis
int check_axes(const wkv_rope_axes *x, bool turned, const void *positions, long long tokens)
{
    if (x->struct_size != sizeof(wkv_rope_axes)) {
        set_error_detail("axes: struct_size %u != %zu", x->struct_size, sizeof(wkv_rope_axes));
        return WKV_ERR_SHAPE;
    }
    if (x->n_axes < 1 || x->position_stride < tokens || !turned) {
        set_error_detail("axes: %d of them, %lld positions to an axis and %lld between two, or no rope", x->n_axes, tokens, (long long)x->position_stride);
        return WKV_ERR_SHAPE;
    }
    if (!x->axis) return missing("axes: axis");
    return positions || tokens == 0 ? WKV_OK : missing("positions");
}
int check_width(int head_dim, const char *what)
{
    if (head_dim <= kAttnMaxHeadDim) return WKV_OK;
    set_error_detail("%s: head_dim %d beyond %d", what, head_dim, kAttnMaxHeadDim);
    return WKV_ERR_UNSUPPORTED;
}
void set_turn(const wkv_head_norm *norm, const wkv_rope_axes *axes, TurnArgs &t)
{
    t.norm = norm != nullptr;
    t.eps = norm ? norm->eps : 0.f;
    t.offset = norm ? norm->offset : 0.f;
    t.q_weight = norm ? norm->q_weight : nullptr;
    t.k_weight = norm ? norm->k_weight : nullptr;
    t.n_axes = axes ? axes->n_axes : 1;
    t.axis = axes ? axes->axis : nullptr;
    t.position_stride = axes ? axes->position_stride : 0;
    t.kind = kPlain;
    t.k_scales = t.v_scales = nullptr;
}

int check_layer(const wkv_cache8 *x, bool values)
{
    if (!x) return missing("layer of the 8-bit cache");
    if (x->struct_size != sizeof(wkv_cache8)) {
        set_error_detail("8-bit cache: struct_size %u != %zu", x->struct_size, sizeof(wkv_cache8));
        return WKV_ERR_SHAPE;
    }
    if (x->type != WKV_CACHE_E4M3 && x->type != WKV_CACHE_I8) {
        set_error_detail("8-bit cache: type %d unknown", x->type);
        return WKV_ERR_DTYPE;
    }
    int st = check_pointer(x->k_codes, "k_codes");
    if (st == WKV_OK && values) st = check_pointer(x->v_codes, "v_codes");
    if (st != WKV_OK) return st;
    if (!x->k_scales || (values && !x->v_scales)) return missing("scales");
    if (values && (x->k_codes == x->v_codes || x->k_scales == x->v_scales)) {
        set_error_detail("8-bit cache: keys and values in one place");
        return WKV_ERR_SHAPE;
    }
    return WKV_OK;
}
int resolve_paged8(const wkv_paged *c, Paged &p)
{
    const int st = resolve_paged(c, p, 1);
    return st != WKV_OK ? st : check_width(c->head_dim, "8-bit cache");
}
// the layers of a call: their pools in one table, K and V in turn
int fill_layers(int n_layers, const wkv_cache8 *layers, bool values, PoolTable &pools, ScaleTable &scales, int &n_tensors)
{
    if (n_layers < 1 || n_layers > WKV_MAX_GROUP_LAYERS) {
        set_error_detail("n_layers %d outside 1..%d", n_layers, WKV_MAX_GROUP_LAYERS);
        return WKV_ERR_LIMIT;
    }
    if (!layers) return missing("layers");
    n_tensors = 0;
    for (int l = 0; l < n_layers; ++l) {
        const int st = check_layer(layers + l, values);
        if (st != WKV_OK) return st;
        if (layers[l].type != layers[0].type) {
            set_error_detail("layer %d is of another type than the first", l);
            return WKV_ERR_DTYPE;
        }
        pools.ptr[n_tensors] = layers[l].k_codes;
        scales.ptr[n_tensors++] = layers[l].k_scales;
        if (!values) continue;
        pools.ptr[n_tensors] = layers[l].v_codes;
        scales.ptr[n_tensors++] = layers[l].v_scales;
    }
    return WKV_OK;
}
Cache8Pages pages_of(const wkv_paged *c)
{
    return {c->block_table, c->max_pages, c->page_size, c->num_pages, c->page_stride, c->head_stride, c->row_stride};
}

constexpr int kFewDraftRows = 64;
constexpr size_t kDraftWithoutBefore = offsetof(wkv_draft, before);
const int32_t *rows_before(const wkv_draft *d) { return d->struct_size == sizeof(wkv_draft) ? d->before : nullptr; }
int check_draft(const wkv_paged *c, const wkv_draft *d)
{
    if (d->struct_size != sizeof(wkv_draft) && d->struct_size != kDraftWithoutBefore) {
        set_error_detail("draft: struct_size %u is neither %zu nor, up to the masks, %zu", d->struct_size, sizeof(wkv_draft), kDraftWithoutBefore);
        return WKV_ERR_SHAPE;
    }
    if (c->max_new > WKV_MAX_DRAFT) {
        set_error_detail("draft: %d tokens of a sequence, at most %d", c->max_new, WKV_MAX_DRAFT);
        return WKV_ERR_LIMIT;
    }
    if (d->words < (c->max_new + 31) / 32) {
        set_error_detail("draft: masks of %d words for %d tokens", d->words, c->max_new);
        return WKV_ERR_SHAPE;
    }
    return d->masks ? WKV_OK : missing("draft: masks");
}

int append(const wkv_paged *c, const wkv_cache8 *layer, const wkv_head_norm *norm, const wkv_rope *rope, const wkv_rope_axes *axes,
           const void *k_new, const void *v_new, const int64_t *kv_strides, const void *q, void *q_out, const int64_t *q_strides,
           const int32_t *positions, const int32_t *lengths, void *k_pool, void *v_pool, int32_t *lengths_out, int32_t *row_positions,
           float *row_weights, const Paged &p, void *cuda_stream)
{
    int st;
    if ((st = check_width(c->head_dim, "norms and rotary positions")) != WKV_OK) return st;
    if (norm && (st = check_norm(norm)) != WKV_OK) return st;
    if (axes && (st = check_axes(axes, rope != nullptr, positions, p.batch_tokens)) != WKV_OK) return st;
    TurnArgs t;
    if ((st = append_args(c, p, rope, k_new, v_new, kv_strides, q, q_out, q_strides, positions, lengths, k_pool, v_pool, lengths_out, row_positions,
                          row_weights, t.r)) != WKV_OK)
        return st;
    set_turn(norm, axes, t);
    if (layer) {
        t.kind = layer->type + 1;
        t.k_scales = layer->k_scales;
        t.v_scales = layer->v_scales;
    }
    return launch_turn(t, c->dtype, static_cast<cudaStream_t>(cuda_stream));
}

int keep_draft(const wkv_paged *c, const Paged &p, const wkv_draft *draft, const PoolTable &pools, const ScaleTable &scales, bool scaled, int n_tensors,
               const int32_t *last, const int32_t *lengths, int32_t *lengths_out, int32_t *row_positions, float *row_weights, void *cuda_stream)
{
    int st;
    if (!draft) return missing("draft");
    // (no new tokens: there are no masks, and the lengths stay)
    const bool none = c->cu_new_host && p.total_new == 0;
    if (!none && (st = check_draft(c, draft)) != WKV_OK) return st;
    if (!last || !lengths || !lengths_out) return missing("last, lengths or lengths_out");
    if (lengths_out == lengths || lengths_out == rows_before(draft)) {
        set_error_detail("lengths_out must not be lengths or the draft's before (other blocks still read them)");
        return WKV_ERR_SHAPE;
    }
    if ((st = check_pools_apart(c)) != WKV_OK) return st;
    DraftArgs a;
    memset(&a, 0, sizeof a);
    a.batch = c->batch;
    a.hkv = c->n_kv_heads;
    a.d = c->head_dim;
    a.elem_bytes = p.pool_eb;
    a.max_q = c->max_new;
    a.total_q = p.total_new;
    a.cu_q = c->cu_new_dev;
    a.masks = none ? nullptr : draft->masks;
    a.words = none ? 0 : draft->words;
    a.pages = pages_of(c);
    a.cap = p.cap;
    a.n_tensors = n_tensors;
    a.scaled = scaled;
    a.last = last;
    a.lengths = lengths;
    a.before = none ? nullptr : rows_before(draft);
    a.lengths_out = lengths_out;
    a.row_positions = row_positions;
    a.row_weights = row_weights;
    return launch_keep_draft(a, pools, scales, static_cast<cudaStream_t>(cuda_stream));
}

}  // namespace

extern "C" {

int wkv_norm_rotate_prompt(const wkv_shape *s, const wkv_head_norm *norm, const wkv_rope *rope, const wkv_rope_axes *axes,
                           const void *q, void *q_out, const int64_t *q_strides, const void *k, void *k_out,
                           const int32_t *positions, void *cuda_stream)
{
    KShape ks;
    int st = resolve(s, ks);
    if (st != WKV_OK) return st;
    if (!norm && !rope) return missing("norm and rope");
    if ((st = check_width(s->head_dim, "norms and rotary positions")) != WKV_OK) return st;
    if (norm && (st = check_norm(norm)) != WKV_OK) return st;
    const bool packed = ks.cu != nullptr;
    const long long tokens = packed ? ks.total_rows : (long long)ks.batch * ks.max_seqlen;
    if (axes && (st = check_axes(axes, rope != nullptr, positions, tokens)) != WKV_OK) return st;
    TurnArgs t;
    if ((st = rotate_args(s, ks, rope, q, q_out, q_strides, k, k_out, positions, t.r)) != WKV_OK) return st;
    set_turn(norm, axes, t);
    return launch_turn(t, s->dtype, static_cast<cudaStream_t>(cuda_stream));
}

int wkv_norm_append_kv_paged(const wkv_paged *c, const wkv_head_norm *norm, const wkv_rope *rope, const wkv_rope_axes *axes,
                             const void *k_new, const void *v_new, const int64_t *kv_strides, const void *q, void *q_out,
                             const int64_t *q_strides, const int32_t *positions, const int32_t *lengths, void *k_pool, void *v_pool,
                             int32_t *lengths_out, int32_t *row_positions, float *row_weights, void *cuda_stream)
{
    Paged p;
    const int st = resolve_paged(c, p);
    if (st != WKV_OK) return st;
    if (!norm && !rope) return missing("norm and rope");
    return append(c, nullptr, norm, rope, axes, k_new, v_new, kv_strides, q, q_out, q_strides, positions, lengths, k_pool, v_pool, lengths_out,
                  row_positions, row_weights, p, cuda_stream);
}

size_t wkv_paged8_workspace_bytes(const wkv_paged *c)
{
    Paged p;
    return resolve_paged8(c, p) == WKV_OK ? plan_paged(c, p).total : 0;
}

int wkv_append_kv_paged8(const wkv_paged *c, const wkv_cache8 *layer, const wkv_head_norm *norm, const wkv_rope *rope,
                         const wkv_rope_axes *axes, const void *k_new, const void *v_new, const int64_t *kv_strides, const void *q,
                         void *q_out, const int64_t *q_strides, const int32_t *positions, const int32_t *lengths,
                         int32_t *lengths_out, int32_t *row_positions, float *row_weights, void *cuda_stream)
{
    Paged p;
    int st = resolve_paged8(c, p);
    if (st != WKV_OK || (st = check_layer(layer, true)) != WKV_OK) return st;
    return append(c, layer, norm, rope, axes, k_new, v_new, kv_strides, q, q_out, q_strides, positions, lengths, layer->k_codes, layer->v_codes, lengths_out,
                  row_positions, row_weights, p, cuda_stream);
}

int wkv_gather_kv_paged8(const wkv_shape *s, const wkv_paged *c, int32_t n_layers, const void *const *k_layers,
                         const void *const *v_layers, const int32_t *window_idx, const wkv_cache8 *layers, void *cuda_stream)
{
    KShape ks;
    Paged p;
    int st = resolve(s, ks);
    if (st != WKV_OK || (st = resolve_paged8(c, p)) != WKV_OK) return st;
    if (c->batch != s->batch || c->n_kv_heads != s->n_kv_heads || c->head_dim != s->head_dim || c->dtype != s->dtype) {
        set_error_detail("8-bit cache of %d sequences, %d KV heads, d %d, type %d for a problem of %d, %d, %d, %d", c->batch, c->n_kv_heads, c->head_dim,
                         c->dtype, s->batch, s->n_kv_heads, s->head_dim, s->dtype);
        return WKV_ERR_SHAPE;
    }
    if (!window_idx) return missing("window_idx");
    if (!k_layers) return missing("k_layers");
    PoolTable pools;
    ScaleTable scales;
    LayerTable src;
    int n_tensors = 0;
    if ((st = fill_layers(n_layers, layers, v_layers != nullptr, pools, scales, n_tensors)) != WKV_OK) return st;
    for (int l = 0, x = 0; l < n_layers; ++l) {
        if ((st = check_pointer(k_layers[l], "a layer's keys")) != WKV_OK) return st;
        src.src[x++] = k_layers[l];
        if (!v_layers) continue;
        if ((st = check_pointer(v_layers[l], "a layer's values")) != WKV_OK) return st;
        src.src[x++] = v_layers[l];
    }
    if (p.cap < wkv_keep_max(s)) {
        set_error_detail("8-bit cache: %d rows of a unit do not cover the %d that it may keep", p.cap, wkv_keep_max(s));
        return WKV_ERR_SHAPE;
    }
    if ((st = check_pools_apart(c)) != WKV_OK) return st;
    return launch_gather8(ks, s->dtype, n_tensors, src, pools, scales, layers[0].type + 1, pages_of(c), window_idx, static_cast<cudaStream_t>(cuda_stream));
}

int wkv_read_kv_paged8(const wkv_paged *c, const wkv_cache8 *layer, const int32_t *first, const int32_t *lengths, int32_t out_dtype,
                       int32_t row_capacity, void *k_out, void *v_out, void *cuda_stream)
{
    Paged p;
    int st = resolve_paged8(c, p);
    if (st != WKV_OK || (st = check_layer(layer, v_out != nullptr)) != WKV_OK) return st;
    if (out_dtype != WKV_F32 && out_dtype != WKV_BF16) {
        set_error_detail("out_dtype %d unknown", out_dtype);
        return WKV_ERR_DTYPE;
    }
    if (!lengths) return missing("lengths");
    if (!k_out && !v_out) return missing("k_out and v_out");
    if ((k_out && (st = check_pointer(k_out, "k_out")) != WKV_OK) || (v_out && (st = check_pointer(v_out, "v_out")) != WKV_OK)) return st;
    if (k_out == v_out || row_capacity < 1) {
        set_error_detail("rows of the 8-bit cache: row_capacity %d, or k_out and v_out in one place", row_capacity);
        return WKV_ERR_SHAPE;
    }
    const void *const codes[2] = {layer->k_codes, layer->v_codes};
    const unsigned char *const scales[2] = {layer->k_scales, layer->v_scales};
    void *const out[2] = {k_out, v_out};
    return launch_read8(c->batch, c->n_kv_heads, c->head_dim, pages_of(c), layer->type + 1, codes, scales, first, lengths, out_dtype, row_capacity, out,
                        static_cast<cudaStream_t>(cuda_stream));
}

int wkv_evict_kv_paged8(const wkv_paged *c, int32_t n_layers, const wkv_cache8 *layers, int32_t budget, const int32_t *budgets,
                        int32_t recent, const float *weights, const int32_t *positions, const int32_t *lengths, float *weights_out,
                        int32_t *positions_out, int32_t *lengths_out, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    Paged p;
    int st = resolve_paged8(c, p), n_tensors = 0;
    if (st != WKV_OK) return st;
    PoolTable pools;
    ScaleTable scales;
    if ((st = check_eviction(budget, recent, weights, positions, lengths, weights_out, positions_out, lengths_out)) != WKV_OK ||
        (st = fill_layers(n_layers, layers, true, pools, scales, n_tensors)) != WKV_OK)
        return st;
    EvictArgs a;
    if ((st = evict_args(c, p, n_tensors, budget, budgets, recent, weights, positions, lengths, weights_out, positions_out, lengths_out, workspace,
                         workspace_bytes, a)) != WKV_OK)
        return st;
    a.scaled = true;
    if ((st = check_once(pools, n_tensors, "pools")) != WKV_OK || (st = check_once(scales, n_tensors, "scales")) != WKV_OK) return st;
    return launch_evict(a, pools, scales, static_cast<cudaStream_t>(cuda_stream));
}

int wkv_draft_masks(const wkv_paged *c, const int32_t *parents, int32_t words, uint32_t *masks, const int32_t *first,
                    int32_t *positions, void *cuda_stream)
{
    Paged p;
    const int st = resolve_paged(c, p);
    if (st != WKV_OK) return st;
    if (c->max_new > WKV_MAX_DRAFT) {
        set_error_detail("draft: %d tokens of a sequence, at most %d", c->max_new, WKV_MAX_DRAFT);
        return WKV_ERR_LIMIT;
    }
    if (words < (c->max_new + 31) / 32) {
        set_error_detail("draft: masks of %d words for %d tokens", words, c->max_new);
        return WKV_ERR_SHAPE;
    }
    if (p.batch_tokens == 0) return WKV_OK;
    if (!parents) return missing("parents");
    if (!masks && !positions) return missing("masks and positions");
    if (positions == parents) {
        set_error_detail("positions must not be parents (other threads still read them)");
        return WKV_ERR_SHAPE;
    }
    return launch_draft_masks(c->batch, c->max_new, p.total_new, c->cu_new_dev, parents, words, masks, first, positions, static_cast<cudaStream_t>(cuda_stream));
}

int wkv_attend_draft_paged(const wkv_paged *c, const wkv_draft *draft, const void *q, const int64_t *q_strides, const void *k_pool,
                           const void *v_pool, const int32_t *lengths, void *out, const int64_t *out_strides, float *lse,
                           void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    Paged p;
    PagedWorkspace w;
    AttnArgs a;
    int st = resolve_paged(c, p);
    if (st != WKV_OK) return st;
    if (!draft) return missing("draft");
    const bool none = c->cu_new_host && p.total_new == 0;
    if (!none && (st = check_draft(c, draft)) != WKV_OK) return st;
    if ((st = attend_args(c, p, q, q_strides, k_pool, v_pool, lengths, out, out_strides, lse, nullptr, nullptr, workspace, workspace_bytes, w, a)) != WKV_OK || none)
        return st;
    a.masks = draft->masks;
    a.mask_words = draft->words;
    a.before = rows_before(draft);
    // A small draft over a short cache: every 16 rows read the keys for themselves, split over the blocks of a cluster, where all of those
    // run at once.  (12 tokens of 32 heads on 8, d = 128: the attention over 992 rows 12.1 us, 22.3 on the tensor cores, 4,000 rows 23.0 and 31.2, 8,000
    // rows, where a block's share reaches kClusterBytes, 38.3 and 36.3.)
    bool clustered = false;
    const int splits = c->dtype == WKV_BF16 && p.rows_max > 16 && p.rows_max <= kFewDraftRows ? plan_splits(c, p, 16, clustered) : 0;
    if (clustered && splits > 1) {
        a.few = a.clustered = true;
        a.splits = splits;
    }
    return launch_attend(c, p, w, a, static_cast<char *>(workspace), static_cast<cudaStream_t>(cuda_stream));
}

int wkv_attend_paged8(const wkv_paged *c, const wkv_cache8 *layer, const wkv_draft *draft, const void *q, const int64_t *q_strides,
                      const int32_t *lengths, void *out, const int64_t *out_strides, float *lse, const float *weights_in,
                      float *weights_out, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    Paged p;
    PagedWorkspace w;
    AttnArgs a;
    int st = resolve_paged8(c, p);
    if (st != WKV_OK || (st = check_layer(layer, true)) != WKV_OK) return st;
    const bool none = c->cu_new_host && p.total_new == 0;
    if (draft && !none && (st = check_draft(c, draft)) != WKV_OK) return st;
    if (draft && (weights_in || weights_out)) {
        set_error_detail("weights of drafted tokens: those that are not kept would count");
        return WKV_ERR_UNSUPPORTED;
    }
    if ((st = attend_args(c, p, q, q_strides, layer->k_codes, layer->v_codes, lengths, out, out_strides, lse, weights_in, weights_out, workspace,
                          workspace_bytes, w, a)) != WKV_OK || (none && !weights_out))
        return st;
    a.kind = layer->type + 1;
    a.k_scales = layer->k_scales;
    a.v_scales = layer->v_scales;
    if (draft && !none) {
        a.masks = draft->masks;
        a.mask_words = draft->words;
        a.before = rows_before(draft);
    }
    return launch_attend(c, p, w, a, static_cast<char *>(workspace), static_cast<cudaStream_t>(cuda_stream));
}

int wkv_keep_draft_paged(const wkv_paged *c, const wkv_draft *draft, int32_t n_layers, void *const *k_pools, void *const *v_pools,
                         const int32_t *last, const int32_t *lengths, int32_t *lengths_out, int32_t *row_positions,
                         float *row_weights, void *cuda_stream)
{
    Paged p;
    int st = resolve_paged(c, p);
    if (st != WKV_OK) return st;
    if (n_layers < 1 || n_layers > WKV_MAX_GROUP_LAYERS) {
        set_error_detail("n_layers %d outside 1..%d", n_layers, WKV_MAX_GROUP_LAYERS);
        return WKV_ERR_LIMIT;
    }
    if (!k_pools) return missing("k_pools");
    PoolTable pools;
    int n_tensors = 0;
    for (int l = 0; l < n_layers; ++l) {
        if ((st = check_pointer(k_pools[l], "a layer's K pool")) != WKV_OK) return st;
        pools.ptr[n_tensors++] = k_pools[l];
        if (!v_pools) continue;
        if ((st = check_pointer(v_pools[l], "a layer's V pool")) != WKV_OK) return st;
        pools.ptr[n_tensors++] = v_pools[l];
    }
    return keep_draft(c, p, draft, pools, ScaleTable(), false, n_tensors, last, lengths, lengths_out, row_positions, row_weights, cuda_stream);
}

int wkv_keep_draft_paged8(const wkv_paged *c, const wkv_draft *draft, int32_t n_layers, const wkv_cache8 *layers, const int32_t *last,
                          const int32_t *lengths, int32_t *lengths_out, int32_t *row_positions, float *row_weights,
                          void *cuda_stream)
{
    Paged p;
    int st = resolve_paged8(c, p), n_tensors = 0;
    if (st != WKV_OK) return st;
    PoolTable pools;
    ScaleTable scales;
    if ((st = fill_layers(n_layers, layers, true, pools, scales, n_tensors)) != WKV_OK) return st;
    return keep_draft(c, p, draft, pools, scales, true, n_tensors, last, lengths, lengths_out, row_positions, row_weights, cuda_stream);
}

}  // extern "C"
