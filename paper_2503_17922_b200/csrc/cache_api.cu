// Host side of the entry points around the selection: rotary positions, the prompt's attention, and the paged cache in use
// (append, attend, evict, row state).  Validation, workspace carve-up and kernel choice; no device memory is allocated here.
#include "cache_common.cuh"

namespace wkv {

int launch_attend(const wkv_paged *c, const Paged &p, const PagedWorkspace &w, const AttnArgs &a, char *ws, cudaStream_t stream)
{
    // Up to 16 rows are one tile of the warp-level kernel, whose time is that of the loads.
    int st = WKV_ERR_UNSUPPORTED;
    if (p.rows_max > (a.kind != kPlain ? kFewRows8 : kFewRows) && !a.few && attn_tc_supported(a, c->dtype))
        st = launch_attn_tc(a, w.pieces ? reinterpret_cast<float *>(ws + w.piece_o_off) : nullptr, reinterpret_cast<float2 *>(ws + w.piece_ml_off),
                            reinterpret_cast<long long *>(ws + w.line_off), stream);
    if (st == WKV_ERR_UNSUPPORTED) {
        st = c->dtype == WKV_F32 ? launch_attn_simt(a, stream) : (a.kind != kPlain ? launch_attn8(a, stream) : launch_attn_mma(a, stream));
        if (st == WKV_OK && !a.clustered && (a.splits > 1 || a.logits)) st = launch_attn_join(a, c->dtype, stream);
    }
    if (st != WKV_OK) return st;
    if (a.weights_out && !a.logits) return c->dtype == WKV_BF16 ? launch_attn_mma_weights(a, stream) : launch_attn_weights(a, stream);
    return WKV_OK;
}

}  // namespace wkv

using namespace wkv;

extern "C" {

int wkv_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_length, double low,
                         double high, uint64_t *turns_out)
{
    if (!turns_out) return missing("turns_out");
    const bool scaled = scaling != WKV_ROPE_NONE;
    if (rot_dim < 2 || rot_dim % 2 || !(base > 0) || !isfinite(base) || scaling < WKV_ROPE_NONE || scaling > WKV_ROPE_BANDS ||
        (scaled && (!(factor > 0) || !isfinite(factor))) ||
        (scaling == WKV_ROPE_BANDS && (!(original_length > 0) || !(high > low) || !isfinite(original_length) || !isfinite(low) || !isfinite(high)))) {
        set_error_detail("rope frequencies: rot_dim %d, base %g, scaling %d, factor %g, original length %g, bands %g .. %g", rot_dim, base,
                         scaling, factor, original_length, low, high);
        return WKV_ERR_SHAPE;
    }
    const long double two_pi = 6.283185307179586476925286766559005768L;
    long double b = base;
    if (scaling == WKV_ROPE_BASE && rot_dim > 2) b *= powl(factor, (long double)rot_dim / (rot_dim - 2));
    for (int i = 0; i < rot_dim / 2; ++i) {
        long double f = powl(b, -2.0L * i / rot_dim);
        if (scaling == WKV_ROPE_LINEAR) f /= factor;
        if (scaling == WKV_ROPE_BANDS) {
            long double t = (original_length * f / two_pi - low) / (high - low);
            t = t < 0 ? 0 : (t > 1 ? 1 : t);
            f *= t + (1 - t) / factor;
        }
        const long double turns = fmodl(f / two_pi, 1.0L);             // whole turns do not matter
        const long double fixed = roundl(ldexpl(turns, 64));
        turns_out[i] = fixed >= ldexpl(1.0L, 64) ? 0 : (uint64_t)fixed;
    }
    return WKV_OK;
}

int wkv_rotate_prompt(const wkv_shape *s, const wkv_rope *rope, const void *q, void *q_out, const int64_t *q_strides,
                      const void *k, void *k_out, const int32_t *positions, void *cuda_stream)
{
    KShape ks;
    RopeArgs a;
    int st = resolve(s, ks);
    if (st != WKV_OK) return st;
    if (!rope) return missing("rope");
    if ((st = rotate_args(s, ks, rope, q, q_out, q_strides, k, k_out, positions, a)) != WKV_OK) return st;
    return launch_rope(a, static_cast<cudaStream_t>(cuda_stream));
}

int wkv_attend_prompt(const wkv_shape *s, const void *q, const int64_t *q_strides, const void *k, const void *v, void *out,
                      const int64_t *out_strides, float *lse, float *lse_obs, int32_t *status, void *cuda_stream)
{
    KShape ks;
    int st = resolve(s, ks);
    if (st != WKV_OK) return st;
    if ((st = check_head_dim(s->head_dim)) != WKV_OK) return st;
    const int eb = elem_bytes(s->dtype);
    if ((st = check_pointer(q, "q")) != WKV_OK || (st = check_pointer(k, "k")) != WKV_OK || (st = check_pointer(v, "v")) != WKV_OK ||
        (st = check_pointer(out, "out")) != WKV_OK)
        return st;
    if ((st = check_strides(q_strides, ks.cu != nullptr, s->head_dim, eb, "q_strides")) != WKV_OK ||
        (st = check_strides(out_strides, ks.cu != nullptr, s->head_dim, eb, "out_strides")) != WKV_OK)
        return st;
    if (out == q || out == k || out == v) {
        set_error_detail("out must not be an input");
        return WKV_ERR_SHAPE;
    }
    if ((st = check_apart(out_strides, ks.batch, ks.hq, ks.cu ? ks.total_rows : ks.max_seqlen, ks.cu != nullptr, ks.d, "out_strides")) != WKV_OK) return st;
    if ((long long)ks.max_seqlen * ks.G > 0x3fffffffLL || (long long)ks.batch * ks.hkv > 0xffffffLL) {
        set_error_detail("attention: %d tokens of %d query heads per KV head, %d sequences", ks.max_seqlen, ks.G, ks.batch);
        return WKV_ERR_LIMIT;
    }
    AttnArgs a;
    memset(&a, 0, sizeof a);
    a.batch = ks.batch;
    a.hq = ks.hq;
    a.hkv = ks.hkv;
    a.G = ks.G;
    a.d = ks.d;
    a.max_q = ks.max_seqlen;
    a.total_q = ks.cu ? ks.total_rows : 0;
    a.cu_q = ks.cu;
    a.q = q;
    a.out = out;
    a.qb = ks.cu ? 0 : q_strides[0];
    a.qh = q_strides[1];
    a.qt = q_strides[2];
    a.ob = ks.cu ? 0 : out_strides[0];
    a.oh = out_strides[1];
    a.ot = out_strides[2];
    a.k = k;
    a.v = v;
    a.kb = ks.sb;
    a.kh = ks.sh;
    a.kt = ks.st;
    a.cap = ks.max_seqlen;
    a.scale_log2 = ks.scale_log2;
    a.lse = lse;
    a.lse_obs = lse_obs;
    a.alpha = ks.alpha;
    a.status = status;
    a.splits = 1;
    a.rows_max = ks.max_seqlen * ks.G;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (lse_obs) {
        bool shorter = false;
        for (int b = 0; b < s->batch; ++b)
            shorter |= (s->cu_seqlens_host ? s->cu_seqlens_host[b + 1] - s->cu_seqlens_host[b] : s->max_seqlen) < s->l_obs;
        if (shorter && (st = launch_attn_lse_obs_fill(a, stream)) != WKV_OK) return st;
    }
    if (attn_tc_supported(a, s->dtype) && (st = launch_attn_tc(a, nullptr, nullptr, nullptr, stream)) != WKV_ERR_UNSUPPORTED) return st;
    return s->dtype == WKV_BF16 ? launch_attn_mma(a, stream) : launch_attn_simt(a, stream);
}

size_t wkv_paged_workspace_bytes(const wkv_paged *c)
{
    Paged p;
    return resolve_paged(c, p) == WKV_OK ? plan_paged(c, p).total : 0;
}

int wkv_append_kv_paged(const wkv_paged *c, const wkv_rope *rope, const void *k_new, const void *v_new,
                        const int64_t *kv_strides, const void *q, void *q_out, const int64_t *q_strides,
                        const int32_t *positions, const int32_t *lengths, void *k_pool, void *v_pool, int32_t *lengths_out,
                        int32_t *row_positions, float *row_weights, void *cuda_stream)
{
    Paged p;
    RopeArgs a;
    int st = resolve_paged(c, p);
    if (st == WKV_OK)
        st = append_args(c, p, rope, k_new, v_new, kv_strides, q, q_out, q_strides, positions, lengths, k_pool, v_pool, lengths_out, row_positions,
                         row_weights, a);
    return st != WKV_OK ? st : launch_rope(a, static_cast<cudaStream_t>(cuda_stream));
}

int wkv_attend_paged(const wkv_paged *c, const void *q, const int64_t *q_strides, const void *k_pool, const void *v_pool,
                     const int32_t *lengths, void *out, const int64_t *out_strides, float *lse, const float *weights_in,
                     float *weights_out, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    Paged p;
    PagedWorkspace w;
    AttnArgs a;
    int st = resolve_paged(c, p);
    if (st == WKV_OK) st = attend_args(c, p, q, q_strides, k_pool, v_pool, lengths, out, out_strides, lse, weights_in, weights_out, workspace, workspace_bytes, w, a);
    if (st != WKV_OK || (c->cu_new_host && p.total_new == 0 && !weights_out)) return st;
    char *const ws = static_cast<char *>(workspace);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return launch_attend(c, p, w, a, ws, stream);
}

int wkv_evict_kv_paged(const wkv_paged *c, int32_t n_layers, void *const *k_pools, void *const *v_pools, int32_t budget,
                       const int32_t *budgets, int32_t recent, const float *weights, const int32_t *positions,
                       const int32_t *lengths, float *weights_out, int32_t *positions_out, int32_t *lengths_out,
                       void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    Paged p;
    int st = resolve_paged(c, p);
    if (st != WKV_OK) return st;
    if (n_layers < 1 || n_layers > WKV_MAX_GROUP_LAYERS) {
        set_error_detail("n_layers %d outside 1..%d", n_layers, WKV_MAX_GROUP_LAYERS);
        return WKV_ERR_LIMIT;
    }
    if (!k_pools) return missing("k_pools");
    if ((st = check_eviction(budget, recent, weights, positions, lengths, weights_out, positions_out, lengths_out)) != WKV_OK) return st;
    PoolTable pools;
    int n_tensors = 0;
    for (int l = 0; l < n_layers; ++l) {
        if ((st = check_pointer(k_pools[l], "a layer's K pool")) != WKV_OK) return st;
        pools.ptr[n_tensors++] = k_pools[l];
        if (!v_pools) continue;
        if ((st = check_pointer(v_pools[l], "a layer's V pool")) != WKV_OK) return st;
        pools.ptr[n_tensors++] = v_pools[l];
    }
    EvictArgs a;
    if ((st = evict_args(c, p, n_tensors, budget, budgets, recent, weights, positions, lengths, weights_out, positions_out, lengths_out, workspace,
                         workspace_bytes, a)) != WKV_OK)
        return st;
    return launch_evict(a, pools, ScaleTable(), static_cast<cudaStream_t>(cuda_stream));
}

int wkv_seed_rows(const wkv_shape *s, const int32_t *window_idx, const float *token_scores, int32_t row_capacity,
                  int32_t *positions, float *weights, void *cuda_stream)
{
    KShape ks;
    int st = resolve(s, ks);
    if (st != WKV_OK) return st;
    if (!window_idx) return missing("window_idx");
    if (!positions && !weights) return missing("positions and weights");
    if (row_capacity < wkv_keep_max(s)) {
        set_error_detail("row_capacity %d smaller than the %d rows a unit may keep", row_capacity, wkv_keep_max(s));
        return WKV_ERR_SHAPE;
    }
    return launch_seed_rows(ks, window_idx, token_scores, row_capacity, positions, weights, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
