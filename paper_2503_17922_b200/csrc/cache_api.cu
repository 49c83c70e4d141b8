// Host side of the entry points around the selection: rotary positions, the prompt's attention, and the paged cache in use
// (append, attend, evict, row state).  Validation, workspace carve-up and kernel choice; no device memory is allocated here.
#include "attn_cluster.cuh"

#include <algorithm>

#include <math.h>
#include <string.h>

namespace wkv {
namespace {

int elem_bytes(int dtype) { return dtype == WKV_F32 ? 4 : 2; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int missing(const char *what)
{
    set_error_detail("%s is NULL", what);
    return WKV_ERR_NULL;
}
int check_pointer(const void *p, const char *what)
{
    if (!p) return missing(what);
    if (aligned16(p)) return WKV_OK;
    set_error_detail("%s is not 16-byte aligned", what);
    return WKV_ERR_ALIGN;
}
// strides of a [B, heads, tokens, d] or packed [T, heads, d] tensor (whose batch stride is not looked at)
int check_strides(const int64_t *st, bool packed, int head_dim, int eb, const char *what)
{
    if (!st) return missing(what);
    for (int i = packed ? 1 : 0; i < 3; ++i)
        if (st[i] < 0 || (st[i] * eb) % 16) {
            set_error_detail("%s: stride #%d = %lld is negative or not 16-byte aligned", what, i, (long long)st[i]);
            return WKV_ERR_ALIGN;
        }
    if (st[2] < head_dim) {
        set_error_detail("%s: token stride smaller than head_dim", what);
        return WKV_ERR_SHAPE;
    }
    return WKV_OK;
}

// The rows of an output lie apart: each dimension, in order of increasing stride, steps over all that the ones before it reach.  (Rows in
// one place are written by several threads, and rotated in place once for each of them.)
struct Dim {
    long long size, stride;
};
int check_apart(Dim x, Dim y, Dim z, int head_dim, const char *what)
{
    Dim dims[3] = {x, y, z};
    std::sort(dims, dims + 3, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    unsigned __int128 reach = (unsigned)head_dim;
    for (const Dim &a : dims) {
        if (a.size <= 1) continue;
        if ((unsigned __int128)a.stride < reach) {
            set_error_detail("%s: a stride of %lld puts rows of an output into one place", what, a.stride);
            return WKV_ERR_SHAPE;
        }
        reach += (unsigned __int128)a.stride * (unsigned long long)(a.size - 1);
    }
    return WKV_OK;
}
// ... of a tensor whose strides check_strides has seen
int check_apart(const int64_t *st, int batch, int heads, long long tokens, bool packed, int head_dim, const char *what)
{
    return check_apart({packed ? 1 : batch, st[0]}, {heads, st[1]}, {tokens, st[2]}, head_dim, what);
}
int check_pools_apart(const wkv_paged *c)
{
    return check_apart({c->num_pages, c->page_stride}, {c->n_kv_heads, c->head_stride}, {c->page_size, c->row_stride}, c->head_dim, "paged cache");
}

// what a call knows about its paged cache
struct Paged {
    int eb, units, cap, total_new, rows_max;
    long long batch_tokens;           // tokens of [B, max_new] or of the packed chunk
};
int resolve_paged(const wkv_paged *c, Paged &p)
{
    if (!c) return missing("cache description");
    if (c->struct_size != sizeof(wkv_paged)) {
        set_error_detail("struct_size %u != %zu", c->struct_size, sizeof(wkv_paged));
        return WKV_ERR_SHAPE;
    }
    if (c->dtype != WKV_F32 && c->dtype != WKV_BF16) {
        set_error_detail("dtype %d unknown", c->dtype);
        return WKV_ERR_DTYPE;
    }
    if (c->batch < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->max_new < 1 || c->page_size < 1 ||
        c->num_pages < 1 || c->max_pages < 1 || c->reserved[0] != 0 || c->reserved[1] != 0) {
        set_error_detail("non-positive size (batch %d, heads %d/%d, d %d, new %d, page %d, pages %d, table %d) or reserved "
                         "words not 0", c->batch, c->n_q_heads, c->n_kv_heads, c->head_dim, c->max_new, c->page_size,
                         c->num_pages, c->max_pages);
        return WKV_ERR_SHAPE;
    }
    if (c->n_q_heads % c->n_kv_heads) {
        set_error_detail("n_q_heads %d not a multiple of n_kv_heads %d", c->n_q_heads, c->n_kv_heads);
        return WKV_ERR_SHAPE;
    }
    p.eb = elem_bytes(c->dtype);
    if (((long long)c->head_dim * p.eb) % 16) {
        set_error_detail("head_dim %d: a row must be a multiple of 16 bytes", c->head_dim);
        return WKV_ERR_ALIGN;
    }
    const int64_t strides[3] = {c->page_stride, c->head_stride, c->row_stride};
    for (int i = 0; i < 3; ++i)
        if (strides[i] < 0 || (strides[i] * p.eb) % 16) {
            set_error_detail("paged cache: stride #%d = %lld is negative or not 16-byte aligned", i, (long long)strides[i]);
            return WKV_ERR_ALIGN;
        }
    if (c->row_stride < c->head_dim) {
        set_error_detail("paged cache: row stride smaller than head_dim");
        return WKV_ERR_SHAPE;
    }
    const long long cap = (long long)c->max_pages * c->page_size, units = (long long)c->batch * c->n_kv_heads;
    const long long rows = (long long)c->max_new * (c->n_q_heads / c->n_kv_heads);
    if (cap > 0x3fffffffLL || units > 0xffffffLL || rows > 0x3fffffffLL || (long long)c->batch * c->n_q_heads > 0x3fffffffLL) {
        set_error_detail("paged cache: %lld rows of a unit (at most 2^30 - 1), %lld units (2^24 - 1), %lld query rows (2^30 - 1)",
                         cap, units, rows);
        return WKV_ERR_LIMIT;
    }
    if (!c->block_table) return missing("block_table");
    if ((c->cu_new_host == nullptr) != (c->cu_new_dev == nullptr)) {
        set_error_detail("host and device copies of cu_new must be given together");
        return WKV_ERR_NULL;
    }
    p.batch_tokens = (long long)c->batch * c->max_new;
    if (c->cu_new_host) {
        for (int b = 0; b < c->batch; ++b) {
            const long long m = (long long)c->cu_new_host[b + 1] - c->cu_new_host[b];
            if (m < 0 || m > c->max_new || (b == 0 && c->cu_new_host[0] != 0)) {
                set_error_detail("cu_new: sequence %d has %lld new tokens (max_new %d)", b, m, c->max_new);
                return WKV_ERR_SHAPE;
            }
        }
        p.batch_tokens = c->cu_new_host[c->batch];
    }
    if (p.batch_tokens > 0x7fffffffLL) {
        set_error_detail("more than 2^31-1 new tokens in the batch");
        return WKV_ERR_LIMIT;
    }
    p.total_new = c->cu_new_host ? (int)p.batch_tokens : 0;
    p.units = (int)units;
    p.cap = (int)cap;
    p.rows_max = (int)rows;
    return WKV_OK;
}

// Workspace of the paged entry points: status word, then what an attention or an eviction leaves between its kernels.
struct PagedWorkspace {
    int splits;
    bool clustered;
    size_t lse_off, ml_off, o_off, logits_off, counts_off, moves_off, places_off, total;
    long long logit_stride;      // 0: the weights are computed from K once more
    int pieces;                  // of the tensor-core kernel
    size_t line_off, piece_o_off, piece_ml_off;
    int moves_max;
};
// Key splits of the kernels that take one tile of rows per block: two blocks for every SM, where each then has a tile of 64
// keys at least; and with 1,024 keys or more to each, up to four times as many, so that sequences of different lengths
// even out.
// With up to 16 rows, a power of two up to eight is preferred: those are clusters, which join their splits themselves, as long as
// all of them run at once (32 sequences of 8 heads x 4-8 K rows: 267 us as clusters of eight, 188 as five splits and a joining
// kernel; one sequence of 8 heads x 992 rows 8.8 and 12.6) and a block has no more than kClusterBytes of keys and values to read.
constexpr int kSplitBlocks = 2 * 148, kSplitKeys = 64, kSplitEven = 1024;
constexpr long long kClusterBytes = 512 << 10;
int plan_splits(const wkv_paged *c, const Paged &p, bool &clustered)
{
    const int tile = p.rows_max <= 16 ? 16 : 64;
    const long long blocks = ((long long)p.rows_max + tile - 1) / tile * p.units;
    long long s = (kSplitBlocks + blocks - 1) / blocks;
    if (s > (p.cap + kSplitKeys - 1) / kSplitKeys) s = (p.cap + kSplitKeys - 1) / kSplitKeys;
    while (blocks * s < 4 * kSplitBlocks && p.cap / (s + 1) >= kSplitEven) ++s;
    if (s < 1) s = 1;
    long long power = 1;
    while (power < s && power < kClusterSplits) power *= 2;
    clustered = tile == 16 && blocks * power <= kSplitBlocks &&
                (s <= power || 2ll * p.cap * c->head_dim * p.eb / kClusterSplits <= kClusterBytes);
    return (int)(clustered ? power : s);
}
// More rows than this go to the tensor-core kernel where it takes the shape (8 new tokens of 32 heads on 8, 32 rows: 4 sequences of 16,384
// keys 171 us on the warp-level kernel, 88 here; one of 4,000 42 and 32).
constexpr int kFewRows = 16;
// Rows per unit whose logits are kept for the weights: 4 bytes for each beside the 2 * d * 2 of K and V, written and read.
constexpr int kLogitRows = 16;
PagedWorkspace plan_paged(const wkv_paged *c, const Paged &p)
{
    PagedWorkspace w;
    w.splits = plan_splits(c, p, w.clustered);
    size_t off = 256;
    w.lse_off = off;
    off = align_up(off + (size_t)c->batch * c->n_q_heads * c->max_new * sizeof(float), 256);
    const bool keeps_logits = p.rows_max <= kLogitRows;
    const size_t parts = !w.clustered && (w.splits > 1 || keeps_logits) ? (size_t)p.units * p.rows_max * w.splits : 0;
    w.ml_off = off;
    off = align_up(off + parts * sizeof(float2), 256);
    w.o_off = off;
    off = align_up(off + parts * c->head_dim * sizeof(float), 256);
    w.logits_off = off;
    w.logit_stride = keeps_logits ? ((long long)p.cap + 3) / 4 * 4 : 0;
    off = align_up(off + (size_t)p.units * p.rows_max * w.logit_stride * sizeof(float), 256);
    w.total = off;
    // (in the place of the parts above: a call runs one kernel or the other)
    off = w.ml_off;
    int rows = 0, items = 0;
    const int G = c->n_q_heads / c->n_kv_heads;
    w.pieces = c->dtype == WKV_BF16 && p.rows_max > kFewRows && G <= 128 && c->head_dim <= 128
                   ? attn_tc_pieces(p.units, c->max_new, G, p.cap, &rows, &items) : 0;
    w.line_off = off;
    off = align_up(off + (w.pieces ? (size_t)(items + 1) * sizeof(long long) : 0), 256);
    w.piece_ml_off = off;
    off = align_up(off + (size_t)w.pieces * rows * sizeof(float2), 256);
    w.piece_o_off = off;
    off = align_up(off + (size_t)w.pieces * rows * c->head_dim * sizeof(float), 256);
    if (off > w.total) w.total = off;
    w.moves_max = p.cap / 2 + 1;
    off = 256;
    w.counts_off = off;
    off = align_up(off + (size_t)p.units * sizeof(int), 256);
    w.moves_off = off;
    off = align_up(off + (size_t)p.units * w.moves_max * sizeof(int2), 256);
    w.places_off = off;
    off = align_up(off + (size_t)p.units * w.moves_max * sizeof(longlong2), 256);
    if (off > w.total) w.total = off;
    return w;
}
int check_workspace(const PagedWorkspace &w, const void *workspace, size_t bytes)
{
    if (!workspace || bytes < w.total) {
        set_error_detail("workspace has %zu bytes, %zu needed", workspace ? bytes : (size_t)0, w.total);
        return WKV_ERR_WORKSPACE;
    }
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) {
        set_error_detail("workspace is not 256-byte aligned");
        return WKV_ERR_WORKSPACE;
    }
    return WKV_OK;
}

int check_rope(const wkv_rope *r, int head_dim)
{
    if (r->struct_size != sizeof(wkv_rope)) {
        set_error_detail("rope: struct_size %u != %zu", r->struct_size, sizeof(wkv_rope));
        return WKV_ERR_SHAPE;
    }
    if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > head_dim || (r->order != WKV_ROPE_HALF && r->order != WKV_ROPE_INTERLEAVED) ||
        !isfinite(r->scale)) {
        set_error_detail("rope: rot_dim %d (even, 2 .. head_dim %d), order %d or scale invalid", r->rot_dim, head_dim, r->order);
        return WKV_ERR_SHAPE;
    }
    if (r->rot_dim > WKV_MAX_ROT_DIM) {
        set_error_detail("rope: rot_dim %d beyond %d", r->rot_dim, WKV_MAX_ROT_DIM);
        return WKV_ERR_LIMIT;
    }
    return r->turns ? WKV_OK : missing("rope: turns");
}
void set_rope(const wkv_rope *r, RopeArgs &a)
{
    a.turns = r ? reinterpret_cast<const unsigned long long *>(r->turns) : nullptr;
    a.rot = r ? r->rot_dim : 0;
    a.order = r ? r->order : WKV_ROPE_HALF;
    a.scale = r ? r->scale : 1.f;
}
int check_head_dim(int d)
{
    if (d <= kAttnMaxHeadDim) return WKV_OK;
    set_error_detail("attention: head_dim %d beyond %d", d, kAttnMaxHeadDim);
    return WKV_ERR_UNSUPPORTED;
}

}  // namespace
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
    int st = resolve(s, ks);
    if (st != WKV_OK) return st;
    if (!rope) return missing("rope");
    if ((st = check_rope(rope, s->head_dim)) != WKV_OK) return st;
    if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (!q && !k)) {
        set_error_detail("q and q_out, k and k_out go together; at least one pair is needed");
        return WKV_ERR_NULL;
    }
    const int eb = elem_bytes(s->dtype);
    if (q) {
        if ((st = check_pointer(q, "q")) != WKV_OK || (st = check_pointer(q_out, "q_out")) != WKV_OK) return st;
        if ((st = check_strides(q_strides, ks.cu != nullptr, s->head_dim, eb, "q_strides")) != WKV_OK) return st;
    }
    if (k && ((st = check_pointer(k, "k")) != WKV_OK || (st = check_pointer(k_out, "k_out")) != WKV_OK)) return st;
    const bool packed = ks.cu != nullptr;
    const long long tokens = packed ? ks.total_rows : ks.max_seqlen;
    if (q && (st = check_apart(q_strides, ks.batch, ks.hq, tokens, packed, ks.d, "q_strides")) != WKV_OK) return st;
    if (k && (st = check_apart({packed ? 1 : ks.batch, ks.sb}, {ks.hkv, ks.sh}, {tokens, ks.st}, ks.d, "k_out")) != WKV_OK) return st;
    RopeArgs a;
    memset(&a, 0, sizeof a);
    a.batch = ks.batch;
    a.d = ks.d;
    a.elem_bytes = eb;
    a.max_q = ks.max_seqlen;
    a.total_q = ks.cu ? ks.total_rows : 0;
    a.cu_q = ks.cu;
    set_rope(rope, a);
    a.positions = positions;
    a.hq = ks.hq;
    a.hkv = ks.hkv;
    a.q = q;
    a.q_out = q_out;
    if (q) {
        a.qb = ks.cu ? 0 : q_strides[0];
        a.qh = q_strides[1];
        a.qt = q_strides[2];
    }
    a.k = k;
    a.k_out = k_out;
    a.kb = ks.sb;
    a.kh = ks.sh;
    a.kt = ks.st;
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
    int st = resolve_paged(c, p);
    if (st != WKV_OK) return st;
    if (rope && (st = check_rope(rope, c->head_dim)) != WKV_OK) return st;
    const void *const ptrs[4] = {k_new, v_new, k_pool, v_pool};
    static const char *const names[4] = {"k_new", "v_new", "k_pool", "v_pool"};
    const bool packed = c->cu_new_host != nullptr, none = packed && p.total_new == 0;      // no new tokens: their tensors may be null
    for (int i = none ? 2 : 0; i < 4; ++i)
        if ((st = check_pointer(ptrs[i], names[i])) != WKV_OK) return st;
    if (!none && (st = check_strides(kv_strides, packed, c->head_dim, p.eb, "kv_strides")) != WKV_OK) return st;
    if (!none && (q == nullptr) != (q_out == nullptr)) return missing(q ? "q_out" : "q");
    if (q && !none) {
        if ((st = check_pointer(q, "q")) != WKV_OK || (st = check_pointer(q_out, "q_out")) != WKV_OK) return st;
        if ((st = check_strides(q_strides, packed, c->head_dim, p.eb, "q_strides")) != WKV_OK) return st;
    }
    if (!lengths) return missing("lengths");
    if (!none && !positions && (rope || row_positions)) return missing("positions");
    if (lengths_out == lengths) {
        set_error_detail("lengths_out must not be lengths (other blocks still read them)");
        return WKV_ERR_SHAPE;
    }
    if (k_pool == v_pool) {
        set_error_detail("k_pool and v_pool are the same");
        return WKV_ERR_SHAPE;
    }
    if ((st = check_pools_apart(c)) != WKV_OK) return st;
    if (q && !none && (st = check_apart(q_strides, c->batch, c->n_q_heads, packed ? p.total_new : c->max_new, packed, c->head_dim, "q_strides")) != WKV_OK)
        return st;
    RopeArgs a;
    memset(&a, 0, sizeof a);
    a.batch = c->batch;
    a.d = c->head_dim;
    a.elem_bytes = p.eb;
    a.max_q = c->max_new;
    a.total_q = p.total_new;
    a.cu_q = c->cu_new_dev;
    set_rope(rope, a);
    a.positions = positions;
    a.hq = c->n_q_heads;
    a.hkv = c->n_kv_heads;
    a.q = q;
    a.q_out = q_out;
    if (q && !none) {
        a.qb = packed ? 0 : q_strides[0];
        a.qh = q_strides[1];
        a.qt = q_strides[2];
    }
    a.k = k_new;
    a.v = v_new;
    a.k_out = k_pool;
    a.v_out = v_pool;
    if (!none) {
        a.kb = packed ? 0 : kv_strides[0];
        a.kh = kv_strides[1];
        a.kt = kv_strides[2];
    }
    a.lengths = lengths;
    a.table = c->block_table;
    a.max_pages = c->max_pages;
    a.page_size = c->page_size;
    a.num_pages = c->num_pages;
    a.cap = p.cap;
    a.page_stride = c->page_stride;
    a.head_stride = c->head_stride;
    a.row_stride = c->row_stride;
    a.lengths_out = lengths_out;
    a.row_positions = row_positions;
    a.row_weights = row_weights;
    return launch_rope(a, static_cast<cudaStream_t>(cuda_stream));
}

int wkv_attend_paged(const wkv_paged *c, const void *q, const int64_t *q_strides, const void *k_pool, const void *v_pool,
                     const int32_t *lengths, void *out, const int64_t *out_strides, float *lse, const float *weights_in,
                     float *weights_out, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    Paged p;
    int st = resolve_paged(c, p);
    if (st != WKV_OK) return st;
    if ((st = check_head_dim(c->head_dim)) != WKV_OK) return st;
    const void *const ptrs[4] = {q, k_pool, v_pool, out};
    static const char *const names[4] = {"q", "k_pool", "v_pool", "out"};
    const bool packed = c->cu_new_host != nullptr, none = packed && p.total_new == 0;      // no new tokens: q and out may be null
    for (int i = 0; i < 4; ++i)
        if (!(none && (i == 0 || i == 3)) && (st = check_pointer(ptrs[i], names[i])) != WKV_OK) return st;
    if (!none && ((st = check_strides(q_strides, packed, c->head_dim, p.eb, "q_strides")) != WKV_OK ||
                  (st = check_strides(out_strides, packed, c->head_dim, p.eb, "out_strides")) != WKV_OK))
        return st;
    if (!lengths) return missing("lengths");
    if (weights_in && !weights_out) return missing("weights_out");
    if (!none && (out == q || out == k_pool || out == v_pool)) {
        set_error_detail("out must not be an input");
        return WKV_ERR_SHAPE;
    }
    if (!none && (st = check_apart(out_strides, c->batch, c->n_q_heads, packed ? p.total_new : c->max_new, packed, c->head_dim, "out_strides")) != WKV_OK)
        return st;
    const PagedWorkspace w = plan_paged(c, p);
    if ((st = check_workspace(w, workspace, workspace_bytes)) != WKV_OK) return st;
    if (none && !weights_out) return WKV_OK;
    char *ws = static_cast<char *>(workspace);
    AttnArgs a;
    memset(&a, 0, sizeof a);
    a.batch = c->batch;
    a.hq = c->n_q_heads;
    a.hkv = c->n_kv_heads;
    a.G = c->n_q_heads / c->n_kv_heads;
    a.d = c->head_dim;
    a.max_q = c->max_new;
    a.total_q = p.total_new;
    a.cu_q = c->cu_new_dev;
    a.q = q;
    a.out = out;
    if (!none) {
        a.qb = packed ? 0 : q_strides[0];
        a.qh = q_strides[1];
        a.qt = q_strides[2];
        a.ob = packed ? 0 : out_strides[0];
        a.oh = out_strides[1];
        a.ot = out_strides[2];
    }
    a.k = k_pool;
    a.v = v_pool;
    a.kb = c->page_stride;
    a.kh = c->head_stride;
    a.kt = c->row_stride;
    a.table = c->block_table;
    a.len = lengths;
    a.max_pages = c->max_pages;
    a.page_size = c->page_size;
    a.num_pages = c->num_pages;
    a.cap = p.cap;
    a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)c->head_dim));
    a.lse = lse ? lse : (weights_out ? reinterpret_cast<float *>(ws + w.lse_off) : nullptr);
    a.status = reinterpret_cast<int *>(ws);
    a.splits = w.splits;
    a.clustered = w.clustered;
    a.part_ml = reinterpret_cast<float2 *>(ws + w.ml_off);
    a.part_o = reinterpret_cast<float *>(ws + w.o_off);
    a.rows_max = p.rows_max;
    a.weights_in = weights_in;
    a.weights_out = weights_out;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (weights_out && w.logit_stride) {
        a.logits = reinterpret_cast<float *>(ws + w.logits_off);
        a.logit_stride = w.logit_stride;
    }
    // Up to 16 rows are one tile of the warp-level kernel, whose time is that of the loads.
    st = WKV_ERR_UNSUPPORTED;
    if (p.rows_max > kFewRows && attn_tc_supported(a, c->dtype))
        st = launch_attn_tc(a, w.pieces ? reinterpret_cast<float *>(ws + w.piece_o_off) : nullptr, reinterpret_cast<float2 *>(ws + w.piece_ml_off),
                            reinterpret_cast<long long *>(ws + w.line_off), stream);
    if (st == WKV_ERR_UNSUPPORTED) {
        st = c->dtype == WKV_BF16 ? launch_attn_mma(a, stream) : launch_attn_simt(a, stream);
        if (st == WKV_OK && !a.clustered && (a.splits > 1 || a.logits)) st = launch_attn_join(a, c->dtype, stream);
    }
    if (st != WKV_OK) return st;
    if (weights_out && !a.logits) return c->dtype == WKV_BF16 ? launch_attn_mma_weights(a, stream) : launch_attn_weights(a, stream);
    return WKV_OK;
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
    if (budget < 0) {
        set_error_detail("budget is negative (%d)", budget);
        return WKV_ERR_BUDGET;
    }
    if (recent < 0) {
        set_error_detail("recent is negative (%d)", recent);
        return WKV_ERR_SHAPE;
    }
    if (!weights || !positions || !lengths || !weights_out || !positions_out || !lengths_out)
        return missing("weights, positions, lengths or one of their outputs");
    PoolTable pools;
    int n_tensors = 0;
    for (int l = 0; l < n_layers; ++l) {
        if ((st = check_pointer(k_pools[l], "a layer's K pool")) != WKV_OK) return st;
        pools.ptr[n_tensors++] = k_pools[l];
        if (!v_pools) continue;
        if ((st = check_pointer(v_pools[l], "a layer's V pool")) != WKV_OK) return st;
        pools.ptr[n_tensors++] = v_pools[l];
    }
    if ((st = check_pools_apart(c)) != WKV_OK) return st;
    const PagedWorkspace w = plan_paged(c, p);
    if ((st = check_workspace(w, workspace, workspace_bytes)) != WKV_OK) return st;
    EvictArgs a;
    memset(&a, 0, sizeof a);
    a.batch = c->batch;
    a.hkv = c->n_kv_heads;
    a.d = c->head_dim;
    a.elem_bytes = p.eb;
    a.table = c->block_table;
    a.max_pages = c->max_pages;
    a.page_size = c->page_size;
    a.num_pages = c->num_pages;
    a.cap = p.cap;
    a.page_stride = c->page_stride;
    a.head_stride = c->head_stride;
    a.row_stride = c->row_stride;
    a.n_tensors = n_tensors;
    a.budget = budget;
    a.recent = recent;
    a.budgets = budgets;
    a.weights = weights;
    a.positions = positions;
    a.lengths = lengths;
    a.weights_out = weights_out;
    a.positions_out = positions_out;
    a.lengths_out = lengths_out;
    a.counts = reinterpret_cast<int *>(static_cast<char *>(workspace) + w.counts_off);
    a.moves = reinterpret_cast<int2 *>(static_cast<char *>(workspace) + w.moves_off);
    a.places = reinterpret_cast<longlong2 *>(static_cast<char *>(workspace) + w.places_off);
    a.moves_max = w.moves_max;
    return launch_evict(a, pools, static_cast<cudaStream_t>(cuda_stream));
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
