// Attention kernels: what a launch knows about queries, keys and values, shared by the whole-prompt and the paged entry points.
//
// The rows of a unit (sequence b, KV head h) are its m_b queries times the G query heads of its group, numbered r = i*G + g, so
// that the heads which share keys and values also share the tiles of them.  Query i attends to the first
// n - m_b + i + 1 of the unit's n rows (a prompt: n = m_b).
#pragma once

#include "wkv_internal.cuh"

#include <atomic>

namespace wkv {

constexpr int kAttnMaxHeadDim = 256;

struct AttnArgs {
    int batch, hq, hkv, G, d;
    int max_q;                   // queries of a sequence: all (dense) or an upper bound (packed)
    int total_q;                 // rows of the packed queries
    const int *cu_q;             // device, or null: dense
    const void *q;
    void *out;
    long long qb, qh, qt, ob, oh, ot;        // element strides
    const void *k, *v;
    long long kb, kh, kt;        // dense or packed: batch, head, token; paged: page, head, slot
    const int *table;            // paged: device [batch][max_pages], else null
    const int *len;              // paged: device [batch][hkv]
    int max_pages, page_size, num_pages;
    int cap;                     // rows of a unit at most
    float scale_log2;            // log2(e)/sqrt(d): logits are handled in base 2
    float *lse;                  // [batch][hq][max_q] natural log, or null
    float *lse_obs;              // prompt: [batch][hq][alpha], or null
    int alpha;
    int *status;                 // or null
    // key splits: `splits` > 1 leaves partial results for the joining kernel
    int splits;
    bool clustered;              // the splits are the blocks of a cluster, which join them: no partial results in memory
    float *part_o;               // [units][rows_max][splits][d]: not yet normalised
    float2 *part_ml;             // [units][rows_max][splits]: (maximum in base 2, sum)
    int rows_max;                // max_q * G
    float *logits;               // [units][rows_max][logit_stride] in base 2, or null: for the weights
    long long logit_stride;      // cap, rounded up to a multiple of four
    const float *weights_in;     // [units][cap] or null
    float *weights_out;          // [units][cap] or null
};

struct AttnSeq {
    int m;            // queries
    int n;            // rows of the unit
    long long q_off;  // first row in packed tensors
};
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs &a, int b, int h)
{
    AttnSeq s;
    if (a.cu_q) {
        // a device copy that disagrees with the host copy must not lead outside the packed tensors
        int lo = a.cu_q[b], hi = a.cu_q[b + 1];
        lo = min(max(lo, 0), a.total_q);
        s.m = min(min(max(hi - lo, 0), a.max_q), a.total_q - lo);
        s.q_off = lo;
    } else {
        s.m = a.max_q;
        s.q_off = 0;
    }
    s.n = a.len ? min(max(a.len[b * a.hkv + h], 0), a.cap) : s.m;
    return s;
}
// element offset of row j of unit (b, h) in K and V, or -1 where its page is none
__device__ __forceinline__ long long attn_row(const AttnArgs &a, int b, int h, long long q_off, int j)
{
    if (a.table) {
        const int pg = j / a.page_size, page = __ldg(a.table + (long long)b * a.max_pages + pg);
        if ((unsigned)page >= (unsigned)a.num_pages) return -1;
        return page * a.kb + h * a.kh + (long long)(j - pg * a.page_size) * a.kt;
    }
    return (q_off + j) * a.kt + b * a.kb + h * a.kh;
}
// log-sum-exp of a row, where it is asked for; lse2 in base 2
__device__ __forceinline__ void attn_store_lse(const AttnArgs &a, int b, int hq, int i, int m, float lse2)
{
    const float l = lse2 * 0.69314718055994531f;
    const long long row = (long long)b * a.hq + hq;
    if (a.lse) a.lse[row * a.max_q + i] = l;
    if (a.lse_obs && i >= m - a.alpha) a.lse_obs[row * a.alpha + (i - m + a.alpha)] = l;
}

// Dynamic shared memory beyond 48 KB has to be asked for once per kernel and device; `asked` remembers for one kernel.
struct SmemAsked {
    std::atomic<uint64_t> devices{0};
};
template <typename K>
inline cudaError_t allow_smem(K kernel, size_t bytes, SmemAsked &asked)
{
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    const uint64_t bit = dev < kMaxDevices ? 1ull << dev : 0;
    if (asked.devices.load(std::memory_order_acquire) & bit) return cudaSuccess;
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (err == cudaSuccess) asked.devices.fetch_or(bit, std::memory_order_release);
    return err;
}

// kernels (each returns a wkv_status)
bool attn_tc_supported(const AttnArgs &a, int dtype);
// WKV_ERR_UNSUPPORTED: a layout that no tensor map describes.  piece_o, piece_ml, line: room for attn_tc_pieces() * rows rows of d
// (256-byte aligned) and of one, and for items + 1 words, or null; with them the blocks share the work evenly where there are few items.
int launch_attn_tc(const AttnArgs &a, float *piece_o, float2 *piece_ml, long long *line, cudaStream_t stream);
int attn_tc_pieces(long long units, int max_q, int G, int cap, int *rows, int *items);
int launch_attn_mma(const AttnArgs &a, cudaStream_t stream);         // bf16
int launch_attn_simt(const AttnArgs &a, cudaStream_t stream);         // fp32
int launch_attn_join(const AttnArgs &a, int dtype, cudaStream_t stream);       // with a.logits: and the weights
int launch_attn_weights(const AttnArgs &a, cudaStream_t stream);      // fp32; reads a.lse
int launch_attn_mma_weights(const AttnArgs &a, cudaStream_t stream);  // bf16; reads a.lse
int launch_attn_lse_obs_fill(const AttnArgs &a, cudaStream_t stream);

// rotary positions
struct RopeArgs {
    int batch, d, elem_bytes;
    int max_q, total_q;
    const int *cu_q;
    int rot, order;
    float scale;
    const unsigned long long *turns;         // null: no rotation
    const int *positions;                    // null: place in the sequence
    int hq, hkv;
    const void *q;
    void *q_out;
    long long qb, qh, qt;
    const void *k, *v;                       // v: append only
    void *k_out, *v_out;                     // rotate: tensors of k's layout; append: the pools
    long long kb, kh, kt;
    // append
    const int *lengths, *table;
    int max_pages, page_size, num_pages, cap;
    long long page_stride, head_stride, row_stride;
    int *lengths_out, *row_positions;
    float *row_weights;
};
int launch_rope(const RopeArgs &a, cudaStream_t stream);

struct EvictArgs {
    int batch, hkv, d, elem_bytes;
    const int *table;
    int max_pages, page_size, num_pages, cap;
    long long page_stride, head_stride, row_stride;
    int n_tensors;
    int budget, recent;
    const int *budgets;
    const float *weights;
    const int *positions, *lengths;
    float *weights_out;
    int *positions_out, *lengths_out;
    int *counts;           // [units] rows that move
    int2 *moves;           // [units][cap / 2 + 1] (to, from)
    longlong2 *places;     // the same rows' element offsets in the pools, -1: no page
    int moves_max;
};
struct PoolTable {
    void *ptr[2 * WKV_MAX_GROUP_LAYERS];
};
int launch_evict(const EvictArgs &a, const PoolTable &pools, cudaStream_t stream);
int launch_seed_rows(const KShape &ks, const int *window_idx, const float *token_scores, int row_capacity, int *positions,
                     float *weights, cudaStream_t stream);

}  // namespace wkv
