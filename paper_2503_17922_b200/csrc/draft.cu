// Drafted tokens: the masks of a tree, and what is kept of a draft once it has been judged.
//
// Masks: a thread per token follows its parents, whose numbers fall at every step, and writes a word when it leaves it.
// Keeping: a token's row moves to that of a lower number or stays, and a row that one token takes is an earlier token's or its own.  So every
// thread walks over the path in ascending order with its own 16 bytes of the rows, a few rows read ahead: what it overwrites it has read before.
//
// Bound by latency, a launch each: of one draft of 12 tokens over 992 rows the masks take 1.5-2.0 us and keeping a path of one layer 4.6 (2.7 where no row moves), of 16 drafts of up to 64 tokens
// 2.0-2.1 and 3.2-3.6, each in a graph of 20.
#include "attn.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 128;
constexpr int kAhead = 4;

__global__ void __launch_bounds__(kThreads) draft_masks_kernel(int batch, int max_q, int total_q, const int *cu_q, const int *parents, int words,
                                                               unsigned *masks, const int *first, int *positions)
{
    pdl_trigger();
    pdl_wait();
    const int b = blockIdx.x;
    long long off = (long long)b * max_q;
    int m = max_q;
    if (cu_q) {
        const int lo = min(max(cu_q[b], 0), total_q);
        m = min(min(max(cu_q[b + 1] - cu_q[b], 0), max_q), total_q - lo);
        off = lo;
    }
    for (int i = threadIdx.x; i < m; i += kThreads) {
        unsigned *mask = masks ? masks + (off + i) * words : nullptr;
        int at = i, word = words - 1, depth = 0;
        unsigned bits = 0u;
        for (;;) {
            while (word > at >> 5) {
                if (mask) mask[word] = bits;
                bits = 0u;
                --word;
            }
            bits |= 1u << (at & 31);
            const int parent = parents[off + at];
            if (parent < 0 || parent >= at) break;
            at = parent;
            ++depth;
        }
        for (; word >= 0; --word, bits = 0u)
            if (mask) mask[word] = bits;
        if (positions) positions[off + i] = (first ? first[b] : 0) + depth;
    }
}

__global__ void __launch_bounds__(kThreads) keep_draft_kernel(const __grid_constant__ DraftArgs a, const __grid_constant__ PoolTable pools,
                                                              const __grid_constant__ ScaleTable scales)
{
    __shared__ short path[WKV_MAX_DRAFT];
    __shared__ int counts[kThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int units = a.batch * a.hkv, unit = (int)blockIdx.x % units, tensor = (int)blockIdx.x / units, b = unit / a.hkv, h = unit - b * a.hkv;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int m = a.max_q;
    long long off = (long long)b * a.max_q;
    if (a.cu_q) {
        const int lo = min(max(a.cu_q[b], 0), a.total_q);
        m = min(min(max(a.cu_q[b + 1] - a.cu_q[b], 0), a.max_q), a.total_q - lo);
        off = lo;
    }
    const int n = min(max(a.lengths[unit], 0), a.cap);
    // rows in front of the draft (negative: its first tokens have no row; given: its last ones may have none)
    const int before = a.before ? min(max(a.before[unit], max(n - m, 0)), n) : n - m;
    const int last = a.last[b];
    const unsigned *mask = (unsigned)last < (unsigned)m ? a.masks + (off + last) * a.words : nullptr;
    // the path's tokens that have a row, in order
    int count = 0;
    for (int j0 = 0; j0 < m && mask; j0 += kThreads) {
        const int j = j0 + tid;
        const bool on = j < m && before + j >= 0 && before + j < n && (mask[j >> 5] >> (j & 31) & 1u);
        const unsigned votes = __ballot_sync(0xffffffffu, on);
        if (lane == 0) counts[warp] = __popc(votes);
        __syncthreads();
        int at = count;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) at += counts[w];
            count += counts[w];
        }
        if (on) path[at + __popc(votes & ((1u << lane) - 1u))] = (short)j;
        __syncthreads();
    }
    const int to0 = max(before, 0);
    auto page_of = [&](int row, int &slot) {
        const int pg = row / a.pages.page_size;
        slot = row - pg * a.pages.page_size;
        return __ldg(a.pages.table + (long long)b * a.pages.max_pages + pg);
    };
    const int vecs = a.d * a.elem_bytes / 16;
    if (tid < vecs + (a.scaled ? 1 : 0)) {
        // a thread's piece: 16 bytes, or the scale
        const bool scale = tid == vecs;
        char *const pool = scale ? reinterpret_cast<char *>(scales.ptr[tensor]) : static_cast<char *>(pools.ptr[tensor]);
        auto place = [&](int row) -> char * {
            int slot;
            const int page = page_of(row, slot);
            if ((unsigned)page >= (unsigned)a.pages.num_pages) return nullptr;
            if (scale) return pool + ((long long)page * a.hkv + h) * a.pages.page_size + slot;
            return pool + (page * a.pages.page_stride + h * a.pages.head_stride + slot * a.pages.row_stride) * a.elem_bytes + tid * 16;
        };
        for (int x0 = 0; x0 < count; x0 += kAhead) {
            int4 v[kAhead];
            char *to[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                to[u] = nullptr;
                if (x0 + u >= count) continue;
                const int from_row = before + path[x0 + u], to_row = to0 + x0 + u;
                const char *from = from_row != to_row ? place(from_row) : nullptr;
                if (!from) continue;
                to[u] = place(to_row);
                if (scale) v[u].x = *reinterpret_cast<const unsigned char *>(from);
                else v[u] = *reinterpret_cast<const int4 *>(from);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (!to[u]) continue;
                if (scale) *reinterpret_cast<unsigned char *>(to[u]) = (unsigned char)v[u].x;
                else *reinterpret_cast<int4 *>(to[u]) = v[u];
            }
        }
    }
    if (tensor != 0) return;
    // the rows' state, by the unit's first block
    for (int x0 = 0; x0 < count; x0 += kThreads) {
        const int x = x0 + tid;
        int position = 0;
        float weight = 0.f;
        const long long base = (long long)unit * a.cap;
        if (x < count) {
            const long long from = base + before + path[x];
            if (a.row_positions) position = a.row_positions[from];
            if (a.row_weights) weight = a.row_weights[from];
        }
        __syncthreads();
        if (x < count) {
            if (a.row_positions) a.row_positions[base + to0 + x] = position;
            if (a.row_weights) a.row_weights[base + to0 + x] = weight;
        }
        __syncthreads();
    }
    if (tid == 0) a.lengths_out[unit] = to0 + count;
}

}  // namespace

int launch_draft_masks(int batch, int max_q, int total_q, const int *cu_q, const int *parents, int words, unsigned *masks, const int *first,
                       int *positions, cudaStream_t stream)
{
    const cudaError_t err = launch_pdl(draft_masks_kernel, dim3((unsigned)batch), kThreads, 0, stream, 1, batch, max_q, total_q, cu_q, parents, words, masks,
                                       first, positions);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "draft masks kernel");
}

int launch_keep_draft(const DraftArgs &a, const PoolTable &pools, const ScaleTable &scales, cudaStream_t stream)
{
    const long long blocks = (long long)a.batch * a.hkv * a.n_tensors;
    if (blocks > 0x7fffffffLL || a.d * a.elem_bytes / 16 + 1 > kThreads) {
        set_error_detail("draft: %lld (unit, tensor) pairs, rows of %d bytes", blocks, a.d * a.elem_bytes);
        return WKV_ERR_LIMIT;
    }
    int st = check_once(pools, a.n_tensors, "pools");
    if (st == WKV_OK && a.scaled) st = check_once(scales, a.n_tensors, "scales");
    if (st != WKV_OK) return st;
    const cudaError_t err = launch_pdl(keep_draft_kernel, dim3((unsigned)blocks), kThreads, 0, stream, 1, a, pools, scales);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "draft kernel");
}

}  // namespace wkv
