// Eviction from the paged cache by accumulated attention weight, and the state that it goes by.
//
// First kernel, a block per unit: rows get 32-bit keys in the order of eviction, the key of the keep-th is found by a radix
// select of 8 bits per pass, and the rows that leave in front of row `keep` and those that stay behind it are listed, pairwise.
// Ties go to the lower row.  Bound by the latency of its steps, of which there are about 20 between barriers.
// Second kernel: every listed row of every layer's K and V is copied over its counterpart.  Targets lie in front of row `keep`
// and sources behind it, so the copies depend on nothing and a call repeated on the same lengths and weights does the same.
#include "attn.cuh"
#include "topk_block.cuh"

#include <algorithm>

namespace wkv {
namespace {

constexpr int kSelThreads = 1024;
constexpr int kMoveThreads = 256;
// Few rows are moved by the first kernel itself: up to so many, and so many vectors of 16 bytes in all.  (8 units of 992 rows, 4 layers, 9
// rows to move 10.1 us with a second kernel, 8.7 without; 25 rows 10.4 and 9.5; 92 rows, 11.8 K vectors, 10.5 and 13.4.)
constexpr int kFewMoves = 256, kFewVecs = 4096;
constexpr int kHeldKeys = 48 * 1024;        // keys that a block holds in shared memory (192 KB); longer lists are re-read

struct SelectSmem {
    int hist[256];
    int equal[32], holes[32], fills[32];
    int newest[32], recent[32];
    unsigned lowest[32], highest[32];
    unsigned prefix;
    int remaining;
};

// A row's place in the order as a key.  With no more recent rows than stay, they all do and have the highest key; with more,
// they alone are chosen among and all others have the lowest.  A weight's own key lies between (NaN: 1; -infinity's is 0x007fffff, infinity's
// 0xff800000).
__device__ __forceinline__ unsigned evict_key(float w, bool is_recent, bool among_recent)
{
    if (is_recent != among_recent) return is_recent ? 0xffffffffu : 0u;
    return w != w ? 1u : topk_order_key(w);
}

// MOVES: the rows are moved here as well, without a second kernel
template <bool MOVES>
__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const __grid_constant__ EvictArgs a, const __grid_constant__ PoolTable pools)
{
    extern __shared__ unsigned held[];
    __shared__ SelectSmem sm;
    __shared__ int2 few[MOVES ? kFewMoves : 1];
    __shared__ longlong2 few_places[MOVES ? kFewMoves : 1];
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x, b = unit / a.hkv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = min(max(a.lengths[unit], 0), a.cap), budget = max(a.budgets ? a.budgets[b] : a.budget, 0), keep = min(n, budget);
    const float *w = a.weights + (long long)unit * a.cap;
    const int *pos = a.positions + (long long)unit * a.cap;
    float *w_out = a.weights_out + (long long)unit * a.cap;
    int *pos_out = a.positions_out + (long long)unit * a.cap;
    if (w_out != w)
        for (int j = tid; j < keep; j += kSelThreads) w_out[j] = w[j];
    if (pos_out != pos)
        for (int j = tid; j < keep; j += kSelThreads) pos_out[j] = pos[j];
    int moved = 0;
    if (keep < n && keep > 0) {
        const bool hold = n <= kHeldKeys;
        int newest = INT_MIN;
        for (int j = tid; j < n; j += kSelThreads) {
            newest = max(newest, pos[j]);
            if (hold) held[j] = __float_as_uint(w[j]);
        }
        newest = __reduce_max_sync(0xffffffffu, newest);
        if (lane == 0) sm.newest[warp] = newest;
        if (tid < 256) sm.hist[tid] = 0;
        __syncthreads();
        newest = __reduce_max_sync(0xffffffffu, sm.newest[lane]);
        const long long recent_from = (long long)newest - a.recent;
        // The keys, for no more recent rows than stay; with more of them, once more.  lo and hi: of the rows that are chosen among.
        unsigned lo = 0xffffffffu, hi = 0u;
        auto range = [&](unsigned key) {
            if (key == 0u || key == 0xffffffffu) return;
            lo = min(lo, key);
            hi = max(hi, key);
        };
        int n_recent = 0;
        for (int j = tid; j < n; j += kSelThreads) {
            const bool is_recent = (long long)pos[j] > recent_from;
            const unsigned key = evict_key(hold ? __uint_as_float(held[j]) : w[j], is_recent, false);
            n_recent += is_recent;
            if (hold) held[j] = key;
            range(key);
        }
        n_recent = __reduce_add_sync(0xffffffffu, n_recent);
        if (lane == 0) sm.recent[warp] = n_recent;
        __syncthreads();
        const int all_recent = __reduce_add_sync(0xffffffffu, sm.recent[lane]);
        const bool among_recent = all_recent > keep;
        auto fresh_key = [&](int j) { return evict_key(w[j], (long long)pos[j] > recent_from, among_recent); };
        auto key_at = [&](int j) { return hold ? held[j] : fresh_key(j); };
        if (among_recent) {
            lo = 0xffffffffu;
            hi = 0u;
            for (int j = tid; j < n; j += kSelThreads) {
                const unsigned key = fresh_key(j);
                if (hold) held[j] = key;
                range(key);
            }
        }
        // Radix select among the rows that are chosen among (keys that are neither lowest nor highest), 8 bits at a time over the bits in
        // which they differ: counted from the top of all 32, nearly all weights share the first eight, and with them
        // one counter (8,192 rows: 26 us).
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        if (lane == 0) {
            sm.lowest[warp] = lo;
            sm.highest[warp] = hi;
        }
        __syncthreads();
        lo = __reduce_min_sync(0xffffffffu, sm.lowest[lane]);
        hi = __reduce_max_sync(0xffffffffu, sm.highest[lane]);
        unsigned prefix = 0u, mask = 0u;                          // of key - lo: bits that are known, and which
        int remaining = among_recent ? keep : keep - all_recent, top = lo <= hi ? 32 - __clz(hi - lo) : 0;
        const bool none = remaining == 0;                         // the recent ones are just as many as stay
#pragma unroll 1
        while (top > 0 && !none) {
            const int low = top > 8 ? top - 8 : 0;
            const unsigned digit = (1u << (top - low)) - 1u;
            for (int j = tid; j < n; j += kSelThreads) {
                const unsigned key = key_at(j), rk = key - lo;
                if (key != 0u && key != 0xffffffffu && (rk & mask) == prefix) atomicAdd(&sm.hist[(rk >> low) & digit], 1);
            }
            __syncthreads();
            if (warp == 0) {
                int c[8], mine = 0;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    c[x] = sm.hist[lane * 8 + x];
                    mine += c[x];
                }
                int upto = mine;                       // in this lane's bins and the higher lanes'
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int t = __shfl_down_sync(0xffffffffu, upto, o);
                    if (lane + o < 32) upto += t;
                }
                int above = upto - mine;
                if (above < remaining && remaining <= upto) {
#pragma unroll
                    for (int x = 7; x >= 0; --x) {
                        if (above < remaining && remaining <= above + c[x]) {
                            sm.prefix = prefix | (unsigned)(lane * 8 + x) << low;
                            sm.remaining = remaining - above;
                        }
                        above += c[x];
                    }
                }
            }
            __syncthreads();
            prefix = sm.prefix;
            remaining = sm.remaining;
            if (tid < 256) sm.hist[tid] = 0;
            __syncthreads();
            mask |= digit << low;
            top = low;
        }
        // the threshold, and how many of the rows that equal it stay (the lower ones)
        const unsigned threshold = none ? 0xffffffffu : prefix + lo;
        if (none) remaining = keep;
        // The rows in order, a part for each warp: which stay, and the two lists.  Three walks, with the warps' counts between them.
        int2 *moves = MOVES ? few : a.moves + (long long)unit * a.moves_max;
        const int moves_max = MOVES ? kFewMoves : a.moves_max;
        const int per = ((n + 31) / 32 + 31) / 32 * 32, part0 = (int)min((long long)warp * per, (long long)n), part1 = (int)min((long long)part0 + per, (long long)n);
        const unsigned lower = (1u << lane) - 1u;
        int equal = 0, holes = 0, fills = 0;
        for (int j0 = part0; j0 < part1; j0 += 32) equal += __popc(__ballot_sync(0xffffffffu, j0 + lane < part1 && key_at(j0 + lane) == threshold));
        if (lane == 0) sm.equal[warp] = equal;
        __syncthreads();
        const int equal_before = __reduce_add_sync(0xffffffffu, lane < warp ? sm.equal[lane] : 0);
        auto walk = [&](auto visit) {                  // visit(row, leaves in front of row `keep`, stays behind it)
            int before = equal_before;
            for (int j0 = part0; j0 < part1; j0 += 32) {
                const int j = j0 + lane;
                const unsigned key = j < part1 ? key_at(j) : 0u;
                const bool same = j < part1 && key == threshold;
                const unsigned votes = __ballot_sync(0xffffffffu, same);
                const bool stays = j < part1 && (key > threshold || (same && before + __popc(votes & lower) < remaining));
                before += __popc(votes);
                visit(j, __ballot_sync(0xffffffffu, j < part1 && j < keep && !stays), __ballot_sync(0xffffffffu, j >= keep && stays));
            }
        };
        walk([&](int, unsigned out, unsigned in) {
            holes += __popc(out);
            fills += __popc(in);
        });
        if (lane == 0) {
            sm.holes[warp] = holes;
            sm.fills[warp] = fills;
        }
        __syncthreads();
        int hole = __reduce_add_sync(0xffffffffu, lane < warp ? sm.holes[lane] : 0), fill = __reduce_add_sync(0xffffffffu, lane < warp ? sm.fills[lane] : 0);
        holes = __reduce_add_sync(0xffffffffu, sm.holes[lane]);
        fills = __reduce_add_sync(0xffffffffu, sm.fills[lane]);
        walk([&](int j, unsigned out, unsigned in) {
            if (out >> lane & 1u && hole + __popc(out & lower) < moves_max) moves[hole + __popc(out & lower)].x = j;
            if (in >> lane & 1u && fill + __popc(in & lower) < moves_max) moves[fill + __popc(in & lower)].y = j;
            hole += __popc(out);
            fill += __popc(in);
        });
        moved = min(min(holes, fills), moves_max);
        __syncthreads();                               // the lists are complete (and the copies above)
        // (where the rows are, for the second kernel: its blocks would each look that up for every tensor)
        longlong2 *places = MOVES ? few_places : a.places + (long long)unit * a.moves_max;
        auto place = [&](int row) -> long long {
            const int pg = row / a.page_size, page = __ldg(a.table + (long long)b * a.max_pages + pg);
            if ((unsigned)page >= (unsigned)a.num_pages) return -1;
            return page * a.page_stride + (unit - b * a.hkv) * a.head_stride + (row - pg * a.page_size) * a.row_stride;
        };
        for (int x = tid; x < moved; x += kSelThreads) {
            const int2 mv = moves[x];
            places[x] = make_longlong2(place(mv.x), place(mv.y));
            w_out[mv.x] = w[mv.y];
            pos_out[mv.x] = pos[mv.y];
        }
    }
    __syncthreads();                                   // lengths_out may be lengths: all have read it (and the places are there)
    if (MOVES) {
        const int vecs = a.d * a.elem_bytes / 16, each = moved * vecs;
        for (int x = tid; x < each * a.n_tensors; x += kSelThreads) {
            const int tensor = x / each, y = x - tensor * each, move = y / vecs, v = y - move * vecs;
            const longlong2 at = few_places[move];
            if (at.x < 0 || at.y < 0) continue;
            char *pool = static_cast<char *>(pools.ptr[tensor]);
            reinterpret_cast<int4 *>(pool + at.x * a.elem_bytes)[v] = reinterpret_cast<const int4 *>(pool + at.y * a.elem_bytes)[v];
        }
    }
    if (tid == 0) {
        a.counts[unit] = moved;
        a.lengths_out[unit] = keep;
    }
}

// A quarter, half or whole warp per row (`lanes` of them), two rows in flight each.  Bound by memory, in pieces of one row: 128 units of
// 4-8 K rows of 256 bytes to 3,932, four layers: 0.68 GB read and written, 146 us with the selection.  Four rows in flight (40
// registers) 148, one 154; with the rows' places looked up here, 204.
constexpr int kAhead = 2;
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictArgs a, const __grid_constant__ PoolTable pools,
                                                                  int lanes_shift)
{
    pdl_trigger();
    pdl_wait();
    const int units = a.batch * a.hkv, unit = blockIdx.x % units, tensor = blockIdx.x / units;
    const int moved = a.counts[unit], lanes = 1 << lanes_shift, lane = threadIdx.x & (lanes - 1);
    const int step = (int)gridDim.y * (kMoveThreads >> lanes_shift), vecs = a.d * a.elem_bytes / 16;
    const longlong2 *places = a.places + (long long)unit * a.moves_max;
    char *pool = static_cast<char *>(pools.ptr[tensor]);
    for (int x0 = (int)blockIdx.y * (kMoveThreads >> lanes_shift) + (threadIdx.x >> lanes_shift); x0 < moved; x0 += step * kAhead) {
        longlong2 at[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) at[u] = x0 + u * step < moved ? places[x0 + u * step] : make_longlong2(-1, -1);
        for (int v = lane; v < vecs; v += lanes) {
            int4 y[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (at[u].x >= 0 && at[u].y >= 0) y[u] = reinterpret_cast<const int4 *>(pool + at[u].y * a.elem_bytes)[v];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (at[u].x >= 0 && at[u].y >= 0) reinterpret_cast<int4 *>(pool + at[u].x * a.elem_bytes)[v] = y[u];
        }
    }
}

__global__ void __launch_bounds__(256) seed_rows_kernel(const __grid_constant__ KShape s, const int *window_idx, const float *token_scores,
                                                        int row_capacity, int *positions, float *weights, int blocks)
{
    pdl_trigger();
    pdl_wait();
    const int unit = (int)blockIdx.x / blocks, part = (int)blockIdx.x - unit * blocks, b = unit / s.hkv;
    const SeqInfo si = seq_info(s, b);
    const int n_r = si.n > s.alpha ? si.n - s.alpha : 0, kw = num_windows(si.n, s.alpha, s.omega);
    const int k = num_selected_capped(si.n, s.alpha, s.omega, si.budget, s.k_max);
    const int *idx = window_idx + (long long)unit * s.k_max;
    int review = k * s.omega;
    if (k > 0 && idx[k - 1] == kw - 1) review -= kw * s.omega - n_r;      // the sequence's short last window
    review = min(review, n_r);
    for (int r = part * (int)blockDim.x + (int)threadIdx.x; r < review + si.n - n_r && r < row_capacity; r += blocks * (int)blockDim.x) {
        int at;
        float w = 0.f;
        if (r < review) {
            const int wi = idx[r / s.omega];
            at = wi * s.omega + r % s.omega;
            if (wi < 0 || wi >= kw || at >= n_r) continue;                // no window of the sequence: the row stays as it is
            if (token_scores) w = token_scores[(long long)unit * s.nr_max + at];
        } else {
            at = n_r + (r - review);
        }
        if (positions) positions[(long long)unit * row_capacity + r] = at;
        if (weights) weights[(long long)unit * row_capacity + r] = w;
    }
}

}  // namespace

int launch_evict(const EvictArgs &a, const PoolTable &pools, cudaStream_t stream)
{
    const int units = a.batch * a.hkv;
    const size_t smem = (size_t)(a.cap < kHeldKeys ? a.cap : kHeldKeys) * sizeof(unsigned);
    const int vecs = a.d * a.elem_bytes / 16;
    // Rows that a unit can have to move: what the budget leaves over, as far as the host knows it.
    long long most_moves = a.moves_max;
    if (!a.budgets) most_moves = std::min(most_moves, (long long)std::min(a.budget, std::max(a.cap - a.budget, 0)));
    const bool here = most_moves <= kFewMoves && most_moves * vecs * a.n_tensors <= kFewVecs;
    static SmemAsked asked[2];
    cudaError_t err = here ? allow_smem(evict_select_kernel<true>, kHeldKeys * 4, asked[1]) : allow_smem(evict_select_kernel<false>, kHeldKeys * 4, asked[0]);
    if (err == cudaSuccess) err = here ? launch_pdl(evict_select_kernel<true>, dim3(units), kSelThreads, smem, stream, 1, a, pools)
                                       : launch_pdl(evict_select_kernel<false>, dim3(units), kSelThreads, smem, stream, 1, a, pools);
    if (err != cudaSuccess) return check_cuda(err, "eviction kernel");
    count_launches(1);
    if (here) return WKV_OK;
    int lanes_shift = 5;
    while (lanes_shift > 2 && (1 << (lanes_shift - 1)) >= vecs) --lanes_shift;
    // several times as many blocks as the GPU holds (eight of 256 threads per SM), so that units of different lengths even out
    const long long pairs = (long long)units * a.n_tensors;
    if (pairs > 0x7fffffffLL) {
        set_error_detail("eviction: %lld (unit, tensor) pairs", pairs);
        return WKV_ERR_LIMIT;
    }
    long long slices = (148 * 64 + pairs - 1) / pairs;
    const long long rows = kAhead * (kMoveThreads >> lanes_shift), most = (most_moves + rows - 1) / rows;
    if (slices > most) slices = most;
    if (slices < 1) slices = 1;
    err = launch_pdl(evict_move_kernel, dim3((unsigned)pairs, (unsigned)slices), kMoveThreads, 0, stream, 1, a, pools, lanes_shift);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "eviction kernel (rows)");
}

int launch_seed_rows(const KShape &ks, const int *window_idx, const float *token_scores, int row_capacity, int *positions,
                     float *weights, cudaStream_t stream)
{
    const long long units = (long long)ks.batch * ks.hkv;
    int blocks = row_capacity > 256 * 16 ? 16 : (row_capacity + 255) / 256;
    if (blocks < 1 || units * blocks > 0x7fffffffLL) blocks = 1;
    if (units > 0x7fffffffLL) {
        set_error_detail("%lld (sequence, KV head) pairs", units);
        return WKV_ERR_LIMIT;
    }
    const cudaError_t err = launch_pdl(seed_rows_kernel, dim3((unsigned)(units * blocks)), 256, 0, stream, 1, ks, window_idx, token_scores,
                                       row_capacity, positions, weights, blocks);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "row state kernel");
}

}  // namespace wkv
