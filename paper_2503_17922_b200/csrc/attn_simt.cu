// Attention on the CUDA cores for fp32, its weights kernel, and the joining kernels of all types.  One block holds ROWS rows of one
// unit in shared memory and walks over the unit's keys in tiles of 64 with a running maximum and sum per row; everything is
// fp32, products in plain multiply-adds of pairs.  A thread has ROWS / 16 rows x 4 keys, then as many rows x d / 16 columns.
//
// Bound by the reads of shared memory (80 % of their peak at 4,096 tokens): 16 bytes to every thread of a warp take four cycles whatever
// the addresses, so that 64 products per thread cost 32 of them with 4 rows to a thread and 24 with 8.  32 heads on 8 of 4,096
// tokens: d = 64 1,815 us (38 TFLOP/s; with 8 rows about an eighth more, a block per SM then instead of two), d = 128 3,440 us with 8 rows
// (40 TFLOP/s; about 4,700 with 4).
//
// ROWS is the largest of 128 (d above 64), 64, 32 and 16 that gives nearly every SM a block.  A prompt without enough of them has its keys split over
// the blocks of a cluster; paged rows are split by the caller.
//
// With S key splits a block walks over one of S parts of the keys and leaves (maximum, sum, unnormalised output) per row for
// the joining kernel.  A row's sums are taken in an order that the launch's sizes give, never in that of arrival.
#include "attn_cluster.cuh"
#include "score_math.cuh"

#include <type_traits>

namespace wkv {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;

__device__ __forceinline__ void from_float(float &y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16 &y, float x) { y = __float2bfloat16_rn(x); }

__device__ __forceinline__ unsigned long long mul_pair(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// four elements of a row of d into shared memory, zeros from d on; `p` null: zeros
template <int DP>
__device__ __forceinline__ void load_row_part(float *dst, const float *p, int d, int part)
{
    const int c = part * 4;
    *reinterpret_cast<float4 *>(dst + c) = p && c < d ? *reinterpret_cast<const float4 *>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
}

// Stages of key tiles: with 16 rows the loads take as long as the arithmetic, and the next tile's come during this one's.  With more
// rows a tile's values come during the product with its keys, and the next keys during that with the values, in half the memory.
template <int DP, int ROWS>
struct SimtSmem {
    static constexpr int kStages = ROWS == 16 && DP <= 128 ? 2 : 1;
    float q[ROWS][DP + 4];
    float k[kStages][kKeys][DP + 4];
    float v[kStages][kKeys][DP];
    float p[ROWS][kKeys + 4];
    int present[2][kKeys];                 // the key's page is one
    float m[ROWS], l[ROWS], lse2[16];
};
template <int DP>
struct WeightsSmem {
    float q[64][DP + 4];
    float k[kKeys][DP + 4];
    float sums[16][kKeys + 1];
    int present[kKeys];
};

// The keys or the values of a tile, on their way; rows from n on and rows without a page are zeros.  A row's vectors lie in neighbouring
// threads, and a thread has EACH rows.  Their pages are looked up some work ahead, as that is a trip to memory.
template <int DP>
struct Fetch {
    static constexpr int kParts = DP / 4, kEach = kKeys * kParts / kThreads, kStep = kThreads / kParts;
    int page[kEach], slot[kEach];
    long long at[kEach];                   // element offsets, -1: none
    __device__ __forceinline__ void look_up(const AttnArgs &a, int b, int n, int j0)
    {
        if (!a.table) return;
#pragma unroll
        for (int x = 0; x < kEach; ++x) {
            const int j = j0 + (int)threadIdx.x / kParts + x * kStep, pg = j / a.page_size;
            slot[x] = j - pg * a.page_size;
            page[x] = j < n ? __ldg(a.table + (long long)b * a.max_pages + pg) : -1;
        }
    }
    __device__ __forceinline__ void place(const AttnArgs &a, int *present, int h, long long dense, int n, int j0)
    {
#pragma unroll
        for (int x = 0; x < kEach; ++x) {
            const int r = (int)threadIdx.x / kParts + x * kStep, j = j0 + r;
            if (a.table) at[x] = (unsigned)page[x] < (unsigned)a.num_pages ? page[x] * a.kb + h * a.kh + slot[x] * a.kt : -1;
            else at[x] = j < n ? dense + j * a.kt : -1;
            if (threadIdx.x % kParts == 0) present[r] = at[x] >= 0;
        }
    }
    __device__ __forceinline__ void issue(const AttnArgs &a, const void *from, float *to, int stride) const
    {
        const int c = (int)(threadIdx.x % kParts) * 4;
#pragma unroll
        for (int x = 0; x < kEach; ++x) {
            const int r = (int)threadIdx.x / kParts + x * kStep;
            const bool have = at[x] >= 0 && c < a.d;
            const float *p = static_cast<const float *>(from) + (have ? at[x] + c : 0);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to + r * stride + c))), "l"(p), "r"(have ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
};
template <int DP>
__device__ __forceinline__ void load_keys(const AttnArgs &a, WeightsSmem<DP> &sm, int b, int h, long long off, int n, int j0)
{
    constexpr int kParts = DP / 4;
    for (int x = threadIdx.x; x < kKeys * kParts; x += kThreads) {
        const int r = x / kParts, part = x - r * kParts, j = j0 + r;
        const long long at = j < n ? attn_row(a, b, h, off, j) : -1;
        load_row_part<DP>(sm.k[r], at >= 0 ? static_cast<const float *>(a.k) + at : nullptr, a.d, part);
        if (part == 0) sm.present[r] = at >= 0;
    }
}
template <int DP, int ROWS>
__device__ __forceinline__ void load_queries(const AttnArgs &a, float (&q)[ROWS][DP + 4], int b, int h, long long off, int row0, int rows)
{
    constexpr int kParts = DP / 4;
    for (int x = threadIdx.x; x < ROWS * kParts; x += kThreads) {
        const int r = x / kParts, part = x - r * kParts, row = row0 + r, i = row / a.G, g = row - i * a.G;
        const float *p = row < rows ? static_cast<const float *>(a.q) + (off + i) * a.qt + b * a.qb + (long long)(h * a.G + g) * a.qh : nullptr;
        load_row_part<DP>(q[r], p, a.d, part);
    }
}
// logits (base 2) of rows ty*RT.. against keys tx + 16 j
template <int DP, int ROWS>
__device__ __forceinline__ void logits(const float (&q)[ROWS][DP + 4], const float (&k)[kKeys][DP + 4], int ty, int tx, float c, float (&s)[ROWS / 16][4])
{
    constexpr int RT = ROWS / 16;
    // products of pairs: sums over the even and the odd elements apart
    unsigned long long sum[RT][4] = {};
#pragma unroll (ROWS >= 128 ? 2 : 4)
    for (int e = 0; e < DP; e += 4) {
        ulonglong2 qv[RT], kv[4];
#pragma unroll
        for (int r = 0; r < RT; ++r) qv[r] = *reinterpret_cast<const ulonglong2 *>(&q[ty * RT + r][e]);
#pragma unroll
        for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const ulonglong2 *>(&k[tx + 16 * j][e]);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum[r][j] = fma_pair(qv[r].x, kv[j].x, sum[r][j]);
                sum[r][j] = fma_pair(qv[r].y, kv[j].y, sum[r][j]);
            }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 x = halves_of(sum[r][j]);
            s[r][j] = (x.x + x.y) * c;
        }
}

template <int DP, int ROWS>
__global__ void __launch_bounds__(kThreads, ROWS == 64 && DP == 64 ? 2 : (DP == 64 && ROWS < 64 ? 3 : 1)) attn_simt_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SimtSmem<DP, ROWS> &sm = *reinterpret_cast<SimtSmem<DP, ROWS> *>(raw);
    constexpr int RT = ROWS / 16, CT = DP / 64, NS = SimtSmem<DP, ROWS>::kStages;
    // The joining kernel may be placed now.  Another of this kind is not to be before this one ends: its blocks would crowd onto the
    // SMs that have room at that time.
    const bool clustered = a.clustered, parts = !clustered && (a.splits > 1 || a.logits);
    if (parts) pdl_trigger();
    pdl_wait();
    const int units = a.batch * a.hkv;
    // the last rows of a prompt have the most keys: they are taken first
    const int splits = a.splits, place = (int)blockIdx.x / splits, split = (int)blockIdx.x - place * splits;
    const int tiles = (int)gridDim.x / splits / units, unit = place % units, tile = tiles - 1 - place / units;
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const AttnSeq sq = attn_seq(a, b, h);
    const int rows = sq.m * a.G, row0 = tile * ROWS;
    if (row0 >= rows) {
        if (clustered) carry_weights(a, unit, (int)((long long)sq.n * split / splits), (int)((long long)sq.n * (split + 1) / splits), kThreads);
        return;
    }
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    const int base = sq.n - sq.m + 1;                                    // keys that query 0 attends to (may be negative)
    const int most = min(base + (min(row0 + ROWS, rows) - 1) / a.G, sq.n);
    const int all_tiles = (max(most, 0) + kKeys - 1) / kKeys;
    const int t0 = (int)((long long)all_tiles * split / splits), t1 = (int)((long long)all_tiles * (split + 1) / splits);
    int limit[RT];
    float m[RT], l[RT];
    unsigned long long o[RT][CT][2];                                     // pairs of columns
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        limit[r] = base + (row0 + ty * RT + r) / a.G;
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int x = 0; x < CT; ++x) o[r][x][0] = o[r][x][1] = 0ull;
    }
    const long long dense = sq.q_off * a.kt + b * a.kb + h * a.kh;
    Fetch<DP> rows_of;
    auto fetch_keys = [&](int t) {
        rows_of.place(a, sm.present[t & 1], h, dense, sq.n, t * kKeys);
        rows_of.issue(a, a.k, &sm.k[t % NS][0][0], DP + 4);
    };
    auto fetch_values = [&](int t) { rows_of.issue(a, a.v, &sm.v[t % NS][0][0], DP); };
    if (t0 < t1) {
        rows_of.look_up(a, b, sq.n, t0 * kKeys);
        fetch_keys(t0);
        fetch_values(t0);
        if (NS == 2) rows_of.look_up(a, b, sq.n, (t0 + 1) * kKeys);
    }
    load_queries<DP, ROWS>(a, sm.q, b, h, sq.q_off, row0, rows);
    if (NS == 1) {
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncthreads();
    }
    const int plain = base + row0 / a.G;                                 // every row attends to the keys before this one
    for (int t = t0; t < t1; ++t) {
        const int j0 = t * kKeys, st = t % NS;
        if (NS == 2) {
            if (t + 1 < t1) {
                fetch_keys(t + 1);
                fetch_values(t + 1);
                rows_of.look_up(a, b, sq.n, j0 + 2 * kKeys);
                asm volatile("cp.async.wait_group 2;" ::: "memory");
            } else {
                asm volatile("cp.async.wait_group 0;" ::: "memory");
            }
            __syncthreads();
        } else {
            rows_of.look_up(a, b, sq.n, j0 + kKeys);
        }
        float s[RT][4];
        logits<DP, ROWS>(sm.q, sm.k[st], ty, tx, a.scale_log2, s);
        if (NS == 1) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();                                             // the values have landed for all, and nobody reads the keys any more
            if (t + 1 < t1) fetch_keys(t + 1);
        }
        const bool guarded = j0 + kKeys > plain;
        if (guarded || a.table) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j0 + tx + 16 * j >= limit[r] || !sm.present[t & 1][tx + 16 * j]) s[r][j] = -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = m[r];
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, s[r][j]);
            if (ROWS == 16 && a.logits && row0 + ty < rows) {
                float *to = a.logits + ((long long)unit * a.rows_max + row0 + ty) * a.logit_stride + j0 + tx;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j0 + tx + 16 * j < sq.n) to[16 * j] = s[r][j];
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
            const float ref = top == -INFINITY ? 0.f : top;              // nothing to attend to so far
            const float keep = exp2f(m[r] - ref);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f(s[r][j] - ref);
                sm.p[ty * RT + r][tx + 16 * j] = p;
                sum += p;
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
            l[r] = l[r] * keep + sum;
            m[r] = top;
            const unsigned long long keep2 = pair_of(keep, keep);
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                o[r][x][0] = mul_pair(o[r][x][0], keep2);
                o[r][x][1] = mul_pair(o[r][x][1], keep2);
            }
        }
        __syncwarp();                                                    // a row's 16 threads are in one warp
        // What stands behind a row's position may be infinite or NaN, and 0 times that is not 0: tiles with such rows go by the rows' limits
        // (a weight of 0 would leave out a seen infinity too; rows without a page are zeros), as far as any row sees them.
        auto product = [&](auto skip_unseen) {
            const int end = decltype(skip_unseen)::value ? min(kKeys, most - j0) : kKeys;
#pragma unroll (decltype(skip_unseen)::value ? 1 : 2)
            for (int j = 0; j < end; j += 4) {
                float4 pp[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) pp[r] = *reinterpret_cast<const float4 *>(&sm.p[ty * RT + r][j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ulonglong2 v[CT];
#pragma unroll
                    for (int x = 0; x < CT; ++x) v[x] = *reinterpret_cast<const ulonglong2 *>(&sm.v[st][j + e][tx * 4 + 64 * x]);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const float p = e == 0 ? pp[r].x : (e == 1 ? pp[r].y : (e == 2 ? pp[r].z : pp[r].w));
                        if (decltype(skip_unseen)::value && j0 + j + e >= limit[r]) continue;
                        const unsigned long long p2 = pair_of(p, p);
#pragma unroll
                        for (int x = 0; x < CT; ++x) {
                            o[r][x][0] = fma_pair(p2, v[x].x, o[r][x][0]);
                            o[r][x][1] = fma_pair(p2, v[x].y, o[r][x][1]);
                        }
                    }
                }
            }
        };
        if (guarded) product(std::true_type{});
        else product(std::false_type{});
        if (NS == 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();                                                 // the next keys have landed for all, and nobody reads the values any more
        if (NS == 1 && t + 1 < t1) fetch_values(t + 1);
    }
    auto columns = [&](int r, int x) {
        const float2 lo = halves_of(o[r][x][0]), hi = halves_of(o[r][x][1]);
        return make_float4(lo.x, lo.y, hi.x, hi.y);
    };
    if (!parts) pdl_trigger();
    if (clustered) {
        __syncthreads();
        float *const all = &sm.q[0][0];                                  // [ROWS][DP + 4]: the queries are not needed any more
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (tx == 0) {
                sm.m[ty * RT + r] = m[r];
                sm.l[ty * RT + r] = l[r];
            }
#pragma unroll
            for (int x = 0; x < CT; ++x) *reinterpret_cast<float4 *>(all + (ty * RT + r) * (DP + 4) + tx * 4 + 64 * x) = columns(r, x);
        }
        cluster_join<float, kThreads, ROWS == 16>(a, sq, unit, b, h, row0, min(ROWS, rows - row0), split, sm.m, sm.l, all, DP + 4, sm.lse2, t0 * kKeys,
                                      min(t1 * kKeys, sq.n));
        return;
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = row0 + ty * RT + r;
        if (row >= rows) continue;
        const int i = row / a.G, hq = h * a.G + row - i * a.G;
        if (parts) {
            const long long at = ((long long)unit * a.rows_max + row) * a.splits + split;
            if (tx == 0) a.part_ml[at] = make_float2(m[r], l[r]);
            if (l[r] == 0.f) continue;
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                const int c = tx * 4 + 64 * x;
                if (c < a.d) *reinterpret_cast<float4 *>(a.part_o + at * a.d + c) = columns(r, x);
            }
            continue;
        }
        if (tx == 0) attn_store_lse(a, b, hq, i, sq.m, l[r] > 0.f || l[r] != l[r] ? m[r] + log2f(l[r]) : -INFINITY);
        const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
        float *dst = static_cast<float *>(a.out) + (sq.q_off + i) * a.ot + b * a.ob + (long long)hq * a.oh;
#pragma unroll
        for (int x = 0; x < CT; ++x) {
            const int c = tx * 4 + 64 * x;
            const float4 y = columns(r, x);
            if (c < a.d) *reinterpret_cast<float4 *>(dst + c) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
        }
    }
}

// Weights that the rows of the cache receive: one block per 64 rows of a unit sums exp2(logit - lse) over all of the unit's
// queries.  The logits are computed once more, from the normalisers that the attention has written; sums in a fixed order.
template <int DP>
__global__ void __launch_bounds__(kThreads) attn_weights_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr int ROWS = 64, RT = ROWS / 16;
    extern __shared__ __align__(16) unsigned char raw[];
    WeightsSmem<DP> &sm = *reinterpret_cast<WeightsSmem<DP> *>(raw);
    pdl_wait();
    const int units = a.batch * a.hkv, unit = (int)blockIdx.x % units, j0 = (int)blockIdx.x / units * kKeys;
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const AttnSeq sq = attn_seq(a, b, h);
    if (j0 >= sq.n) return;
    const int rows = sq.m * a.G, base = sq.n - sq.m + 1;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    load_keys<DP>(a, sm, b, h, sq.q_off, sq.n, j0);
    float got[4] = {0.f, 0.f, 0.f, 0.f};
    // queries in front of the tile's first key do not attend to any of it
    const long long first = base > j0 ? 0 : (long long)(j0 - base + 1) * a.G;
    for (int row0 = (int)(first / ROWS * ROWS); row0 < rows; row0 += ROWS) {
        __syncthreads();
        load_queries<DP, ROWS>(a, sm.q, b, h, sq.q_off, row0, rows);
        __syncthreads();
        float s[RT][4];
        logits<DP, ROWS>(sm.q, sm.k, ty, tx, a.scale_log2, s);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = row0 + ty * RT + r, i = row / a.G, hq = h * a.G + row - i * a.G;
            if (row >= rows) continue;
            const float lse2 = a.lse[((long long)b * a.hq + hq) * a.max_q + i] * 1.44269504088896341f;
            if (lse2 == -INFINITY) continue;                             // nothing to attend to, or logits of -infinity alone
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j0 + tx + 16 * j < base + i && sm.present[tx + 16 * j]) got[j] += exp2f(s[r][j] - lse2);
        }
    }
    pdl_trigger();
#pragma unroll
    for (int j = 0; j < 4; ++j) sm.sums[ty][tx + 16 * j] = got[j];
    __syncthreads();
    if (threadIdx.x < kKeys && j0 + (int)threadIdx.x < sq.n) {
        float w = 0.f;
#pragma unroll
        for (int y = 0; y < 16; ++y) w += sm.sums[y][threadIdx.x];
        const long long at = (long long)unit * a.cap + j0 + threadIdx.x;
        a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + w;
    }
}

// Joins the parts of up to 16 rows: o = sum exp2(m_s - M) o_s / sum exp2(m_s - M) l_s.  The parts' factors first, a warp per row; then
// every thread sums four columns of a row over the parts, in order, several of them in flight (one after the other 16 parts
// took 12 us, of which the memory's latency was all).
constexpr int kJoinParts = 64;               // factors in shared memory at a time
struct JoinSmem {
    float factor[16][kJoinParts];
    float top[16], sum[16], lse2[16];
};
template <typename T>
__device__ __forceinline__ void join_rows(const AttnArgs &a, JoinSmem &sm, const AttnSeq &sq, int unit, int b, int h, int row0, int n, bool write)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int r = warp; r < n; r += kThreads / 32) {
        const long long at = ((long long)unit * a.rows_max + row0 + r) * a.splits;
        float top = -INFINITY, l = 0.f;
        for (int s = lane; s < a.splits; s += 32) top = fmaxf(top, a.part_ml[at + s].x);
#pragma unroll
        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        const float ref = top == -INFINITY ? 0.f : top;
        // every lane its parts, then over the lanes: one order, whatever the launch
        for (int s = lane; s < a.splits; s += 32) {
            const float2 ml = a.part_ml[at + s];
            l += ml.y * exp2f(ml.x - ref);
        }
#pragma unroll
        for (int x = 16; x; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
        if (lane == 0) {
            sm.top[r] = ref;
            sm.sum[r] = l;
            sm.lse2[r] = l > 0.f || l != l ? top + log2f(l) : -INFINITY;
        }
    }
    __syncthreads();
    if (!write) return;
    const int cols = a.d / 4;
    for (int x0 = 0; x0 < n * cols; x0 += kThreads) {
        const int x = x0 + threadIdx.x, r = x / cols, c = (x - r * cols) * 4;
        const long long at = ((long long)unit * a.rows_max + row0 + r) * a.splits;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = 0; s0 < a.splits; s0 += kJoinParts) {
            const int parts = min(kJoinParts, a.splits - s0);
            __syncthreads();
            for (int y = threadIdx.x; y < n * parts; y += kThreads) {
                const int fr = y / parts, fs = y - fr * parts;
                const float2 ml = a.part_ml[((long long)unit * a.rows_max + row0 + fr) * a.splits + s0 + fs];
                sm.factor[fr][fs] = ml.y == 0.f ? -1.f : exp2f(ml.x - sm.top[fr]);      // -1: a part without weight, which has no output
            }
            __syncthreads();
            if (x >= n * cols) continue;
            const float *from = a.part_o + (at + s0) * a.d + c;
#pragma unroll 8
            for (int s = 0; s < parts; ++s) {
                const float f = sm.factor[r][s];
                float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
                // (a factor of 0 does not leave a part out: an infinity or NaN in its output counts)
                if (!(f < 0.f)) p = *reinterpret_cast<const float4 *>(from + (long long)s * a.d);
                o.x = fmaf(f, p.x, o.x);
                o.y = fmaf(f, p.y, o.y);
                o.z = fmaf(f, p.z, o.z);
                o.w = fmaf(f, p.w, o.w);
            }
        }
        if (x >= n * cols) continue;
        const int row = row0 + r, i = row / a.G, hq = h * a.G + row - i * a.G;
        if (c == 0) attn_store_lse(a, b, hq, i, sq.m, sm.lse2[r]);
        const float l = sm.sum[r], inv = l == 0.f ? 0.f : 1.f / l;
        T *dst = static_cast<T *>(a.out) + (sq.q_off + i) * a.ot + b * a.ob + (long long)hq * a.oh + c;
        T y[4];
        from_float(y[0], o.x * inv);
        from_float(y[1], o.y * inv);
        from_float(y[2], o.z * inv);
        from_float(y[3], o.w * inv);
        if (sizeof(T) == 4) *reinterpret_cast<float4 *>(dst) = *reinterpret_cast<float4 *>(y);
        else *reinterpret_cast<uint2 *>(dst) = *reinterpret_cast<uint2 *>(y);
    }
}
// block (unit, y): 16 rows from 16 y on
template <typename T>
__global__ void __launch_bounds__(kThreads) attn_join_kernel(const __grid_constant__ AttnArgs a)
{
    __shared__ JoinSmem sm;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x % (a.batch * a.hkv), b = unit / a.hkv, h = unit - b * a.hkv, row0 = (int)(blockIdx.x / (a.batch * a.hkv)) * 16;
    const AttnSeq sq = attn_seq(a, b, h);
    const int n = min(16, sq.m * a.G - row0);
    if (n > 0) join_rows<T>(a, sm, sq, unit, b, h, row0, n, true);
}
// The same for up to 16 rows whose logits are in the workspace: block (y, unit) also adds up the weights of kJoinKeys keys.  Every
// block of a unit needs the rows' normalisers and joins the few parts for itself; block 0 writes the rows.
constexpr int kJoinKeys = 4 * kThreads;
template <typename T>
__global__ void __launch_bounds__(kThreads) attn_join_weights_kernel(const __grid_constant__ AttnArgs a)
{
    __shared__ JoinSmem sm;
    pdl_trigger();
    pdl_wait();
    const int units = a.batch * a.hkv, unit = (int)blockIdx.x % units, part = (int)blockIdx.x / units - 1, b = unit / a.hkv, h = unit - b * a.hkv;
    const AttnSeq sq = attn_seq(a, b, h);
    const int rows = sq.m * a.G, j = part * kJoinKeys + threadIdx.x * 4;
    if (part < 0) {                                               // the first block writes the rows, the others weights
        join_rows<T>(a, sm, sq, unit, b, h, 0, rows, true);
        return;
    }
    if (part * kJoinKeys >= sq.n) return;
    join_rows<T>(a, sm, sq, unit, b, h, 0, rows, false);
    if (j >= sq.n) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    bool nan = false;
    const float *x = a.logits + (long long)unit * a.rows_max * a.logit_stride + j;
#pragma unroll 4
    for (int row = 0; row < rows; ++row) {
        const float ref = sm.lse2[row];
        nan |= ref != ref;
        if (!(fabsf(ref) < INFINITY)) continue;                          // the row has no weight, or is NaN
        const float4 s = *reinterpret_cast<const float4 *>(x + row * a.logit_stride);
        w[0] += exp2f(s.x - ref);
        w[1] += exp2f(s.y - ref);
        w[2] += exp2f(s.z - ref);
        w[3] += exp2f(s.w - ref);
    }
    if (nan)                                                             // a NaN for the keys that such a row sees: the others' logits are -infinity
        for (int row = 0; row < rows; ++row) {
            const float ref = sm.lse2[row];
            if (ref == ref) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (x[row * a.logit_stride + e] != -INFINITY) w[e] = ref;
        }
    const long long at = (long long)unit * a.cap + j;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (j + e < sq.n) a.weights_out[at + e] = (a.weights_in ? a.weights_in[at + e] : 0.f) + w[e];
}

// -infinity where an observation row would lie in front of its sequence
__global__ void lse_obs_fill_kernel(const __grid_constant__ AttnArgs a)
{
    pdl_trigger();
    pdl_wait();
    const long long x = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (x >= (long long)a.batch * a.hq * a.alpha) return;
    const int i = (int)(x % a.alpha), b = (int)(x / ((long long)a.alpha * a.hq));
    if (i < a.alpha - attn_seq(a, b, 0).m) a.lse_obs[x] = -INFINITY;
}

template <typename K>
int launch(K kernel, dim3 grid, size_t smem, const AttnArgs &a, cudaStream_t stream, const char *what, int cluster = 1)
{
    cudaError_t err = smem > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) : cudaSuccess;
    if (err == cudaSuccess) err = launch_pdl(kernel, grid, kThreads, smem, stream, cluster, a);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, what);
}
template <int ROWS>
int launch_rows(const AttnArgs &a, cudaStream_t stream)
{
    const long long tiles = ((long long)a.rows_max + ROWS - 1) / ROWS, blocks = tiles * a.batch * a.hkv * a.splits;
    if (blocks > 0x7fffffffLL) {
        set_error_detail("attention: %lld blocks", blocks);
        return WKV_ERR_LIMIT;
    }
    const dim3 grid((unsigned)blocks);
    const int cluster = a.clustered ? a.splits : 1;
    if constexpr (ROWS == 128) {
        return launch(attn_simt_kernel<128, ROWS>, grid, sizeof(SimtSmem<128, ROWS>), a, stream, "attention kernel", cluster);
    } else {
        if (a.d <= 64) return launch(attn_simt_kernel<64, ROWS>, grid, sizeof(SimtSmem<64, ROWS>), a, stream, "attention kernel", cluster);
        if (a.d <= 128) return launch(attn_simt_kernel<128, ROWS>, grid, sizeof(SimtSmem<128, ROWS>), a, stream, "attention kernel", cluster);
        return launch(attn_simt_kernel<256, ROWS>, grid, sizeof(SimtSmem<256, ROWS>), a, stream, "attention kernel", cluster);
    }
}
int launch_weights(const AttnArgs &a, cudaStream_t stream)
{
    const long long blocks = ((long long)a.cap + kKeys - 1) / kKeys * a.batch * a.hkv;
    if (blocks > 0x7fffffffLL) {
        set_error_detail("attention weights: %lld blocks", blocks);
        return WKV_ERR_LIMIT;
    }
    const dim3 grid((unsigned)blocks);
    if (a.d <= 64) return launch(attn_weights_kernel<64>, grid, sizeof(WeightsSmem<64>), a, stream, "attention weights kernel");
    if (a.d <= 128) return launch(attn_weights_kernel<128>, grid, sizeof(WeightsSmem<128>), a, stream, "attention weights kernel");
    return launch(attn_weights_kernel<256>, grid, sizeof(WeightsSmem<256>), a, stream, "attention weights kernel");
}

}  // namespace

int launch_attn_simt(const AttnArgs &args, cudaStream_t stream)
{
    AttnArgs a = args;
    const long long units = (long long)a.batch * a.hkv;
    const auto blocks = [&](int rows) { return ((long long)a.rows_max + rows - 1) / rows * units * a.splits; };
    if (!a.table) {
        // A prompt's keys are split over a cluster: until there are 200 blocks of 64 rows, and two for every SM as long as each keeps 1.5
        // key tiles or more, of which the rows see half on average (4 heads on 2, d = 64, 1,024 tokens: 64 blocks x 2 51 us, x 4 37,
        // x 8 44; 2,000 tokens at d = 128: x 2 271 us, x 4 178).
        while (a.splits < kClusterSplits && (blocks(64) < 200 || (blocks(64) < 2 * 148 && a.cap >= 6 * kKeys * a.splits)) && a.splits * kKeys < a.cap)
            a.splits *= 2;
        a.clustered = a.splits > 1;
    }
    if (a.rows_max <= 16 || blocks(32) < 120) return launch_rows<16>(a, stream);
    // (128 rows: a fragment of keys or values serves twice as many products, and shared memory bounds them)
    if (a.d > 64 && a.d <= 128 && blocks(128) >= 120) return launch_rows<128>(a, stream);
    return blocks(64) < 120 ? launch_rows<32>(a, stream) : launch_rows<64>(a, stream);
}
int launch_attn_weights(const AttnArgs &a, cudaStream_t stream) { return launch_weights(a, stream); }
int launch_attn_join(const AttnArgs &a, int dtype, cudaStream_t stream)
{
    const int units = a.batch * a.hkv;
    if (a.logits) {
        const long long blocks = (1ll + (a.cap + kJoinKeys - 1) / kJoinKeys) * units;
        if (blocks > 0x7fffffffLL) {
            set_error_detail("attention weights: %lld blocks", blocks);
            return WKV_ERR_LIMIT;
        }
        const dim3 grid((unsigned)blocks);
        return dtype == WKV_F32 ? launch(attn_join_weights_kernel<float>, grid, 0, a, stream, "attention joining kernel")
                                : launch(attn_join_weights_kernel<__nv_bfloat16>, grid, 0, a, stream, "attention joining kernel");
    }
    const long long blocks = ((long long)a.rows_max + 15) / 16 * units;
    if (blocks > 0x7fffffffLL) {
        set_error_detail("attention: %lld blocks", blocks);
        return WKV_ERR_LIMIT;
    }
    const dim3 grid((unsigned)blocks);
    return dtype == WKV_F32 ? launch(attn_join_kernel<float>, grid, 0, a, stream, "attention joining kernel")
                            : launch(attn_join_kernel<__nv_bfloat16>, grid, 0, a, stream, "attention joining kernel");
}
int launch_attn_lse_obs_fill(const AttnArgs &a, cudaStream_t stream)
{
    const long long n = (long long)a.batch * a.hq * a.alpha;
    return launch(lse_obs_fill_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)), 0, a, stream, "log-sum-exp fill kernel");
}

}  // namespace wkv
