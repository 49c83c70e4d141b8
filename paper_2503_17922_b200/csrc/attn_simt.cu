// Attention on the CUDA cores for fp32, its weights kernel, and the joining kernels of all types.  One block holds ROWS rows of one
// unit in shared memory and walks over the unit's keys in tiles of 64 with a running maximum and sum per row; everything is
// fp32, products in plain multiply-adds, which bound it (2 * 64 * d per row and tile).  A tile's keys and values come by asynchronous copies
// while the one before is worked on.
//
// ROWS is the largest of 64, 32 and 16 that gives every SM a block (4 heads of 1,024 tokens, d = 64: 122 us with 64 rows in 64 blocks).
//
// With S key splits a block walks over one of S parts of the keys and leaves (maximum, sum, unnormalised output) per row for
// the joining kernel.  A row's sums are taken in one order whatever else the launch holds, so results do not depend
// on the other sequences of a batch.
#include "attn_cluster.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;

__device__ __forceinline__ void from_float(float &y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16 &y, float x) { y = __float2bfloat16_rn(x); }

// four elements of a row of d into shared memory, zeros from d on; `p` null: zeros
template <int DP>
__device__ __forceinline__ void load_row_part(float *dst, const float *p, int d, int part)
{
    const int c = part * 4;
    *reinterpret_cast<float4 *>(dst + c) = p && c < d ? *reinterpret_cast<const float4 *>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
}

// Stages of key tiles: two where they fit.
__host__ __device__ constexpr int simt_stages(int dp) { return dp <= 128 ? 2 : 1; }
template <int DP, int ROWS>
struct SimtSmem {
    float q[ROWS][DP + 4];
    float k[simt_stages(DP)][kKeys][DP + 4];
    float v[simt_stages(DP)][kKeys][DP];
    float p[ROWS][kKeys + 4];
    int present[simt_stages(DP)][kKeys];       // the key's page is one
    float m[16], l[16], lse2[16];
};
template <int DP>
struct WeightsSmem {
    float q[64][DP + 4];
    float k[kKeys][DP + 4];
    float sums[16][kKeys + 1];
    int present[kKeys];
};

// the keys and values of one tile, on their way; rows from n on and rows without a page are zeros
template <int DP, int ROWS>
__device__ __forceinline__ void fetch_keys(const AttnArgs &a, SimtSmem<DP, ROWS> &sm, int st, int b, int h, long long off, int n, int j0)
{
    // a row's vectors lie in neighbouring threads; the rows' places first, so that their looking up (a trip to memory where paged) overlaps
    constexpr int kParts = DP / 4, kEach = kKeys * kParts / kThreads;
    const int c = (int)(threadIdx.x % kParts) * 4, r0 = threadIdx.x / kParts;
    long long at[kEach];
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        const int j = j0 + r0 + x * (kThreads / kParts);
        at[x] = j < n ? attn_row(a, b, h, off, j) : -1;
    }
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        const int r = r0 + x * (kThreads / kParts);
        const bool have = at[x] >= 0 && c < a.d;
        const int size = have ? 16 : 0;
        const float *kp = static_cast<const float *>(a.k) + (have ? at[x] + c : 0), *vp = static_cast<const float *>(a.v) + (have ? at[x] + c : 0);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(&sm.k[st][r][c]))), "l"(kp), "r"(size) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(&sm.v[st][r][c]))), "l"(vp), "r"(size) : "memory");
        if (c == 0) sm.present[st][r] = at[x] >= 0;
    }
}
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
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[r][j] = 0.f;
#pragma unroll 4
    for (int e = 0; e < DP; e += 4) {
        float4 qv[RT], kv[4];
#pragma unroll
        for (int r = 0; r < RT; ++r) qv[r] = *reinterpret_cast<const float4 *>(&q[ty * RT + r][e]);
#pragma unroll
        for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4 *>(&k[tx + 16 * j][e]);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[r][j] = fmaf(qv[r].x, kv[j].x, s[r][j]);
                s[r][j] = fmaf(qv[r].y, kv[j].y, s[r][j]);
                s[r][j] = fmaf(qv[r].z, kv[j].z, s[r][j]);
                s[r][j] = fmaf(qv[r].w, kv[j].w, s[r][j]);
            }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[r][j] *= c;
}

template <int DP, int ROWS>
__global__ void __launch_bounds__(kThreads) attn_simt_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char raw[];
    SimtSmem<DP, ROWS> &sm = *reinterpret_cast<SimtSmem<DP, ROWS> *>(raw);
    constexpr int RT = ROWS / 16, CT = DP / 64, NS = simt_stages(DP);
    // The joining kernel may be placed now.  Another of this kind is not to be before this one ends: its blocks would crowd onto the
    // SMs that have room at that time.
    const bool clustered = ROWS == 16 && a.clustered, parts = !clustered && (a.splits > 1 || a.logits);
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
    float4 o[RT][CT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        limit[r] = base + (row0 + ty * RT + r) / a.G;
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int x = 0; x < CT; ++x) o[r][x] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (t0 < t1) fetch_keys(a, sm, 0, b, h, sq.q_off, sq.n, t0 * kKeys);
    asm volatile("cp.async.commit_group;" ::: "memory");
    load_queries<DP, ROWS>(a, sm.q, b, h, sq.q_off, row0, rows);
    const int plain = base + row0 / a.G;                                 // every row attends to the keys before this one
    for (int t = t0; t < t1; ++t) {
        const int j0 = t * kKeys, st = NS == 2 ? (t - t0) & 1 : 0;
        if (NS == 2 && t + 1 < t1) fetch_keys(a, sm, st ^ 1, b, h, sq.q_off, sq.n, j0 + kKeys);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(NS - 1) : "memory");
        __syncthreads();
        float s[RT][4];
        logits<DP, ROWS>(sm.q, sm.k[st], ty, tx, a.scale_log2, s);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = m[r];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j0 + tx + 16 * j >= limit[r] || !sm.present[st][tx + 16 * j]) s[r][j] = -INFINITY;
                top = fmaxf(top, s[r][j]);
            }
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
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                o[r][x].x *= keep;
                o[r][x].y *= keep;
                o[r][x].z *= keep;
                o[r][x].w *= keep;
            }
        }
        __syncwarp();                                                    // a row's 16 threads are in one warp
        const bool guarded = j0 + kKeys > plain;
#pragma unroll 2
        for (int j = 0; j < kKeys; j += 4) {
            float4 pp[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) pp[r] = *reinterpret_cast<const float4 *>(&sm.p[ty * RT + r][j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float4 vv[CT];
#pragma unroll
                for (int x = 0; x < CT; ++x) vv[x] = *reinterpret_cast<const float4 *>(&sm.v[st][j + e][tx * 4 + 64 * x]);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const float p = e == 0 ? pp[r].x : (e == 1 ? pp[r].y : (e == 2 ? pp[r].z : pp[r].w));
                    // what stands behind a row's position may be infinite or NaN: 0 times it is not 0
                    if (guarded && p == 0.f) continue;
#pragma unroll
                    for (int x = 0; x < CT; ++x) {
                        o[r][x].x = fmaf(p, vv[x].x, o[r][x].x);
                        o[r][x].y = fmaf(p, vv[x].y, o[r][x].y);
                        o[r][x].z = fmaf(p, vv[x].z, o[r][x].z);
                        o[r][x].w = fmaf(p, vv[x].w, o[r][x].w);
                    }
                }
            }
        }
        __syncthreads();
        if (NS == 1 && t + 1 < t1) fetch_keys(a, sm, 0, b, h, sq.q_off, sq.n, j0 + kKeys);
    }
    if (!parts) pdl_trigger();
    if (clustered) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        float *const all = &sm.k[0][0][0];                               // [16][DP + 4]
        if (tx == 0) {
            sm.m[ty] = m[0];
            sm.l[ty] = l[0];
        }
#pragma unroll
        for (int x = 0; x < CT; ++x) *reinterpret_cast<float4 *>(all + ty * (DP + 4) + tx * 4 + 64 * x) = o[0][x];
        cluster_join<float, kThreads>(a, sq, unit, b, h, row0, min(16, rows - row0), split, sm.m, sm.l, all, DP + 4, sm.lse2, t0 * kKeys,
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
                if (c < a.d) *reinterpret_cast<float4 *>(a.part_o + at * a.d + c) = o[r][x];
            }
            continue;
        }
        if (tx == 0) attn_store_lse(a, b, hq, i, sq.m, l[r] > 0.f || l[r] != l[r] ? m[r] + log2f(l[r]) : -INFINITY);
        const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
        float *dst = static_cast<float *>(a.out) + (sq.q_off + i) * a.ot + b * a.ob + (long long)hq * a.oh;
#pragma unroll
        for (int x = 0; x < CT; ++x) {
            const int c = tx * 4 + 64 * x;
            if (c < a.d) *reinterpret_cast<float4 *>(dst + c) = make_float4(o[r][x].x * inv, o[r][x].y * inv, o[r][x].z * inv, o[r][x].w * inv);
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
                sm.factor[fr][fs] = ml.y == 0.f ? 0.f : exp2f(ml.x - sm.top[fr]);       // (a part without a key of the row has no output)
            }
            __syncthreads();
            if (x >= n * cols) continue;
            const float *from = a.part_o + (at + s0) * a.d + c;
#pragma unroll 8
            for (int s = 0; s < parts; ++s) {
                const float f = sm.factor[r][s];
                float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
                if (f != 0.f) p = *reinterpret_cast<const float4 *>(from + (long long)s * a.d);
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
// The same for up to 16 rows whose logits are in the workspace: block (unit, y) also adds up the weights of kJoinKeys keys.  Every
// block of a unit needs the rows' normalisers and joins the few parts for itself; block 0 writes the rows.
constexpr int kJoinKeys = 4 * kThreads;
template <typename T>
__global__ void __launch_bounds__(kThreads) attn_join_weights_kernel(const __grid_constant__ AttnArgs a)
{
    __shared__ JoinSmem sm;
    pdl_trigger();
    pdl_wait();
    const int unit = blockIdx.x, b = unit / a.hkv, h = unit - b * a.hkv;
    const AttnSeq sq = attn_seq(a, b, h);
    const int rows = sq.m * a.G, j = ((int)blockIdx.y - 1) * kJoinKeys + threadIdx.x * 4;
    if (blockIdx.y == 0) {                                               // the first block writes the rows, the others weights
        join_rows<T>(a, sm, sq, unit, b, h, 0, rows, true);
        return;
    }
    if (((int)blockIdx.y - 1) * kJoinKeys >= sq.n) return;
    join_rows<T>(a, sm, sq, unit, b, h, 0, rows, false);
    if (j >= sq.n) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    const float *x = a.logits + (long long)unit * a.rows_max * a.logit_stride + j;
#pragma unroll 4
    for (int row = 0; row < rows; ++row) {
        const float ref = sm.lse2[row];
        if (ref == -INFINITY) continue;                                  // the row attends to nothing
        const float4 s = *reinterpret_cast<const float4 *>(x + row * a.logit_stride);
        w[0] += exp2f(s.x - ref);
        w[1] += exp2f(s.y - ref);
        w[2] += exp2f(s.z - ref);
        w[3] += exp2f(s.w - ref);
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
    const int cluster = ROWS == 16 && a.clustered ? a.splits : 1;
    if (a.d <= 64) return launch(attn_simt_kernel<64, ROWS>, grid, sizeof(SimtSmem<64, ROWS>), a, stream, "attention kernel", cluster);
    if (a.d <= 128) return launch(attn_simt_kernel<128, ROWS>, grid, sizeof(SimtSmem<128, ROWS>), a, stream, "attention kernel", cluster);
    return launch(attn_simt_kernel<256, ROWS>, grid, sizeof(SimtSmem<256, ROWS>), a, stream, "attention kernel", cluster);
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

int launch_attn_simt(const AttnArgs &a, cudaStream_t stream)
{
    const long long units = (long long)a.batch * a.hkv * a.splits, enough = 120;
    if (a.rows_max <= 16 || ((long long)a.rows_max + 31) / 32 * units < enough) return launch_rows<16>(a, stream);
    return ((long long)a.rows_max + 63) / 64 * units < enough ? launch_rows<32>(a, stream) : launch_rows<64>(a, stream);
}
int launch_attn_weights(const AttnArgs &a, cudaStream_t stream) { return launch_weights(a, stream); }
int launch_attn_join(const AttnArgs &a, int dtype, cudaStream_t stream)
{
    const int units = a.batch * a.hkv;
    if (a.logits) {
        const int blocks = 1 + (a.cap + kJoinKeys - 1) / kJoinKeys;
        if (blocks > 65535) {
            set_error_detail("attention weights: %d rows of a unit", a.cap);
            return WKV_ERR_LIMIT;
        }
        const dim3 grid(units, blocks);
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
