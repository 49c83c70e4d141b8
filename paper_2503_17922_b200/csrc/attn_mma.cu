// Attention on warp-level matrix instructions (m16n8k16, bf16): single tokens and short chunks over the paged cache, where the
// bytes of K and V bound the time, and the shapes that the tcgen05 kernel does not take (head dimensions beyond 128,
// pages of sizes that eight does not divide).
//
// A block of four warps walks over the keys of one unit (or a split of them) in tiles of 64, which come through a ring of
// asynchronous 16-byte copies: one tile is in flight while another is worked on (three for d up to 64).  What keeps memory busy
// is three blocks per SM: 32 sequences of 4-8 K rows, one token of 32 heads on 8, with weights, 160 us with two tiles in the ring
// and about 190 with a deeper one and two blocks; the kernel itself reads 5.6 TB/s.  Rows (position x head of the group) sit on the M
// side of the instruction:
//   FEW    up to 16 rows, all in every warp; a warp takes 16 of the tile's keys and keeps a maximum and a sum of its own, joined
//          once at the end
//   else   64 rows, 16 per warp, every warp takes all keys
// Rows that do not exist cost nothing that counts: with 4 rows of 16 the instructions take a third of the time of the loads.
//
// P is rounded to bf16 for the product (as its operand has to be); logits, maxima, sums and outputs are fp32, the sum of the unrounded P.
//
// Where weights are wanted (FEW), the logits go to the workspace (4 bytes per row and key beside the 512 of K and V) and the joining
// kernel adds up exp2(logit - lse), instead of K being read once more.
#include "attn_cluster.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 128;
constexpr int kKeys = 64;
__host__ __device__ constexpr int stages_for(int dp) { return dp == 64 ? 4 : 2; }

template <int DP>
struct MmaSmem {
    __align__(128) __nv_bfloat16 k[stages_for(DP)][kKeys][DP];
    __align__(128) __nv_bfloat16 v[stages_for(DP)][kKeys][DP];
    long long at[2][kKeys];                    // element offsets of a tile's rows, -1: none
    int missing[stages_for(DP) + 1][2];        // of a tile's two halves: some row has no page
    float m[4][16], l[4][16], lse2[16];
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// 16-byte chunks of a row are XORed with the row modulo 8, so that eight rows of one chunk lie in different banks
template <int DP>
__device__ __forceinline__ uint32_t chunk_addr(uint32_t base, int row, int chunk)
{
    return base + (uint32_t)(row * DP * 2 + ((chunk ^ (row & 7)) << 4));
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int DP, bool FEW>
__global__ void __launch_bounds__(kThreads) attn_mma_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(128) unsigned char raw[];
    MmaSmem<DP> &sm = *reinterpret_cast<MmaSmem<DP> *>(raw);
    constexpr int NS = stages_for(DP), kRows = FEW ? 16 : 64, kSteps = DP / 16, kGroups = FEW ? 1 : 4;   // 16-key groups per warp
    // The joining kernel may be placed now.  Another of this kind is not to be before this one ends: its blocks would crowd onto the
    // SMs that have room at that time.
    const bool clustered = FEW && a.clustered, parts = !clustered && (a.splits > 1 || a.logits);
    if (parts) pdl_trigger();
    pdl_wait();
    const int units = a.batch * a.hkv;
    // the last rows of a prompt have the most keys: they are taken first
    const int splits = a.splits, place_of = (int)blockIdx.x / splits, split = (int)blockIdx.x - place_of * splits;
    const int tiles = (int)gridDim.x / splits / units, unit = place_of % units, tile = tiles - 1 - place_of / units;
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const AttnSeq sq = attn_seq(a, b, h);
    const int rows = sq.m * a.G, row0 = tile * kRows;
    if (row0 >= rows) {
        if (clustered) carry_weights(a, unit, (int)((long long)sq.n * split / splits), (int)((long long)sq.n * (split + 1) / splits), kThreads);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = lane >> 2, ql = lane & 3;
    const int base = sq.n - sq.m + 1;                                    // keys that query 0 attends to (may be negative)
    const int most = min(base + (min(row0 + kRows, rows) - 1) / a.G, sq.n);
    const int all_tiles = (max(most, 0) + kKeys - 1) / kKeys;
    const int t0 = (int)((long long)all_tiles * split / splits), t1 = (int)((long long)all_tiles * (split + 1) / splits);
    const int plain = base + row0 / a.G;                                 // every row attends to the keys before this one

    // rows of this thread: `quad` and quad + 8 of the warp's sixteen
    const int my_row[2] = {row0 + (FEW ? 0 : warp * 16) + quad, row0 + (FEW ? 0 : warp * 16) + quad + 8};
    int limit[2];
    uint32_t q[kSteps][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int row = my_row[x], i = row / a.G, g = row - i * a.G;
        limit[x] = row < rows ? base + i : 0;
        const __nv_bfloat16 *p = static_cast<const __nv_bfloat16 *>(a.q) + (sq.q_off + i) * a.qt + b * a.qb + (long long)(h * a.G + g) * a.qh;
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int c = s * 16 + y * 8 + ql * 2;
                q[s][2 * y + x] = row < rows && c < a.d ? *reinterpret_cast<const uint32_t *>(p + c) : 0u;
            }
    }
    float o[DP / 8][4];
#pragma unroll
    for (int x = 0; x < DP / 8; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) o[x][y] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    // ---- the ring of key tiles -----------------------------------------------------------------
    // The rows' places are looked up a tile ahead of their loads (a trip to memory for paged rows).
    auto place = [&](int t) -> long long {
        const int j = t * kKeys + tid;
        return t < t1 && tid < kKeys && j < sq.n ? attn_row(a, b, h, sq.q_off, j) : -1;
    };
    auto keep_place = [&](int t, long long at) {
        if (tid >= kKeys) return;
        sm.at[t & 1][tid] = at;
        const unsigned there = __ballot_sync(0xffffffffu, at >= 0);
        if (lane == 0) sm.missing[t % (NS + 1)][warp] = there != 0xffffffffu;
    };
    constexpr int kChunks = DP / 8, kRowsAtOnce = kThreads / kChunks;
    const int chunk = tid % kChunks;
    const bool real = chunk * 8 < a.d;
    auto load = [&](int t) {
        if (t < t1) {
            const int st = t % NS;
            const uint32_t ks = smem_addr(&sm.k[st][0][0]), vs = smem_addr(&sm.v[st][0][0]);
#pragma unroll
            for (int r = tid / kChunks; r < kKeys; r += kRowsAtOnce) {
                const long long at = sm.at[t & 1][r];
                const bool have = at >= 0 && real;
                const __nv_bfloat16 *kp = static_cast<const __nv_bfloat16 *>(a.k) + (have ? at + chunk * 8 : 0);
                const __nv_bfloat16 *vp = static_cast<const __nv_bfloat16 *>(a.v) + (have ? at + chunk * 8 : 0);
                const int size = have ? 16 : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(chunk_addr<DP>(ks, r, chunk)), "l"(kp), "r"(size) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(chunk_addr<DP>(vs, r, chunk)), "l"(vp), "r"(size) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    keep_place(t0, place(t0));
    for (int x = 0; x < NS - 1; ++x) {
        const long long next = place(t0 + x + 1);
        __syncthreads();
        load(t0 + x);
        keep_place(t0 + x + 1, next);
    }
    for (int t = t0; t < t1; ++t) {
        const int st = t % NS;
        const long long next = place(t + NS);
        asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
        __syncthreads();                      // tile t has landed for all; the stage of tile t - 1 is free; places of t + NS - 1 are there
        load(t + NS - 1);
        const int j0 = t * kKeys;
        const bool masked = j0 + kKeys > plain || sm.missing[t % (NS + 1)][0] || sm.missing[t % (NS + 1)][1];
        const uint32_t ks = smem_addr(&sm.k[st][0][0]), vs = smem_addr(&sm.v[st][0][0]);
#pragma unroll
        for (int grp = 0; grp < kGroups; ++grp) {
            const int key0 = (FEW ? warp : grp) * 16;
            // (two sums over every other step of the head dimension: half the chain of dependent instructions)
            float s[2][4] = {}, s1[2][4] = {};
#pragma unroll
            for (int c = 0; c < kSteps; c += 2) {
                uint32_t kf[4], kg[4];
                ldmatrix4(chunk_addr<DP>(ks, key0 + (lane & 7) + ((lane >> 4) << 3), 2 * c + ((lane >> 3) & 1)), kf);
                ldmatrix4(chunk_addr<DP>(ks, key0 + (lane & 7) + ((lane >> 4) << 3), 2 * c + 2 + ((lane >> 3) & 1)), kg);
                mma(s[0], q[c], kf[0], kf[1]);
                mma(s[1], q[c], kf[2], kf[3]);
                mma(s1[0], q[c + 1], kg[0], kg[1]);
                mma(s1[1], q[c + 1], kg[2], kg[3]);
            }
            bool unseen = false;              // some key that exists is not seen by some row
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[y][e] = (s[y][e] + s1[y][e]) * a.scale_log2;
            if (masked) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int jj = key0 + y * 8 + ql * 2 + e, j = j0 + jj;
                        bool there = j < sq.n;
                        // (the places of the tile at hand have been written over: its pages are looked up again, where some are missing)
                        if (there && a.table && (sm.missing[t % (NS + 1)][0] | sm.missing[t % (NS + 1)][1])) there = attn_row(a, b, h, sq.q_off, j) >= 0;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const bool sees = there && j < limit[x];
                            unseen |= there && !sees;
                            if (!sees) s[y][2 * x + e] = -INFINITY;
                        }
                    }
            }
            if (FEW && a.logits) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (my_row[x] < rows) {
                        float *to = a.logits + ((long long)unit * a.rows_max + my_row[x]) * a.logit_stride + j0 + key0 + ql * 2;
#pragma unroll
                        for (int y = 0; y < 2; ++y)
                            if (j0 + key0 + y * 8 + ql * 2 < sq.n) *reinterpret_cast<float2 *>(to + y * 8) = make_float2(s[y][2 * x], s[y][2 * x + 1]);
                    }
            }
            uint32_t p[4];
            float pf[2][4];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float top = fmaxf(fmaxf(s[0][2 * x], s[0][2 * x + 1]), fmaxf(s[1][2 * x], s[1][2 * x + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(m[x], fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)));
                const float ref = top == -INFINITY ? 0.f : top, keep = ex2(m[x] - ref);
                m[x] = top;
                float sum = 0.f;
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        pf[y][2 * x + e] = ex2(s[y][2 * x + e] - ref);
                        sum += pf[y][2 * x + e];
                    }
                l[x] = l[x] * keep + sum;                 // this thread's keys; joined over the quad at the end
                if (keep != 1.f) {
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d) {
                        o[d][2 * x] *= keep;
                        o[d][2 * x + 1] *= keep;
                    }
                }
            }
            p[0] = pack(pf[0][0], pf[0][1]);
            p[1] = pack(pf[0][2], pf[0][3]);
            p[2] = pack(pf[1][0], pf[1][1]);
            p[3] = pack(pf[1][2], pf[1][3]);
            bool plain_product = true;
            if (masked && __any_sync(0xffffffffu, unseen)) {
                // 0 times an infinity or NaN is not 0: are there any among the values?
                uint32_t bad = 0;
                for (int x = lane; x < 16 * kChunks; x += 32) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned char *>(&sm.v[st][key0][0]) + x * 16);
                    const uint32_t all = 0x7f807f80u;
                    bad |= __vcmpeq2(w.x & all, all) | __vcmpeq2(w.y & all, all) | __vcmpeq2(w.z & all, all) | __vcmpeq2(w.w & all, all);
                }
                plain_product = !__any_sync(0xffffffffu, bad != 0);
            }
            // (then such elements count as 0 in the product, and are added to the rows that do see them)
            const uint32_t e = 0x7f807f80u;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                uint32_t vf[4];
                ldmatrix4_trans(chunk_addr<DP>(vs, key0 + (lane & 15), 2 * d + (lane >> 4)), vf);
                if (!plain_product) {
#pragma unroll
                    for (int y = 0; y < 4; ++y) vf[y] &= ~__vcmpeq2(vf[y] & e, e);
                }
                mma(o[2 * d], p, vf[0], vf[1]);
                mma(o[2 * d + 1], p, vf[2], vf[3]);
            }
            if (!plain_product) {
                for (int kk = 0; kk < 16; ++kk) {
                    const int row = key0 + kk;
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d) {
                        const __nv_bfloat162 w = *reinterpret_cast<const __nv_bfloat162 *>(
                            reinterpret_cast<const unsigned char *>(&sm.v[st][row][0]) + ((d ^ (row & 7)) << 4) + ql * 4);
                        const float w0 = __low2float(w), w1 = __high2float(w);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            if (j0 + row >= limit[x]) continue;
                            if (!(fabsf(w0) < INFINITY)) o[d][2 * x] += w0;
                            if (!(fabsf(w1) < INFINITY)) o[d][2 * x + 1] += w1;
                        }
                    }
                }
            }
        }
        keep_place(t + NS, next);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!parts) pdl_trigger();
    if (FEW) {
        // ---- the four warps' sums, in order -------------------------------------------------------
        __syncthreads();
        constexpr int kPad = DP + 4;
        float *const all = reinterpret_cast<float *>(&sm.k[0][0][0]);          // [4][16][kPad]
        static_assert(4 * 16 * kPad * 4 <= sizeof(sm.k) + sizeof(sm.v), "the ring holds the warps' outputs");
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int r = quad + 8 * x;
            if (ql == 0) {
                sm.m[warp][r] = m[x];
                sm.l[warp][r] = l[x];
            }
#pragma unroll
            for (int d = 0; d < DP / 8; ++d)
                *reinterpret_cast<float2 *>(all + (warp * 16 + r) * kPad + d * 8 + ql * 2) = make_float2(o[d][2 * x], o[d][2 * x + 1]);
        }
        __syncthreads();
        const int live = min(16, rows - row0);
        for (int x = tid; x < live * (DP / 4); x += kThreads) {
            const int r = x / (DP / 4), c = (x - r * (DP / 4)) * 4;
            const float top = fmaxf(fmaxf(sm.m[0][r], sm.m[1][r]), fmaxf(sm.m[2][r], sm.m[3][r])), ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = ex2(sm.m[w][r] - ref);
                const float4 part = *reinterpret_cast<const float4 *>(all + (w * 16 + r) * kPad + c);
                sum += f * sm.l[w][r];
                if (sm.l[w][r] == 0.f) continue;           // a warp without a key of the row
                y.x = fmaf(f, part.x, y.x);
                y.y = fmaf(f, part.y, y.y);
                y.z = fmaf(f, part.z, y.z);
                y.w = fmaf(f, part.w, y.w);
            }
            if (clustered) {
                *reinterpret_cast<float4 *>(all + r * kPad + c) = y;          // (in the place of the first warp's, which this thread has read)
                continue;
            }
            const int row = row0 + r, i = row / a.G, hq = h * a.G + row - i * a.G;
            if (parts) {
                const long long at = ((long long)unit * a.rows_max + row) * a.splits + split;
                if (c == 0) a.part_ml[at] = make_float2(top, sum);
                if (c < a.d && sum != 0.f) *reinterpret_cast<float4 *>(a.part_o + at * a.d + c) = y;
                continue;
            }
            if (c == 0) attn_store_lse(a, b, hq, i, sq.m, sum > 0.f || sum != sum ? top + log2f(sum) : -INFINITY);
            if (c >= a.d) continue;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + (sq.q_off + i) * a.ot + b * a.ob + (long long)hq * a.oh + c;
            *reinterpret_cast<uint2 *>(dst) = make_uint2(pack(y.x * inv, y.y * inv), pack(y.z * inv, y.w * inv));
        }
        if (clustered) {
            __syncthreads();
            float top = 0.f, sum = 0.f;
            if (tid < 16) {
                top = fmaxf(fmaxf(sm.m[0][tid], sm.m[1][tid]), fmaxf(sm.m[2][tid], sm.m[3][tid]));
                const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int w = 0; w < 4; ++w) sum += ex2(sm.m[w][tid] - ref) * sm.l[w][tid];
                sm.m[0][tid] = top;
                sm.l[0][tid] = sum;
            }
            cluster_join<__nv_bfloat16, kThreads, true>(a, sq, unit, b, h, row0, live, split, sm.m[0], sm.l[0], all, kPad, sm.lse2, t0 * kKeys,
                                                  min(t1 * kKeys, sq.n));
        }
    } else {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int row = my_row[x];
            if (row >= rows) continue;
            const int i = row / a.G, hq = h * a.G + row - i * a.G;
            if (parts) {
                const long long at = ((long long)unit * a.rows_max + row) * a.splits + split;
                if (ql == 0) a.part_ml[at] = make_float2(m[x], l[x]);
                if (l[x] == 0.f) continue;
#pragma unroll
                for (int d = 0; d < DP / 8; ++d)
                    if (d * 8 + ql * 2 < a.d) *reinterpret_cast<float2 *>(a.part_o + at * a.d + d * 8 + ql * 2) = make_float2(o[d][2 * x], o[d][2 * x + 1]);
                continue;
            }
            if (ql == 0) attn_store_lse(a, b, hq, i, sq.m, l[x] > 0.f || l[x] != l[x] ? m[x] + log2f(l[x]) : -INFINITY);
            const float inv = l[x] == 0.f ? 0.f : 1.f / l[x];
            __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + (sq.q_off + i) * a.ot + b * a.ob + (long long)hq * a.oh;
#pragma unroll
            for (int d = 0; d < DP / 8; ++d)
                if (d * 8 + ql * 2 < a.d) *reinterpret_cast<uint32_t *>(dst + d * 8 + ql * 2) = pack(o[d][2 * x] * inv, o[d][2 * x + 1] * inv);
        }
    }
}

// ---- weights that the rows of the cache receive from longer chunks --------------------------------
// A block takes WARPS * 16 * F keys of a unit and sums exp2(logit - lse) over all of the unit's queries that see them: the logits are
// computed once more, from the normalisers that the attention has written.  The keys sit on the M side of the instruction and
// stay in registers, 16 F for each warp; the queries come through a ring in tiles of 64, and every fragment of them serves F
// instructions.  Sums are fp32, over a thread's queries in order and then over the four threads of a key: one order, no atomics.
//
// Bound by the instructions: 2 * keys * rows * d.  Four sequences of 10-16 K rows and up to 512 new tokens of 32 heads, d = 128: 580 us
// beside 327 of the attention (on the CUDA cores 4,650); of up to 64 tokens 101 us (660).
constexpr int kWeightRows = 64, kWeightStages = 3;
template <int DP>
struct WeightsSmem {
    __align__(128) __nv_bfloat16 q[kWeightStages][kWeightRows][DP];
    __align__(16) float lse[kWeightStages][kWeightRows];
    __align__(16) int limit[kWeightStages][kWeightRows];           // keys that the row sees; 0: there is no such row
};
template <int DP, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 16 / WARPS) attn_mma_weights_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(128) unsigned char raw[];
    WeightsSmem<DP> &sm = *reinterpret_cast<WeightsSmem<DP> *>(raw);
    constexpr int F = DP == 256 ? 1 : 2, NS = kWeightStages, kSteps = DP / 16, kBlockKeys = WARPS * 16 * F, kBlock = WARPS * 32;
    pdl_wait();
    const int units = a.batch * a.hkv, unit = (int)blockIdx.x % units, j0 = (int)blockIdx.x / units * kBlockKeys;
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const AttnSeq sq = attn_seq(a, b, h);
    if (j0 >= sq.n) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = lane >> 2, ql = lane & 3;
    const int rows = sq.m * a.G, base = sq.n - sq.m + 1;
    const int key0 = j0 + warp * 16 * F + quad;                    // this thread's keys: key0 + 16 f + 8 x

    // queries in front of the block's first key do not attend to any of it
    const int first = base > j0 ? 0 : (int)min((long long)(j0 - base + 1) * a.G, (long long)rows), tiles = (rows - first + kWeightRows - 1) / kWeightRows;
    constexpr int kChunks = DP / 8, kRowsAtOnce = kBlock / kChunks;
    const int chunk = tid % kChunks;
    auto load = [&](int t) {
        if (t < tiles) {
            const int st = t % NS;
            const uint32_t qs = smem_addr(&sm.q[st][0][0]);
#pragma unroll
            for (int r = tid / kChunks; r < kWeightRows; r += kRowsAtOnce) {
                const int row = first + t * kWeightRows + r, i = row / a.G, g = row - i * a.G;
                const bool have = row < rows && chunk * 8 < a.d;
                const __nv_bfloat16 *p = static_cast<const __nv_bfloat16 *>(a.q);
                if (have) p += (sq.q_off + i) * a.qt + b * a.qb + (long long)(h * a.G + g) * a.qh + chunk * 8;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(chunk_addr<DP>(qs, r, chunk)), "l"(p), "r"(have ? 16 : 0) : "memory");
            }
            if (tid < kWeightRows) {
                const int row = first + t * kWeightRows + tid, i = row / a.G, g = row - i * a.G;
                const float *p = a.lse;
                if (row < rows) p += ((long long)b * a.hq + h * a.G + g) * a.max_q + i;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_addr(&sm.lse[st][tid])), "l"(p), "r"(row < rows ? 4 : 0) : "memory");
                sm.limit[st][tid] = row < rows ? base + i : 0;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int x = 0; x < NS - 1; ++x) load(x);

    uint32_t k[F][kSteps][4];
    bool there[F][2];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int j = key0 + 16 * f + 8 * x;
            const long long at = j < sq.n ? attn_row(a, b, h, sq.q_off, j) : -1;
            there[f][x] = at >= 0;
            const __nv_bfloat16 *p = static_cast<const __nv_bfloat16 *>(a.k) + (at >= 0 ? at : 0);
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int c = s * 16 + y * 8 + ql * 2;
                    k[f][s][2 * y + x] = at >= 0 && c < a.d ? __ldg(reinterpret_cast<const uint32_t *>(p + c)) : 0u;
                }
        }
    float sum[F][2] = {};
    for (int t = 0; t < tiles; ++t) {
        const int st = t % NS, row0 = first + t * kWeightRows;
        asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
        __syncthreads();                      // tile t has landed for all; the stage of tile t - 1 is free
        load(t + NS - 1);
        const bool masked = j0 + kBlockKeys > base + row0 / a.G || row0 + kWeightRows > rows;
        const uint32_t qs = smem_addr(&sm.q[st][0][0]);
#pragma unroll 1
        for (int g = 0; g < kWeightRows; g += 16) {
            float s[F][2][4] = {};
#pragma unroll
            for (int c = 0; c < kSteps; ++c) {
                uint32_t qf[4];
                ldmatrix4(chunk_addr<DP>(qs, g + (lane & 7) + ((lane >> 4) << 3), 2 * c + ((lane >> 3) & 1)), qf);
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    mma(s[f][0], k[f][c], qf[0], qf[1]);
                    mma(s[f][1], k[f][c], qf[2], qf[3]);
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int r = g + y * 8 + ql * 2;
                const float2 lse = *reinterpret_cast<const float2 *>(&sm.lse[st][r]);
                // (a row of logits of -infinity has no weight: infinity in the place of its normaliser)
                const float ref[2] = {lse.x == -INFINITY ? INFINITY : lse.x * 1.44269504088896341f, lse.y == -INFINITY ? INFINITY : lse.y * 1.44269504088896341f};
                const int2 limit = masked ? *reinterpret_cast<const int2 *>(&sm.limit[st][r]) : make_int2(INT_MAX, INT_MAX);
#pragma unroll
                for (int f = 0; f < F; ++f)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int j = key0 + 16 * f + 8 * x;
                        const float w0 = ex2(fmaf(s[f][y][2 * x], a.scale_log2, -ref[0])), w1 = ex2(fmaf(s[f][y][2 * x + 1], a.scale_log2, -ref[1]));
                        if (j < limit.x) sum[f][x] += w0;
                        if (j < limit.y) sum[f][x] += w1;
                    }
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    pdl_trigger();
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float w = sum[f][x];
            w += __shfl_xor_sync(0xffffffffu, w, 1);
            w += __shfl_xor_sync(0xffffffffu, w, 2);
            const int j = key0 + 16 * f + 8 * x;
            const long long at = (long long)unit * a.cap + j;
            if (ql == 0 && j < sq.n) a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + (there[f][x] ? w : 0.f);
        }
}

template <int DP, bool FEW>
int launch_dp(const AttnArgs &a, cudaStream_t stream)
{
    static SmemAsked asked;
    constexpr int kRows = FEW ? 16 : 64;
    const long long tiles = ((long long)a.rows_max + kRows - 1) / kRows, blocks = tiles * a.batch * a.hkv * a.splits;
    if (blocks > 0x7fffffffLL) {
        set_error_detail("attention: %lld blocks", blocks);
        return WKV_ERR_LIMIT;
    }
    cudaError_t err = allow_smem(attn_mma_kernel<DP, FEW>, sizeof(MmaSmem<DP>), asked);
    if (err == cudaSuccess) err = launch_pdl(attn_mma_kernel<DP, FEW>, dim3((unsigned)blocks), kThreads, sizeof(MmaSmem<DP>), stream,
                                             FEW && a.clustered ? a.splits : 1, a);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "attention kernel");
}

template <int DP, int WARPS>
int launch_weights(const AttnArgs &a, cudaStream_t stream)
{
    static SmemAsked asked;
    constexpr int kBlockKeys = WARPS * 16 * (DP == 256 ? 1 : 2);
    const long long blocks = ((long long)a.cap + kBlockKeys - 1) / kBlockKeys * a.batch * a.hkv;
    // (half as many keys to a block where that leaves SMs without one)
    if (WARPS > 4 && blocks < 2 * 148) return launch_weights<DP, 4>(a, stream);
    if (blocks > 0x7fffffffLL) {
        set_error_detail("attention weights: %lld blocks", blocks);
        return WKV_ERR_LIMIT;
    }
    cudaError_t err = allow_smem(attn_mma_weights_kernel<DP, WARPS>, sizeof(WeightsSmem<DP>), asked);
    if (err == cudaSuccess) err = launch_pdl(attn_mma_weights_kernel<DP, WARPS>, dim3((unsigned)blocks), WARPS * 32, sizeof(WeightsSmem<DP>), stream, 1, a);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "attention weights kernel");
}

}  // namespace

int launch_attn_mma_weights(const AttnArgs &a, cudaStream_t stream)
{
    return a.d <= 64 ? launch_weights<64, 8>(a, stream) : a.d <= 128 ? launch_weights<128, 8>(a, stream) : launch_weights<256, 8>(a, stream);
}
int launch_attn_mma(const AttnArgs &a, cudaStream_t stream)
{
    if (a.rows_max <= 16) return a.d <= 64 ? launch_dp<64, true>(a, stream) : a.d <= 128 ? launch_dp<128, true>(a, stream) : launch_dp<256, true>(a, stream);
    return a.d <= 64 ? launch_dp<64, false>(a, stream) : a.d <= 128 ? launch_dp<128, false>(a, stream) : launch_dp<256, false>(a, stream);
}

}  // namespace wkv
