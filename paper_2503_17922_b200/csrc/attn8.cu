// Attention over the 8-bit cache on warp-level matrix instructions (m16n8k16, f16): single tokens, short chunks and drafts, and the
// shapes that the tcgen05 kernel does not take.
//
// A block of four warps walks over the keys of one unit (or a split of them) in tiles of 128, which come through a ring of asynchronous
// 16-byte copies, codes as they are; a warp takes 32 of a tile's keys and keeps a maximum and a sum of its own, joined once at the end.
//   S^T = K Q^T     16 keys x 8 rows (position x head of the group) per instruction, K's codes as operand A
//   O^T += V^T P^T  16 columns x 8 rows, V's codes as operand A
// Keys and columns are on the M side, so that the few rows that share them fill N = 8 and not a quarter of M = 16; the accumulator of the
// one product becomes the operand of the other by two 8 x 8 transpositions.
//
// Codes become f16 in registers, exactly, an instruction or two to a pair, and scales stay out of the products: a logit is multiplied by
// its key's 2^e, a weight by its value's.  Queries are scaled by a power of two per row, so that their largest element is in
// 2^14 .. 2^15: exact down to 2^-29 of that.  Weights p 2^e go into the second product as f16, relative to a power of two per row, that of the
// largest p 2^e that the row has met (its seen keys' alone: a scale that another row sees, or one of next to no weight, takes no bits), and times
// 2^14: rounded to 2^-11 of themselves at most, half a step, down to 2^-28 of that, where bf16 has 2^-8.  Sums, maxima, logits and outputs are fp32, the sum of the
// unrounded p.
//
// Which 16-byte chunk of a row a thread reads is free, as long as Q and K agree on the order of the columns: a thread reads whole chunks and takes them
// apart into the operands of four (K) or eight (V) instructions.  Chunks are XORed with the row so that eight lanes meet eight
// different ones.
//
// Bound by the instructions that make operands of codes, half of them on the half-rate integer pipe, and by what few warps can hide: 32 sequences of 4-8 K rows of 8
// heads, d = 128, one token of 32 heads (int8, 423 MB): 92 us = 4.6 TB/s, with the rows' weights 105-112; issue slots 54 % busy, integer pipe 46 %, tensor pipe 13 %, 11 warps
// per SM: the ring of 70 KB per block of four warps admits three.  With tiles of 64 keys, one group to a warp, 137 with weights.  With one reference for all of a
// warp's rows, seen keys or not, 0.7 % less time, with 16 rows 5 % less, and wrong where a row does not see the largest value (16 drafts over 4-8 K rows,
// 64 rows at most: 142 and 135 us).  One token over 992 rows of one sequence: 7.7 us.
#include "attn_cluster.cuh"
#include "cache8.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 128;
constexpr int kKeys = 128;
constexpr int kGroups = 2;                     // of 16 keys, of a warp
__host__ __device__ constexpr int stages_for(int dp) { return dp == 64 ? 3 : 2; }

template <int DP>
struct Smem8 {
    __align__(128) unsigned char k[stages_for(DP)][kKeys * DP];
    __align__(128) unsigned char v[stages_for(DP)][kKeys * DP];
    long long at[2][kKeys];                    // byte offsets of a tile's rows, -1: none
    float scale[stages_for(DP)][2][kKeys];     // of K and V; 0: the row has no page
    __align__(16) int missing[stages_for(DP) + 1][4];        // of a tile's four quarters: some row has no page
    float m[4][16], l[4][16], lse2[16];
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// byte offset of 16-byte chunk `chunk` of a row: in the row's line of 128 bytes, eight chunks are permuted
template <int DP, bool VALUES>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk)
{
    const int linear = row * (DP / 16) + chunk;
    return (uint32_t)(VALUES ? linear ^ ((row >> 1 & 3) << 1) : (DP == 64 ? linear : linear ^ ((row & 1) << 2))) << 4;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
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
// codes that are NaN, as bytes of ones
template <int KIND>
__device__ __forceinline__ uint32_t nan_codes(uint32_t w)
{
    return KIND == kE4m3 ? __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu) : 0u;
}

// NT: tiles of eight rows.  DRAFT: the rows go by their masks.
template <int DP, int KIND, int NT, bool DRAFT>
__global__ void __launch_bounds__(kThreads, DP == 256 ? 1 : (DP == 64 && NT == 1 ? 4 : 3)) attn8_kernel(const __grid_constant__ AttnArgs a, int page_shift)
{
    extern __shared__ __align__(128) unsigned char raw[];
    Smem8<DP> &sm = *reinterpret_cast<Smem8<DP> *>(raw);
    constexpr int NS = stages_for(DP), kRows = 8 * NT, kBlocks = DP / 64, kCols = DP / 8, kTiles = DP / 16;      // kCols: columns of V of a thread
    // The joining kernel may be placed now.  Another of this kind is not to be before this one ends: its blocks would crowd onto the
    // SMs that have room at that time.
    const bool clustered = a.clustered, parts = !clustered && (a.splits > 1 || a.logits);
    if (parts) pdl_trigger();
    pdl_wait();
    const int units = a.batch * a.hkv;
    const int splits = a.splits, place_of = (int)blockIdx.x / splits, split = (int)blockIdx.x - place_of * splits;
    // (a unit's row tiles are neighbours: they read the same keys at about the same time, from L2)
    const int tiles = (int)gridDim.x / splits / units, unit = place_of / tiles, tile = place_of - unit * tiles;
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const AttnSeq sq = attn_seq(a, b, h);
    const int rows = sq.m * a.G, row0 = tile * kRows;
    if (row0 >= rows) {
        if (clustered) carry_weights(a, unit, (int)((long long)sq.n * split / splits), (int)((long long)sq.n * (split + 1) / splits), kThreads);
        return;
    }
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = lane >> 2, ql = lane & 3;
    const int base = attn_before<DRAFT>(a, sq, unit) + 1;                // keys that query 0 attends to (may be negative)
    const int most = DRAFT ? sq.n : min(base + (min(row0 + kRows, rows) - 1) / a.G, sq.n);
    const int all_tiles = (max(most, 0) + kKeys - 1) / kKeys;
    const int t0 = (int)((long long)all_tiles * split / splits), t1 = (int)((long long)all_tiles * (split + 1) / splits);
    const int plain = DRAFT ? base - 1 : base + row0 / a.G;              // every row attends to the keys before this one

    // queries: row `quad` of every tile, 16 columns of each 64
    uint32_t q[NT][kBlocks][8];
    float back[NT];                                                      // logit scale of the row: what the power of two took away, in base 2
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = row0 + t * 8 + quad, i = row / a.G, g = row - i * a.G;
        const __nv_bfloat16 *p = static_cast<const __nv_bfloat16 *>(a.q) + (sq.q_off + i) * a.qt + b * a.qb + (long long)(h * a.G + g) * a.qh;
        float x[kBlocks][16];
        unsigned top = 0u;
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) {
            const int d0 = c * 64 + ql * 16;
            uint4 w[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
            if (row < rows && d0 < a.d) {                                // (a row is a multiple of 16 elements)
                w[0] = *reinterpret_cast<const uint4 *>(p + d0);
                w[1] = *reinterpret_cast<const uint4 *>(p + d0 + 8);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[c][e] = __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(w)[e]);
                const unsigned bits = magnitude(x[c][e]);
                if (bits < 0x7f800000u) top = max(top, bits);
            }
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int shift = top == 0u ? 0 : min(14 + 127 - (int)(top >> 23), 120);
        const float by = __uint_as_float((unsigned)(127 + shift) << 23);
        back[t] = a.scale_log2 * __uint_as_float((unsigned)(127 - shift) << 23);
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) q[t][c][e] = pack_f16(x[c][2 * e] * by, x[c][2 * e + 1] * by);
    }
    // accumulators have rows 2 ql and 2 ql + 1 of a tile
    float scale_of[NT][2];
    int limit[NT][2];
    const unsigned *mask[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            scale_of[t][e] = __shfl_sync(0xffffffffu, back[t], (2 * ql + e) * 4);
            const int row = row0 + t * 8 + 2 * ql + e, i = row / a.G;
            limit[t][e] = row < rows ? (DRAFT ? base - 1 : base + i) : 0;
            mask[t][e] = DRAFT && row < rows ? attn_mask(a, sq, b, i) : nullptr;
        }
    auto sees = [&](int t, int e, int j) {                               // row (t, e) and key j < n, whose page is one
        if (j < limit[t][e]) return true;
        if (!DRAFT || !mask[t][e]) return false;
        const int at = j - (base - 1);                                   // token of the draft (limit is base - 1)
        return at < sq.m && (__ldg(mask[t][e] + (at >> 5)) >> (at & 31) & 1u) != 0u;
    };
    float o[NT][kTiles][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) o[t][x][y] = 0.f;
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            m[t][e] = -INFINITY;
            l[t][e] = 0.f;
        }
    // O is in units of v_ref / 2^14, a power of two that the row's p 2^e (p relative to m) have not passed twofold.  Of a float the upper half
    // says enough: those of a tile's two rows are one word, and compared by one instruction.
    constexpr unsigned kLeastRef = (unsigned)(kScaleBias + kLeastExponent - 10) << 7, kMostRef = 253u << 7, kBoth = 0x10001u;
    unsigned v_ref[NT];
    auto ref_bits = [](unsigned both, int e) { return e ? both & 0xffff0000u : both << 16; };
#pragma unroll
    for (int t = 0; t < NT; ++t) v_ref[t] = kLeastRef * kBoth;

    // ---- the ring of key tiles -----------------------------------------------------------------
    // A thread has a row of the tile: its place is looked up a tile ahead of its load, its scales a tile behind that: a trip to memory each.
    const int *const table = a.table + (long long)b * a.max_pages;
    auto page_of = [&](int j, int &slot) {
        const int pg = page_shift >= 0 ? j >> page_shift : j / a.page_size;
        slot = j - pg * a.page_size;
        return __ldg(table + pg);
    };
    int page = -1, slot = 0;
    auto look_up = [&](int t) {
        const int j = t * kKeys + tid;
        page = -1;
        if (t < t1 && j < sq.n) page = page_of(j, slot);
    };
    int byte[2] = {-1, -1};                   // scales of the row whose place was kept last
    auto keep_place = [&](int t) {
        const bool have = (unsigned)page < (unsigned)a.num_pages;
        sm.at[t & 1][tid] = have ? page * a.kb + h * a.kh + (long long)slot * a.kt : -1;
        const unsigned there = __ballot_sync(0xffffffffu, have);
        if (lane == 0) sm.missing[t % (NS + 1)][warp] = there != 0xffffffffu;
        byte[0] = byte[1] = -1;
        if (have) {
            const long long at = ((long long)page * a.hkv + h) * a.page_size + slot;
            byte[0] = a.k_scales[at];
            byte[1] = a.v_scales[at];
        }
    };
    auto keep_scales = [&](int t) {
#pragma unroll
        for (int x = 0; x < 2; ++x) sm.scale[t % NS][x][tid] = byte[x] < 0 ? 0.f : scale_value(byte[x]);
    };
    constexpr int kChunks = DP / 16, kRowsAtOnce = kThreads / kChunks;
    const int chunk = tid % kChunks, row_of = tid / kChunks;
    const bool real = chunk * 16 < a.d;
    const unsigned char *const k_from = static_cast<const unsigned char *>(a.k) + chunk * 16, *const v_from = static_cast<const unsigned char *>(a.v) + chunk * 16;
    // (the permutations of a line's chunks repeat every eight rows, and kRowsAtOnce rows on is the same place in them, or the same but for known bits)
    auto load = [&](int t) {
        if (t < t1) {
            const int st = t % NS;
            const uint32_t ks = smem_addr(&sm.k[st][0]), vs = smem_addr(&sm.v[st][0]);
#pragma unroll
            for (int r = 0; r < kKeys; r += kRowsAtOnce) {
                const long long at = sm.at[t & 1][row_of + r];
                const bool have = at >= 0 && real;
                const long long off = have ? at : 0;
                const int size = have ? 16 : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ks + chunk_at<DP, false>(row_of + r, chunk)), "l"(k_from + off), "r"(size) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(vs + chunk_at<DP, true>(row_of + r, chunk)), "l"(v_from + off), "r"(size) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    look_up(t0);
    keep_place(t0);
    for (int x = 0; x < NS - 1; ++x) {
        look_up(t0 + x + 1);
        __syncthreads();
        load(t0 + x);
        keep_scales(t0 + x);
        keep_place(t0 + x + 1);
    }
    // where this row's logits go, less the keys of the block's first tile
    float *logits[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int row = row0 + n * 8 + 2 * ql + e;
            logits[n][e] = a.logits && row < rows ? a.logits + ((long long)unit * a.rows_max + row) * a.logit_stride + warp * 32 + quad : nullptr;
        }
    for (int t = t0; t < t1; ++t) {
        const int st = t % NS;
        look_up(t + NS);
        asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
        __syncthreads();                      // tile t has landed for all; the stage of tile t - 1 is free; places of t + NS - 1 are there
        load(t + NS - 1);
        const int j0 = t * kKeys + warp * 32;                            // the warp's first key
        const int4 gaps = *reinterpret_cast<const int4 *>(&sm.missing[t % (NS + 1)][0]);
        const bool holes = gaps.x | gaps.y | gaps.z | gaps.w, masked = (t + 1) * kKeys > plain || holes;
        // ---- logits: keys quad and quad + 8 of each group ----------------------------------------------
        float s[kGroups][NT][4] = {};
        float v_scale[kGroups][2];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int key0 = warp * 32 + g * 16;
            const float k_scale[2] = {sm.scale[st][0][key0 + quad], sm.scale[st][0][key0 + quad + 8]};
            v_scale[g][0] = sm.scale[st][1][key0 + quad];
            v_scale[g][1] = sm.scale[st][1][key0 + quad + 8];
#pragma unroll
            for (int c = 0; c < kBlocks; ++c) {
                const uint4 k0 = *reinterpret_cast<const uint4 *>(&sm.k[st][chunk_at<DP, false>(key0 + quad, c * 4 + ql)]);
                const uint4 k1 = *reinterpret_cast<const uint4 *>(&sm.k[st][chunk_at<DP, false>(key0 + quad + 8, c * 4 + ql)]);
                const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t f[4];
                    codes_to_f16<KIND>(w0[i], f[0], f[2]);
                    codes_to_f16<KIND>(w1[i], f[1], f[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_f16(s[g][n], f, q[n][c][2 * i], q[n][c][2 * i + 1]);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int y = 0; y < 4; ++y) s[g][n][y] *= scale_of[n][y & 1] * k_scale[y >> 1];
        }
        unsigned hidden = 0u;                 // bit (g NT + n) 4 + y: the row does not see the key
        bool unseen = false;                  // ... and there are such a key and such a row
        if (masked) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int y = 0; y < 4; y += 2) {
                    const int j = j0 + g * 16 + quad + 4 * y;
                    bool there = j < sq.n;
                    if (there && holes) {
                        int unused;
                        there = (unsigned)page_of(j, unused) < (unsigned)a.num_pages;
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            if (there && sees(n, e, j)) continue;
                            s[g][n][y + e] = -INFINITY;
                            hidden |= 1u << ((g * NT + n) * 4 + y + e);
                            unseen |= there;
                        }
                }
        }
        if (a.logits) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (logits[n][y & 1] && j0 + g * 16 + quad + 8 * (y >> 1) < sq.n) logits[n][y & 1][t * kKeys + g * 16 + 8 * (y >> 1)] = s[g][n][y];
        }
        // ---- weights ---------------------------------------------------------------------------------
        uint32_t p[kGroups][NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float w[kGroups][4], keep[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = fmaxf(fmaxf(s[0][n][e], s[0][n][2 + e]), fmaxf(s[1][n][e], s[1][n][2 + e]));
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                top = fmaxf(m[n][e], top);
                const float ref = top == -INFINITY ? 0.f : top;
                keep[e] = ex2(m[n][e] - ref);
                m[n][e] = top;
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float x = ex2(s[g][n][2 * y + e] - ref);
                        sum += x;
                        w[g][2 * y + e] = x * v_scale[g][y];
                    }
                l[n][e] = l[n][e] * keep[e] + sum;                       // this thread's keys; joined over the quads at the end
            }
            if (masked) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (hidden >> ((g * NT + n) * 4 + y) & 1u) w[g][y] = 0.f;          // (0 times a NaN scale is not 0)
            }
            // the rows' largest p 2^e
            const float w_top[2] = {fmaxf(fmaxf(w[0][0], w[0][2]), fmaxf(w[1][0], w[1][2])), fmaxf(fmaxf(w[0][1], w[0][3]), fmaxf(w[1][1], w[1][3]))};
            unsigned tops = __byte_perm(__float_as_uint(w_top[0]), __float_as_uint(w_top[1]), 0x7632);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) tops = __vmaxu2(tops, __shfl_xor_sync(0xffffffffu, tops, x));
#pragma unroll
            for (int e = 0; e < 2; ++e) keep[e] *= __uint_as_float(ref_bits(v_ref[n], e));
            tops = __vmaxu2(tops, __byte_perm(__float_as_uint(keep[0]), __float_as_uint(keep[1]), 0x7632));
            v_ref[n] = __vminu2(__vmaxu2(tops, kLeastRef * kBoth), kMostRef * kBoth) & 0xff80ff80u;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float inverse = __uint_as_float((254u << 23) - ref_bits(v_ref[n], e));
                keep[e] *= inverse;
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    w[g][e] *= inverse * 16384.f;
                    w[g][2 + e] *= inverse * 16384.f;
                }
            }
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                p[g][n][0] = transposed(pack_f16(w[g][0], w[g][1]));
                p[g][n][1] = transposed(pack_f16(w[g][2], w[g][3]));
            }
            if (__any_sync(0xffffffffu, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
                for (int x = 0; x < kTiles; ++x) {
                    o[n][x][0] *= keep[0];
                    o[n][x][1] *= keep[1];
                    o[n][x][2] *= keep[0];
                    o[n][x][3] *= keep[1];
                }
            }
        }
        // ---- O^T += V^T P^T: keys 2 ql, 2 ql + 1 and those plus 8, columns quad * 16 .. of each 128 (or quad * 8 .. of 64) ----------------
        // (0 times a NaN code is not 0: where some row does not see some key, such codes count as 0 and are added to the rows that see them)
        bool poisoned = false;
        const bool look = KIND == kE4m3 && masked && __any_sync(0xffffffffu, unseen);
        constexpr int kWords = DP == 64 ? 2 : 4;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int c = 0; c < kCols / (4 * kWords); ++c) {
                uint32_t w[4][kWords];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int row = warp * 32 + g * 16 + 2 * ql + (x & 1) + (x >> 1) * 8;
                    if constexpr (DP == 64) {
                        const uint2 y = *reinterpret_cast<const uint2 *>(&sm.v[st][chunk_at<DP, true>(row, quad >> 1) + (quad & 1) * 8]);
                        w[x][0] = y.x;
                        w[x][1] = y.y;
                    } else {
                        const uint4 y = *reinterpret_cast<const uint4 *>(&sm.v[st][chunk_at<DP, true>(row, c * 8 + quad)]);
                        w[x][0] = y.x;
                        w[x][1] = y.y;
                        w[x][2] = y.z;
                        w[x][3] = y.w;
                    }
                }
                if (look) {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int i = 0; i < kWords; ++i) {
                            const uint32_t bad = nan_codes<KIND>(w[x][i]);
                            poisoned |= bad != 0u;
                            w[x][i] &= ~bad;
                        }
                }
#pragma unroll
                for (int i = 0; i < kWords; ++i) {
                    uint32_t f[2][4];             // columns 4 i, 4 i + 1 and 4 i + 2, 4 i + 3
                    codes_to_f16<KIND>(__byte_perm(w[0][i], w[1][i], 0x5140), f[0][0], f[0][1]);
                    codes_to_f16<KIND>(__byte_perm(w[2][i], w[3][i], 0x5140), f[0][2], f[0][3]);
                    codes_to_f16<KIND>(__byte_perm(w[0][i], w[1][i], 0x7362), f[1][0], f[1][1]);
                    codes_to_f16<KIND>(__byte_perm(w[2][i], w[3][i], 0x7362), f[1][2], f[1][3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_f16(o[n][(c * kWords + i) * 2], f[0], p[g][n][0], p[g][n][1]);
                        mma_f16(o[n][(c * kWords + i) * 2 + 1], f[1], p[g][n][0], p[g][n][1]);
                    }
                }
            }
        if (look && __any_sync(0xffffffffu, poisoned)) {
            for (int kk = 0; kk < 32; ++kk) {
                const int row = warp * 32 + kk, j = j0 + kk;
                if (j >= sq.n) break;
#pragma unroll
                for (int x = 0; x < kTiles; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int col = DP == 64 ? quad * 8 + 2 * x + y : (x >> 3) * 128 + quad * 16 + (x & 7) * 2 + y;
                        const unsigned char code = sm.v[st][chunk_at<DP, true>(row, col >> 4) + (col & 15)];
                        if ((code & 0x7f) != 0x7f) continue;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (sees(n, e, j)) o[n][x][2 * y + e] = __uint_as_float(0x7fffffffu);
                    }
            }
        }
        keep_scales(t + NS - 1);
        keep_place(t + NS);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!parts) pdl_trigger();
    // ---- the four warps' sums, in order -----------------------------------------------------------
    __syncthreads();
    constexpr int kPad = DP + 4;
    float *const all = reinterpret_cast<float *>(&sm.k[0][0]);             // [4][kRows][kPad]
    static_assert(4 * kRows * kPad * 4 <= sizeof(sm.k) + sizeof(sm.v), "the ring holds the warps' outputs");
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = n * 8 + 2 * ql + e;
            const float by = __uint_as_float(ref_bits(v_ref[n], e)) * (1.f / 16384.f);
            if (quad == 0) {
                sm.m[warp][r] = m[n][e];
                sm.l[warp][r] = l[n][e];
            }
#pragma unroll
            for (int x = 0; x < kTiles; ++x) {
                const int col = DP == 64 ? quad * 8 + 2 * x : (x >> 3) * 128 + quad * 16 + (x & 7) * 2;
                *reinterpret_cast<float2 *>(all + (warp * kRows + r) * kPad + col) = make_float2(o[n][x][e] * by, o[n][x][2 + e] * by);
            }
        }
    __syncthreads();
    const int live = min(kRows, rows - row0);
    for (int x = tid; x < live * (DP / 4); x += kThreads) {
        const int r = x / (DP / 4), c = (x - r * (DP / 4)) * 4;
        const float top = fmaxf(fmaxf(sm.m[0][r], sm.m[1][r]), fmaxf(sm.m[2][r], sm.m[3][r])), ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = ex2(sm.m[w][r] - ref);
            const float4 part = *reinterpret_cast<const float4 *>(all + (w * kRows + r) * kPad + c);
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
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv));
    }
    if (clustered) {
        __syncthreads();
        float top = 0.f, sum = 0.f;
        if (tid < kRows) {
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
}

template <int DP, int KIND, int NT, bool DRAFT>
int launch8(const AttnArgs &a, cudaStream_t stream)
{
    static SmemAsked asked;
    const long long tiles = ((long long)a.rows_max + 8 * NT - 1) / (8 * NT), blocks = tiles * a.batch * a.hkv * a.splits;
    if (blocks > 0x7fffffffLL) {
        set_error_detail("attention: %lld blocks", blocks);
        return WKV_ERR_LIMIT;
    }
    const int page_shift = (a.page_size & (a.page_size - 1)) == 0 ? __builtin_ctz(a.page_size) : -1;
    cudaError_t err = allow_smem(attn8_kernel<DP, KIND, NT, DRAFT>, sizeof(Smem8<DP>), asked);
    if (err == cudaSuccess) err = launch_pdl(attn8_kernel<DP, KIND, NT, DRAFT>, dim3((unsigned)blocks), kThreads, sizeof(Smem8<DP>), stream,
                                             a.clustered ? a.splits : 1, a, page_shift);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "attention kernel (8-bit cache)");
}
template <int DP, int KIND>
int launch_kind(const AttnArgs &a, cudaStream_t stream)
{
    if (a.masks) return a.rows_max <= 8 ? launch8<DP, KIND, 1, true>(a, stream) : launch8<DP, KIND, 2, true>(a, stream);
    return a.rows_max <= 8 ? launch8<DP, KIND, 1, false>(a, stream) : launch8<DP, KIND, 2, false>(a, stream);
}
template <int DP>
int launch_dp(const AttnArgs &a, cudaStream_t stream)
{
    return a.kind == kE4m3 ? launch_kind<DP, kE4m3>(a, stream) : launch_kind<DP, kI8>(a, stream);
}

}  // namespace

int launch_attn8(const AttnArgs &a, cudaStream_t stream)
{
    if (a.d <= 64) return launch_dp<64>(a, stream);
    return a.d <= 128 ? launch_dp<128>(a, stream) : launch_dp<256>(a, stream);
}

}  // namespace wkv
