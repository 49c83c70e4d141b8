// Attention on the tensor cores (tcgen05, tensor memory, TMA): bf16, head dimensions up to 128, whole prompts and chunks of new
// tokens over a paged cache.
//
// An item is two query tiles of up to 128 rows of one unit (row = position x query head of the group, so one key tile serves
// every head that shares it), against the unit's keys in tiles of 128, in ascending order:
//   S = Q K^T    128 x 128 per query tile, in tensor memory
//   P = exp2(S c - m c), in bf16 over S's first columns; one thread per row keeps the maximum m and the sum of P
//   O += P V     128 x d in tensor memory
// The two query tiles alternate: while one's P is computed, the tensor cores work on the other.  m follows the row's maximum
// only when that has grown by more than 2^8: a sum that is too large by at most that factor loses nothing in fp32, and O has to
// be read, scaled and written back only then.
//
// P is rounded to bf16 for the product (as its operand has to be); sum, maximum and O are fp32, the sum of the unrounded P.
//
// Warps: 0-3 and 4-7 the softmax of the two query tiles (thread = row), 8 issues the MMAs, 9 the TMA loads (keys and values of a
// tile in turn through one ring), 10 and 11 load the queries and look through the values of tiles that hold rows which some query
// does not see: P is 0 there, but 0 times an infinity or NaN is not.  Such elements are replaced by 0 in shared memory, and the rows that do see them
// get them added at the end.
//
// Bound by the chain of one query tile, product - weights - product, of which two are in flight (tensor memory holds no third): 32 heads on 8 of 8,192
// tokens, d = 128, 492 us = 1.12 PFLOP/s in a run of 25 ms at 1,965 MHz, 555-575 us = 0.97 PFLOP/s in long runs, which the power limit holds at
// 1,600 to 1,800; tensor pipe 51 % of cycles, special functions 45 %; 32,768 tokens 8.2-8.5 ms = 1.05 PFLOP/s.  Of a chain's 4,000 cycles the
// weights take 2,500, the products 1,100.  Sixteen warps for the weights, two to a row, were slower (600 us where eight took 575): they
// have to agree on the maximum.
//
// Blocks are persistent, one per SM; the items come in order of descending work and are dealt to the blocks back and forth.
// Every wait is bounded; on expiry the block sets bit 0 of the status word, lets its loads land, frees its tensor memory and returns.
#include "attn.cuh"
#include "score_math.cuh"
#include "tc_common.cuh"
#include "tensor_map.cuh"

#include <type_traits>

namespace wkv {
namespace {

using namespace tc;

constexpr int kTile = 128;
constexpr int kThreads = 384;
constexpr int kRegion = kTile * 128;          // bytes of 64 columns of a tile
constexpr uint32_t kTmemCols = 512;           // all of it: S/P of the two query tiles (128 columns each), O of both (128 each)
constexpr int kMaxStages = 8;
constexpr int kMaskSlots = 8;
constexpr int kFmaEvery = 8;                  // one pair of exponentials in so many on the FMA pipe, see exp2_pair_fma()
constexpr int kFirst = 2;                     // 32-key pieces of a tile whose product begins while the others' weights are computed
                                              // (32 heads on 8 of 8,192 tokens, long runs: one 556 us, two 554, three 565; d = 64: 434, 428, 424)
constexpr float kLazy = 8.f;                  // exponent by which the maximum may be outgrown
__host__ __device__ constexpr int stages_for(int kb) { return kb == 2 ? 5 : 8; }
struct TcAttnArgs {
    AttnArgs a;
    int ppt;                 // positions of a query tile: 128 / G
    int max_pairs;           // items of a unit at most
    long long items;
    int k_slot[3];           // tensor-map coordinates of (token, head, batch) / (slot, head, page)
    int box_rows;            // rows of a key box
    bool wide_out;           // rows of the output begin on 32 bytes
    bool by_work;            // kWorkBlocks blocks share the items' key tiles evenly; otherwise items are dealt out whole
    float *piece_o;          // by_work: [2 * blocks][256][d] and
    float2 *piece_ml;        // [2 * blocks][256], what a block has of an item that it does not have all of
    long long *line;         // [items + 1]: where the items begin on the line of work, for the joining kernel
};

struct Shared {
    uint64_t q_full, q_empty;
    uint64_t full[kMaxStages], empty[kMaxStages], look[kMaxStages], clean[kMaxStages];
    uint64_t s_full[2], p_part[2], p_full[2], pv_done[2], o_free[2];
    uint32_t tmem_base;
    int abort;
    int poison[kMaskSlots];                        // item whose values held an infinity or NaN in a tile that was looked through
    uint4 present[kMaskSlots];                     // of the tiles' 128 rows: those with a page
};

struct Item {
    int unit, b, h;
    AttnSeq sq;
    int pos0;                // first position of the first query tile
    int rows[2];             // positions in each
    int tiles[2];            // key tiles of each
    int base;                // keys that query 0 sees
    int looked;              // key tiles from here on are looked through
    int n_tiles;
    int begin, end;          // key tiles that this block takes
    int piece;               // where it leaves what it has of the item, -1: it has all of it
};
__device__ __forceinline__ bool get_item(const TcAttnArgs &t, long long k, Item &im)
{
    const AttnArgs &a = t.a;
    const int units = a.batch * a.hkv;
    const int rank = (int)(k / units);
    im.unit = (int)(k - (long long)rank * units);
    im.b = im.unit / a.hkv;
    im.h = im.unit - im.b * a.hkv;
    im.sq = attn_seq(a, im.b, im.h);
    const int per = 2 * t.ppt, pairs = (im.sq.m + per - 1) / per, pair = pairs - 1 - rank;
    if (pair < 0) return false;
    im.pos0 = pair * per;
    im.base = im.sq.n - im.sq.m + 1;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int first = im.pos0 + x * t.ppt;
        im.rows[x] = min(max(im.sq.m - first, 0), t.ppt);
        const int most = im.rows[x] > 0 ? min(im.base + first + im.rows[x] - 1, im.sq.n) : 0;
        im.tiles[x] = (max(most, 0) + kTile - 1) / kTile;
    }
    im.looked = max(im.base + im.pos0, 0) / kTile;       // every row sees all of the tiles in front of this one
    im.n_tiles = max(im.tiles[0], im.tiles[1]);
    im.begin = 0;
    im.end = im.n_tiles;
    im.piece = -1;
    return true;
}

// Sharing by work: the items, one after the other, are a line of (tiles + kItemCost) each, of which every block takes an equal length.
// An item that lies across blocks is computed in pieces and joined by the kernel behind this one, which finds the pieces by the same
// arithmetic.
constexpr int kItemCost = 4;            // what an item costs beside its key tiles, in tiles
constexpr int kWorkItems = 4 * 148;     // with more items than this they are dealt out whole
constexpr int kWorkKeys = 2048;         // ... and where a unit has fewer keys at most
constexpr int kWorkBlocks = 148;
__device__ __forceinline__ long long item_cost(const TcAttnArgs &t, long long k)
{
    Item im;
    return k < t.items && get_item(t, k, im) ? im.n_tiles + kItemCost : 0;
}
// By a whole warp, 32 items at a time: the length of the line; and, at a place on it, the item there and where that begins.
__device__ __forceinline__ long long line_length(const TcAttnArgs &t, int lane)
{
    long long sum = 0;
    for (int x = lane; x < t.items; x += 32) sum += item_cost(t, x);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}
template <typename F>
__device__ __forceinline__ void walk_line(const TcAttnArgs &t, int lane, F visit)      // visit(item, where it begins, where it ends): enough?
{
    long long before = 0;
    for (int x0 = 0; x0 < t.items; x0 += 32) {
        const long long c = item_cost(t, x0 + lane);
        long long end = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, end, o);
            if (lane >= o) end += v;
        }
        end += before;
        if (visit(x0 + lane, end - c, end)) return;
        before = __shfl_sync(0xffffffffu, end, 31);
    }
}
// what block c has of an item at `at` on a line of `total`: tiles begin .. end - 1
__device__ __forceinline__ void piece_of(long long total, int c, long long at, int n_tiles, int &begin, int &end)
{
    const long long lo = total * c / kWorkBlocks - at, hi = total * (c + 1) / kWorkBlocks - at;
    begin = (int)min(max(lo - kItemCost, 0ll), (long long)n_tiles);
    end = (int)min(max(hi - kItemCost, 0ll), (long long)n_tiles);
}
__device__ __forceinline__ int piece_slot(int c, int begin) { return 2 * c + (begin == 0); }

// a block's items: back and forth over the list, or its share of the line
struct Walk {
    long long k0 = 0;
    int round = 0, seq = 0;       // seq: items with key tiles so far
    long long at = 0, total = -1;
    __device__ __forceinline__ bool next(const TcAttnArgs &t, Item &im)
    {
        if (t.by_work) return next_share(t, im);
        while (k0 < t.items) {
            const long long k = k0 + (round & 1 ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
            k0 += gridDim.x;
            ++round;
            if (k < t.items && get_item(t, k, im)) return true;
        }
        return false;
    }
    __device__ __forceinline__ bool next_share(const TcAttnArgs &t, Item &im)
    {
        if (total < 0) {
            const int lane = threadIdx.x & 31;
            total = line_length(t, lane);
            const long long lo = total * blockIdx.x / kWorkBlocks;
            long long k = t.items, from = 0;
            walk_line(t, lane, [&](int item, long long start, long long end) {
                const unsigned there = __ballot_sync(0xffffffffu, end > lo);
                if (!there) return false;
                k = __shfl_sync(0xffffffffu, item, __ffs(there) - 1);
                from = __shfl_sync(0xffffffffu, start, __ffs(there) - 1);
                return true;
            });
            k0 = k;
            at = from;
        }
        const long long lo = total * blockIdx.x / kWorkBlocks, hi = total * (blockIdx.x + 1) / kWorkBlocks;
        while (k0 < t.items && at < hi) {
            if (!get_item(t, k0, im)) {
                ++k0;
                continue;
            }
            const long long here = at;
            ++k0;
            at += im.n_tiles + kItemCost;
            if (at <= lo) continue;
            piece_of(total, blockIdx.x, here, im.n_tiles, im.begin, im.end);
            if (im.n_tiles == 0) {
                if (here >= lo) return true;              // nothing to see: its rows are written where it begins
                continue;
            }
            if (im.begin >= im.end) continue;
            if (im.end - im.begin < im.n_tiles) im.piece = piece_slot(blockIdx.x, im.begin);
            return true;
        }
        return false;
    }
};

// ---- tensor memory and MMA forms that only this kernel uses -------------------------------------
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                 "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void umma_bf16_ta_if(uint32_t leader, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                                uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "setp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 :
                 : "r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader)
                 : "memory");
}
// Values as B operand: N (the head dimension) runs along the 128-byte rows, K (the keys) across them.  Stride byte offset: 8 keys
// (1024 bytes); leading byte offset: the next 64 columns (a region).
__device__ __forceinline__ uint64_t value_desc(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr >> 4) & 0x3FFFu) | ((uint64_t)(kRegion >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
constexpr uint32_t kBTransposed = 1u << 16;
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ void store32(void *p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h)
                 : "memory");
}
__device__ __forceinline__ void store32(float *p, float a, float b, float c, float d, float e, float f, float g, float h)
{
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(a), "f"(b), "f"(c), "f"(d), "f"(e), "f"(f), "f"(g), "f"(h)
                 : "memory");
}

// ---- the softmax of one query tile ------------------------------------------------------------
// S is read twice, 32 columns at a time, for the maximum and for the exponentials: a row of 128 in registers takes more of them than
// a thread has (168 for each of 384), and the code of a row in one piece more than the instruction cache holds.
struct RowMask {
    uint4 bits;              // of the tile's 128 keys: those that the row sees
    __device__ __forceinline__ uint32_t of(int y) const { return y == 0 ? bits.x : (y == 1 ? bits.y : (y == 2 ? bits.z : bits.w)); }
};
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? ~0u : (n <= 0 ? 0u : (1u << n) - 1u); }
__device__ __forceinline__ void hide(float (&v)[32], uint32_t seen)
{
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = seen >> j & 1u ? v[j] : -INFINITY;
}

// 2^x of two values on the FMA pipe, which is half idle where the special functions are not (32 heads on 8 of 8,192 tokens, long runs: none
// 567 us, one pair in eight 554, in four 554, in two 612; d = 64: 485, 428, 436, 497): 2^t * 2^f with t the nearest integer, 2^f by a polynomial of degree five (a Remez fit of the
// relative error on [-1/2, 1/2], 7.5e-8; evaluated in fp32 2.1e-7).  x is at most kLazy; below -127 it counts as -127,
// whose factor 2^t is 0, so that the weight is 0 below -126.5, as with the special functions; a NaN stays one.
__device__ __forceinline__ unsigned long long exp2_pair_fma(unsigned long long x2)
{
    float2 x = halves_of(x2);
    asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x.x));      // -127
    asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x.y));
    auto both = [](float v) { return pair_of(v, v); };
    x2 = pair_of(x.x, x.y);
    const unsigned long long shifted = add_pair(x2, both(12582912.f));            // 1.5 * 2^23: the integer is in the low bits
    const unsigned long long f = fma_pair(add_pair(shifted, both(-12582912.f)), both(-1.f), x2);
    unsigned long long p = both(1.3276472e-3f);
    p = fma_pair(p, f, both(9.675541e-3f));
    p = fma_pair(p, f, both(5.550713e-2f));
    p = fma_pair(p, f, both(2.402212e-1f));
    p = fma_pair(p, f, both(6.9314694e-1f));
    p = fma_pair(p, f, both(1.0000001f));
    const float2 s = halves_of(shifted);
    return fma_pair(p, pair_of(__int_as_float((__float_as_int(s.x) << 23) + 0x3f800000), __int_as_float((__float_as_int(s.y) << 23) + 0x3f800000)),
                    0ull);
}

__device__ __forceinline__ float largest(float top, const float (&v)[32])
{
    float t0 = top, t1 = v[0];
#pragma unroll
    for (int j = 1; j < 31; j += 2) {
        if (j & 2) t0 = fmaxf(t0, fmaxf(v[j], v[j + 1]));
        else t1 = fmaxf(t1, fmaxf(v[j], v[j + 1]));
    }
    return fmaxf(t0, fmaxf(t1, v[31]));
}

// WHOLE: the head dimension is KB * 64.  Otherwise the columns from it on are zeros in shared memory, and the products leave out the
// steps and columns of 16 that hold nothing else.
template <int KB, bool WHOLE>
__device__ __forceinline__ void softmax_warps(const TcAttnArgs &t, Shared &sh, int x, uint32_t tmem)
{
    const AttnArgs &a = t.a;
    const int D = WHOLE ? KB * 64 : a.d;
    const int lane = threadIdx.x & 31, quarter = (threadIdx.x >> 5) & 3, row = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lanes + x * kTile, o_addr = lanes + 2 * kTile + x * kTile;
    const int place = row / a.G, head = row - place * a.G;
    const bool of_tile = row < t.ppt * a.G;
    const float c = a.scale_log2;
    const unsigned long long c2 = pair_of(c, c);
    uint32_t turn = 0, tiles_before = 0;            // tiles of S taken so far; key tiles of the items so far
    volatile int *const abort_flag = &sh.abort;
    Walk walk;
    Item im;
    while (walk.next(t, im)) {
        const int pos = im.pos0 + x * t.ppt + place, tiles = min(x ? im.tiles[1] : im.tiles[0], im.end);
        const bool mine = of_tile && place < (x ? im.rows[1] : im.rows[0]);
        const int limit = mine ? min(im.base + pos, im.sq.n) : 0;
        const int plain = (im.base + im.pos0 + x * t.ppt) / kTile;         // tiles that every row of this query tile sees all of
        float m = -INFINITY, l = 0.f;
        for (int u = im.begin; u < tiles; ++u, ++turn) {
            if (!warp_wait(&sh.s_full[x], turn & 1, abort_flag)) return;
            tc_fence_after_sync();
            RowMask seen = {make_uint4(~0u, ~0u, ~0u, ~0u)};
            bool masked = u >= plain;
            if (a.table) {
                seen.bits = sh.present[(tiles_before + u - im.begin) % kMaskSlots];
                masked |= (seen.bits.x & seen.bits.y & seen.bits.z & seen.bits.w) != ~0u;
            }
            if (masked) {
                const int in_tile = limit - u * kTile;
                seen.bits.x &= first_bits(in_tile);
                seen.bits.y &= first_bits(in_tile - 32);
                seen.bits.z &= first_bits(in_tile - 64);
                seen.bits.w &= first_bits(in_tile - 96);
            }
            // (A load in flight never crosses a branch: its registers must not be touched, or moved, before the wait.)
            float grown = m;
            if (!masked) {
                float v0[32], v1[32];
                tmem_ld32_issue(s_addr, v0);
#pragma unroll
                for (int y = 0; y < 4; y += 2) {
                    tmem_ld_wait(v0);
                    tmem_ld32_issue(s_addr + y * 32 + 32, v1);
                    grown = largest(grown, v0);
                    tmem_ld_wait(v1);
                    if (y == 0) tmem_ld32_issue(s_addr + 64, v0);
                    grown = largest(grown, v1);
                }
            } else {
#pragma unroll 1
                for (int y = 0; y < 4; ++y) {
                    float v[32];
                    tmem_ld32(s_addr + y * 32, v);
                    hide(v, seen.of(y));
                    grown = largest(grown, v);
                }
            }
            const bool follow = (grown - m) * c > kLazy;          // (also from -infinity on)
            if (u == im.begin) {
                m = grown;
            } else if (__any_sync(0xffffffffu, follow)) {
                if (!warp_wait(&sh.pv_done[x], (turn - 1) & 1, abort_flag)) return;
                tc_fence_after_sync();
                const float f = follow ? exp2f((m - grown) * c) : 1.f;
                if (follow) m = grown;
                l *= f;
#pragma unroll 1
                for (int y = 0; y < (D + 15) / 16; ++y) {
                    float o[16];
                    tmem_ld16(o_addr + y * 16, o);
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(o[j] * f);
                    tmem_st16(o_addr + y * 16, w);
                }
            }
            const float ref = m == -INFINITY ? 0.f : -m * c;
            const unsigned long long ref2 = pair_of(ref, ref);
            unsigned long long sum0 = 0ull, sum1 = 0ull;
            auto weights = [&](float(&v)[32], int y, auto all_seen) {
                uint32_t p[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const unsigned long long e2 = fma_pair(pair_of(v[2 * j], v[2 * j + 1]), c2, ref2), w2 = decltype(all_seen)::value && j % kFmaEvery == kFmaEvery - 1 ? exp2_pair_fma(e2) : exp2_pair(e2);
                    if (j & 1) sum1 = add_pair(sum1, w2);
                    else sum0 = add_pair(sum0, w2);
                    const float2 w = halves_of(w2);
                    p[j] = pack_bf16(w.x, w.y);
                }
                tmem_st16(s_addr + y * 16, p);
            };
            // the product of the first keys may begin while the others' weights are computed
            auto first_part = [&]() {
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_part[x]);
            };
            if (!masked) {
                float v0[32], v1[32];
                tmem_ld32_issue(s_addr, v0);
#pragma unroll
                for (int y = 0; y < 4; y += 2) {
                    tmem_ld_wait(v0);
                    tmem_ld32_issue(s_addr + y * 32 + 32, v1);
                    weights(v0, y, std::true_type{});
                    if (y + 1 == kFirst) first_part();
                    tmem_ld_wait(v1);
                    if (y == 0) tmem_ld32_issue(s_addr + 64, v0);
                    weights(v1, y + 1, std::true_type{});
                    if (y + 2 == kFirst) first_part();
                }
            } else {
#pragma unroll 1
                for (int y = 0; y < 4; ++y) {
                    float v[32];
                    tmem_ld32(s_addr + y * 32, v);
                    hide(v, seen.of(y));
                    weights(v, y, std::false_type{});
                    if (y + 1 == kFirst) first_part();
                }
            }
            tmem_st_wait();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.p_full[x]);
            const float2 s0 = halves_of(sum0), s1 = halves_of(sum1);
            l += (s0.x + s0.y) + (s1.x + s1.y);
        }
        // ---- the item's rows: O / l -------------------------------------------------------------
        const bool any = tiles > im.begin;
        const int hq = im.h * a.G + head;
        __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + (im.sq.q_off + pos) * a.ot + im.b * a.ob + (long long)hq * a.oh;
        if (any) {
            if (!warp_wait(&sh.pv_done[x], (turn - 1) & 1, abort_flag)) return;
            tc_fence_after_sync();
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const bool poisoned = any && *static_cast<volatile int *>(&sh.poison[walk.seq % kMaskSlots]) == walk.seq + 1;
        const long long left = ((long long)im.piece * 2 * kTile + x * kTile + row);      // row of the pieces
#pragma unroll 1
        for (int y = 0; y < (D + 31) / 32; ++y) {
            float o[32];
            if (any) {
                tmem_ld32(o_addr + y * 32, o);
                const float f = im.piece >= 0 ? 1.f : inv;
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = l == 0.f ? 0.f : o[j] * f;
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = 0.f;
            }
            if (poisoned) {
                for (int j = max(im.looked, im.begin) * kTile; j < min(limit, im.end * kTile); ++j) {
                    const long long at = attn_row(a, im.b, im.h, im.sq.q_off, j);
                    if (at < 0) continue;
                    const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(a.v) + at + y * 32;
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        if (!WHOLE && y * 32 + e >= D) break;
                        const float ve = __bfloat162float(v[e]);
                        if (!(fabsf(ve) < INFINITY)) o[e] += ve;
                    }
                }
            }
            if (!mine) continue;
            if (im.piece >= 0) {
                float *to = t.piece_o + left * D + y * 32;
#pragma unroll
                for (int j = 0; j < 32; j += 8)
                    if (WHOLE || y * 32 + j < D) store32(to + j, o[j], o[j + 1], o[j + 2], o[j + 3], o[j + 4], o[j + 5], o[j + 6], o[j + 7]);
            } else if (t.wide_out) {
                // (32 bytes a store are whole sectors: 16 take twice as many of L2's write cycles)
#pragma unroll
                for (int j = 0; j < 32; j += 16)
                    if (WHOLE || y * 32 + j < D) store32(dst + y * 32 + j, pack_bf16(o[j], o[j + 1]), pack_bf16(o[j + 2], o[j + 3]), pack_bf16(o[j + 4], o[j + 5]),
                            pack_bf16(o[j + 6], o[j + 7]), pack_bf16(o[j + 8], o[j + 9]), pack_bf16(o[j + 10], o[j + 11]),
                            pack_bf16(o[j + 12], o[j + 13]), pack_bf16(o[j + 14], o[j + 15]));
            } else {
#pragma unroll
                for (int j = 0; j < 32; j += 8)
                    if (WHOLE || y * 32 + j < D) *reinterpret_cast<uint4 *>(dst + y * 32 + j) = make_uint4(pack_bf16(o[j], o[j + 1]), pack_bf16(o[j + 2], o[j + 3]),
                                                                              pack_bf16(o[j + 4], o[j + 5]), pack_bf16(o[j + 6], o[j + 7]));
            }
        }
        if (any) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.o_free[x]);
        }
        if (mine) {
            if (im.piece >= 0) t.piece_ml[left] = make_float2(m * c, l);
            else attn_store_lse(a, im.b, hq, pos, im.sq.m, l > 0.f || l != l ? m * c + log2f(l) : -INFINITY);
        }
        walk.seq += im.end > im.begin;
        tiles_before += im.end - im.begin;
    }
}

// ---- MMAs --------------------------------------------------------------------------------------
// One warp issues for both query tiles in turn, which keeps them half a step apart: with a warp for each they fell into step, both
// at their exponentials or both at their products (8,192 tokens of 32 heads: 11 % more time).
template <int KB, bool WHOLE>
__device__ __forceinline__ void mma_warp(const TcAttnArgs &t, Shared &sh, uint8_t *q_img, uint8_t *ring, uint32_t tmem)
{
    constexpr int NS = stages_for(KB), kStage = KB * kRegion;
    const int lane = threadIdx.x & 31;
    const uint32_t leader = elect_one();
    volatile int *const abort_flag = &sh.abort;
    const uint64_t q_desc0 = umma_desc_sw128(smem_u32(q_img)), k_desc0 = umma_desc_sw128(smem_u32(ring)), v_desc0 = value_desc(smem_u32(ring));
    const int steps = WHOLE ? KB * 4 : (t.a.d + 15) / 16;        // of 16 columns
    constexpr uint32_t s_idesc = umma_idesc_bf16(kTile, kTile);
    const uint32_t o_idesc = umma_idesc_bf16(kTile, steps * 16) | kBTransposed;
    uint32_t entry = 0, clean_phase = 0;               // ring entries so far; parity per stage of the looked-through tiles
    uint32_t turn[2] = {0, 0}, outs[2] = {0, 0};       // tiles and items of each query tile so far
    Walk walk;
    Item im;
    auto scores = [&](int x, int stage) {
        const uint64_t kd = k_desc0 + (uint64_t)((uint32_t)(stage * kStage) >> 4), qd = q_desc0 + (uint64_t)((uint32_t)(x * kStage) >> 4);
#pragma unroll
        for (int ks = 0; ks < KB * 4; ++ks) {
            if (!WHOLE && ks >= steps) break;
            const uint32_t at = (uint32_t)((ks >> 2) * kRegion + (ks & 3) * 32) >> 4;
            umma_bf16_if(leader, tmem + x * kTile, qd + at, kd + at, s_idesc, ks > 0);
        }
        umma_commit_if(leader, &sh.s_full[x]);
    };
    while (walk.next(t, im)) {
        if (im.end == im.begin) continue;
        const int tiles[2] = {min(im.tiles[0], im.end), min(im.tiles[1], im.end)};
        if (!warp_wait(&sh.q_full, walk.seq & 1, abort_flag)) return;
        const int first = entry % NS;
        if (!warp_wait(&sh.full[first], (entry / NS) & 1, abort_flag)) return;
        tc_fence_after_sync();
        // (S of the last item's last tile has been read: its P was waited for)
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (tiles[x] > im.begin) scores(x, first);
        umma_commit_if(leader, &sh.empty[first]);
        if (im.end - im.begin == 1) umma_commit_if(leader, &sh.q_empty);
        ++entry;
        for (int u = im.begin; u < im.end; ++u) {
            const int v_stage = entry % NS;
            if (!warp_wait(&sh.full[v_stage], (entry / NS) & 1, abort_flag)) return;
            const bool looked = u >= im.looked;
            if (looked && lane == 0) mbar_arrive(&sh.look[v_stage]);
            ++entry;
            const bool more = u + 1 < im.end;
            const int k_stage = entry % NS;
            if (more && !warp_wait(&sh.full[k_stage], (entry / NS) & 1, abort_flag)) return;
            if (looked) {
                if (!warp_wait(&sh.clean[v_stage], clean_phase >> v_stage & 1u, abort_flag)) return;
                clean_phase ^= 1u << v_stage;
            }
            const uint64_t vd = v_desc0 + (uint64_t)((uint32_t)(v_stage * kStage) >> 4);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (u >= tiles[x]) continue;
                const uint32_t s_tmem = tmem + x * kTile, o_tmem = tmem + 2 * kTile + x * kTile;
                if (u == im.begin) {
                    if (outs[x] > 0 && !warp_wait(&sh.o_free[x], (outs[x] - 1) & 1, abort_flag)) return;
                    ++outs[x];
                }
                if (!warp_wait(&sh.p_part[x], turn[x] & 1, abort_flag)) return;
                tc_fence_after_sync();
#pragma unroll
                for (int ks = 0; ks < 2 * kFirst; ++ks)
                    umma_bf16_ta_if(leader, o_tmem, s_tmem + ks * 8, vd + (uint64_t)((ks * 2048) >> 4), o_idesc, u > im.begin || ks > 0);
                if (!warp_wait(&sh.p_full[x], turn[x] & 1, abort_flag)) return;
                tc_fence_after_sync();
#pragma unroll
                for (int ks = 2 * kFirst; ks < kTile / 16; ++ks)
                    umma_bf16_ta_if(leader, o_tmem, s_tmem + ks * 8, vd + (uint64_t)((ks * 2048) >> 4), o_idesc, 1);
                umma_commit_if(leader, &sh.pv_done[x]);
                ++turn[x];
                if (u + 1 < tiles[x]) scores(x, k_stage);
            }
            umma_commit_if(leader, &sh.empty[v_stage]);
            if (more) {
                umma_commit_if(leader, &sh.empty[k_stage]);
                ++entry;
                if (u + 2 == im.end) umma_commit_if(leader, &sh.q_empty);
            }
        }
        ++walk.seq;
    }
}

// ---- loads --------------------------------------------------------------------------------------
template <int KB>
__device__ __forceinline__ uint32_t load_warp(const TcAttnArgs &t, Shared &sh, const CUtensorMap *k_map, const CUtensorMap *v_map, uint8_t *ring)
{
    constexpr int NS = stages_for(KB), kStage = KB * kRegion;
    const AttnArgs &a = t.a;
    const int lane = threadIdx.x & 31;
    volatile int *const abort_flag = &sh.abort;
    uint32_t entry = 0;
    Walk walk;
    Item im;
    const int boxes = kTile / t.box_rows;             // of a tile
    const uint32_t leader = elect_one();
    // One box into a stage.  One lane issues, and every operand is the same in all lanes: the instruction takes them from
    // uniform registers, so that an address which varies from lane to lane is another lane's.
    auto put_box = [&](const CUtensorMap *map, int stage, int box, int tok, int h, int third) {
        const int c1 = t.k_slot[0] == 1 ? tok : (t.k_slot[1] == 1 ? h : third);
        const int c2 = t.k_slot[0] == 2 ? tok : (t.k_slot[1] == 2 ? h : third);
        const int c3 = t.k_slot[0] == 3 ? tok : (t.k_slot[1] == 3 ? h : third);
        uint8_t *to = ring + stage * kStage + box * t.box_rows * 128;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) tma_load_4d_if(leader, to + kb * kRegion, map, &sh.full[stage], kb * 64, c1, c2, c3);
    };
    while (walk.next(t, im)) {
        for (int u = im.begin; u < im.end; ++u) {
            // Where the tile's rows are: dense, one box; paged, one box per page or part of one, and rows without a page are
            // zeros (a page beyond the pool's).  Lane i looks up box i.
            int tok = (int)im.sq.q_off + u * kTile, third = a.cu_q ? 0 : im.b;
            if (a.table) {
                const int row = u * kTile + lane * t.box_rows;
                int page = -1;
                tok = 0;
                if (lane < boxes && row < im.sq.n) {
                    const int pg = row / a.page_size;
                    page = __ldg(a.table + (long long)im.b * a.max_pages + pg);
                    tok = row - pg * a.page_size;
                }
                const bool have = (unsigned)page < (unsigned)a.num_pages;
                third = have ? page : a.num_pages;
                // bit j of word w: row 32 w + j has a page (rows from the length on: no matter)
                const uint32_t votes = __ballot_sync(0xffffffffu, have), all = (1u << boxes) - 1u;
                uint32_t bits = ~0u;
                if ((votes & all) != all) {
                    if (boxes >= 4) {
                        bits = 0;
                        for (int j = 0; j < 32; ++j) bits |= (votes >> (((lane & 3) * 32 + j) / t.box_rows) & 1u) << j;
                    } else {
                        bits = votes >> ((lane & 3) * boxes / 4) & 1u ? ~0u : 0u;
                    }
                }
                if (lane < 4) reinterpret_cast<uint32_t *>(&sh.present[(entry >> 1) % kMaskSlots])[lane] = bits;
                __syncwarp();
            }
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const int stage = entry % NS;
                if (entry >= NS && !warp_wait(&sh.empty[stage], (entry / NS - 1) & 1, abort_flag)) return entry;
                mbar_arrive_expect_tx_if(leader, &sh.full[stage], kStage);
                for (int box = 0; box < boxes; ++box) {
                    const int bt = __shfl_sync(0xffffffffu, tok, box), b3 = __shfl_sync(0xffffffffu, third, box);
                    if (kv == 0) put_box(k_map, stage, box, bt, im.h, b3);
                    else put_box(v_map, stage, box, bt, im.h, b3);
                }
                ++entry;
            }
        }
    }
    return entry;
}

// ---- queries, and values of tiles that some row does not see whole -----------------------------------
// Rows of a query tile (one to each of the two warps) into shared memory, in the 128-byte swizzle that the MMAs read; rows that no query
// has are zeros.  An item's first product waits for it: row and address go on by steps, without a division or a product per row (with
// them the rows of an item took 20,000 cycles, a sixth of the time of 8,192 tokens).
template <int KB>
__device__ __forceinline__ void load_queries(const TcAttnArgs &t, const Item &im, uint8_t *q_img, int x, int lane)
{
    constexpr int kChunks = KB * 8, kRows = 32 / kChunks;        // of 16 bytes, in a row; rows at a time
    const AttnArgs &a = t.a;
    const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(a.q) + im.sq.q_off * a.qt + im.b * a.qb + (long long)im.h * a.G * a.qh;
    const int chunk = lane % kChunks, row0 = lane / kChunks, rows = x ? im.rows[1] : im.rows[0];
    const int place_step = kRows / a.G, head_step = kRows - place_step * a.G;
    const long long step = place_step * a.qt + head_step * a.qh, next_place = a.qt - a.G * a.qh;
    int place = row0 / a.G, head = row0 - place * a.G;
    const __nv_bfloat16 *from = q + (long long)(im.pos0 + x * t.ppt + place) * a.qt + head * a.qh + chunk * 8;
    const uint32_t to = smem_u32(q_img + x * KB * kRegion + (chunk >> 3) * kRegion);
    const bool column = chunk * 8 < a.d;
    for (int r = row0; r < kTile; r += 8) {
#pragma unroll
        for (int y = 0; y < 8; y += kRows) {
            const bool there = column && place < rows;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + swz128_offset(r + y, chunk & 7)), "l"(there ? from : q), "r"(there ? 16 : 0)
                         : "memory");
            from += step;
            place += place_step;
            head += head_step;
            if (head >= a.G) {
                head -= a.G;
                ++place;
                from += next_place;
            }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}
template <int KB>
__device__ __forceinline__ void helper_warp(const TcAttnArgs &t, Shared &sh, uint8_t *q_img, uint8_t *ring, int which)
{
    constexpr int NS = stages_for(KB), kStage = KB * kRegion;
    const int lane = threadIdx.x & 31;
    volatile int *const abort_flag = &sh.abort;
    uint32_t entry = 0, look_phase = 0;
    Walk walk;
    Item im;
    if (t.by_work && blockIdx.x == 0 && which == 1)
        walk_line(t, lane, [&](int item, long long start, long long end) {
            if (item < t.items) t.line[item] = start;
            if (item == t.items - 1) t.line[item + 1] = end;
            return false;
        });
    while (walk.next(t, im)) {
        if (im.end == im.begin) continue;
        if (walk.seq > 0 && !warp_wait(&sh.q_empty, (walk.seq - 1) & 1, abort_flag)) return;
        load_queries<KB>(t, im, q_img, which, lane);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full);
        for (int u = im.begin; u < im.end; ++u, entry += 2) {
            if (u < im.looked) continue;
            const int stage = (entry + 1) % NS;
            // The MMA warp says when: it has seen the tile land and does not go on before this is done, so that the stage's
            // barrier stands at this entry's phase and not two away.
            if (!warp_wait(&sh.look[stage], look_phase >> stage & 1u, abort_flag)) return;
            look_phase ^= 1u << stage;
            if (!warp_wait(&sh.full[stage], ((entry + 1) / NS) & 1, abort_flag)) return;
            uint4 *tile = reinterpret_cast<uint4 *>(ring + stage * kStage) + which * (kStage / 32);
            uint32_t found = 0;
#pragma unroll 8
            for (int y = lane; y < kStage / 32; y += 32) {
                const uint4 v = tile[y];
                const uint32_t e = 0x7f807f80u;
                const uint32_t bx = __vcmpeq2(v.x & e, e), by = __vcmpeq2(v.y & e, e), bz = __vcmpeq2(v.z & e, e), bw = __vcmpeq2(v.w & e, e);
                if (bx | by | bz | bw) {
                    found = 1;
                    tile[y] = make_uint4(v.x & ~bx, v.y & ~by, v.z & ~bz, v.w & ~bw);
                }
            }
            if (found) *static_cast<volatile int *>(&sh.poison[walk.seq % kMaskSlots]) = walk.seq + 1;
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.clean[stage]);
        }
        ++walk.seq;
    }
}

template <int KB, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 1)
attn_tc_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ TcAttnArgs t)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ Shared sh;
    constexpr int NS = stages_for(KB), kStage = KB * kRegion;
    uint8_t *q_img = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023u) & ~uintptr_t(1023u));
    uint8_t *ring = q_img + 2 * kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();
    if (threadIdx.x == 0) {
        mbar_init(&sh.q_full, 2);
        mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < NS; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 1);
            mbar_init(&sh.look[i], 1);
            mbar_init(&sh.clean[i], 2);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sh.s_full[x], 1);
            mbar_init(&sh.p_part[x], 4);
            mbar_init(&sh.p_full[x], 4);
            mbar_init(&sh.pv_done[x], 1);
            mbar_init(&sh.o_free[x], 4);
        }
        fence_barrier_init();
        sh.abort = 0;
        for (int i = 0; i < kMaskSlots; ++i) sh.poison[i] = 0;
    }
    // Tensor memory only behind the wait: the kernel in front may still need all of it on this SM.
    pdl_wait();
    if (warp == 8) tmem_alloc(&sh.tmem_base, kTmemCols);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;
    if (warp < 8) {
        softmax_warps<KB, WHOLE>(t, sh, warp >> 2, tmem);
    } else if (warp == 8) {
        mma_warp<KB, WHOLE>(t, sh, q_img, ring, tmem);
    } else if (warp == 9) {
        if (lane == 0) {
            tma_prefetch_desc(&k_map);
            tma_prefetch_desc(&v_map);
        }
        const uint32_t issued = load_warp<KB>(t, sh, &k_map, &v_map, ring);
        // nothing of this block may be in flight when it ends: the last MMAs must have released their stages; after a
        // failed wait, the loads already issued must still land
        for (uint32_t e = issued > NS ? issued - NS : 0; e < issued; ++e) {
            const int st = e % NS;
            if (!warp_wait(&sh.empty[st], (e / NS) & 1, &sh.abort)) {
                volatile int never = 0;
                warp_wait(&sh.full[st], (e / NS) & 1, &never);
            }
        }
        if (lane == 0 && *static_cast<volatile int *>(&sh.abort) && t.a.status) atomicOr(t.a.status, kStatusWaitExpired);
    } else {
        helper_warp<KB>(t, sh, q_img, ring, warp - 10);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 8) tmem_dealloc(sh.tmem_base, kTmemCols);
}

// Joins the pieces of the items that lie across blocks: block (item, y) takes 8 * RPW of its 256 rows, RPW to a warp.  With few
// items each is in many pieces, whose reading is trips to memory: a row per warp then (8 items of 32 rows over 16,384 keys: 44
// us with the kernel in front, 66 with 32 rows per block).  With many there are two pieces or so, and fewer blocks look for them
// more seldom (160 items: 101 us with 8 rows, 96 with 32).
constexpr int kFewItems = 128;
template <int RPW>                      // rows of a warp, all in flight together
__global__ void __launch_bounds__(256) attn_tc_join_kernel(const __grid_constant__ TcAttnArgs t)
{
    pdl_trigger();
    pdl_wait();
    __shared__ int slots[kWorkBlocks];
    __shared__ int n_slots;
    const AttnArgs &a = t.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Item im;
    if (!get_item(t, blockIdx.x, im) || im.n_tiles == 0) return;
    const int first_row = (int)blockIdx.y * 8 * RPW, x = first_row / kTile;
    if ((first_row - x * kTile) / a.G >= (x ? im.rows[1] : im.rows[0])) return;                // (no row of this block's)
    const long long at = t.line[blockIdx.x], total = t.line[t.items];
    // the pieces, in order: 32 blocks at a time, by the first warp
    if (warp == 0) {
        int n = 0, whole = 0;
        const int from = (int)(at * kWorkBlocks / total), to = (int)min((at + im.n_tiles + kItemCost) * kWorkBlocks / total + 1, (long long)kWorkBlocks);
        for (int c0 = from; c0 < to; c0 += 32) {
            const int c = c0 + lane;
            int begin = 0, end = 0;
            if (c < to) piece_of(total, c, at, im.n_tiles, begin, end);
            const unsigned some = __ballot_sync(0xffffffffu, begin < end);
            whole |= __any_sync(0xffffffffu, end - begin == im.n_tiles);
            if (begin < end) slots[n + __popc(some & ((1u << lane) - 1u))] = piece_slot(c, begin);
            n += __popc(some);
        }
        if (lane == 0) n_slots = whole ? 0 : n;           // (one block has it whole, and has written its rows)
    }
    __syncthreads();
    const int n = n_slots;
    if (n == 0) return;
    int row[RPW];
    bool there[RPW];
    float top[RPW], l[RPW];
    float4 o[RPW];
#pragma unroll
    for (int k = 0; k < RPW; ++k) {
        row[k] = first_row - x * kTile + warp + 8 * k;
        const int place = row[k] / a.G;
        there[k] = place < t.ppt && place < (x ? im.rows[1] : im.rows[0]);
        top[k] = -INFINITY;
        l[k] = 0.f;
        o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int i = lane; i < n; i += 32) {
        const float2 *from = t.piece_ml + (long long)slots[i] * 2 * kTile + x * kTile;
#pragma unroll
        for (int k = 0; k < RPW; ++k)
            if (there[k]) top[k] = fmaxf(top[k], from[row[k]].x);
    }
#pragma unroll
    for (int k = 0; k < RPW; ++k)
#pragma unroll
        for (int y = 16; y; y >>= 1) top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], y));
#pragma unroll (RPW == 1 ? 8 : 2)
    for (int i = 0; i < n; ++i) {
        const long long from = (long long)slots[i] * 2 * kTile + x * kTile;
        float2 ml[RPW];
        float4 p[RPW];
#pragma unroll
        for (int k = 0; k < RPW; ++k) {
            ml[k] = make_float2(0.f, 0.f);
            p[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (!there[k]) continue;
            ml[k] = t.piece_ml[from + row[k]];
            if (lane * 4 < a.d) p[k] = *reinterpret_cast<const float4 *>(t.piece_o + (from + row[k]) * a.d + lane * 4);
        }
#pragma unroll
        for (int k = 0; k < RPW; ++k) {
            // (only a piece without weight is left out: with a factor of 0, NaN in its sum and infinities in its output still count)
            if (ml[k].y == 0.f) continue;
            const float f = exp2f(ml[k].x - (top[k] == -INFINITY ? 0.f : top[k]));
            l[k] += f * ml[k].y;
            o[k].x = fmaf(f, p[k].x, o[k].x);
            o[k].y = fmaf(f, p[k].y, o[k].y);
            o[k].z = fmaf(f, p[k].z, o[k].z);
            o[k].w = fmaf(f, p[k].w, o[k].w);
        }
    }
#pragma unroll
    for (int k = 0; k < RPW; ++k) {
        if (!there[k]) continue;
        const int place = row[k] / a.G, pos = im.pos0 + x * t.ppt + place, hq = im.h * a.G + row[k] - place * a.G;
        if (lane == 0) attn_store_lse(a, im.b, hq, pos, im.sq.m, l[k] > 0.f || l[k] != l[k] ? top[k] + log2f(l[k]) : -INFINITY);
        const float inv = l[k] == 0.f ? 0.f : 1.f / l[k];
        __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + (im.sq.q_off + pos) * a.ot + im.b * a.ob + (long long)hq * a.oh;
        if (lane * 4 < a.d)
            *reinterpret_cast<uint2 *>(dst + lane * 4) = make_uint2(pack_bf16(o[k].x * inv, o[k].y * inv), pack_bf16(o[k].z * inv, o[k].w * inv));
    }
}

template <int KB, bool WHOLE>
int launch_kb(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream)
{
    constexpr size_t smem = 1024 + (size_t)(2 + stages_for(KB)) * KB * kRegion;
    static_assert(smem + sizeof(Shared) <= 232448, "shared memory of a block");
    static SmemAsked asked;
    int dev = 0, sms = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (err == cudaSuccess) err = allow_smem(attn_tc_kernel<KB, WHOLE>, smem, asked);
    const long long grid = t.by_work ? kWorkBlocks : (t.items < sms ? t.items : sms);
    if (err == cudaSuccess) err = launch_pdl(attn_tc_kernel<KB, WHOLE>, dim3((unsigned)grid), kThreads, smem, stream, 1, k_map, v_map, t);
    if (err == cudaSuccess) count_launches(1);
    if (err == cudaSuccess && t.by_work) {
        const auto join = [&](auto kernel, int rows) { return launch_pdl(kernel, dim3((unsigned)t.items, 2 * kTile / rows), 256, 0, stream, 1, t); };
        err = t.items <= kFewItems ? join(attn_tc_join_kernel<1>, 8) : join(attn_tc_join_kernel<4>, 32);
        if (err == cudaSuccess) count_launches(1);
    }
    return check_cuda(err, "tensor-core attention kernel");
}

}  // namespace

// A tile's rows come in boxes that never cross a page's end: the largest power of two that a page is a multiple of, eight at
// least, since the swizzle's pattern repeats every eight rows.  (Four sequences of 10-16 K rows, up to
// 512 new tokens of 32 heads, a short run: 327 us in pages of 128 rows, 403 in pages of 24 and so boxes of eight; in pages of seven, on the
// warp-level kernel, 2,310.)
static int box_of_page(int page_size) { return std::min(page_size & -page_size, kTile); }

// Shapes that the kernel takes; a layout that no tensor map describes is found out at launch (WKV_ERR_UNSUPPORTED).
bool attn_tc_supported(const AttnArgs &a, int dtype)
{
    if (dtype != WKV_BF16 || a.d > 128 || a.G > kTile) return false;
    // a key tile is one box: tensors of fewer rows are left to the other kernels, which are as fast there
    if (!a.table && (a.cu_q ? a.total_q : a.max_q) < kTile) return false;
    if (a.table && box_of_page(a.page_size) < 8) return false;
    int dev = 0, major = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    return major == 10;
}

int attn_tc_pieces(long long units, int max_q, int G, int cap, int *rows, int *items)
{
    const int ppt = kTile / G;
    *rows = 2 * kTile;
    *items = kWorkItems;
    return units * ((max_q + 2 * ppt - 1) / (2 * ppt)) <= kWorkItems && cap >= kWorkKeys ? 2 * kWorkBlocks : 0;
}

int launch_attn_tc(const AttnArgs &a, float *piece_o, float2 *piece_ml, long long *line, cudaStream_t stream)
{
    TcAttnArgs t;
    t.a = a;
    t.ppt = kTile / a.G;
    const long long units = (long long)a.batch * a.hkv;
    t.max_pairs = (a.max_q + 2 * t.ppt - 1) / (2 * t.ppt);
    t.items = units * t.max_pairs;
    t.box_rows = a.table ? box_of_page(a.page_size) : kTile;
    t.wide_out = a.d % 16 == 0 && (reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ot * 2) | (uintptr_t)(a.oh * 2) | (uintptr_t)(a.ob * 2)) % 32 == 0;
    int rows = 0, most = 0;
    t.by_work = piece_o && attn_tc_pieces(units, a.max_q, a.G, a.cap, &rows, &most);
    t.piece_o = piece_o;
    t.piece_ml = piece_ml;
    t.line = line;
    alignas(64) CUtensorMap k_map, v_map;
    const unsigned long long tokens = a.cu_q ? a.total_q : a.max_q, batch = a.cu_q ? 1 : a.batch;
    if (a.cu_q && a.total_q == 0) return WKV_OK;
    const RowDim k_dims[3] = {{a.table ? (unsigned long long)a.page_size : tokens, (unsigned long long)a.kt * 2, (unsigned)t.box_rows},
                              {(unsigned long long)a.hkv, (unsigned long long)a.kh * 2, 1},
                              {a.table ? (unsigned long long)a.num_pages : batch, (unsigned long long)a.kb * 2, 1}};
    if (!make_row_tensor_map(a.k, a.d, k_dims, &k_map, t.k_slot) || !make_row_tensor_map(a.v, a.d, k_dims, &v_map, t.k_slot))
        return WKV_ERR_UNSUPPORTED;
    if (a.d > 64) return a.d == 128 ? launch_kb<2, true>(t, k_map, v_map, stream) : launch_kb<2, false>(t, k_map, v_map, stream);
    return a.d == 64 ? launch_kb<1, true>(t, k_map, v_map, stream) : launch_kb<1, false>(t, k_map, v_map, stream);
}

}  // namespace wkv
