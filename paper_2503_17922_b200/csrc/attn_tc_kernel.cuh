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
// EIGHT: keys and values of 8 bits.  Warps 12-15 make bf16 tiles of them, exactly (a row's scale is a power of two), in the place where TMA otherwise puts
// them; TMA's own tiles of codes have a ring in front of that.  What follows is the same.  Bound by those four warps' instructions beside the softmax's, on one
// half-rate integer pipe and one instruction cache: four sequences of 8-16 K keys, 512 new tokens of 32 heads on 8, d = 128: 456-464 us (329 over bf16 rows; 386 in a copy that
// converts nothing: the rest of the difference, with rings of three and four stages where the plain form has one of five, is not explained); issue slots 49 % busy, tensor pipe
// 32 %.  P is rounded to bf16 as in the plain form: 1.7e-3 from the 64-bit value over a whole output of the case above, where weights of fp32 would leave the output's own
// 1.5e-3.  The loop over a tile is kept small, as the softmax's code fills the cache: unrolled, 738 us.
// DRAFT: the rows go by their masks, as far as the new tokens' rows are concerned: every row's keys reach to the unit's last one.  (16 drafts of 64 tokens over 4-8 K
// rows of 8 bits, 32 heads on 8: 224-231 us; 197 in a copy that converts nothing.)
//
// Blocks are persistent, one per SM; the items come in order of descending work and are dealt to the blocks back and forth.
// Every wait is bounded; on expiry the block sets bit 0 of the status word, lets its loads land, frees its tensor memory and returns.
#pragma once

#include "cache8.cuh"
#include "score_math.cuh"
#include "tc_common.cuh"
#include "tensor_map.cuh"

#include <type_traits>

namespace wkv {

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

namespace {

using namespace tc;

constexpr int kTile = 128;
constexpr int threads_for(bool eight) { return eight ? 512 : 384; }
// Registers of a thread (EIGHT): of the 512 x 128 that the block is launched with, the softmax's two warpgroups take 168 each, the others keep 88.
constexpr int kSoftmaxRegs = 168, kOtherRegs = 88;
static_assert(256 * kSoftmaxRegs + 256 * kOtherRegs <= 512 * 128, "what the block is launched with");
constexpr int kRegion = kTile * 128;          // bytes of 64 columns of a tile
constexpr uint32_t kTmemCols = 512;           // all of it: S/P of the two query tiles (128 columns each), O of both (128 each)
constexpr int kMaxStages = 8;
constexpr int kMaskSlots = 8;
constexpr int kFmaEvery = 8;                  // one pair of exponentials in so many on the FMA pipe, see exp2_pair_fma()
constexpr int kFirst = 2;                     // 32-key pieces of a tile whose product begins while the others' weights are computed
                                              // (32 heads on 8 of 8,192 tokens, long runs: one 556 us, two 554, three 565; d = 64: 434, 428, 424)
constexpr float kLazy = 8.f;                  // exponent by which the maximum may be outgrown
__host__ __device__ constexpr int stages_for(int kb, bool eight) { return kb == 2 ? (eight ? 3 : 5) : 8; }
constexpr int kRawStages = 4;                 // tiles of codes on their way (EIGHT)
__host__ __device__ constexpr int raw_bytes(int kb) { return kTile * kb * 64; }
struct Shared {
    uint64_t q_full, q_empty;
    uint64_t full[kMaxStages], empty[kMaxStages], look[kMaxStages], clean[kMaxStages];
    uint64_t s_full[2], p_part[2], p_full[2], pv_done[2], o_free[2];
    uint32_t tmem_base;
    int abort;
    int poison[kMaskSlots];                        // item whose values held an infinity or NaN in a tile that was looked through
    uint4 present[kMaskSlots];                     // of the tiles' 128 rows: those with a page
    uint64_t raw_full[kRawStages], raw_empty[kRawStages];          // EIGHT
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
template <bool DRAFT>
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
    im.base = attn_before<DRAFT>(a, im.sq, im.unit) + 1;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int first = im.pos0 + x * t.ppt;
        im.rows[x] = min(max(im.sq.m - first, 0), t.ppt);
        const int most = im.rows[x] > 0 ? (DRAFT ? im.sq.n : min(im.base + first + im.rows[x] - 1, im.sq.n)) : 0;
        im.tiles[x] = (max(most, 0) + kTile - 1) / kTile;
    }
    im.looked = max(DRAFT ? im.base - 1 : im.base + im.pos0, 0) / kTile;       // every row sees all of the tiles in front of this one
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
template <bool DRAFT>
__device__ __forceinline__ long long item_cost(const TcAttnArgs &t, long long k)
{
    Item im;
    return k < t.items && get_item<DRAFT>(t, k, im) ? im.n_tiles + kItemCost : 0;
}
// By a whole warp, 32 items at a time: the length of the line; and, at a place on it, the item there and where that begins.
template <bool DRAFT>
__device__ __forceinline__ long long line_length(const TcAttnArgs &t, int lane)
{
    long long sum = 0;
    for (int x = lane; x < t.items; x += 32) sum += item_cost<DRAFT>(t, x);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}
template <bool DRAFT, typename F>
__device__ __forceinline__ void walk_line(const TcAttnArgs &t, int lane, F visit)      // visit(item, where it begins, where it ends): enough?
{
    long long before = 0;
    for (int x0 = 0; x0 < t.items; x0 += 32) {
        const long long c = item_cost<DRAFT>(t, x0 + lane);
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
template <bool DRAFT>
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
            if (k < t.items && get_item<DRAFT>(t, k, im)) return true;
        }
        return false;
    }
    __device__ __forceinline__ bool next_share(const TcAttnArgs &t, Item &im)
    {
        if (total < 0) {
            const int lane = threadIdx.x & 31;
            total = line_length<DRAFT>(t, lane);
            const long long lo = total * blockIdx.x / kWorkBlocks;
            long long k = t.items, from = 0;
            walk_line<DRAFT>(t, lane, [&](int item, long long start, long long end) {
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
            if (!get_item<DRAFT>(t, k0, im)) {
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
//
// 32 bits of a draft's mask from token `at` on (which may be negative: those are zeros)
__device__ __forceinline__ uint32_t mask_window(const unsigned *mask, int words, int at)
{
    const int w = at >> 5;
    const uint32_t lo = w >= 0 && w < words ? __ldg(mask + w) : 0u, hi = w + 1 >= 0 && w + 1 < words ? __ldg(mask + w + 1) : 0u;
    return __funnelshift_r(lo, hi, at & 31);
}
template <int KB, bool WHOLE, bool EIGHT, bool DRAFT>
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
    Walk<DRAFT> walk;
    Item im;
    while (walk.next(t, im)) {
        const int pos = im.pos0 + x * t.ppt + place, tiles = min(x ? im.tiles[1] : im.tiles[0], im.end);
        const bool mine = of_tile && place < (x ? im.rows[1] : im.rows[0]);
        const int limit = mine ? (DRAFT ? im.base - 1 : min(im.base + pos, im.sq.n)) : 0;
        const unsigned *const mask = DRAFT && mine ? attn_mask(a, im.sq, im.b, pos) : nullptr;
        const int plain = DRAFT ? max(im.base - 1, 0) / kTile : (im.base + im.pos0 + x * t.ppt) / kTile;         // tiles that every row of this query tile sees all of
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
                if constexpr (DRAFT) {
                    const int there = im.sq.n - u * kTile;
                    auto bits = [&](int y) {
                        return first_bits(in_tile - y) | (mask ? mask_window(mask, a.mask_words, y - in_tile) & first_bits(there - y) : 0u);
                    };
                    seen.bits.x &= bits(0);
                    seen.bits.y &= bits(32);
                    seen.bits.z &= bits(64);
                    seen.bits.w &= bits(96);
                } else {
                    seen.bits.x &= first_bits(in_tile);
                    seen.bits.y &= first_bits(in_tile - 32);
                    seen.bits.z &= first_bits(in_tile - 64);
                    seen.bits.w &= first_bits(in_tile - 96);
                }
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
                const int upto = DRAFT ? (mine ? im.sq.n : 0) : limit;
                for (int j = max(im.looked, im.begin) * kTile; j < min(upto, im.end * kTile); ++j) {
                    if (DRAFT && j >= limit && !(mask_window(mask, a.mask_words, j - limit) & 1u)) continue;
                    const long long at = attn_row(a, im.b, im.h, im.sq.q_off, j);
                    if (at < 0) continue;
                    if constexpr (EIGHT) {
                        const unsigned char *v = static_cast<const unsigned char *>(a.v) + at + y * 32;
                        const float by = scale_value(a.v_scales[attn_scale(a, im.b, im.h, j)]);
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (!WHOLE && y * 32 + e >= D) break;
                            const float ve = codes_to_float(v[e], a.kind).x * by;
                            if (!(fabsf(ve) < INFINITY)) o[e] += ve;
                        }
                    } else {
                        const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(a.v) + at + y * 32;
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (!WHOLE && y * 32 + e >= D) break;
                            const float ve = __bfloat162float(v[e]);
                            if (!(fabsf(ve) < INFINITY)) o[e] += ve;
                        }
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
template <int KB, bool WHOLE, bool EIGHT, bool DRAFT>
__device__ __forceinline__ void mma_warp(const TcAttnArgs &t, Shared &sh, uint8_t *q_img, uint8_t *ring, uint32_t tmem)
{
    constexpr int NS = stages_for(KB, EIGHT), kStage = KB * kRegion;
    const int lane = threadIdx.x & 31;
    const uint32_t leader = elect_one();
    volatile int *const abort_flag = &sh.abort;
    const uint64_t q_desc0 = umma_desc_sw128(smem_u32(q_img)), k_desc0 = umma_desc_sw128(smem_u32(ring)), v_desc0 = value_desc(smem_u32(ring));
    const int steps = WHOLE ? KB * 4 : (t.a.d + 15) / 16;        // of 16 columns
    constexpr uint32_t s_idesc = umma_idesc_bf16(kTile, kTile);
    const uint32_t o_idesc = umma_idesc_bf16(kTile, steps * 16) | kBTransposed;
    uint32_t entry = 0, clean_phase = 0;               // ring entries so far; parity per stage of the looked-through tiles
    uint32_t turn[2] = {0, 0}, outs[2] = {0, 0};       // tiles and items of each query tile so far
    Walk<DRAFT> walk;
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
// `ring`: of the tiles as the products take them, or of codes (EIGHT)
template <int KB, bool EIGHT, bool DRAFT>
__device__ __forceinline__ uint32_t load_warp(const TcAttnArgs &t, Shared &sh, const CUtensorMap *k_map, const CUtensorMap *v_map, uint8_t *ring)
{
    constexpr int NS = EIGHT ? kRawStages : stages_for(KB, false), kStage = EIGHT ? raw_bytes(KB) : KB * kRegion;
    uint64_t *const full = EIGHT ? sh.raw_full : sh.full, *const empty = EIGHT ? sh.raw_empty : sh.empty;
    const AttnArgs &a = t.a;
    const int lane = threadIdx.x & 31;
    volatile int *const abort_flag = &sh.abort;
    uint32_t entry = 0;
    Walk<DRAFT> walk;
    Item im;
    const int boxes = kTile / t.box_rows;             // of a tile
    const uint32_t leader = elect_one();
    // One box into a stage.  One lane issues, and every operand is the same in all lanes: the instruction takes them from
    // uniform registers, so that an address which varies from lane to lane is another lane's.
    auto put_box = [&](const CUtensorMap *map, int stage, int box, int tok, int h, int third) {
        const int c1 = t.k_slot[0] == 1 ? tok : (t.k_slot[1] == 1 ? h : third);
        const int c2 = t.k_slot[0] == 2 ? tok : (t.k_slot[1] == 2 ? h : third);
        const int c3 = t.k_slot[0] == 3 ? tok : (t.k_slot[1] == 3 ? h : third);
        uint8_t *to = ring + stage * kStage + box * t.box_rows * (EIGHT ? KB * 64 : 128);
#pragma unroll
        for (int kb = 0; kb < (EIGHT ? 1 : KB); ++kb) tma_load_4d_if(leader, to + kb * kRegion, map, &full[stage], kb * 64, c1, c2, c3);
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
                if (entry >= NS && !warp_wait(&empty[stage], (entry / NS - 1) & 1, abort_flag)) return entry;
                mbar_arrive_expect_tx_if(leader, &full[stage], kStage);
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
template <int KB, bool EIGHT, bool DRAFT>
__device__ __forceinline__ void helper_warp(const TcAttnArgs &t, Shared &sh, uint8_t *q_img, uint8_t *ring, int which)
{
    constexpr int NS = stages_for(KB, EIGHT), kStage = KB * kRegion;
    const int lane = threadIdx.x & 31;
    volatile int *const abort_flag = &sh.abort;
    uint32_t entry = 0, look_phase = 0;
    Walk<DRAFT> walk;
    Item im;
    if (t.by_work && blockIdx.x == 0 && which == 1)
        walk_line<DRAFT>(t, lane, [&](int item, long long start, long long end) {
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

// ---- codes to bf16 ------------------------------------------------------------------------------------
// A warp makes 32 rows of a tile, a lane a row, 16 codes at a time: so its scale stays in a register.  The lanes take their row's codes in different orders
// (the i-th of a lane is i ^ turn), in which any eight neighbours read from, and write to, eight different sixteenths of the banks.  A small loop with
// the next codes on their way: the instructions of a whole row in one piece, beside those of the softmax, do not fit the cache in front of the issue (4
// sequences of 10-16 K rows, up to 512 new tokens of 32 heads, d = 128: 738 us against 484).
// PLAIN: every row is there, and its scale an f16.
template <int KB, int KIND, bool PLAIN>
__device__ __forceinline__ void convert_tile(const uint8_t *raw, uint8_t *tile, int row, float s)
{
    const int k = row >> 1 & 3, turn = KB == 2 ? row & 7 : (k << 1 ^ k) & 2 | k >> 1;
    const uint32_t from = smem_u32(raw) + row * (KB * 64) + turn * 16;
    const uint32_t to = smem_u32(tile) + row * 128 + ((turn * 32 & 127) ^ (row & 7) << 4), near = to + (turn >> 2) * kRegion, far = to + (turn >> 2 ^ 1) * kRegion;
    const F16Scale<KIND> scale(PLAIN ? s : 1.f);
    auto fetch = [&](int i) {
        uint4 w;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(from ^ i * 16));
        return w;
    };
    auto put = [](uint32_t at, uint2 x, uint2 y) {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(y.x), "r"(y.y) : "memory");
    };
    auto make = [&](uint4 w, uint32_t at) {
        if (PLAIN) {
            put(at, scale.four(w.x), scale.four(w.y));
            put(at ^ 16u, scale.four(w.z), scale.four(w.w));
        } else {
            if (s < 0.f) w = make_uint4(0, 0, 0, 0);             // (whatever stands there)
            put(at, codes_to_bf16<KIND>(w.x, s), codes_to_bf16<KIND>(w.y, s));
            put(at ^ 16u, codes_to_bf16<KIND>(w.z, s), codes_to_bf16<KIND>(w.w, s));
        }
    };
    constexpr int kPairs = KB * 2;
    uint4 a = fetch(0), b = fetch(1);
#pragma unroll 1
    for (int i = 0; i < kPairs; ++i) {
        const uint4 x = a, y = b;
        const uint32_t at = (i < 2 ? near : far) ^ (i & 1) * 64;
        if (i + 1 < kPairs) {
            a = fetch(2 * i + 2);
            b = fetch(2 * i + 3);
        }
        make(x, at);
        make(y, at ^ 32u);
    }
}
template <int KB, bool DRAFT>
__device__ __forceinline__ void convert_warp(const TcAttnArgs &t, Shared &sh, const uint8_t *raw, uint8_t *ring, int which)
{
    constexpr int NS = stages_for(KB, true), kStage = KB * kRegion;
    const AttnArgs &a = t.a;
    const int lane = threadIdx.x & 31;
    volatile int *const abort_flag = &sh.abort;
    uint32_t entry = 0;
    Walk<DRAFT> walk;
    Item im;
    bool ok = true;
    while (ok && walk.next(t, im)) {
        // this lane's row of a tile: its page, then its scales; -1: no such row
        const int *const table = a.table + (long long)im.b * a.max_pages;
        auto page_of = [&](int u) {
            const int j = u * kTile + which * 32 + lane;
            return u < im.end && j < im.sq.n ? __ldg(table + j / a.page_size) : -1;
        };
        int byte[2];
        auto look_up = [&](int u, int page) {
            const int j = u * kTile + which * 32 + lane;
            byte[0] = byte[1] = -1;
            if ((unsigned)page >= (unsigned)a.num_pages) return;
            const long long at = ((long long)page * a.hkv + im.h) * a.page_size + j % a.page_size;
            byte[0] = a.k_scales[at];
            byte[1] = a.v_scales[at];
        };
        look_up(im.begin, page_of(im.begin));
        int page = page_of(im.begin + 1);
        for (int u = im.begin; ok && u < im.end; ++u) {
            const int mine[2] = {byte[0], byte[1]};
            look_up(u + 1, page);
            page = page_of(u + 2);
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv, ++entry) {
                const int from = entry % kRawStages, to = entry % NS, code = kv ? mine[1] : mine[0];
                const float s = code < 0 ? -1.f : scale_value(code);
                const bool plain = __all_sync(0xffffffffu, code >= kLeastF16 && code <= kMostF16);
                ok = warp_wait(&sh.raw_full[from], (entry / kRawStages) & 1, abort_flag) &&
                     (entry < NS || warp_wait(&sh.empty[to], (entry / NS - 1) & 1, abort_flag));
                if (!ok) break;
                const uint8_t *const codes = raw + from * raw_bytes(KB);
                uint8_t *const tile = ring + to * kStage;
                if (a.kind == kE4m3) plain ? convert_tile<KB, kE4m3, true>(codes, tile, which * 32 + lane, s) : convert_tile<KB, kE4m3, false>(codes, tile, which * 32 + lane, s);
                else plain ? convert_tile<KB, kI8, true>(codes, tile, which * 32 + lane, s) : convert_tile<KB, kI8, false>(codes, tile, which * 32 + lane, s);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.full[to]);
                    mbar_arrive(&sh.raw_empty[from]);
                }
            }
        }
    }
    // (the last products have released their stages before the block ends)
    if (which == 0)
        for (uint32_t e = entry > NS ? entry - NS : 0; ok && e < entry; ++e) ok = warp_wait(&sh.empty[e % NS], (e / NS) & 1, abort_flag);
}

template <int KB, bool WHOLE, bool EIGHT, bool DRAFT>
__global__ void __launch_bounds__(threads_for(EIGHT), 1)
attn_tc_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ TcAttnArgs t)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ Shared sh;
    constexpr int NS = stages_for(KB, EIGHT), kStage = KB * kRegion;
    uint8_t *q_img = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023u) & ~uintptr_t(1023u));
    uint8_t *ring = q_img + 2 * kStage, *raw = ring + NS * kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();
    if (threadIdx.x == 0) {
        mbar_init(&sh.q_full, 2);
        mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < NS; ++i) {
            mbar_init(&sh.full[i], EIGHT ? 4 : 1);
            mbar_init(&sh.empty[i], 1);
            mbar_init(&sh.look[i], 1);
            mbar_init(&sh.clean[i], 2);
        }
        if (EIGHT)
            for (int i = 0; i < kRawStages; ++i) {
                mbar_init(&sh.raw_full[i], 1);
                mbar_init(&sh.raw_empty[i], 4);
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
    if constexpr (EIGHT) {
        if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    }
    if (warp < 8) {
        softmax_warps<KB, WHOLE, EIGHT, DRAFT>(t, sh, warp >> 2, tmem);
    } else if (warp == 8) {
        mma_warp<KB, WHOLE, EIGHT, DRAFT>(t, sh, q_img, ring, tmem);
    } else if (warp == 9) {
        if (lane == 0) {
            tma_prefetch_desc(&k_map);
            tma_prefetch_desc(&v_map);
        }
        const uint32_t issued = load_warp<KB, EIGHT, DRAFT>(t, sh, &k_map, &v_map, EIGHT ? raw : ring);
        // nothing of this block may be in flight when it ends: the last MMAs (EIGHT: conversions) must have released their stages; after a
        // failed wait, the loads already issued must still land
        constexpr uint32_t LS = EIGHT ? kRawStages : NS;
        uint64_t *const full = EIGHT ? sh.raw_full : sh.full, *const empty = EIGHT ? sh.raw_empty : sh.empty;
        for (uint32_t e = issued > LS ? issued - LS : 0; e < issued; ++e) {
            const int st = e % LS;
            if (!warp_wait(&empty[st], (e / LS) & 1, &sh.abort)) {
                volatile int never = 0;
                warp_wait(&full[st], (e / LS) & 1, &never);
            }
        }
        if (lane == 0 && *static_cast<volatile int *>(&sh.abort) && t.a.status) atomicOr(t.a.status, kStatusWaitExpired);
    } else if (!EIGHT || warp < 12) {
        helper_warp<KB, EIGHT, DRAFT>(t, sh, q_img, ring, warp - 10);
    } else if constexpr (EIGHT) {
        convert_warp<KB, DRAFT>(t, sh, raw, ring, warp - 12);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 8) tmem_dealloc(sh.tmem_base, kTmemCols);
}

template <int KB, bool WHOLE, bool EIGHT, bool DRAFT>
cudaError_t launch_tc_kernel(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream)
{
    constexpr size_t smem = 1024 + (size_t)(2 + stages_for(KB, EIGHT)) * KB * kRegion + (EIGHT ? kRawStages * raw_bytes(KB) : 0);
    static_assert(smem + sizeof(Shared) <= 232448, "shared memory of a block");
    static SmemAsked asked;
    int dev = 0, sms = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (err == cudaSuccess) err = allow_smem(attn_tc_kernel<KB, WHOLE, EIGHT, DRAFT>, smem, asked);
    const long long grid = t.by_work ? kWorkBlocks : (t.items < sms ? t.items : sms);
    if (err == cudaSuccess) err = launch_pdl(attn_tc_kernel<KB, WHOLE, EIGHT, DRAFT>, dim3((unsigned)grid), threads_for(EIGHT), smem, stream, 1, k_map, v_map, t);
    return err;
}

}  // namespace

// the kernel's forms, by what the call needs
cudaError_t launch_tc_plain(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream);
cudaError_t launch_tc_draft(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream);
cudaError_t launch_tc_eight(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream);
cudaError_t launch_tc_eight_draft(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream);
template <bool EIGHT, bool DRAFT>
inline cudaError_t launch_tc_form(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream)
{
    if (t.a.d > 64) return t.a.d == 128 ? launch_tc_kernel<2, true, EIGHT, DRAFT>(t, k_map, v_map, stream) : launch_tc_kernel<2, false, EIGHT, DRAFT>(t, k_map, v_map, stream);
    return t.a.d == 64 ? launch_tc_kernel<1, true, EIGHT, DRAFT>(t, k_map, v_map, stream) : launch_tc_kernel<1, false, EIGHT, DRAFT>(t, k_map, v_map, stream);
}

}  // namespace wkv
