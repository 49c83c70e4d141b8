// Attention on the tensor cores: the form for whole prompts and chunks over a cache of plain rows, the kernel that joins shared items, and the choice of form.
#include "attn_tc_kernel.cuh"

namespace wkv {
namespace {

// Joins the pieces of the items that lie across blocks: block (item, y) takes 8 * RPW of its 256 rows, RPW to a warp.  With few
// items each is in many pieces, whose reading is trips to memory: a row per warp then (8 items of 32 rows over 16,384 keys: 44
// us with the kernel in front, 66 with 32 rows per block).  With many there are two pieces or so, and fewer blocks look for them
// more seldom (160 items: 101 us with 8 rows, 96 with 32).
constexpr int kFewItems = 128;
template <int RPW, bool DRAFT>          // rows of a warp, all in flight together
__global__ void __launch_bounds__(256) attn_tc_join_kernel(const __grid_constant__ TcAttnArgs t)
{
    pdl_trigger();
    pdl_wait();
    __shared__ int slots[kWorkBlocks];
    __shared__ int n_slots;
    const AttnArgs &a = t.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Item im;
    if (!get_item<DRAFT>(t, blockIdx.x, im) || im.n_tiles == 0) return;
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

static int launch_forms(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream)
{
    const bool eight = t.a.kind != kPlain;
    cudaError_t err = eight ? (t.a.masks ? launch_tc_eight_draft : launch_tc_eight)(t, k_map, v_map, stream)
                            : (t.a.masks ? launch_tc_draft : launch_tc_plain)(t, k_map, v_map, stream);
    if (err == cudaSuccess) count_launches(1);
    if (err == cudaSuccess && t.by_work) {
        const auto join = [&](auto kernel, int rows) { return launch_pdl(kernel, dim3((unsigned)t.items, 2 * kTile / rows), 256, 0, stream, 1, t); };
        if (t.a.masks) err = t.items <= kFewItems ? join(attn_tc_join_kernel<1, true>, 8) : join(attn_tc_join_kernel<4, true>, 32);
        else err = t.items <= kFewItems ? join(attn_tc_join_kernel<1, false>, 8) : join(attn_tc_join_kernel<4, false>, 32);
        if (err == cudaSuccess) count_launches(1);
    }
    return check_cuda(err, "tensor-core attention kernel");
}
cudaError_t launch_tc_plain(const TcAttnArgs &t, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream)
{
    return launch_tc_form<false, false>(t, k_map, v_map, stream);
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
    const int eb = a.kind != kPlain ? 1 : 2, codes = a.kind != kPlain ? (a.d > 64 ? 128 : 64) : 0;
    const RowDim k_dims[3] = {{a.table ? (unsigned long long)a.page_size : tokens, (unsigned long long)a.kt * eb, (unsigned)t.box_rows},
                              {(unsigned long long)a.hkv, (unsigned long long)a.kh * eb, 1},
                              {a.table ? (unsigned long long)a.num_pages : batch, (unsigned long long)a.kb * eb, 1}};
    if (!make_row_tensor_map(a.k, a.d, k_dims, &k_map, t.k_slot, codes) || !make_row_tensor_map(a.v, a.d, k_dims, &v_map, t.k_slot, codes))
        return WKV_ERR_UNSUPPORTED;
    return launch_forms(t, k_map, v_map, stream);
}

}  // namespace wkv
