// Rotary positions of queries and keys, of a prompt in its tensors or of new tokens on their way into the paged cache.
//
// A block takes a few tokens: cosines and sines of a token's rot/2 pairs are computed once (sincospif of the angle in half
// turns) and serve all of its heads; then every thread turns one 16-byte vector of first partners with the vector of
// second partners (HALF order) or one vector of whole pairs (INTERLEAVED).  The angle is position * turns mod 2^64 in
// integers: exact at any position, where the product in fp32 would be off by 2^-24 of itself, 0.04 radians at position 10^6.
// Each thread reads what it writes, so an output may be its input.  Bound by memory.
#include "attn.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 2048;          // rot/2 at most, per block: cosines and sines in shared memory (16 KB)

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float &y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16 &y, float x) { y = __float2bfloat16_rn(x); }

struct Token {
    int b, i, m;          // sequence, place in its chunk, tokens of the sequence
    long long off;        // first row of the sequence in packed tensors
};
// sequence of packed row t: the last b with cu[b] <= t
__device__ __forceinline__ bool find_token(const RopeArgs &a, long long t, Token &tok)
{
    if (!a.cu_q) {
        tok.b = (int)(t / a.max_q);
        tok.i = (int)(t - (long long)tok.b * a.max_q);
        tok.m = a.max_q;
        tok.off = 0;
        return true;
    }
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.cu_q[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int first = a.cu_q[lo], last = a.cu_q[lo + 1];
    tok.b = lo;
    tok.i = (int)(t - first);
    tok.m = min(last - first, a.max_q);
    tok.off = first;
    // (a device copy that disagrees with the host copy: not beyond what the host copy allowed for)
    return first >= 0 && t < last && tok.i < tok.m;
}

// VEC elements of 16 bytes (fast path), or single elements
template <typename T, int VEC>
__device__ __forceinline__ void load(const T *p, float (&x)[VEC])
{
    if (VEC == 1) {
        x[0] = to_float(p[0]);
    } else {
        const int4 raw = *reinterpret_cast<const int4 *>(p);
        const T *e = reinterpret_cast<const T *>(&raw);
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] = to_float(e[i]);
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store(T *p, const float (&x)[VEC])
{
    if (VEC == 1) {
        from_float(p[0], x[0]);
    } else {
        int4 raw;
        T *e = reinterpret_cast<T *>(&raw);
#pragma unroll
        for (int i = 0; i < VEC; ++i) from_float(e[i], x[i]);
        *reinterpret_cast<int4 *>(p) = raw;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void copy(const T *p, T *q)
{
    if (VEC == 1) q[0] = p[0];
    else *reinterpret_cast<int4 *>(q) = *reinterpret_cast<const int4 *>(p);
}

// VEC = 16 bytes where vectors do not straddle the two halves or the end of the turned part; else single elements
// (single pairs in INTERLEAVED order).
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeArgs a, int tokens_per_block, long long tokens)
{
    __shared__ float2 turn[kMaxPairs];
    __shared__ Token token[16];
    __shared__ int there[16];
    pdl_trigger();
    pdl_wait();
    const int half = a.turns ? a.rot / 2 : 0, rot = 2 * half;
    const long long t0 = (long long)blockIdx.x * tokens_per_block;
    const int n = (int)min((long long)tokens_per_block, tokens - t0);
    if (a.lengths_out)
        // the units' new lengths, by the blocks in turn
        for (long long u = (long long)blockIdx.x * kThreads + threadIdx.x; u < (long long)a.batch * a.hkv; u += (long long)gridDim.x * kThreads) {
            const int b = (int)(u / a.hkv);
            int m = a.max_q;
            if (a.cu_q) m = min(min(max(a.cu_q[b + 1] - a.cu_q[b], 0), a.max_q), a.total_q);
            a.lengths_out[u] = (int)min((long long)max(a.lengths[u], 0) + m, (long long)a.cap);
        }
    if ((int)threadIdx.x < n) {
        Token tok;
        there[threadIdx.x] = find_token(a, t0 + threadIdx.x, tok);
        token[threadIdx.x] = tok;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < n * half; x += kThreads) {
        const int w = x / half, p = x - w * half;
        const long long pos = a.positions ? a.positions[t0 + w] : token[w].i;
        const unsigned long long angle = (unsigned long long)pos * a.turns[p];
        float sine, cosine;
        sincospif((float)(int)(angle >> 32) * (1.f / 2147483648.f), &sine, &cosine);      // angle in half turns, -1 .. 1
        turn[x] = make_float2(cosine * a.scale, sine * a.scale);
    }
    __syncthreads();
    // pieces of a row: HALF: `half/VEC` pairs of vectors; INTERLEAVED: rot/VEC vectors of pairs (rot/2 pairs if VEC = 1); the rest copied
    const bool inter = a.order == WKV_ROPE_INTERLEAVED;
    const int turned = inter && VEC > 1 ? rot / VEC : half / VEC, pieces = turned + (a.d - rot) / VEC;
    const int v_pieces = a.v ? a.d / VEC : 0;
    const int hq = a.q ? a.hq : 0, hk = a.k ? a.hkv : 0;
    const int per_token = (hq + hk) * pieces + hk * v_pieces;
    for (int x = threadIdx.x; x < n * per_token; x += kThreads) {
        const int w = x / per_token;
        int y = x - w * per_token;
        if (!there[w]) continue;
        const Token tok = token[w];
        int kind = 0, head, piece;
        if (y < hq * pieces) {
            head = y / pieces;
            piece = y - head * pieces;
        } else if ((y -= hq * pieces) < hk * pieces) {
            kind = 1;
            head = y / pieces;
            piece = y - head * pieces;
        } else {
            y -= hk * pieces;
            kind = 2;
            head = y / v_pieces;
            piece = y - head * v_pieces;
        }
        const T *src;
        T *dst;
        if (kind == 0) {
            const long long at = (tok.off + tok.i) * a.qt + tok.b * a.qb + head * a.qh;
            src = static_cast<const T *>(a.q) + at;
            dst = static_cast<T *>(a.q_out) + at;
        } else {
            const long long at = (tok.off + tok.i) * a.kt + tok.b * a.kb + head * a.kh;
            src = static_cast<const T *>(kind == 1 ? a.k : a.v) + at;
            if (a.table) {
                const long long unit = (long long)tok.b * a.hkv + head, row = (long long)max(a.lengths[unit], 0) + tok.i;
                if (row >= a.cap) continue;
                const int pg = (int)row / a.page_size, page = __ldg(a.table + (long long)tok.b * a.max_pages + pg);
                if (kind == 1 && piece == 0) {
                    if (a.row_positions) a.row_positions[unit * a.cap + row] = a.positions[t0 + w];
                    if (a.row_weights) a.row_weights[unit * a.cap + row] = 0.f;
                }
                if ((unsigned)page >= (unsigned)a.num_pages) continue;
                dst = static_cast<T *>(kind == 1 ? a.k_out : a.v_out) + page * a.page_stride + head * a.head_stride +
                      (row - (long long)pg * a.page_size) * a.row_stride;
            } else {
                dst = static_cast<T *>(a.k_out) + at;
            }
        }
        if (kind == 2) {
            copy<T, VEC>(src + piece * VEC, dst + piece * VEC);
            continue;
        }
        if (piece >= turned) {
            const int c = rot + (piece - turned) * VEC;
            if (src != dst) copy<T, VEC>(src + c, dst + c);
            continue;
        }
        const float2 *tr = turn + w * half;
        if (!inter || VEC == 1) {
            const int j = inter ? 2 * piece : piece * VEC, k = inter ? j + 1 : j + half;
            float p[VEC], q[VEC], u[VEC], v[VEC];
            load<T, VEC>(src + j, p);
            load<T, VEC>(src + k, q);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float2 cs = tr[piece * VEC + e];
                u[e] = p[e] * cs.x - q[e] * cs.y;
                v[e] = q[e] * cs.x + p[e] * cs.y;
            }
            store<T, VEC>(dst + j, u);
            store<T, VEC>(dst + k, v);
        } else {
            constexpr int kPairs = VEC > 1 ? VEC / 2 : 1;
            float p[VEC], u[VEC];
            load<T, VEC>(src + piece * VEC, p);
#pragma unroll
            for (int e = 0; e < kPairs; ++e) {
                const float2 cs = tr[piece * kPairs + e];
                u[2 * e] = p[2 * e] * cs.x - p[(2 * e + 1) % VEC] * cs.y;
                u[(2 * e + 1) % VEC] = p[(2 * e + 1) % VEC] * cs.x + p[2 * e] * cs.y;
            }
            store<T, VEC>(dst + piece * VEC, u);
        }
    }
}

template <typename T>
int launch(const RopeArgs &a, cudaStream_t stream)
{
    constexpr int kVec = 16 / sizeof(T);
    const int half = a.turns ? a.rot / 2 : 0;
    const long long tokens = a.cu_q ? a.total_q : (long long)a.batch * a.max_q;
    // vectors must end where the turned part does, and in HALF order where its first half does
    const bool vectors = a.order == WKV_ROPE_HALF ? half % kVec == 0 : (2 * half) % kVec == 0;
    // Tokens of a block: several where there are plenty, so that the threads that have no pair to compute angles for wait less
    long long per = tokens / (148 * 8);
    per = per < 1 ? 1 : (per > 4 ? 4 : per);
    if (half > 0 && per * half > kMaxPairs) per = kMaxPairs / half;
    const long long blocks = (tokens + per - 1) / per;
    if (blocks > 0x7fffffffLL) {
        set_error_detail("rotary positions: %lld tokens", tokens);
        return WKV_ERR_LIMIT;
    }
    const dim3 grid((unsigned)(blocks > 0 ? blocks : 1));
    const cudaError_t err = vectors ? launch_pdl(rope_kernel<T, kVec>, grid, kThreads, 0, stream, 1, a, (int)per, tokens)
                                    : launch_pdl(rope_kernel<T, 1>, grid, kThreads, 0, stream, 1, a, (int)per, tokens);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "rotary positions kernel");
}

}  // namespace

int launch_rope(const RopeArgs &a, cudaStream_t stream)
{
    return a.elem_bytes == 4 ? launch<float>(a, stream) : launch<__nv_bfloat16>(a, stream);
}

}  // namespace wkv
