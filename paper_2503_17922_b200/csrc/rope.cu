// Rotary positions of queries and keys, of a prompt in its tensors or of new tokens on their way into the paged cache.
//
// A block takes a few tokens: cosines and sines of a token's rot/2 pairs are computed once (sincospif of the angle in half
// turns) and serve all of its heads; then every thread turns vectors of first partners with the vectors of second
// partners (HALF order) or vectors of whole pairs (INTERLEAVED).  The angle is position * turns mod 2^64 in
// integers: exact at any position, where the product in fp32 would be off by 2^-24 of itself, 0.04 radians at position 10^6.
// Each thread reads what it writes, so an output may be its input.
//
// Bound by memory: 32,768 tokens of 40 rows of 128 in bf16, 64 of each turned, take 116 us, 5.8 TB/s read and written, and 120 us
// with all 128 turned in HALF order; 8,192 tokens 35 us, with 62 turned 36, and in HALF order, element by element, 61.  Two rows
// in flight per thread leave room for seven or eight blocks per SM; four rows (half as many blocks) took 12 % more, one 7 %; four
// tokens per block: eight took 3 % more.  When each thread worked out its own addresses, piece by piece, the divisions and strides took
// as long as the memory (186 us).
#include "attn.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = WKV_MAX_ROT_DIM / 2;          // per block: cosines and sines in shared memory (16 KB)

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

// VEC elements as they stand in memory: 2 to 16 bytes
template <int BYTES> struct Bits;
template <> struct Bits<2> { typedef unsigned short type; };
template <> struct Bits<4> { typedef unsigned type; };
template <> struct Bits<8> { typedef uint2 type; };
template <> struct Bits<16> { typedef uint4 type; };
template <typename T, int VEC>
struct Vec {
    typedef typename Bits<VEC * sizeof(T)>::type Raw;
    Raw raw;
    __device__ __forceinline__ void load(const T *p) { raw = *reinterpret_cast<const Raw *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<Raw *>(p) = raw; }
    __device__ __forceinline__ float get(int i) const { return to_float(reinterpret_cast<const T *>(&raw)[i]); }
    __device__ __forceinline__ void set(int i, float x) { from_float(reinterpret_cast<T *>(&raw)[i], x); }
};

// A row on its way: where it is read and written (null: nowhere), and its token's cosines and sines (-1: copied as it is)
struct Row {
    const void *src;
    void *dst;
};

// The rows of a block's tokens are listed in shared memory, one per thread and kThreads at a time: the divisions, the strides
// and the look-up of the page are done once for a row, not once for each of its pieces.  A thread keeps to one piece of the rows and
// takes a few at a time, loads first.  Pieces of a row:
//   PAIRS (INTERLEAVED order)  16-byte vectors, whose pairs from rot on stay as they are
//   else (HALF order)          half / VEC pairs of vectors, VEC the largest of which a half is a multiple; from rot on single vectors of
//                              VEC as far as the next 16 bytes, then 16-byte vectors
template <typename T, int VEC, bool PAIRS, bool TAIL = false>      // TAIL: the turned part ends inside a vector of pairs
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeArgs a, int tokens_per_block, long long tokens)
{
    constexpr int kWide = 16 / sizeof(T), kBatch = VEC > 1 ? 2 : 4;       // rows in flight
    __shared__ __align__(16) float2 turn[kMaxPairs];
    __shared__ Row list[kThreads];
    __shared__ int list_token[kThreads];
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
    const int turned = PAIRS ? (rot + VEC - 1) / VEC : half / VEC, wide_from = (rot + kWide - 1) / kWide * kWide;
    const int single = PAIRS ? 0 : (wide_from - rot) / VEC;                       // vectors of VEC behind the turned part
    const int pieces = PAIRS ? a.d / VEC : turned + single + (a.d - wide_from) / kWide;
    const int hq = a.q ? a.hq : 0, hk = a.k ? a.hkv : 0, hv = a.v ? a.hkv : 0, rows = hq + hk + hv;
    const int width = min(pieces, kThreads), step = kThreads / width, slot = threadIdx.x / width;
    for (int y0 = 0; y0 < n * rows; y0 += kThreads) {
        const int listed = min(n * rows - y0, kThreads);
        if (y0 > 0) __syncthreads();
        if ((int)threadIdx.x < listed) {
            const int y = y0 + threadIdx.x, w = y / rows, row = y - w * rows;
            const Token tok = token[w];
            Row r = {nullptr, nullptr};
            int kind = w;
            if (there[w]) {
                if (row < hq) {
                    const long long off = (tok.off + tok.i) * a.qt + tok.b * a.qb + row * a.qh;
                    r.src = static_cast<const T *>(a.q) + off;
                    r.dst = static_cast<T *>(a.q_out) + off;
                } else {
                    const bool value = row >= hq + hk;
                    const int head = row - hq - (value ? hk : 0);
                    const long long off = (tok.off + tok.i) * a.kt + tok.b * a.kb + head * a.kh;
                    r.src = static_cast<const T *>(value ? a.v : a.k) + off;
                    if (value) kind = -1;
                    if (a.table) {
                        const long long unit = (long long)tok.b * a.hkv + head, at = (long long)max(a.lengths[unit], 0) + tok.i;
                        if (at < a.cap) {
                            const int pg = (int)at / a.page_size, page = __ldg(a.table + (long long)tok.b * a.max_pages + pg);
                            if (!value) {
                                if (a.row_positions) a.row_positions[unit * a.cap + at] = a.positions[t0 + w];
                                if (a.row_weights) a.row_weights[unit * a.cap + at] = 0.f;
                            }
                            if ((unsigned)page < (unsigned)a.num_pages)
                                r.dst = static_cast<T *>(value ? a.v_out : a.k_out) + page * a.page_stride + head * a.head_stride +
                                        (at - (long long)pg * a.page_size) * a.row_stride;
                        }
                    } else {
                        r.dst = static_cast<T *>(a.k_out) + off;
                    }
                }
            }
            list[threadIdx.x] = r;
            list_token[threadIdx.x] = kind;
        }
        __syncthreads();
        if (slot < step)
            for (int piece = threadIdx.x - slot * width; piece < pieces; piece += width) {
                const bool turns = piece < turned;
                const bool wide = !PAIRS && piece >= turned + single;
                const int j = PAIRS || turns ? piece * VEC : (wide ? wide_from + (piece - turned - single) * kWide : rot + (piece - turned) * VEC);
                const int k = j + half;                                          // the second vector of a pair
                const float2 *tr = turn + (PAIRS ? piece * (VEC / 2) : piece * VEC);
                for (int x0 = slot; x0 < listed; x0 += step * kBatch) {
                    Vec<T, VEC> first[kBatch], second[PAIRS ? 1 : kBatch];
                    Vec<T, kWide> whole[PAIRS || VEC == kWide ? 1 : kBatch];
                    constexpr bool kOther = !PAIRS && VEC != kWide;              // wide vectors are of another size
                    T *dst[kBatch];
                    int w[kBatch];
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) {
                        const int x = x0 + u * step;
                        dst[u] = nullptr;
                        w[u] = -1;
                        if (x >= listed) continue;
                        const T *src = static_cast<const T *>(list[x].src);
                        dst[u] = static_cast<T *>(list[x].dst);
                        w[u] = list_token[x];
                        if (!dst[u]) continue;
                        if (kOther && wide) {
                            whole[kOther ? u : 0].load(src + j);
                            continue;
                        }
                        first[u].load(src + j);
                        if (!PAIRS && turns) second[PAIRS ? 0 : u].load(src + k);
                    }
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) {
                        if (!dst[u]) continue;
                        if (kOther && wide) {
                            whole[kOther ? u : 0].store(dst[u] + j);
                            continue;
                        }
                        if (turns && w[u] >= 0) {
                            const float2 *cs = tr + w[u] * half;
#pragma unroll
                            for (int e = 0; e < VEC; e += PAIRS ? 2 : 1) {
                                Vec<T, VEC> &to = PAIRS ? first[u] : second[PAIRS ? 0 : u];
                                constexpr int kNext = PAIRS ? 1 : 0;
                                if (PAIRS && TAIL && piece * VEC + e >= rot) break;
                                const float2 t = cs[PAIRS ? e / 2 : e];
                                const float p = first[u].get(e), q = to.get(e + kNext);
                                first[u].set(e, p * t.x - q * t.y);
                                to.set(e + kNext, q * t.x + p * t.y);
                            }
                        }
                        first[u].store(dst[u] + j);
                        if (!PAIRS && turns) second[PAIRS ? 0 : u].store(dst[u] + k);
                    }
                }
            }
    }
}

template <typename T>
int launch(const RopeArgs &a, cudaStream_t stream)
{
    constexpr int kVec = 16 / sizeof(T);
    const int half = a.turns ? a.rot / 2 : 0;
    const long long tokens = a.cu_q ? a.total_q : (long long)a.batch * a.max_q;
    // Tokens of a block: several where there are plenty, so that the threads that have no pair to compute angles for wait less
    long long per = tokens / (148 * 8);
    per = per < 1 ? 1 : (per > 4 ? 4 : per);
    if (half > 0 && per * half > kMaxPairs) per = kMaxPairs / half;
    const long long blocks = (tokens + per - 1) / per;
    if (blocks > 0x7fffffffLL) {
        set_error_detail("rotary positions: %lld tokens", tokens);
        return WKV_ERR_LIMIT;
    }
    if ((a.hq + 2ll * a.hkv) * per > 0x3fffffffLL) {
        set_error_detail("rotary positions: %d query and %d KV heads", a.hq, a.hkv);
        return WKV_ERR_LIMIT;
    }
    const dim3 grid((unsigned)(blocks > 0 ? blocks : 1));
    auto go = [&](auto kernel) { return launch_pdl(kernel, grid, kThreads, 0, stream, 1, a, (int)per, tokens); };
    cudaError_t err;
    if (a.order == WKV_ROPE_INTERLEAVED) err = (2 * half) % kVec ? go(rope_kernel<T, kVec, true, true>) : go(rope_kernel<T, kVec, true>);
    else if (half % kVec == 0) err = go(rope_kernel<T, kVec, false>);
    else if (half % (kVec / 2) == 0) err = go(rope_kernel<T, kVec / 2, false>);
    else if (half % 2 == 0) err = go(rope_kernel<T, 2, false>);
    else err = go(rope_kernel<T, 1, false>);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "rotary positions kernel");
}

}  // namespace

int launch_rope(const RopeArgs &a, cudaStream_t stream)
{
    return a.elem_bytes == 4 ? launch<float>(a, stream) : launch<__nv_bfloat16>(a, stream);
}

}  // namespace wkv
