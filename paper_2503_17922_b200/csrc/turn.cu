// Per-head norms and rotary positions of queries and keys in one pass, of a prompt in its tensors or of new tokens on their way into the
// paged cache, of plain rows or of 8 bits.
//
//   y = x / sqrt(mean(x^2) + eps) * (weight + offset), then pairs turned by their axis' position; into an 8-bit cache the row's
//   largest magnitude gives its scale
//
// Both sums need the whole row before the first element can be written.  So a row is taken by a group of lanes of one warp, as many as it has pieces
// (a power of two up to 32), and stays in their registers between load and store: 16 elements per lane at most, two rows in flight.  A
// piece is a vector of first partners with that of the second partners (HALF order), or a vector of whole pairs.  Cosines and sines
// of a block's tokens and the weights are computed once into shared memory and serve all heads, as in the kernel without norms.
#include "cache8.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxDim = kAttnMaxHeadDim;
constexpr int kMaxTokens = 4;                // of a block
constexpr int kAhead = 2;                    // rows of a group in flight

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float &y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16 &y, float x) { y = __float2bfloat16_rn(x); }

template <int BYTES> struct Bits;
template <> struct Bits<1> { typedef unsigned char type; };
template <> struct Bits<2> { typedef unsigned short type; };
template <> struct Bits<4> { typedef unsigned type; };
template <> struct Bits<8> { typedef uint2 type; };
template <> struct Bits<16> { typedef uint4 type; };

struct Token {
    int b, i;             // sequence, place in its chunk; b < 0: none
    long long off;        // first row of the sequence in packed tensors
};
__device__ __forceinline__ Token find_token(const RopeArgs &a, long long t)
{
    Token tok;
    if (!a.cu_q) {
        tok.b = (int)(t / a.max_q);
        tok.i = (int)(t - (long long)tok.b * a.max_q);
        tok.off = 0;
        return tok;
    }
    int lo = 0, hi = a.batch;                // the last b with cu[b] <= t
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.cu_q[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int first = a.cu_q[lo], last = a.cu_q[lo + 1];
    tok.b = lo;
    tok.i = (int)(t - first);
    tok.off = first;
    // (a device copy that disagrees with the host copy: not beyond what the host copy allowed for)
    if (!(first >= 0 && t < last && tok.i < a.max_q)) tok.b = -1;
    return tok;
}

struct Row {
    const void *src;
    void *dst;                // null: nowhere
    unsigned char *scale;     // 8-bit rows
    int token, kind;          // 0 query, 1 key, 2 value
};

template <typename T, int VEC, bool PAIRS>
__global__ void __launch_bounds__(kThreads) turn_kernel(const __grid_constant__ TurnArgs p, int tokens_per_block, long long tokens, int lanes_shift)
{
    typedef typename Bits<VEC * sizeof(T)>::type Raw;
    typedef typename Bits<VEC>::type Codes;
    constexpr int kEach = VEC >= 8 ? 1 : 8 / VEC, kSides = PAIRS ? 1 : 2;       // pieces of a lane at most; vectors of a piece
    const RopeArgs &a = p.r;
    __shared__ __align__(16) float2 turn[kMaxTokens][kMaxDim / 2];
    __shared__ __align__(16) float weight[2][kMaxDim];
    __shared__ Row list[kThreads];
    __shared__ Token token[kMaxTokens];
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
    if ((int)threadIdx.x < n) token[threadIdx.x] = find_token(a, t0 + threadIdx.x);
    if (p.norm)
        for (int x = threadIdx.x; x < 2 * a.d; x += kThreads) {
            const int which = x >= a.d, c = x - which * a.d;
            const T *w = static_cast<const T *>(which ? p.k_weight : p.q_weight);
            weight[which][c] = w ? to_float(w[c]) + p.offset : 1.f;
        }
    __syncthreads();
    for (int x = threadIdx.x; x < n * half; x += kThreads) {
        const int w = x / half, pair = x - w * half;
        long long pos = token[w].i;
        if (a.positions) {
            const int axis = p.axis ? p.axis[pair] : 0;
            pos = (unsigned)axis < (unsigned)p.n_axes ? a.positions[axis * p.position_stride + t0 + w] : 0;
        }
        const unsigned long long angle = (unsigned long long)pos * a.turns[pair];
        float sine, cosine;
        sincospif((float)(int)(angle >> 32) * (1.f / 2147483648.f), &sine, &cosine);      // angle in half turns, -1 .. 1
        turn[w][pair] = make_float2(cosine * a.scale, sine * a.scale);
    }
    const int turned = PAIRS ? (rot + VEC - 1) / VEC : half / VEC, pieces = PAIRS ? a.d / VEC : turned + (a.d - rot) / VEC;
    const int hq = a.q ? a.hq : 0, hk = a.k ? a.hkv : 0, hv = a.v ? a.hkv : 0, rows = hq + hk + hv;
    const int lanes = 1 << lanes_shift, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> lanes_shift, groups = kThreads >> lanes_shift;
    for (int y0 = 0; y0 < n * rows; y0 += kThreads) {
        const int listed = min(n * rows - y0, kThreads);
        if (y0 > 0) __syncthreads();
        if ((int)threadIdx.x < listed) {
            const int y = y0 + threadIdx.x, w = y / rows, row = y - w * rows;
            const Token tok = token[w];
            Row r = {nullptr, nullptr, nullptr, w, row < hq ? 0 : (row < hq + hk ? 1 : 2)};
            if (tok.b >= 0) {
                if (r.kind == 0) {
                    const long long off = (tok.off + tok.i) * a.qt + tok.b * a.qb + row * a.qh;
                    r.src = static_cast<const T *>(a.q) + off;
                    r.dst = static_cast<T *>(a.q_out) + off;
                } else {
                    const int head = row - hq - (r.kind == 2 ? hk : 0);
                    const long long off = (tok.off + tok.i) * a.kt + tok.b * a.kb + head * a.kh;
                    r.src = static_cast<const T *>(r.kind == 2 ? a.v : a.k) + off;
                    if (a.table) {
                        const long long unit = (long long)tok.b * a.hkv + head, at = (long long)max(a.lengths[unit], 0) + tok.i;
                        if (at < a.cap) {
                            const int pg = (int)at / a.page_size, slot = (int)at - pg * a.page_size, page = __ldg(a.table + (long long)tok.b * a.max_pages + pg);
                            if (r.kind == 1) {
                                if (a.row_positions) a.row_positions[unit * a.cap + at] = a.positions[t0 + w];
                                if (a.row_weights) a.row_weights[unit * a.cap + at] = 0.f;
                            }
                            if ((unsigned)page < (unsigned)a.num_pages) {
                                const long long to = page * a.page_stride + head * a.head_stride + slot * a.row_stride;
                                char *pool = static_cast<char *>(r.kind == 2 ? a.v_out : a.k_out);
                                r.dst = pool + to * (p.kind == kPlain ? (int)sizeof(T) : 1);
                                if (p.kind != kPlain) r.scale = (r.kind == 2 ? p.v_scales : p.k_scales) + ((long long)page * a.hkv + head) * a.page_size + slot;
                            }
                        }
                    } else {
                        r.dst = static_cast<T *>(a.k_out) + off;
                    }
                }
            }
            list[threadIdx.x] = r;
        }
        __syncthreads();
        for (int x0 = 0; x0 < listed; x0 += groups * kAhead) {             // (the same number of turns for all lanes: they exchange sums)
            Raw raw[kAhead][kEach][kSides];
            Row row[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int x = x0 + u * groups + group;
                row[u].dst = nullptr;
                if (x < listed) row[u] = list[x];
                if (!row[u].dst) continue;
                const T *src = static_cast<const T *>(row[u].src);
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    const int piece = lane + k * lanes, j = PAIRS || piece < turned ? piece * VEC : rot + (piece - turned) * VEC;
                    if (piece >= pieces) continue;
                    raw[u][k][0] = *reinterpret_cast<const Raw *>(src + j);
                    if (!PAIRS && piece < turned) raw[u][k][kSides - 1] = *reinterpret_cast<const Raw *>(src + j + half);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (!__any_sync(0xffffffffu, row[u].dst != nullptr)) continue;
                float v[kEach][kSides][VEC];
                float squares = 0.f;
#pragma unroll
                for (int k = 0; k < kEach; ++k)
#pragma unroll
                    for (int s = 0; s < kSides; ++s) {
                        const int piece = lane + k * lanes;
                        const bool have = row[u].dst && piece < (s == 0 ? pieces : turned);
                        const T *e = reinterpret_cast<const T *>(&raw[u][k][s]);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) {
                            v[k][s][i] = have ? to_float(e[i]) : 0.f;
                            squares = fmaf(v[k][s][i], v[k][s][i], squares);
                        }
                    }
                float by = 1.f;
                if (p.norm) {
                    for (int o = 1; o < lanes; o <<= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
                    by = 1.f / sqrtf(squares / (float)a.d + p.eps);
                }
                const bool turns = row[u].dst && row[u].kind < 2;
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    const int piece = lane + k * lanes, j = PAIRS || piece < turned ? piece * VEC : rot + (piece - turned) * VEC;
                    if (!turns || piece >= pieces) continue;
                    if (p.norm) {
#pragma unroll
                        for (int s = 0; s < kSides; ++s) {
                            if (s == 1 && piece >= turned) continue;
                            const float *w = &weight[row[u].kind][j + s * half];
#pragma unroll
                            for (int i = 0; i < VEC; ++i) v[k][s][i] = v[k][s][i] * by * w[i];
                        }
                    }
                    if (piece < turned) {
                        const float2 *cs = &turn[row[u].token][PAIRS ? piece * (VEC / 2) : piece * VEC];
#pragma unroll
                        for (int i = 0; i < VEC; i += PAIRS ? 2 : 1) {
                            if (PAIRS && j + i >= rot) break;
                            float &first = v[k][0][i], &second = PAIRS ? v[k][0][PAIRS ? i + 1 : i] : v[k][kSides - 1][i];
                            const float2 t = cs[PAIRS ? i / 2 : i];
                            const float f = first, g = second;
                            first = f * t.x - g * t.y;
                            second = g * t.x + f * t.y;
                        }
                    }
                }
                const bool codes = row[u].scale && row[u].kind > 0;
                float inverse = 0.f;
                if (p.kind != kPlain) {
                    unsigned most = 0u;
#pragma unroll
                    for (int k = 0; k < kEach; ++k)
#pragma unroll
                        for (int s = 0; s < kSides; ++s)
#pragma unroll
                            for (int i = 0; i < VEC; ++i) most = max(most, magnitude(v[k][s][i]));
                    for (int o = 1; o < lanes; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
                    const int byte = scale_byte(most, p.kind);
                    inverse = scale_inverse(byte);
                    if (row[u].dst && codes && lane == 0) *row[u].scale = (unsigned char)byte;
                }
                if (!row[u].dst) continue;
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    const int piece = lane + k * lanes, j = PAIRS || piece < turned ? piece * VEC : rot + (piece - turned) * VEC;
                    if (piece >= pieces) continue;
#pragma unroll
                    for (int s = 0; s < kSides; ++s) {
                        if (s == 1 && piece >= turned) continue;
                        if (codes) {
                            unsigned char *dst = static_cast<unsigned char *>(row[u].dst) + j + s * half;
                            __align__(8) unsigned w[(VEC + 3) / 4];
#pragma unroll
                            for (int i = 0; i < VEC; i += 4)
                                w[i / 4] = quantise4(v[k][s][i], VEC > 1 ? v[k][s][(i + 1) % VEC] : 0.f, VEC > 2 ? v[k][s][(i + 2) % VEC] : 0.f,
                                                     VEC > 2 ? v[k][s][(i + 3) % VEC] : 0.f, inverse, p.kind);
                            *reinterpret_cast<Codes *>(dst) = *reinterpret_cast<const Codes *>(w);
                        } else {
                            T *dst = static_cast<T *>(row[u].dst) + j + s * half;
                            Raw out;
#pragma unroll
                            for (int i = 0; i < VEC; ++i) from_float(reinterpret_cast<T *>(&out)[i], v[k][s][i]);
                            *reinterpret_cast<Raw *>(dst) = out;
                        }
                    }
                }
            }
        }
    }
}

template <typename T>
int launch(const TurnArgs &p, cudaStream_t stream)
{
    constexpr int kVec = 16 / sizeof(T);
    const RopeArgs &a = p.r;
    const int half = a.turns ? a.rot / 2 : 0;
    const long long tokens = a.cu_q ? a.total_q : (long long)a.batch * a.max_q;
    // tokens of a block: several where there are plenty, so that the threads that have no pair to compute angles for wait less
    long long per = tokens / (148 * 8);
    per = per < 1 ? 1 : (per > kMaxTokens ? kMaxTokens : per);
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
    auto go = [&](auto kernel, int vec, bool pairs) {
        const int pieces = pairs ? a.d / vec : half / vec + (a.d - 2 * half) / vec;
        int shift = 0;
        while (shift < 5 && (1 << shift) < pieces) ++shift;
        return launch_pdl(kernel, grid, kThreads, 0, stream, 1, p, (int)per, tokens, shift);
    };
    cudaError_t err;
    if (half == 0 || a.order == WKV_ROPE_INTERLEAVED) err = go(turn_kernel<T, kVec, true>, kVec, true);
    else if (half % kVec == 0) err = go(turn_kernel<T, kVec, false>, kVec, false);
    else if (half % (kVec / 2) == 0) err = go(turn_kernel<T, kVec / 2, false>, kVec / 2, false);
    else if (half % 2 == 0) err = go(turn_kernel<T, 2, false>, 2, false);
    else err = go(turn_kernel<T, 1, false>, 1, false);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "norm and rotary positions kernel");
}

}  // namespace

int launch_turn(const TurnArgs &a, int dtype, cudaStream_t stream)
{
    return dtype == WKV_F32 ? launch<float>(a, stream) : launch<__nv_bfloat16>(a, stream);
}

}  // namespace wkv
