// Per-head norms and rotary positions of queries and keys in one pass, of a prompt in its tensors or of new tokens on their way into the
// paged cache, of plain rows or of 8 bits.
//
//   y = x / sqrt(mean(x^2) + eps) * (weight + offset), then pairs turned by their axis' position; into an 8-bit cache the row's
//   largest magnitude gives its scale
//
// Both sums need the whole row before the first element can be written.  So a row is taken by a group of lanes of one warp, as many as it has pieces
// (a power of two up to 32), and stays in their registers between load and store: 16 elements per lane at most, two rows in flight.  A
// piece is a vector of first partners with that of the second partners (HALF order), or a vector of whole pairs.  Cosines and sines
// of a block's tokens and the weights are computed once into shared memory and serve all heads, as in the kernel without norms; the first
// rows are on their way while the angles are computed.
//
// Bound by the instructions between load and store: 32,768 tokens, 32 query heads and 8 key heads of 128, bf16, three axes, 671 MB: 154-159 us = 4.3 TB/s with norms,
// 81 % of issue slots busy; without norms 120 us = 5.6 TB/s.  With the tables read where they stand, neighbours in one bank, 177 us.  1,024 tokens of 4 query and 2 key heads, d = 64, fp32, as
// every small call: 8 us, a launch and its trips to memory.  An element is unpacked twice, once for the squares and once for its product, and the
// tables are read for every row.
// In HALF order the whole row goes by the largest vector that half the turned dimensions are a multiple of: of 32,768 tokens as above with 124 dimensions turned (vectors of
// two) 405 us, with 126, 62 or 34 (single elements) 620-650.
#include "cache8.cuh"

namespace wkv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxDim = kAttnMaxHeadDim;
constexpr int kMaxTokens = 4;                // of a block

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

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

// N neighbouring elements in registers as floats, and back
template <int N>
__device__ __forceinline__ void unpack(const float *e, float *x)
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = e[i];
}
template <int N>
__device__ __forceinline__ void pack(float *e, const float *x)
{
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = x[i];
}
template <int N>
__device__ __forceinline__ void unpack(const __nv_bfloat16 *e, float *x)
{
    if constexpr (N == 1) {
        x[0] = __bfloat162float(e[0]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint32_t w = reinterpret_cast<const uint32_t *>(e)[i];
            x[2 * i] = __uint_as_float(w << 16);
            x[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
}
template <int N>
__device__ __forceinline__ void pack(__nv_bfloat16 *e, const float *x)
{
    if constexpr (N == 1) {
        e[0] = __float2bfloat16_rn(x[0]);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) reinterpret_cast<uint32_t *>(e)[i] = pack_pair_bf16(x[2 * i], x[2 * i + 1]);
    }
}
// Floats that lane `piece` reads N at a time, four in one access: the lanes' fours stand side by side (in pieces one after the other
// neighbours would meet in the same banks: two thirds of a kernel's shared-memory cycles).
template <int N>
__device__ __forceinline__ int spread(int piece, int e, int pieces)
{
    return N <= 4 ? piece * N + e : ((e >> 2) * pieces + piece) * 4 + (e & 3);
}
// ... count of them, from the e-th on
template <int N, int COUNT>
__device__ __forceinline__ void read(float *to, const float *from, int piece, int e, int pieces)
{
    if constexpr (COUNT % 4 == 0) {
#pragma unroll
        for (int i = 0; i < COUNT; i += 4) *reinterpret_cast<float4 *>(to + i) = *reinterpret_cast<const float4 *>(from + spread<N>(piece, e + i, pieces));
    } else if constexpr (COUNT % 2 == 0) {
#pragma unroll
        for (int i = 0; i < COUNT; i += 2) *reinterpret_cast<float2 *>(to + i) = *reinterpret_cast<const float2 *>(from + spread<N>(piece, e + i, pieces));
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) to[i] = from[spread<N>(piece, e + i, pieces)];
    }
}

// EIGHT: keys and values go into an 8-bit cache
template <typename T, int VEC, bool PAIRS, bool EIGHT>
__global__ void __launch_bounds__(kThreads, EIGHT ? 3 : (sizeof(T) == 4 ? 4 : 5)) turn_kernel(const __grid_constant__ TurnArgs p, int tokens_per_block, long long tokens, int lanes_shift)
{
    typedef typename Bits<VEC * sizeof(T)>::type Raw;
    typedef typename Bits<VEC>::type Codes;
    constexpr int kEach = VEC >= 8 ? 1 : 8 / VEC, kSides = PAIRS ? 1 : 2;       // pieces of a lane at most; vectors of a piece
    constexpr int kAhead = 2;                                                  // rows of a group in flight
    const RopeArgs &a = p.r;
    constexpr int kPairsOf = PAIRS ? VEC / 2 : VEC;                            // pairs of a piece
    __shared__ __align__(16) float turn[kMaxTokens][kMaxDim + 8];              // cosines and sines, spread()
    __shared__ __align__(16) float weight[2][kSides][kMaxDim];                 // spread()
    __shared__ Row list[kThreads];
    __shared__ Token token[kMaxTokens];
    pdl_trigger();
    pdl_wait();
    const int half = a.turns ? a.rot / 2 : 0, rot = 2 * half;
    const int turned = PAIRS ? (rot + VEC - 1) / VEC : half / VEC, pieces = PAIRS ? a.d / VEC : turned + (a.d - rot + 2 * VEC - 1) / (2 * VEC);
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
            const int behind = c - rot, side = PAIRS ? 0 : (behind < 0 ? c >= half : behind / VEC & 1);
            const int piece = PAIRS ? c / VEC : (behind < 0 ? (c - side * half) / VEC : turned + behind / (2 * VEC)), e = PAIRS || behind >= 0 ? c % VEC : (c - side * half) % VEC;
            weight[which][side ? kSides - 1 : 0][spread<VEC>(piece, e, pieces)] = w ? to_float(w[c]) + p.offset : 1.f;
        }
    __syncthreads();
    const int hq = a.q ? a.hq : 0, hk = a.k ? a.hkv : 0, hv = a.v ? a.hkv : 0, rows = hq + hk + hv;
    // A group of lanes keeps to one token: its rows in turn with those of the token's other groups
    const int lanes = 1 << lanes_shift, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> lanes_shift, groups = kThreads >> lanes_shift;
    const int of_token = groups / tokens_per_block, mine = group / of_token, sub = group - mine * of_token, at_once = kThreads / tokens_per_block;
    const float inverse_d = 1.f / (float)a.d;
    // where a piece's vectors begin: two of a turned piece, a half apart; behind the turned dimensions two neighbours, of which the last may be alone
    auto place = [&](int piece) { return PAIRS || piece < turned ? piece * VEC : rot + (piece - turned) * 2 * VEC; };
    auto other = [&](int piece) { return piece < turned ? half : VEC; };
    auto two = [&](int piece) { return !PAIRS && (piece < turned || rot + (piece - turned) * 2 * VEC + VEC < a.d); };
    auto angles = [&]() {
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
            const int at = spread<2 * kPairsOf>(pair / kPairsOf, pair % kPairsOf * 2, turned);
        turn[w][at] = cosine * a.scale;
        turn[w][at + 1] = sine * a.scale;
        }
    };
    for (int r0 = 0; r0 < rows; r0 += at_once) {
        const int listed = min(rows - r0, at_once);
        if (r0 > 0) __syncthreads();
        const int of = (int)threadIdx.x / at_once, nth = (int)threadIdx.x - of * at_once;
        if (of < n && nth < listed) {
            const int row = r0 + nth;
            const Token tok = token[of];
            Row r = {nullptr, nullptr, nullptr, of, row < hq ? 0 : (row < hq + hk ? 1 : 2)};
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
                                if (a.row_positions) a.row_positions[unit * a.cap + at] = a.positions[t0 + of];
                                if (a.row_weights) a.row_weights[unit * a.cap + at] = 0.f;
                            }
                            if ((unsigned)page < (unsigned)a.num_pages) {
                                const long long to = page * a.page_stride + head * a.head_stride + slot * a.row_stride;
                                char *pool = static_cast<char *>(r.kind == 2 ? a.v_out : a.k_out);
                                r.dst = pool + to * (EIGHT ? 1 : (int)sizeof(T));
                                if (EIGHT) r.scale = (r.kind == 2 ? p.v_scales : p.k_scales) + ((long long)page * a.hkv + head) * a.page_size + slot;
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
        Raw raw[kAhead][kEach][kSides];
        int at[kAhead];                                                    // where the row stands in the list, -1: none
        auto fetch = [&](int x0) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int x = x0 + u * of_token;
                at[u] = mine < n && x < listed && list[mine * at_once + x].dst ? mine * at_once + x : -1;
                if (at[u] < 0) continue;
                const T *src = static_cast<const T *>(list[at[u]].src);
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    if (k * lanes >= pieces) break;
                    const int piece = lane + k * lanes, j = place(piece);
                    if (piece >= pieces) continue;
                    raw[u][k][0] = *reinterpret_cast<const Raw *>(src + j);
                    if (two(piece)) raw[u][k][kSides - 1] = *reinterpret_cast<const Raw *>(src + j + other(piece));
                }
            }
        };
        fetch(sub);
        if (r0 == 0) {                                                     // (while the first rows are on their way)
            angles();
            __syncthreads();
        }
        for (int x0 = sub; x0 - sub < listed; x0 += of_token * kAhead) {   // (the same number of turns for all lanes: they exchange sums)
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (!__any_sync(0xffffffffu, at[u] >= 0)) continue;
                const Row &row = list[max(at[u], 0)];
                const int kind = at[u] >= 0 ? row.kind : 2;
                const bool turns = kind < 2, codes = EIGHT && at[u] >= 0 && kind > 0;
                float by = 1.f;
                if (p.norm) {
                    float squares = 0.f;
#pragma unroll
                    for (int k = 0; k < kEach; ++k) {
                        if (k * lanes >= pieces) break;
#pragma unroll
                        for (int s = 0; s < kSides; ++s) {
                            const int piece = lane + k * lanes;
                            if (!turns || piece >= pieces || (s == 1 && !two(piece))) continue;
                            float x[VEC];
                            unpack<VEC>(reinterpret_cast<const T *>(&raw[u][k][s]), x);
#pragma unroll
                            for (int i = 0; i < VEC; ++i) squares = fmaf(x[i], x[i], squares);
                        }
                    }
                    for (int o = 1; o < lanes; o <<= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
                    by = rsqrtf(fmaf(squares, inverse_d, p.eps));
                }
                // A few elements of both partners at a time, each written back where it came from; or kept until their scale is known
                float v[EIGHT ? kEach : 1][EIGHT ? kSides : 1][EIGHT ? VEC : 1] = {};
                constexpr int kStep = VEC < 4 ? VEC : 4;
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    if (k * lanes >= pieces) break;
                    const int piece = lane + k * lanes, j = place(piece);
                    if (at[u] < 0 || piece >= pieces || (!EIGHT && !turns)) continue;
                    const bool both = two(piece);
                    T *e[2] = {reinterpret_cast<T *>(&raw[u][k][0]), reinterpret_cast<T *>(&raw[u][k][kSides - 1])};
#pragma unroll
                    for (int i0 = 0; i0 < VEC; i0 += kStep) {
                        float x[2][kStep];
                        unpack<kStep>(e[0] + i0, x[0]);
                        if (both) unpack<kStep>(e[1] + i0, x[1]);
                        if (turns) {
                            if (p.norm) {
                                float w[kStep];
                                read<VEC, kStep>(w, weight[kind][0], piece, i0, pieces);
#pragma unroll
                                for (int i = 0; i < kStep; ++i) x[0][i] = x[0][i] * by * w[i];
                                if (both) {
                                    read<VEC, kStep>(w, weight[kind][kSides - 1], piece, i0, pieces);
#pragma unroll
                                    for (int i = 0; i < kStep; ++i) x[1][i] = x[1][i] * by * w[i];
                                }
                            }
                            if (piece < turned) {
                                constexpr int kPairs = PAIRS ? kStep / 2 : kStep;
                                float cs[2 * kPairs];
                                read<2 * kPairsOf, 2 * kPairs>(cs, turn[row.token], piece, PAIRS ? i0 : 2 * i0, turned);
#pragma unroll
                                for (int i = 0; i < kPairs; ++i) {
                                    if (PAIRS && j + i0 + 2 * i >= rot) break;
                                    float &first = x[0][PAIRS ? 2 * i : i], &second = PAIRS ? x[0][PAIRS ? 2 * i + 1 : 0] : x[1][i];
                                    const float f = first, g = second;
                                    // (as the kernel without norms rounds)
                                    first = fmaf(f, cs[2 * i], -(g * cs[2 * i + 1]));
                                    second = fmaf(f, cs[2 * i + 1], g * cs[2 * i]);
                                }
                            }
                        }
                        if constexpr (EIGHT) {
#pragma unroll
                            for (int i = 0; i < kStep; ++i) {
                                v[k][0][i0 + i] = x[0][i];
                                if (both) v[k][kSides - 1][i0 + i] = x[1][i];
                            }
                        }
                        if (turns) {
                            pack<kStep>(e[0] + i0, x[0]);
                            if (both) pack<kStep>(e[1] + i0, x[1]);
                        }
                    }
                }
                int byte = 0;
                if constexpr (EIGHT) {
                    if (__any_sync(0xffffffffu, codes)) {
                        float top = 0.f;
#pragma unroll
                        for (int k = 0; k < kEach; ++k)
#pragma unroll
                            for (int s = 0; s < kSides; ++s)
#pragma unroll
                                for (int i = 0; i < VEC; ++i) top = largest_nan(top, v[k][s][i]);
                        unsigned most = magnitude(top);
                        for (int o = 1; o < lanes; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
                        byte = scale_byte(most, p.kind);
                        if (codes && lane == 0) *row.scale = (unsigned char)byte;
                    }
                }
                if (at[u] < 0) continue;
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    if (k * lanes >= pieces) break;
                    const int piece = lane + k * lanes, j = place(piece), second = other(piece);
                    if (piece >= pieces) continue;
#pragma unroll
                    for (int s = 0; s < kSides; ++s) {
                        if (s == 1 && !two(piece)) continue;
                        if (codes) {
                            if constexpr (EIGHT) {
                                unsigned char *dst = static_cast<unsigned char *>(row.dst) + j + s * second;
                                __align__(8) unsigned c[(VEC + 3) / 4];
                                quantise<VEC>(v[k][s], c, byte, p.kind);
                                *reinterpret_cast<Codes *>(dst) = *reinterpret_cast<const Codes *>(c);
                            }
                        } else {
                            *reinterpret_cast<Raw *>(static_cast<T *>(row.dst) + j + s * second) = raw[u][k][s];
                        }
                    }
                }
            }
            fetch(x0 + of_token * kAhead);
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
    // Tokens of a block: one, two or four, as many as leave every SM several blocks
    long long per = 1;
    while (2 * per <= kMaxTokens && tokens >= 148 * 4 * 2 * per) per *= 2;
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
    const bool eight = p.kind != kPlain;
    auto go = [&](auto plain, auto codes, int vec, bool pairs) {
        const auto kernel = eight ? codes : plain;
        const int pieces = pairs ? a.d / vec : half / vec + (a.d - 2 * half + 2 * vec - 1) / (2 * vec);
        int shift = 0;
        while (shift < 5 && (1 << shift) < pieces) ++shift;
        return launch_pdl(kernel, grid, kThreads, 0, stream, 1, p, (int)per, tokens, shift);
    };
    cudaError_t err;
    if (half == 0 || a.order == WKV_ROPE_INTERLEAVED) err = go(turn_kernel<T, kVec, true, false>, turn_kernel<T, kVec, true, true>, kVec, true);
    else if (half % kVec == 0) err = go(turn_kernel<T, kVec, false, false>, turn_kernel<T, kVec, false, true>, kVec, false);
    else if (half % (kVec / 2) == 0) err = go(turn_kernel<T, kVec / 2, false, false>, turn_kernel<T, kVec / 2, false, true>, kVec / 2, false);
    else if (half % 2 == 0) err = go(turn_kernel<T, 2, false, false>, turn_kernel<T, 2, false, true>, 2, false);
    else err = go(turn_kernel<T, 1, false, false>, turn_kernel<T, 1, false, true>, 1, false);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "norm and rotary positions kernel");
}

}  // namespace

int launch_turn(const TurnArgs &a, int dtype, cudaStream_t stream)
{
    return dtype == WKV_F32 ? launch<float>(a, stream) : launch<__nv_bfloat16>(a, stream);
}

}  // namespace wkv
