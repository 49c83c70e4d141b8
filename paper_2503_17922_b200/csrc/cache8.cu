// The gather behind the selection into an 8-bit cache, and rows of the cache read back.
//
// A block takes kRows rows of one unit of one tensor.  Where they come from and go to is looked up once for each, a row per thread (window, table
// entry), into shared memory; then a group of lanes takes a row, a vector to a lane, and a few rows at a time, loads first.  The row's
// largest magnitude, by which its scale goes, is found over the lanes of the group: a row is read once.
//
// Bound by waiting rather than by a pipe: of the gather's issue slots 47 % are busy, with 26 warps on an SM; places come before the first load, and two
// rows of a group are in flight.  Two layers of eight prompts of up to 12,289 rows, 30 % kept, d = 128, bf16 into int8 codes, and all of it read back,
// 142 MB: 38.5 us, of which the gather (one launch) 20.9 and the two reads (one per layer) 18.3, each timed alone; with one vector to a lane 44 in all.  Reading back with 16 codes to a
// lane instead of eight was slower.
#include "cache8.cuh"

#include <algorithm>
#include <type_traits>

namespace wkv {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// element offset of a row of unit (b, h) in the pools, -1: no page; and where its scale stands
__device__ __forceinline__ long long place(const Cache8Pages &c, int hkv, int b, int h, int row, long long &scale)
{
    const int pg = row / c.page_size, slot = row - pg * c.page_size, page = pg < c.max_pages ? __ldg(c.table + (long long)b * c.max_pages + pg) : -1;
    if ((unsigned)page >= (unsigned)c.num_pages) return -1;
    scale = ((long long)page * hkv + h) * c.page_size + slot;
    return page * c.page_stride + h * c.head_stride + slot * c.row_stride;
}

struct Gather8Args {
    KShape s;
    LayerTable src;
    PoolTable codes;
    ScaleTable scales;
    Cache8Pages pages;
    const int *window_idx;
    int kind, lanes_shift, units;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) gather8_kernel(const __grid_constant__ Gather8Args a)
{
    // two vectors to a lane: half as many lanes share a row's largest magnitude, scale and place
    constexpr int kVec = 16 / sizeof(T), kEach = 2, kAhead = 2;
    static_assert(kAttnMaxHeadDim / kVec <= 32 * kEach, "a row in the lanes of a warp");
    __shared__ long long from[kRows], to[kRows], to_scale[kRows];
    const KShape &s = a.s;
    pdl_trigger();
    pdl_wait();
    const int unit = (int)blockIdx.x % a.units, tensor = (int)blockIdx.x / a.units, row0 = (int)blockIdx.y * kRows;
    const int b = unit / s.hkv, h = unit - b * s.hkv;
    const SeqInfo si = seq_info(s, b);
    const int n_r = si.n > s.alpha ? si.n - s.alpha : 0, kw = num_windows(si.n, s.alpha, s.omega);
    const int k = num_selected_capped(si.n, s.alpha, s.omega, si.budget, s.k_max);
    const int *idx = a.window_idx + (long long)unit * s.k_max;
    // rows of the unit: the selected windows (only the sequence's last window can be short, and it is selected last), then the observation rows
    int review = k * s.omega;
    if (k > 0 && idx[k - 1] == kw - 1) review -= kw * s.omega - n_r;
    review = min(review, n_r);
    const int rows = min(review + si.n - n_r - row0, kRows);
    if (rows <= 0) return;
    if ((int)threadIdx.x < rows) {
        const int r = row0 + threadIdx.x;
        int at = n_r + (r - review);
        if (r < review) {
            const int wi = idx[r / s.omega];
            at = wi * s.omega + r % s.omega;
            if (wi < 0 || wi >= kw || at >= n_r) at = -1;                 // no window of the sequence: the row stays as it is
        }
        long long scale = 0;
        const long long dst = place(a.pages, s.hkv, b, h, r, scale);
        from[threadIdx.x] = at < 0 || dst < 0 ? -1 : (si.off + at) * s.st + b * s.sb + h * s.sh;
        to[threadIdx.x] = dst;
        to_scale[threadIdx.x] = scale;
    }
    __syncthreads();
    const T *src = static_cast<const T *>(a.src.src[tensor]);
    unsigned char *codes = static_cast<unsigned char *>(a.codes.ptr[tensor]), *scales = a.scales.ptr[tensor];
    const int lanes = 1 << a.lanes_shift, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_shift, groups = kThreads >> a.lanes_shift;
    const int pieces = s.d / kVec;
    for (int x0 = 0; x0 < rows; x0 += groups * kAhead) {                      // (the same number of turns for all lanes: they exchange maxima)
        uint4 raw[kAhead][kEach];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int x = x0 + u * groups + group;
            const long long at = x < rows ? from[x] : -1;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                raw[u][e] = make_uint4(0, 0, 0, 0);
                if (at >= 0 && lane + e * lanes < pieces) raw[u][e] = __ldg(reinterpret_cast<const uint4 *>(src + at) + lane + e * lanes);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < kEach; ++e)
#pragma unroll
                for (int i = 0; i < kVec; ++i) top = largest_nan(top, to_float(reinterpret_cast<const T *>(&raw[u][e])[i]));
            unsigned most = magnitude(top);
            for (int o = 1; o < lanes; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
            const int x = x0 + u * groups + group, byte = scale_byte(most, a.kind);
            if (x >= rows || from[x] < 0) continue;
            if (lane == 0) scales[to_scale[x]] = (unsigned char)byte;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int piece = lane + e * lanes;
                if (piece >= pieces) continue;
                float v[kVec];
                __align__(8) unsigned c[kVec / 4];
#pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] = to_float(reinterpret_cast<const T *>(&raw[u][e])[i]);
                quantise<kVec>(v, c, byte, a.kind);
                typename std::conditional<kVec == 8, uint2, unsigned>::type out;
                out = *reinterpret_cast<const decltype(out) *>(c);
                *reinterpret_cast<decltype(out) *>(codes + to[x] + piece * kVec) = out;
            }
        }
    }
}

struct Read8Args {
    int batch, hkv, d, kind, cap, row_capacity, lanes_shift, units;
    Cache8Pages pages;
    const unsigned char *codes[2], *scales[2];
    void *out[2];
    const int *first, *lengths;
};
// eight codes as what they stand for
__device__ __forceinline__ void store8(float *p, uint2 w, float by, int kind)
{
    const float4 x = codes_to_float(w.x, kind), y = codes_to_float(w.y, kind);
    reinterpret_cast<float4 *>(p)[0] = make_float4(x.x * by, x.y * by, x.z * by, x.w * by);
    reinterpret_cast<float4 *>(p)[1] = make_float4(y.x * by, y.y * by, y.z * by, y.w * by);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, uint2 w, float by, int kind)
{
    // (exact: eight bits of a code at most, and a power of two)
    const uint2 x = kind == kE4m3 ? codes_to_bf16<kE4m3>(w.x, by) : codes_to_bf16<kI8>(w.x, by), y = kind == kE4m3 ? codes_to_bf16<kE4m3>(w.y, by) : codes_to_bf16<kI8>(w.y, by);
    *reinterpret_cast<uint4 *>(p) = make_uint4(x.x, x.y, y.x, y.y);
}
template <typename T>
__global__ void __launch_bounds__(kThreads) read8_kernel(const __grid_constant__ Read8Args a)
{
    constexpr int kAhead = 4;
    __shared__ long long from[kRows], from_scale[kRows];
    pdl_trigger();
    pdl_wait();
    const int unit = (int)blockIdx.x % a.units, which = (int)blockIdx.x / a.units, row0 = (int)blockIdx.y * kRows, kv = a.out[0] ? which : 1;
    const int b = unit / a.hkv, h = unit - b * a.hkv;
    const int first = a.first ? max(a.first[unit], 0) : 0, n = min(a.lengths[unit], a.cap);
    const int rows = (int)min(min((long long)n - first, (long long)a.row_capacity) - row0, (long long)kRows);
    if (rows <= 0) return;
    const unsigned char *codes = a.codes[kv], *scales = a.scales[kv];
    if ((int)threadIdx.x < rows) {
        long long scale = 0;
        from[threadIdx.x] = place(a.pages, a.hkv, b, h, first + row0 + threadIdx.x, scale);
        from_scale[threadIdx.x] = scale;
    }
    __syncthreads();
    // eight codes to a lane
    const int lanes = 1 << a.lanes_shift, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.lanes_shift, groups = kThreads >> a.lanes_shift;
    if (lane * 8 >= a.d) return;
    T *out = static_cast<T *>(a.out[kv]) + ((long long)unit * a.row_capacity + row0) * a.d + lane * 8;
    for (int x0 = group; x0 < rows; x0 += groups * kAhead) {
        uint2 raw[kAhead];
        int byte[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int x = x0 + u * groups;
            const long long at = x < rows ? from[x] : -1;
            byte[u] = -1;
            if (at < 0) continue;
            raw[u] = *reinterpret_cast<const uint2 *>(codes + at + lane * 8);
            byte[u] = scales[from_scale[x]];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (byte[u] >= 0) store8(out + (long long)(x0 + u * groups) * a.d, raw[u], scale_value(byte[u]), a.kind);
    }
}

int shift_for(int pieces)
{
    int shift = 0;
    while (shift < 5 && (1 << shift) < pieces) ++shift;
    return shift;
}
int check_grid(long long blocks, long long parts, const char *what)
{
    if (blocks <= 0x7fffffffLL && parts <= 65535) return WKV_OK;
    set_error_detail("%s: %lld x %lld blocks", what, blocks, parts);
    return WKV_ERR_LIMIT;
}

}  // namespace

int launch_gather8(const KShape &ks, int dtype, int n_tensors, const LayerTable &src, const PoolTable &codes, const ScaleTable &scales,
                   int kind, const Cache8Pages &pages, const int *window_idx, cudaStream_t stream)
{
    Gather8Args a;
    a.s = ks;
    a.src = src;
    a.codes = codes;
    a.scales = scales;
    a.pages = pages;
    a.window_idx = window_idx;
    a.kind = kind;
    a.units = ks.batch * ks.hkv;
    a.lanes_shift = shift_for((ks.d * (dtype == WKV_F32 ? 4 : 2) / 16 + 1) / 2);
    const long long most = (long long)ks.k_max * ks.omega + ks.alpha, parts = (std::min(most, (long long)ks.max_seqlen) + kRows - 1) / kRows;
    const long long blocks = (long long)a.units * n_tensors;
    if (const int st = check_grid(blocks, parts, "gather into the 8-bit cache")) return st;
    const dim3 grid((unsigned)blocks, (unsigned)(parts > 0 ? parts : 1));
    const cudaError_t err = dtype == WKV_F32 ? launch_pdl(gather8_kernel<float>, grid, kThreads, 0, stream, 1, a)
                                             : launch_pdl(gather8_kernel<__nv_bfloat16>, grid, kThreads, 0, stream, 1, a);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "gather into the 8-bit cache");
}

int launch_read8(int batch, int hkv, int d, const Cache8Pages &pages, int kind, const void *const (&codes)[2],
                 const unsigned char *const (&scales)[2], const int *first, const int *lengths, int out_dtype, int row_capacity,
                 void *const (&out)[2], cudaStream_t stream)
{
    Read8Args a;
    a.batch = batch;
    a.hkv = hkv;
    a.d = d;
    a.kind = kind;
    a.cap = pages.max_pages * pages.page_size;
    a.row_capacity = row_capacity;
    a.units = batch * hkv;
    a.pages = pages;
    a.lanes_shift = shift_for(d / 8);
    for (int x = 0; x < 2; ++x) {
        a.codes[x] = static_cast<const unsigned char *>(codes[x]);
        a.scales[x] = scales[x];
        a.out[x] = out[x];
    }
    a.first = first;
    a.lengths = lengths;
    const long long blocks = (long long)a.units * ((out[0] != nullptr) + (out[1] != nullptr)), parts = ((long long)std::min(row_capacity, a.cap) + kRows - 1) / kRows;
    if (const int st = check_grid(blocks, parts, "rows of the 8-bit cache")) return st;
    const dim3 grid((unsigned)blocks, (unsigned)parts);
    const cudaError_t err = out_dtype == WKV_F32 ? launch_pdl(read8_kernel<float>, grid, kThreads, 0, stream, 1, a)
                                                 : launch_pdl(read8_kernel<__nv_bfloat16>, grid, kThreads, 0, stream, 1, a);
    if (err == cudaSuccess) count_launches(1);
    return check_cuda(err, "rows of the 8-bit cache");
}

}  // namespace wkv
