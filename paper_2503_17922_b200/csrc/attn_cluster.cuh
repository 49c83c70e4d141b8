// Joining the key splits of a block's rows inside one launch: the splits are the blocks of a cluster, and each reads the others'
// maxima, sums and outputs from their shared memory.  It takes the place of a kernel behind this one (one token over 992 rows:
// 12.6 us with it), as far as a cluster reaches: eight blocks.
#pragma once

#include "attn.cuh"

namespace wkv {

constexpr int kClusterSplits = 8;

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the same place in the shared memory of block `rank` of the cluster
__device__ __forceinline__ uint32_t in_block(uint32_t addr, int rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float remote_float(uint32_t addr)
{
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ float4 remote_float4(uint32_t addr)
{
    float4 x;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ void store_four(float *p, float a, float b, float c, float d) { *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store_four(__nv_bfloat16 *p, float a, float b, float c, float d)
{
    uint2 r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.x) : "f"(b), "f"(a));
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.y) : "f"(d), "f"(c));
    *reinterpret_cast<uint2 *>(p) = r;
}

// By all threads of all blocks of the cluster (1 .. kClusterSplits blocks, whose rank is their split): `n` rows from row0 on, m, l [n] and
// o [n][stride] in shared memory at the same places in all of them, m in base 2, o relative to m.  With WEIGHTS and a.logits (16 rows at most) the block also adds up
// the weights of the keys [key0, key1), whose logits it has written.  lse2 [16]: shared memory.
template <typename T, int THREADS, bool WEIGHTS>
__device__ __forceinline__ void cluster_join(const AttnArgs &a, const AttnSeq &sq, int unit, int b, int h, int row0, int n, int rank, const float *m,
                                             const float *l, const float *o, int stride, float *lse2, int key0, int key1)
{
    const int S = a.splits;
    if (S > 1) cluster_sync();
    else __syncthreads();
    const uint32_t ms = static_cast<uint32_t>(__cvta_generic_to_shared(m)), ls = static_cast<uint32_t>(__cvta_generic_to_shared(l)),
                   os = static_cast<uint32_t>(__cvta_generic_to_shared(o));
    // every block takes a share of the columns, and (for the weights) all rows' normalisers
    const int cols = a.d / 4, share = (n * cols + S - 1) / S;
    for (int y = threadIdx.x; y < share; y += THREADS) {
        const int x = rank * share + y;
        if (x >= n * cols) break;
        const int r = x / cols, c = (x - r * cols) * 4;
        float mm[kClusterSplits], ll[kClusterSplits], top = -INFINITY;
#pragma unroll
        for (int s = 0; s < kClusterSplits; ++s) {
            mm[s] = s < S ? remote_float(in_block(ms + r * 4, s)) : -INFINITY;
            ll[s] = s < S ? remote_float(in_block(ls + r * 4, s)) : 0.f;
        }
#pragma unroll
        for (int s = 0; s < kClusterSplits; ++s) top = fmaxf(top, mm[s]);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int s = 0; s < kClusterSplits; ++s) {
            if (s >= S || ll[s] == 0.f) continue;
            const float f = exp2f(mm[s] - ref);
            const float4 p = remote_float4(in_block(os + (r * stride + c) * 4, s));
            sum += f * ll[s];
            v.x = fmaf(f, p.x, v.x);
            v.y = fmaf(f, p.y, v.y);
            v.z = fmaf(f, p.z, v.z);
            v.w = fmaf(f, p.w, v.w);
        }
        const int row = row0 + r, i = row / a.G, hq = h * a.G + row - i * a.G;
        if (c == 0) attn_store_lse(a, b, hq, i, sq.m, sum > 0.f || sum != sum ? top + log2f(sum) : -INFINITY);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        store_four(static_cast<T *>(a.out) + (sq.q_off + i) * a.ot + b * a.ob + (long long)hq * a.oh + c, v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    }
    if (WEIGHTS && a.logits) {
        if ((int)threadIdx.x < n) {
            const int r = threadIdx.x;
            float mm[kClusterSplits], ll[kClusterSplits], top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int s = 0; s < kClusterSplits; ++s) {                   // (all trips to the other blocks at once)
                mm[s] = s < S ? remote_float(in_block(ms + r * 4, s)) : -INFINITY;
                ll[s] = s < S ? remote_float(in_block(ls + r * 4, s)) : 0.f;
                top = fmaxf(top, mm[s]);
            }
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int s = 0; s < kClusterSplits; ++s)
                if (s < S) sum += exp2f(mm[s] - ref) * ll[s];
            lse2[r] = sum > 0.f || sum != sum ? top + log2f(sum) : -INFINITY;
        }
        __syncthreads();
        const float *x = a.logits + ((long long)unit * a.rows_max + row0) * a.logit_stride;
        for (int j = key0 + (int)threadIdx.x * 2; j < key1; j += THREADS * 2) {
            float w0 = 0.f, w1 = 0.f;
            bool nan = false;
#pragma unroll 4
            for (int r = 0; r < n; ++r) {
                const float ref = lse2[r];
                const float2 s = *reinterpret_cast<const float2 *>(x + r * a.logit_stride + j);
                nan |= ref != ref;
                if (!(fabsf(ref) < INFINITY)) continue;                  // the row has no weight, or is NaN
                w0 += exp2f(s.x - ref);
                w1 += exp2f(s.y - ref);
            }
            if (nan)                                                     // a NaN for the keys that such a row sees: the others' logits are -infinity
                for (int r = 0; r < n; ++r) {
                    const float ref = lse2[r];
                    if (ref == ref) continue;
                    const float2 s = *reinterpret_cast<const float2 *>(x + r * a.logit_stride + j);
                    if (s.x != -INFINITY) w0 = ref;
                    if (s.y != -INFINITY) w1 = ref;
                }
            const long long at = (long long)unit * a.cap + j;
            a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + w0;
            if (j + 1 < key1) a.weights_out[at + 1] = (a.weights_in ? a.weights_in[at + 1] : 0.f) + w1;
        }
    }
    if (S > 1) cluster_sync();           // nobody leaves while its shared memory is read
}
// a unit without new tokens, or without rows: its weights are carried over by the same shares of the keys
__device__ __forceinline__ void carry_weights(const AttnArgs &a, int unit, int key0, int key1, int threads)
{
    if (!a.logits) return;
    for (int j = key0 + (int)threadIdx.x; j < key1; j += threads) {
        const long long at = (long long)unit * a.cap + j;
        a.weights_out[at] = a.weights_in ? a.weights_in[at] : 0.f;
    }
}

}  // namespace wkv
