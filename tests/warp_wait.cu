// A block whose warps wait for barriers that nobody arrives at (and for one that is complete): the wait of the attention kernel on
// its own, which ends by itself after its limit.
#include "tc_common.cuh"

using namespace wkv::tc;

__global__ void waits(int *result, unsigned long long *ns, int *abort_out)
{
    __shared__ uint64_t done, never[2];
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        mbar_init(&done, 1);
        mbar_init(&never[0], 1);
        mbar_init(&never[1], 1);
        fence_barrier_init();
        abort_flag = 0;
        mbar_arrive(&done);
    }
    __syncthreads();
    const bool before = warp_wait(&done, 0, &abort_flag);
    const unsigned long long t0 = global_timer_ns();
    const bool there = warp_wait(&never[warp & 1], 0, &abort_flag);
    ns[threadIdx.x] = global_timer_ns() - t0;
    result[threadIdx.x] = (before ? 1 : 0) | (there ? 2 : 0);
    __syncthreads();
    if (threadIdx.x == 0) *abort_out = abort_flag;
}

extern "C" int run_waits(int *result, unsigned long long *ns, int *abort_out, void *stream)
{
    waits<<<1, 128, 0, static_cast<cudaStream_t>(stream)>>>(result, ns, abort_out);
    return (int)cudaGetLastError();
}
