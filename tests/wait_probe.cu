// Waits of tree attention's warps on barriers that nothing completes, and on such that are complete (tests/test_gpu_waits.py).
#include "gva_waits.cuh"

// Barrier 0 is complete, barrier 1 never will be.  mode 0: wait on 0; 1: on 1; 2: on 0 and 1 together; 3: on 1 without a flag.
// result[lane] = what the lane's wait said, elapsed[lane] = ns it took.
__global__ void wait_probe_kernel(int mode, int flag, int *result, unsigned long long *elapsed) {
    __shared__ __align__(8) unsigned long long bars[2];
    __shared__ volatile int abort_flag;
    const uint32_t done = gva::smem_u32(&bars[0]), open = gva::smem_u32(&bars[1]);
    if (threadIdx.x == 0) {
        gva::mbar_init(done, 1);
        gva::mbar_init(open, 1);
        gva::mbar_arrive(done);
        abort_flag = flag;
    }
    __syncthreads();
    const unsigned long long t0 = gva::global_timer_ns();
    bool ok;
    if (mode == 0) ok = gva::warp_wait(done, 0, &abort_flag);
    else if (mode == 1) ok = gva::warp_wait(open, 0, &abort_flag);
    else if (mode == 2) ok = gva::warp_wait(done, 0, open, 0, &abort_flag);
    else ok = gva::warp_wait(open, 0, nullptr);
    result[threadIdx.x] = ok;
    elapsed[threadIdx.x] = gva::global_timer_ns() - t0;
}

extern "C" int wait_probe(int mode, int flag, int *result, unsigned long long *elapsed, void *stream) {
    wait_probe_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(mode, flag, result, elapsed);
    return cudaGetLastError() == cudaSuccess ? 0 : 1;
}
