// Kernels for tests/test_gpu_operator_waits.py: warps that leave a walk together.
#include "../paper_2103_07454_b200/csrc/eg_ops.cuh"

using namespace eg;

// Two warps walk and meet twice a turn; block b's flag is raised in turn b % 61 by warp b & 1, sooner or later within the turn.
__global__ void k_walk(int* turns, int most) {
    __shared__ volatile int s_abort;
    if (threadIdx.x == 0) s_abort = 0;
    __syncthreads();
    const int warp = threadIdx.x >> 5;
    int t = 0;
    for (; t < most; ++t) {
        if (op_leave_together(1, 64, &s_abort)) break;
        const bool mine = warp == (int)(blockIdx.x & 1) && t == (int)(blockIdx.x % 61);
        if (mine && (blockIdx.x & 2)) s_abort = 1;
        op_named_barrier(1, 64);
        const long long begin = clock64();
        while (mine && clock64() - begin < (long long)(blockIdx.x / 61)) {}
        if (mine && !(blockIdx.x & 2)) s_abort = 1;
    }
    if ((threadIdx.x & 31) == 0) turns[2 * blockIdx.x + warp] = t;
}

extern "C" int walk(int* turns, int blocks, int most, void* stream) {
    k_walk<<<blocks, 64, 0, static_cast<cudaStream_t>(stream)>>>(turns, most);
    return (int)cudaGetLastError();
}
