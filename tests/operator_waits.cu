// Kernels for tests/test_gpu_operator_waits.py: warps that leave a walk together, a slow predecessor.
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

// Lets its successor in the stream start at once, and ends after so many nanoseconds (3 s at most).
__global__ void k_slow(unsigned long long ns) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
    if (ns > 3000000000ull) ns = 3000000000ull;
    const long long begin = clock64();
    do {
        asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    } while (t - t0 < ns && clock64() - begin < 8000000000ll);
}

extern "C" int slow(unsigned long long ns, void* stream) {
    k_slow<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(ns);
    return (int)cudaGetLastError();
}

extern "C" int walk(int* turns, int blocks, int most, void* stream) {
    k_walk<<<blocks, 64, 0, static_cast<cudaStream_t>(stream)>>>(turns, most);
    return (int)cudaGetLastError();
}
