// Shared by the operators around the step (eg_residual_norm.cu, eg_feed_forward.cu): value types,
// 16-byte accesses, launches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/eventgrad.h"

namespace eg {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Two values <-> one 32-bit word of 16-bit ones.
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// VEC consecutive values at p: 16 bytes at once (p on a 16-byte boundary) or one by one (VEC == 1).
template <typename T, int VEC> __device__ __forceinline__ void load_vec(const T* p, float* v) {
    if constexpr (VEC == 1) {
        v[0] = to_f32(*p);
    } else {
        static_assert(VEC * sizeof(T) == 16, "one 16-byte access");
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (sizeof(T) == 4) {
                v[q] = __uint_as_float(w[q]);
            } else {
                const float2 f = unpack2<T>(w[q]);
                v[2 * q] = f.x;
                v[2 * q + 1] = f.y;
            }
        }
    }
}
template <typename T, int VEC> __device__ __forceinline__ void store_vec(T* p, const float* v) {
    if constexpr (VEC == 1) {
        *p = from_f32<T>(v[0]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (sizeof(T) == 4) w[q] = __float_as_uint(v[q]);
            else w[q] = pack2<T>(v[2 * q], v[2 * q + 1]);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Two fp32 values in one register pair: one instruction for both (sm_100's packed fp32 arithmetic).
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack_f2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ f32x2 pack_f2(float2 v) { return pack_f2(v.x, v.y); }
__device__ __forceinline__ float2 unpack_f2(f32x2 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Launch that may begin while its predecessor in the stream finishes; the kernel calls
// griddepcontrol.wait before it reads what that one wrote.
template <typename... KArgs, typename... Args>
cudaError_t launch_after(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Multiprocessors of the current device, asked for once per device.
inline int sm_count() {
    static int known[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64 && known[dev]) return known[dev];
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < 64) known[dev] = n;
    return n;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace eg

// ---------------------------------------------------------------------------------------
// Shared-memory barriers with bounded waits.  A wait that runs out sets kErrWaitTimeout in the
// operators' error word (eg_operator_status) and raises the CTA's abort flag, so that the other
// waits of the CTA end too; the kernel then drains its copies and returns.
// ---------------------------------------------------------------------------------------
namespace eg {

constexpr unsigned kOpErrWaitTimeout = 8u;
constexpr long long kOpWaitCycles = 2000000000ll;   // about one second

unsigned int* operator_error_word();                // device address on the current device, nullptr on failure

__device__ __forceinline__ uint32_t op_smem(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void op_mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(op_smem(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void op_mbar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(op_smem(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void op_mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(op_smem(bar)) : "memory");
}
__device__ __forceinline__ bool op_mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(op_smem(bar)), "r"(parity), "r"(1000u)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool op_mbar_wait(uint64_t* bar, uint32_t parity, volatile int* s_abort, unsigned int* err,
                                             long long cycles = kOpWaitCycles) {
    if (op_mbar_test(bar, parity)) return true;
    const long long t0 = clock64();
    unsigned spins = 0;
    while (!op_mbar_test(bar, parity)) {
        if ((++spins & 63u) != 0) continue;
        if (*s_abort) return false;
        if (clock64() - t0 > cycles) {
            *s_abort = 1;
            atomicOr(err, kOpErrWaitTimeout);
            return false;
        }
    }
    return true;
}
// The same for a barrier that the other CTA of a cluster arrives on.
__device__ __forceinline__ bool op_mbar_wait_cluster(uint64_t* bar, uint32_t parity, volatile int* s_abort, unsigned int* err,
                                                     long long cycles = kOpWaitCycles) {
    const long long t0 = clock64();
    for (unsigned spins = 1;; ++spins) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(op_smem(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if ((spins & 63u) != 0) continue;
        if (*s_abort) return false;
        if (clock64() - t0 > cycles) {
            *s_abort = 1;
            atomicOr(err, kOpErrWaitTimeout);
            return false;
        }
    }
}
// 1-D bulk copy global -> shared; both addresses and the size multiples of 16 bytes.
__device__ __forceinline__ void op_bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(op_smem(dst)),
                 "l"(src), "r"(bytes), "r"(op_smem(bar))
                 : "memory");
}
__device__ __forceinline__ void op_named_barrier(int id, int threads) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

}  // namespace eg
