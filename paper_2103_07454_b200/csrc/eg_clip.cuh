// The gradient norm of a replica over all its tensors, and clipping:
//   norm_i = sqrt( sum over the tensors t and elements e of g[i][t][e]^2 ),
//   c_i = min(1, max_norm / norm_i),   out = c_i * g.
//
// Two kernels.  Both cut the P * n_tiles tiles into one contiguous run per CTA (the same cut), so
// that a CTA meets few replicas: k_clip_sums leaves one partial sum per (replica, CTA) pair that
// meet, k_clip_scale adds up those of its replica once per replica -- every CTA in the same order,
// hence the same bits -- and scales its tiles, last tile first: those are the ones that the first
// kernel has just left in the L2.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "eg_common.cuh"

namespace eg {

constexpr int kClipCtasPerSm = 8;

struct ClipArgs {
    const void* grads;        // [P][stride], float, bf16 or fp16
    float* out;               // [P][stride]; may be `grads` itself when that is fp32
    TileTable tt;             // tiles of kNormTile elements
    int P;
    long long stride;
    double max_norm;
    int zero_nonfinite;       // a replica whose norm is not finite gets zeros
    double* partials;         // [P + CTAs]
    float* norms;             // [P]
};

// 16 bytes of gradients, widened.
template <typename T> struct ClipVec;
template <> struct ClipVec<float> {
    static constexpr int kN = 4;
    __device__ static void load(const float* p, float* v) {
        const float4 a = ld_stream(p);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    }
};
template <> struct ClipVec<__nv_bfloat16> {
    static constexpr int kN = 8;
    __device__ static void load(const __nv_bfloat16* p, float* v) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[2 * q] = __uint_as_float(w[q] << 16);
            v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
        }
    }
};
template <> struct ClipVec<__half> {
    static constexpr int kN = 8;
    __device__ static void load(const __half* p, float* v) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[q]));
            v[2 * q] = f.x;
            v[2 * q + 1] = f.y;
        }
    }
};

// First of the W units that CTA b of G works on.
__device__ __forceinline__ long long clip_first(long long W, int b, int G) { return W * b / G; }

// CTA b and replica i meet at most once along the (monotone) walk of the units, so i + b numbers
// the pairs without a gap.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_clip_sums(const ClipArgs a) {
    pdl_release();
    __shared__ double s_warp[kWarps];
    using V = ClipVec<T>;
    constexpr int kIter = kNormTile / (kThreads * V::kN);
    const int n_tiles = a.tt.n_tiles, b = blockIdx.x, G = gridDim.x;
    const long long W = (long long)a.P * n_tiles;
    const long long u0 = clip_first(W, b, G), u1 = clip_first(W, b + 1, G);
    if (u0 >= u1) return;
    int i = (int)(u0 / n_tiles), tile = (int)(u0 % n_tiles);
    double acc = 0.0;
    for (long long u = u0; u < u1; ++u) {
        if (!tile_ok(a.tt, tile, 0x7fffffff, a.stride, kNormTile)) return;   // bounds-checked build only
        const int len = a.tt.length[tile];
        const T* g = static_cast<const T*>(a.grads) + (long long)i * a.stride + a.tt.offset[tile];
        float v[kIter][V::kN];
#pragma unroll
        for (int q = 0; q < kIter; ++q) {
            const int local = (q * kThreads + threadIdx.x) * V::kN;
            if (local < len) {
                V::load(g + local, v[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < kIter; ++q) {
            const int local = (q * kThreads + threadIdx.x) * V::kN;
#pragma unroll
            for (int e = 0; e < V::kN; ++e)
                if (local + e < len) acc = __fma_rn((double)v[q][e], (double)v[q][e], acc);
        }
        if (++tile == n_tiles || u + 1 == u1) {
            const double total = block_sum(acc, s_warp);
            if (threadIdx.x == 0) a.partials[i + b] = total;
            __syncthreads();
            acc = 0.0;
            if (tile == n_tiles) { tile = 0; ++i; }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_clip_scale(const ClipArgs a) {
    __shared__ double s_warp[kWarps];
    using V = ClipVec<T>;
    constexpr int kIter = kNormTile / (kThreads * V::kN);
    const int n_tiles = a.tt.n_tiles, b = blockIdx.x, G = gridDim.x;
    const long long W = (long long)a.P * n_tiles;
    const long long u0 = clip_first(W, b, G), u1 = clip_first(W, b + 1, G);
    pdl_wait();                 // the partial sums come from the kernel before this one
    if (u0 >= u1) return;
    const bool in_place = a.grads == (const void*)a.out;
    int i = (int)((u1 - 1) / n_tiles), tile = (int)((u1 - 1) % n_tiles);
    bool fresh = true;
    float scale = 1.f;
    double wide = 1.0;
    for (long long u = u1 - 1; u >= u0; --u) {
        if (fresh) {
            // CTAs that met replica i: those whose run holds one of [i * n_tiles, (i + 1) * n_tiles)
            const long long first = (long long)i * n_tiles, last = first + n_tiles - 1;
            int b0 = (int)(first * G / W), b1 = (int)(last * G / W);
            while (clip_first(W, b0 + 1, G) <= first) ++b0;      // the quotients are off by one at most
            while (b0 > 0 && clip_first(W, b0, G) > first) --b0;
            while (clip_first(W, b1 + 1, G) <= last) ++b1;
            while (b1 > 0 && clip_first(W, b1, G) > last) --b1;
            double acc = 0.0;
            for (int q = b0 + (int)threadIdx.x; q <= b1; q += kThreads)
                if (clip_first(W, q, G) < clip_first(W, q + 1, G)) acc = __dadd_rn(acc, a.partials[i + q]);
            __syncthreads();
            const double total = block_sum(acc, s_warp);
            if (threadIdx.x == 0) s_warp[0] = total;
            __syncthreads();
            const double norm = __dsqrt_rn(s_warp[0]);
            if (u == (long long)i * n_tiles + n_tiles - 1 && threadIdx.x == 0) a.norms[i] = (float)norm;
            wide = norm > a.max_norm ? a.max_norm / norm : 1.0;
            if (isnan(norm)) wide = norm;
            if (a.zero_nonfinite && !isfinite(norm)) wide = 0.0;
            scale = (float)wide;
            fresh = false;
        }
        if (!tile_ok(a.tt, tile, 0x7fffffff, a.stride, kNormTile)) return;   // bounds-checked build only
        const int len = a.tt.length[tile];
        const long long base = (long long)i * a.stride + a.tt.offset[tile];
        const T* g = static_cast<const T*>(a.grads) + base;
        float* o = a.out + base;
        const bool zero = a.zero_nonfinite && wide == 0.0;
        // below the normal range the factor itself would lose bits: multiply in 64 bits there
        const bool tiny = wide < 1.1754943508222875e-38;
        if (!(in_place && wide == 1.0)) {
            float v[kIter][V::kN];
#pragma unroll
            for (int q = 0; q < kIter; ++q) {
                const int local = (q * kThreads + threadIdx.x) * V::kN;
                if (local < len && !zero) V::load(g + local, v[q]);
            }
#pragma unroll
            for (int q = 0; q < kIter; ++q) {
                const int local = (q * kThreads + threadIdx.x) * V::kN;
                if (local >= len) continue;
#pragma unroll
                for (int e = 0; e < V::kN; ++e)
                    v[q][e] = zero ? 0.f : tiny ? (float)__dmul_rn(wide, (double)v[q][e]) : __fmul_rn(scale, v[q][e]);
#pragma unroll
                for (int e = 0; e < V::kN; e += 4) {
                    if (local + e + 4 <= len)
                        st_stream(o + local + e, make_float4(v[q][e], v[q][e + 1], v[q][e + 2], v[q][e + 3]));
                    else
                        for (int w = e; w < e + 4; ++w)
                            if (local + w < len) o[local + w] = v[q][w];
                }
            }
        }
        if (--tile < 0) { tile = n_tiles - 1; --i; fresh = true; }
    }
}

}  // namespace eg
