// The gradient norm of a replica over all its tensors, and clipping:
//   norm_i = sqrt( sum over the tensors t and elements e of g[i][t][e]^2 ),
//   c_i = min(1, max_norm / norm_i),   out = c_i * g.
//
// Two kernels.  k_clip_sums cuts the P * n_tiles tiles into one contiguous run per CTA, so that a CTA
// meets few replicas, and leaves one partial sum per (replica, CTA) pair that meet; the CTA that is last to
// finish adds up those of every replica -- in the order of the CTAs, hence the same bits every time -- and
// writes norms and factors.  k_clip_scale multiplies, one tile per CTA, last tile first: those are the
// ones that the first kernel has just left in the L2.
//
// Bound by memory: the gradients are read twice (nothing on the chip holds 715 MB) and written once.  Measured:
// fp32, 16 replicas of 11.2 M, 126 us (5.7 TB/s) + 204 us (6.5 TB/s, the copy rate); bf16, 8 replicas of 52 M, 153 us
// (5.4 TB/s) + 366 us (6.7 TB/s).  Tried and slower: factors formed by every CTA of a scaling kernel that walks the
// same runs (252 us: registers for two tiles, half the CTAs), 16-bit values fetched 16 bytes a thread in the
// scaling (437 us: its two 16-byte stores then leave half a sector each).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "eg_common.cuh"

namespace eg {

constexpr int kClipCtasPerSm = 4;         // resident at once: both kernels then walk all runs side by side
constexpr long long kClipKeepBytes = 80ll << 20;   // of the 126 MB L2

struct ClipArgs {
    const void* grads;        // [P][stride], float, bf16 or fp16
    float* out;               // [P][stride]; may be `grads` itself when that is fp32
    TileTable tt;             // tiles of kNormTile elements
    int P;
    long long stride;
    double max_norm;
    int zero_nonfinite;       // a replica whose norm is not finite gets zeros
    double* partials;         // [P + CTAs]
    double* factors;          // [P]
    int* first_cta;           // [P] CTA of k_clip_sums whose run holds the first tile of a replica
    unsigned int* done;       // CTAs of k_clip_sums that have finished; zero between calls
    float* norms;             // [P]
};

// 16 bytes of gradients, widened.
template <typename T> __device__ __forceinline__ void clip_widen(const uint4& a, float (&v)[16 / sizeof(T)]) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (std::is_same<T, float>::value) {
            v[q] = __uint_as_float(w[q]);
        } else if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[q]));
            v[2 * q] = f.x;
            v[2 * q + 1] = f.y;
        } else {
            v[2 * q] = __uint_as_float(w[q] << 16);
            v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
        }
    }
}

// A tile's values of one thread, on their way from memory.  Both kernels fetch the next tiles before they work on
// one: a thread alone has too few bytes in flight to keep the memory busy.
template <typename T> struct ClipTile {
    static constexpr int kN = 16 / (int)sizeof(T), kIter = kNormTile / (kThreads * kN);
    int len;
    long long base;
    uint4 raw[kIter];

    __device__ __forceinline__ double sum_of_squares() const {
        double sum[2] = {0.0, 0.0};
        const bool whole = len == kNormTile;
#pragma unroll
        for (int q = 0; q < kIter; ++q) {
            float v[kN];
            clip_widen<T>(raw[q], v);
            const int local = (q * kThreads + threadIdx.x) * kN;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < kN; ++e) v[e] = local + e < len ? v[e] : 0.f;
            }
#pragma unroll
            for (int e = 0; e < kN; ++e) sum[e & 1] = __fma_rn((double)v[e], (double)v[e], sum[e & 1]);
        }
        return __dadd_rn(sum[0], sum[1]);
    }

    // keep: leave the lines in the L2
    __device__ __forceinline__ void fetch(const ClipArgs& a, int i, int tile, bool keep) {
        len = 0;
        if (!tile_ok(a.tt, tile, 0x7fffffff, a.stride, kNormTile)) return;   // bounds-checked build only
        len = a.tt.length[tile];
        base = (long long)i * a.stride + a.tt.offset[tile];
        const T* g = static_cast<const T*>(a.grads) + base;
#pragma unroll
        for (int q = 0; q < kIter; ++q) {
            const int local = (q * kThreads + threadIdx.x) * kN;
            raw[q] = make_uint4(0, 0, 0, 0);
            if (local < len)
                raw[q] = keep ? __ldg(reinterpret_cast<const uint4*>(g + local)) : __ldcs(reinterpret_cast<const uint4*>(g + local));
        }
    }
};

// First of the W units that CTA b of G works on.
__device__ __forceinline__ long long clip_first(long long W, int b, int G) { return W * b / G; }

// CTA b and replica i meet at most once along the (monotone) walk of the units, so i + b numbers
// the pairs without a gap.
template <typename T>
__global__ void __launch_bounds__(kThreads, kClipCtasPerSm) k_clip_sums(const ClipArgs a) {
    pdl_release();
    __shared__ double s_warp[kWarps];
    using Tile = ClipTile<T>;
    constexpr int DEPTH = sizeof(T) == 2 ? 3 : 2;             // tiles in flight
    const int n_tiles = a.tt.n_tiles, b = blockIdx.x, G = gridDim.x;
    const long long W = (long long)a.P * n_tiles;
    const long long u0 = clip_first(W, b, G), u1 = clip_first(W, b + 1, G);
    if (u0 >= u1) return;
    // the end of the run stays in the L2 for the second kernel, which begins there
    const long long keep_from = u1 - kClipKeepBytes / (kNormTile * (long long)sizeof(T)) / G;
    int i = (int)(u0 / n_tiles), tile = (int)(u0 % n_tiles), ai = i, atile = tile;
    long long au = u0;                                        // next tile to fetch: au = (ai, atile)
    Tile t[DEPTH];
    auto ahead = [&](Tile& to) {
        if (au < u1) to.fetch(a, ai, atile, au >= keep_from);
        ++au;
        if (++atile == n_tiles) { atile = 0; ++ai; }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) ahead(t[d]);
    // Replica r owns the slots r + first_cta[r] .. r + first_cta[r + 1]; the last one stays without a CTA where
    // replica r + 1 begins a run.
    if (threadIdx.x == 0 && tile == 0) {
        a.first_cta[i] = b;
        if (i > 0) a.partials[i - 1 + b] = 0.0;
    }
    double acc = 0.0;
    for (long long u = u0; u < u1;) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (u >= u1) break;
            acc = __dadd_rn(acc, t[d].sum_of_squares());
            ahead(t[d]);
            ++u;
            if (++tile == n_tiles || u == u1) {
                const double total = block_sum(acc, s_warp);
                if (threadIdx.x == 0) a.partials[i + b] = total;
                __syncthreads();
                acc = 0.0;
                if (tile == n_tiles) {
                    tile = 0;
                    ++i;
                    if (u < u1 && threadIdx.x == 0) a.first_cta[i] = b;
                }
            }
        }
    }
    // the last CTA to come here forms norms and factors, one warp per replica
    __shared__ bool s_last;
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(a.done, 1u) + 1 == (unsigned)G;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    for (int r = threadIdx.x >> 5; r < a.P; r += kWarps) {
        const int from = r + __ldcg(a.first_cta + r), to = r + (r + 1 < a.P ? __ldcg(a.first_cta + r + 1) : G - 1);
        double total = 0.0;
        for (int q = from + (int)(threadIdx.x & 31); q <= to; q += 32) total = __dadd_rn(total, __ldcg(a.partials + q));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total = __dadd_rn(total, __shfl_down_sync(0xffffffffu, total, o));
        if ((threadIdx.x & 31) != 0) continue;
        const double norm = __dsqrt_rn(total);
        a.norms[r] = (float)norm;
        double factor = norm > a.max_norm ? a.max_norm / norm : 1.0;
        if (isnan(norm)) factor = norm;
        if (a.zero_nonfinite && !isfinite(norm)) factor = 0.0;
        a.factors[r] = factor;
    }
    if (threadIdx.x == 0) *a.done = 0;
}

// Four values a thread and access, so that the 16 bytes a thread writes follow those of its neighbour.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_clip_scale(const ClipArgs a) {
    constexpr int kN = 4, kIter = kNormTile / (kThreads * kN);
    const int i = a.P - 1 - (int)blockIdx.y, tile = a.tt.n_tiles - 1 - (int)blockIdx.x;
    if (!tile_ok(a.tt, tile, 0x7fffffff, a.stride, kNormTile)) return;       // bounds-checked build only
    const int len = a.tt.length[tile];
    const long long base = (long long)i * a.stride + a.tt.offset[tile];
    const T* g = static_cast<const T*>(a.grads) + base;
    float* o = a.out + base;
    pdl_wait();                 // the factors come from the kernel before this one
    const double wide = a.factors[i];
    const bool zero = a.zero_nonfinite && wide == 0.0;
    if (a.grads == (const void*)a.out && wide == 1.0) return;
    float v[kIter][kN];
#pragma unroll
    for (int q = 0; q < kIter; ++q) {
        const int local = (q * kThreads + threadIdx.x) * kN;
        if (local >= len) continue;
        if constexpr (sizeof(T) == 4) {
            const float4 x = ld_stream(reinterpret_cast<const float*>(g) + local);
            v[q][0] = x.x; v[q][1] = x.y; v[q][2] = x.z; v[q][3] = x.w;
        } else {
            const uint2 x = __ldcs(reinterpret_cast<const uint2*>(g + local));
            float both[8];
            clip_widen<T>(make_uint4(x.x, x.y, 0, 0), both);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[q][e] = both[e];
        }
    }
    const float scale = (float)wide;
    // below the normal range the factor itself would lose bits: 64 bits there
    const bool tiny = wide < 1.1754943508222875e-38;
#pragma unroll
    for (int q = 0; q < kIter; ++q) {
        const int local = (q * kThreads + threadIdx.x) * kN;
        if (local >= len) continue;
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            if (tiny) v[q][e] = zero ? 0.f : (float)__dmul_rn(wide, (double)v[q][e]);
            else v[q][e] = __fmul_rn(scale, v[q][e]);
        }
        if (local + kN <= len) {
            st_stream(o + local, make_float4(v[q][0], v[q][1], v[q][2], v[q][3]));
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (local + e < len) o[local + e] = v[q][e];
        }
    }
}

}  // namespace eg
