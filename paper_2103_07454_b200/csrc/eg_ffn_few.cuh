// The feed-forward block for few tokens: the weights are read once and little is computed with each of
// them, so the two kernels here are streams of weights, as wide as the memory allows, and not tiles.
//
//   k_few_mma   16-bit weights on 16-byte rows: mma.sync m16n8k16 with the weights as A (16 outputs) and 8
//               tokens as B.  The order of K inside a step is free as long as both operands follow it, so a
//               thread's fragments of two steps are 16 consecutive bytes of a weight row and of a token.
//               (tcgen05 would stage the weights in shared memory only to multiply them with a
//               tile of which 128 - n rows are empty.)
//   k_few_dot   everything else (fp32; 16-bit rows off the 16-byte boundaries): dot products in fp32, lanes along K.
//
// Bound by the memory: 1 token, 4 replicas, 1024 x 2816 in bf16: 10.3 us (4.5 TB/s) + 7.1 us (3.3 TB/s), of which some 2 us
// each are the launch and the first load's latency.  Tried and slower: one unit of outputs per CTA (15.3 + 10.9 us:
// every CTA begins with an empty memory pipe), two sixteens of outputs a warp for 32 tokens (46 us, 40 with one).
//
// Both split K over the warps of a CTA and add the warps' sums in order in shared memory.  They run twice:
// for H = act(x Wg^T) * (x Wu^T) and for y = H Wd^T, the second as a dependent launch that fetches its first
// weights before it waits for H.
#pragma once
#include "eg_gemm.cuh"

namespace eg {

struct FewArgs {
    const void *wa, *wb;              // weights: gate and up, or down alone
    long long wa_rep, wa_row, wb_rep, wb_row;
    const void* x;                    // tokens x K
    long long x_rep, x_row;
    void* out;                        // tokens x rows
    long long out_rep, out_row;
    int P, n, rows, K, act;
    int splits;                       // k_few_dot: warps that share the rows of a unit
};

template <typename T> __device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                                  uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T> __device__ __forceinline__ float few_result(int act, float g, float u) {
    float h = 0.f;
    with_act(act, [&](auto which) { h = act_value<T, decltype(which)::value>(g) * u; });
    return h;
}

// The first kernel of a call waits for whatever came before and only then lets the second one start: the second
// reads its first weights without waiting, and what came before the call may have written them.
template <bool GATE> __device__ __forceinline__ void few_begin() {
    if (GATE) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A unit is 16 outputs of a replica; a CTA takes units blockIdx.x, blockIdx.x + gridDim.x, ...  The weights of the
// next unit are on their way while the sums of this one are put together.  NT: eights of tokens.
template <typename T, int NT, bool GATE>
__global__ void __launch_bounds__(256, 2) k_few_mma(const FewArgs a) {
    constexpr int W = GATE ? 2 : 1, BATCH = GATE ? 4 : 6;
    constexpr int ROW = NT * 8 + 1, WARPS = 8;
    __shared__ float s_part[WARPS][W][16][ROW];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, q = lane & 3;
    const int steps = (a.K + 31) / 32, blocks = (a.rows + 15) / 16;
    const long long units = (long long)a.P * blocks;
    uint4 wv[BATCH][W][2];
    // weights of steps s0, s0 + WARPS, ... of a unit
    auto fetch = [&](long long unit, int s0) {
        const int p = (int)(unit / blocks), row = (int)(unit % blocks) * 16 + g;
#pragma unroll
        for (int m = 0; m < W; ++m) {
            const long long stride = m ? a.wb_row : a.wa_row;
            const T* w = static_cast<const T*>(m ? a.wb : a.wa) + p * (m ? a.wb_rep : a.wa_rep) + row * stride + q * 8;
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int k = (s0 + u * WARPS) * 32;
                const bool in = k + q * 8 < a.K;
                wv[u][m][0] = in && row < a.rows ? __ldcs(reinterpret_cast<const uint4*>(w + k)) : make_uint4(0, 0, 0, 0);
                wv[u][m][1] = in && row + 8 < a.rows ? __ldcs(reinterpret_cast<const uint4*>(w + 8 * stride + k)) : make_uint4(0, 0, 0, 0);
            }
        }
    };
    long long unit = blockIdx.x;
    few_begin<GATE>();
    if (unit < units) fetch(unit, warp);
    if (!GATE) asm volatile("griddepcontrol.wait;" ::: "memory");
    for (; unit < units; unit += gridDim.x) {
        const int p = (int)(unit / blocks), row0 = (int)(unit % blocks) * 16;
        const T* x = static_cast<const T*>(a.x) + p * a.x_rep + g * a.x_row + q * 8;
        float acc[W][NT][4];
#pragma unroll
        for (int m = 0; m < W; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[m][t][e] = 0.f;
        for (int s0 = warp; s0 < steps; s0 += WARPS * BATCH) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int k = (s0 + u * WARPS) * 32;
                const bool in = k + q * 8 < a.K;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    uint4 xv = make_uint4(0, 0, 0, 0);
                    if (in && t * 8 + g < a.n) xv = *reinterpret_cast<const uint4*>(x + t * 8 * a.x_row + k);
#pragma unroll
                    for (int m = 0; m < W; ++m) {
                        const uint4 &lo = wv[u][m][0], &hi = wv[u][m][1];
                        mma_16x8x16<T>(acc[m][t], lo.x, hi.x, lo.y, hi.y, xv.x, xv.y);
                        mma_16x8x16<T>(acc[m][t], lo.z, hi.z, lo.w, hi.w, xv.z, xv.w);
                    }
                }
            }
            if (s0 + WARPS * BATCH < steps) fetch(unit, s0 + WARPS * BATCH);
        }
        if (unit + gridDim.x < units) fetch(unit + gridDim.x, warp);
#pragma unroll
        for (int m = 0; m < W; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) s_part[warp][m][g + (e >> 1) * 8][t * 8 + q * 2 + (e & 1)] = acc[m][t][e];
        __syncthreads();
        for (int o = threadIdx.x; o < 16 * a.n; o += blockDim.x) {
            const int r = o % 16, token = o / 16;
            float sum[W];
#pragma unroll
            for (int m = 0; m < W; ++m) {
                sum[m] = 0.f;
#pragma unroll
                for (int v = 0; v < WARPS; ++v) sum[m] += s_part[v][m][r][token];
            }
            if (row0 + r < a.rows)
                static_cast<T*>(a.out)[p * a.out_rep + token * a.out_row + row0 + r] =
                    from_f32<T>(GATE ? few_result<T>(a.act, sum[0], sum[W - 1]) : sum[0]);
        }
        __syncthreads();
    }
}

// grid (CTAs, P, groups of N tokens), 256 threads.  A unit is R weight rows: gate and up of R / 2 outputs, or R outputs -- more of
// them for more tokens, so that a token's values serve several rows once they are in registers.
// Elements VEC * (32 * split + lane) ... of K belong to lane `lane` of the unit's warp `split`.
template <typename T, int VEC, int N, int R, bool GATE>
__global__ void __launch_bounds__(256) k_few_dot(const FewArgs a) {
    constexpr int OUT = GATE ? R / 2 : R;             // outputs of a unit
    __shared__ float s_part[8][R * N];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, p = blockIdx.y;
    const int unit = blockIdx.x * (8 / a.splits) + warp / a.splits, split = warp % a.splits;
    const int r0 = unit * OUT, count = min(OUT, a.rows - r0);
    const T* wa = static_cast<const T*>(a.wa) + p * a.wa_rep + (long long)r0 * a.wa_row;
    const T* wb = GATE ? static_cast<const T*>(a.wb) + p * a.wb_rep + (long long)r0 * a.wb_row : wa;
    const int t0 = blockIdx.z * N, n = a.n - t0;
    const T* x = static_cast<const T*>(a.x) + p * a.x_rep + t0 * a.x_row;
    float acc[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < N; ++t) acc[r][t] = 0.f;
    const int stride = a.splits * 32 * VEC;
    few_begin<GATE>();
    bool waited = GATE;
    if (count > 0) {
        constexpr int BATCH = R * N <= 4 ? 4 : R * N <= 16 ? 2 : 1;
        for (int k0 = (split * 32 + lane) * VEC; k0 < a.K; k0 += stride * BATCH) {
            float v[BATCH][R][VEC];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int k = k0 + u * stride;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int row = GATE ? r / 2 : r;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[u][r][e] = 0.f;
                    if (k < a.K && row < count) load_vec<T, VEC>((GATE && r & 1 ? wb + row * a.wb_row : wa + row * a.wa_row) + k, v[u][r]);
                }
            }
            if (!waited) {
                asm volatile("griddepcontrol.wait;" ::: "memory");
                waited = true;
            }
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                const int k = k0 + u * stride;
                if (k >= a.K) continue;
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    if (t >= n) continue;
                    float xv[VEC];
                    load_vec<T, VEC>(x + t * a.x_row + k, xv);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) acc[r][t] = fmaf(v[u][r][e], xv[e], acc[r][t]);
                }
            }
        }
    }
    __syncwarp();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < N; ++t) {
            float v = acc[r][t];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0) s_part[warp][r * N + t] = v;
        }
    __syncthreads();
    if (split != 0) return;
    for (int o = lane; o < count * N; o += 32) {
        const int r = o / N, t = o % N;
        if (t >= n) continue;
        float g = 0.f, u = 0.f;
        for (int v = 0; v < a.splits; ++v) {
            g += s_part[warp + v][(GATE ? 2 * r : r) * N + t];
            if (GATE) u += s_part[warp + v][(2 * r + 1) * N + t];
        }
        T* out = static_cast<T*>(a.out) + p * a.out_rep + (t0 + t) * a.out_row + r0 + r;
        *out = from_f32<T>(GATE ? few_result<T>(a.act, g, u) : g);
    }
}

constexpr int kFewMmaTokens = 16, kFewDotTokens32 = 8, kFewDotTokens16 = 2;

template <typename T, bool GATE> cudaError_t launch_few_mma(const FewArgs& a, cudaStream_t stream) {
    const long long units = (long long)a.P * ((a.rows + 15) / 16), most = 2ll * sm_count();
    auto go = [&](auto kernel) {
        const dim3 grid((unsigned)(units < most ? units : most));
        return launch_after(kernel, grid, dim3(256), 0, stream, a);
    };
    return a.n <= 8 ? go(k_few_mma<T, 1, GATE>) : go(k_few_mma<T, 2, GATE>);
}

template <typename T, int VEC, bool GATE> cudaError_t launch_few_dot(FewArgs a, int P, cudaStream_t stream) {
    auto go = [&](auto kernel, int N, int R) {
        const int outs = GATE ? R / 2 : R, units = (a.rows + outs - 1) / outs;
        // warps per unit: enough of them to fill the multiprocessors, each with some K to work on
        a.splits = 8;
        while (a.splits > 1 && ((long long)units * P * a.splits > 32ll * sm_count() || a.K < a.splits * 32 * VEC)) a.splits /= 2;
        const int per = 8 / a.splits;
        const dim3 grid((units + per - 1) / per, P, (a.n + N - 1) / N), block(256);
        return launch_after(kernel, grid, block, 0, stream, a);
    };
    if (a.n <= 1) return go(k_few_dot<T, VEC, 1, 2, GATE>, 1, 2);
    if constexpr (sizeof(T) == 4) {
        if (a.n > 4) return go(k_few_dot<T, VEC, 8, 8, GATE>, 8, 8);
        if (a.n > 2) return go(k_few_dot<T, VEC, 4, 4, GATE>, 4, 4);
    }
    return go(k_few_dot<T, VEC, 2, 4, GATE>, 2, 4);
}

}  // namespace eg
