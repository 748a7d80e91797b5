// The norm between two residual blocks (eg_residual_norm) and its gradients.
//
//   forward   yh = y * inv1,  inv1 = 1 / sqrt(mean(y^2) + eps)
//             r' = scale * r + a * yh,   a = sigmoid(gate) * w_post
//             o  = r' * inv2 * w_pre,    inv2 = 1 / sqrt(mean(r'^2) + eps)
//   backward  dn = d_o * w_pre,  rh = r' * inv2,  c3 = mean(dn * rh)
//             dR = d_r' + inv2 * (dn - rh * c3)                 gradient of r'
//             dr = scale * dR
//             dy = inv1 * (a * dR - yh * c4),  c4 = mean(a * dR * yh)
//             sums over the rows:  C = sum dR * yh,  D = sum dR * r,  W = sum d_o * rh
//             d_w_post = sigmoid(gate) * C,  d_gate = w_post * sigmoid' * C,  d_scale = D,  d_w_pre = W
//
// Bound by memory: the forward call moves four rows per token, the backward call six.  Both keep a
// row on chip between its one load and its stores; the backward call recomputes r' from y and r
// (12 instead of 14 bytes per element in 16-bit types, and nothing is saved by the forward call).
#include "eg_ops.cuh"

namespace eg {
namespace {

constexpr int kMaxWidth = EG_NORM_MAX_WIDTH;
constexpr int kFwdThreads = 256;
constexpr int kBwdThreads = 512;          // consumer threads of the backward kernel at most
constexpr int kBwdMaxCtas = 160;          // one per multiprocessor; bounds the workspace
constexpr int kSmemMax = 227 * 1024;

struct Mat {
    void* p;
    long long rep, row;                   // strides in elements
};

struct NormArgs {
    int P;
    long long rows;
    int d;
    float eps, inv_d;
    Mat in[4];                            // y, r, d_r', d_o
    Mat w_post, gate, scale, w_pre, r_out, o, dy, dr;
    float* partials;
    unsigned int* err;
    int stages, group_rows, slot_bytes;   // backward: ring of shared-memory stages
};

__device__ __forceinline__ float sigmoid_f(float g) { return 1.f / (1.f + expf(-g)); }

template <typename T> __device__ __forceinline__ T* row_of(const Mat& m, int i, long long t) {
    return static_cast<T*>(m.p) + (long long)i * m.rep + t * m.row;
}

// Sums K values over the TPR threads of a group; every thread gets the result.  Groups wider than a
// warp meet at the named barrier 1 + group; `red` (this group's slots, one per warp, K values padded
// to a multiple of 4) must not be the one of the previous call.
template <int K>
__device__ __forceinline__ void group_sum(float (&v)[K], int tpr, int t, int group, float* red) {
    const int width = tpr < 32 ? tpr : 32;
    for (int o = width >> 1; o > 0; o >>= 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
    if (tpr <= 32) return;
    constexpr int KP = (K + 3) & ~3;
    const int warps = tpr >> 5;
    if ((t & 31) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) red[(t >> 5) * KP + k] = v[k];
    }
    op_named_barrier(1 + group, tpr);
    if (K == 1) {
        // padded to four floats per warp only so that both forms share one buffer size
        float s = 0.f;
        for (int w = 0; w < warps; ++w) s += red[w * KP];
        v[0] = s;
    } else {
        float s[KP];
#pragma unroll
        for (int k = 0; k < KP; ++k) s[k] = 0.f;
        for (int w = 0; w < warps; ++w) {
#pragma unroll
            for (int q = 0; q < KP; q += 4) {
                const float4 a = *reinterpret_cast<const float4*>(red + w * KP + q);
                s[q] += a.x; s[q + 1] += a.y; s[q + 2] += a.z; s[q + 3] += a.w;
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = s[k];
    }
}

// Threads that share a row of width d with E elements each: a power of two below a warp, whole
// warps above.
inline int threads_per_row(int d, int E) {
    const int need = (d + E - 1) / E;
    if (need <= 8) return 8;
    if (need <= 16) return 16;
    return (need + 31) / 32 * 32;
}

// ----------------------------------------------------------------------------------- forward
// A CTA holds blockDim / tpr groups; each takes one row at a time of the CTA's run of rows.
// E elements per thread: vector v of the row's VEC-element vectors v * tpr + t.
template <typename T, int VEC, int E>
__global__ void __launch_bounds__(512) k_norm_forward(const __grid_constant__ NormArgs a, int tpr, long long rows_per_cta) {
    constexpr int NV = E / VEC;
    __shared__ float4 s_red[2][16];
    const int group = threadIdx.x / tpr, t = threadIdx.x % tpr, groups = blockDim.x / tpr;
    const long long W = (long long)a.P * a.rows;
    const long long u0 = blockIdx.x * rows_per_cta, u1 = min(W, u0 + rows_per_cta);
    const bool post = a.w_post.p != nullptr, has_y = a.in[0].p != nullptr, pre = a.o.p != nullptr;
    long long u = u0 + group;
    int i = (int)(u / a.rows);
    long long row = u % a.rows;
    int have = -1;                                   // replica whose factors are held
    float fa[E], fs[E];
    float* red0 = reinterpret_cast<float*>(s_red[0] + (group * tpr >> 5));
    float* red1 = reinterpret_cast<float*>(s_red[1] + (group * tpr >> 5));
    // every group makes the same number of turns: the groups of a warp shuffle together
    for (long long base = u0; base < u1; base += groups, u += groups, row += groups) {
        while (row >= a.rows) { row -= a.rows; ++i; }
        const bool active = u < u1 && group < groups;
        float y[E], r[E];
        float sum[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * tpr + t) * VEC;
            const bool in = active && c < a.d;
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[v * VEC + e] = r[v * VEC + e] = 0.f;
            if (in && has_y) load_vec<T, VEC>(row_of<T>(a.in[0], i, row) + c, y + v * VEC);
            if (in) load_vec<T, VEC>(row_of<T>(a.in[1], i, row) + c, r + v * VEC);
        }
        if (active && have != i) {
            have = i;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * tpr + t) * VEC;
#pragma unroll
                for (int e = 0; e < VEC; ++e) fa[v * VEC + e] = fs[v * VEC + e] = 1.f;
                if (c >= a.d) continue;
                if (post) load_vec<T, VEC>(row_of<T>(a.w_post, i, 0) + c, fa + v * VEC);
                if (a.gate.p) {
                    float g[VEC];
                    load_vec<T, VEC>(row_of<T>(a.gate, i, 0) + c, g);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) fa[v * VEC + e] *= sigmoid_f(g[e]);
                }
                if (a.scale.p) load_vec<T, VEC>(row_of<T>(a.scale, i, 0) + c, fs + v * VEC);
            }
        }
        float inv1 = 1.f;
        if (post && has_y) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] = fmaf(y[e], y[e], sum[0]);
            group_sum<1>(sum, tpr, t, group, red0);
            inv1 = __frsqrt_rn(fmaf(sum[0], a.inv_d, a.eps));
        }
        sum[0] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float sr = fs[e] * r[e];
            r[e] = has_y ? fmaf(fa[e], y[e] * inv1, sr) : sr;
            if (!active) r[e] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * tpr + t) * VEC;
            if (active && c < a.d && a.r_out.p) store_vec<T, VEC>(row_of<T>(a.r_out, i, row) + c, r + v * VEC);
            if (c >= a.d)
#pragma unroll
                for (int e = 0; e < VEC; ++e) r[v * VEC + e] = 0.f;
        }
        if (!pre) continue;
#pragma unroll
        for (int e = 0; e < E; ++e) sum[0] = fmaf(r[e], r[e], sum[0]);
        group_sum<1>(sum, tpr, t, group, red1);
        const float inv2 = __frsqrt_rn(fmaf(sum[0], a.inv_d, a.eps));
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * tpr + t) * VEC;
            if (!active || c >= a.d) continue;
            float w[VEC];
            load_vec<T, VEC>(row_of<T>(a.w_pre, i, 0) + c, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) w[e] *= r[v * VEC + e] * inv2;
            store_vec<T, VEC>(row_of<T>(a.o, i, row) + c, w);
        }
    }
}

// ----------------------------------------------------------------------------------- backward
// First of the W rows (replica after replica) that CTA b of G works on.
__host__ __device__ __forceinline__ long long cut(long long W, int b, int G) { return W * b / G; }

// One CTA per multiprocessor.  The producer warp streams rows of y, r, d_r', d_o through a ring of
// shared-memory stages (bulk copies); a stage holds one row for each group of consumer threads.
// Unaligned rows are copied from the 16-byte boundary below them and read from the remainder.
// A thread owns the same columns of every row: its three column sums stay in registers until the
// replica changes, are then added up over the groups in shared memory (in the place of the factors
// a, scale, w_pre, which the next replica reloads) and left as one partial sum per (replica, CTA)
// pair that meet; along the walk i + b numbers these pairs without a gap.
template <typename T, int VEC, int E>
__global__ void __launch_bounds__(kBwdThreads + 32, 1) k_norm_backward(const __grid_constant__ NormArgs a, int tpr) {
    constexpr int NV = E / VEC;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t s_full[4], s_empty[4];
    __shared__ float4 s_red[2][2 * (kBwdThreads / 32)];
    __shared__ volatile int s_abort;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int R = a.group_rows, S = a.stages, d = a.d;
    const int nc = (R * tpr + 31) & ~31;            // consumer threads
    float* fac = reinterpret_cast<float*>(smem);    // [3][d]: a, scale, w_pre; later the column sums
    unsigned char* ring = smem + ((3 * d * (int)sizeof(float) + 127) & ~127);
    const int array_bytes = R * a.slot_bytes, stage_bytes = 4 * array_bytes;
    const long long W = (long long)a.P * a.rows;
    const int b = blockIdx.x, G = gridDim.x;
    const long long u0 = cut(W, b, G), u1 = cut(W, b + 1, G);
    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int s = 0; s < S; ++s) {
            op_mbar_init(&s_full[s], 32);
            op_mbar_init(&s_empty[s], nc / 32);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x >= nc) {
        // ------------------------------------------------------------------ producer warp
        if (warp != nc / 32) return;
        int s = 0, round = 0;
        bool ok = true;
        for (long long u = u0; u < u1 && ok;) {
            const int i = (int)(u / a.rows);
            const long long end = min(u1, (long long)(i + 1) * a.rows);
            for (; u < end; u += R) {
                const int n = (int)min((long long)R, end - u);
                ok = round == 0 || op_mbar_wait(&s_empty[s], (round - 1) & 1, &s_abort, a.err);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                unsigned char* stage = ring + s * stage_bytes;
                uint32_t bytes = 0;
                for (int q = lane; q < 4 * n; q += 32) {
                    const Mat& m = a.in[q / n];
                    if (!m.p) continue;
                    const uintptr_t p = (uintptr_t)row_of<T>(m, i, u - (long long)i * a.rows + q % n);
                    bytes += (uint32_t)(((p + (uintptr_t)d * sizeof(T) + 15) & ~(uintptr_t)15) - (p & ~(uintptr_t)15));
                }
                op_mbar_expect(&s_full[s], bytes);
                for (int q = lane; q < 4 * n; q += 32) {
                    const int k = q / n, g = q % n;
                    const Mat& m = a.in[k];
                    if (!m.p) continue;
                    const uintptr_t p = (uintptr_t)row_of<T>(m, i, u - (long long)i * a.rows + g);
                    const uintptr_t from = p & ~(uintptr_t)15;
                    op_bulk_load(stage + k * array_bytes + g * a.slot_bytes, (const void*)from,
                                 (uint32_t)(((p + (uintptr_t)d * sizeof(T) + 15) & ~(uintptr_t)15) - from), &s_full[s]);
                }
                if (++s == S) { s = 0; ++round; }
            }
            u = end;
        }
        if (!ok) {      // a wait ran out: let the copies in flight land (with a limit) before the memory is given back
            for (int q = 0; q < S; ++q) {
                const int uses = round + (q < s ? 1 : 0);       // of stage q so far
                for (int tries = 0; uses > 0 && tries < 2000 && !op_mbar_test(&s_full[q], (uses - 1) & 1); ++tries) {}
            }
        }
        return;
    }

    // ---------------------------------------------------------------------- consumers
    const int group = threadIdx.x / tpr, t = threadIdx.x % tpr;
    const bool post = a.w_post.p != nullptr && a.in[0].p != nullptr, has_y = a.in[0].p != nullptr;
    const bool has_dr = a.in[2].p != nullptr, has_do = a.in[3].p != nullptr;
    float* red0 = reinterpret_cast<float*>(&s_red[0][0]) + (group * tpr >> 5) * 8;
    float* red1 = reinterpret_cast<float*>(&s_red[1][0]) + (group * tpr >> 5) * 8;
    float accC[E], accD[E], accW[E];
    int s = 0, round = 0;
    for (long long u = u0; u < u1;) {
        const int i = (int)(u / a.rows);
        const long long end = min(u1, (long long)(i + 1) * a.rows);
        op_named_barrier(15, nc);                    // the sums of the previous replica are written
        for (int c = threadIdx.x; c < d; c += nc) {
            float fa = has_y ? 1.f : 0.f;
            if (a.w_post.p) fa *= to_f32(row_of<T>(a.w_post, i, 0)[c]);
            if (a.gate.p) fa *= sigmoid_f(to_f32(row_of<T>(a.gate, i, 0)[c]));
            fac[c] = fa;
            fac[d + c] = a.scale.p ? to_f32(row_of<T>(a.scale, i, 0)[c]) : 1.f;
            fac[2 * d + c] = has_do ? to_f32(row_of<T>(a.w_pre, i, 0)[c]) : 0.f;
        }
        op_named_barrier(15, nc);
#pragma unroll
        for (int e = 0; e < E; ++e) accC[e] = accD[e] = accW[e] = 0.f;
        for (; u < end; u += R) {
            const int n = (int)min((long long)R, end - u);
            // after a time-out the walk goes on without waiting, so that no barrier is missed
            (void)op_mbar_wait(&s_full[s], round & 1, &s_abort, a.err);
            const bool active = group < n;
            const long long row = u - (long long)i * a.rows + group;
            const unsigned char* stage = ring + s * stage_bytes + group * a.slot_bytes;
            const T* in[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uintptr_t p = active && a.in[k].p ? (uintptr_t)row_of<T>(a.in[k], i, row) : 0;
                in[k] = reinterpret_cast<const T*>(stage + k * array_bytes + (p & 15));
            }
            float one[1] = {0.f};
            float inv1 = 1.f;
            if (post) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int c = (v * tpr + t) * VEC;
                    float y[VEC];
                    if (active && c < d) {
                        load_vec<T, VEC>(in[0] + c, y);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) one[0] = fmaf(y[e], y[e], one[0]);
                    }
                }
                group_sum<1>(one, tpr, t, group, red0);
                inv1 = __frsqrt_rn(fmaf(one[0], a.inv_d, a.eps));
            }
            // sums of rn^2, dn*rn, a*yh*d_r, a*yh*dn, a*yh*rn: c3 and c4 follow from them
            float five[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * tpr + t) * VEC;
                if (NV * VEC > 8) asm volatile("" ::: "memory");   // one vector's values at a time: registers
                if (!active || c >= d) continue;
                float y[VEC], r[VEC], g[VEC], o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) y[e] = g[e] = o[e] = 0.f;
                if (has_y) load_vec<T, VEC>(in[0] + c, y);
                load_vec<T, VEC>(in[1] + c, r);
                if (has_dr) load_vec<T, VEC>(in[2] + c, g);
                if (has_do) load_vec<T, VEC>(in[3] + c, o);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float ay = fac[c + e] * (y[e] * inv1);
                    const float rn = fmaf(fac[d + c + e], r[e], ay), dn = fac[2 * d + c + e] * o[e];
                    five[0] = fmaf(rn, rn, five[0]);
                    five[1] = fmaf(dn, rn, five[1]);
                    five[2] = fmaf(ay, g[e], five[2]);
                    five[3] = fmaf(ay, dn, five[3]);
                    five[4] = fmaf(ay, rn, five[4]);
                }
            }
            group_sum<5>(five, tpr, t, group, red1);
            const float inv2 = has_do ? __frsqrt_rn(fmaf(five[0], a.inv_d, a.eps)) : 0.f;
            const float c3 = has_do ? inv2 * inv2 * five[1] * a.inv_d : 0.f;      // inv2 * mean(dn * rh)
            const float c4 = post ? (five[2] + inv2 * (five[3] - c3 * five[4])) * a.inv_d : 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * tpr + t) * VEC;
                if (NV * VEC > 8) asm volatile("" ::: "memory");   // one vector's values at a time: registers
                if (!active || c >= d) continue;
                float y[VEC], r[VEC], g[VEC], o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) y[e] = g[e] = o[e] = 0.f;
                if (has_y) load_vec<T, VEC>(in[0] + c, y);
                load_vec<T, VEC>(in[1] + c, r);
                if (has_dr) load_vec<T, VEC>(in[2] + c, g);
                if (has_do) load_vec<T, VEC>(in[3] + c, o);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float fa = fac[c + e], fs = fac[d + c + e];
                    const float yh = y[e] * inv1;
                    const float rn = fmaf(fs, r[e], fa * yh), dn = fac[2 * d + c + e] * o[e];
                    const float dR = has_do ? fmaf(inv2, dn - rn * c3, g[e]) : g[e];
                    accC[v * VEC + e] = fmaf(dR, yh, accC[v * VEC + e]);
                    accD[v * VEC + e] = fmaf(dR, r[e], accD[v * VEC + e]);
                    accW[v * VEC + e] = fmaf(o[e], rn * inv2, accW[v * VEC + e]);
                    r[e] = fs * dR;
                    y[e] = inv1 * (fa * dR - yh * c4);
                }
                if (a.dr.p) store_vec<T, VEC>(row_of<T>(a.dr, i, row) + c, r);
                if (a.dy.p) store_vec<T, VEC>(row_of<T>(a.dy, i, row) + c, y);
            }
            __syncwarp();
            if (lane == 0) op_mbar_arrive(&s_empty[s]);
            if (++s == S) { s = 0; ++round; }
        }
        u = end;
        // column sums of this replica: first the groups inside a warp, then group after group
        op_named_barrier(15, nc);
        for (int o = tpr; o < 32; o <<= 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                accC[e] += __shfl_xor_sync(0xffffffffu, accC[e], o);
                accD[e] += __shfl_xor_sync(0xffffffffu, accD[e], o);
                accW[e] += __shfl_xor_sync(0xffffffffu, accW[e], o);
            }
        }
        const int turn_threads = tpr < 32 ? 32 : tpr, turns = nc / turn_threads;
        const int my_turn = threadIdx.x / turn_threads;
        const bool writer = tpr >= 32 || lane < tpr;
        for (int turn = 0; turn < turns; ++turn) {
            if (turn == my_turn && writer) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int c = (v * tpr + t) * VEC;
                    if (c >= d) continue;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        float* f = fac + c + e;
                        const int q = v * VEC + e;
                        f[0] = turn ? f[0] + accC[q] : accC[q];
                        f[d] = turn ? f[d] + accD[q] : accD[q];
                        f[2 * d] = turn ? f[2 * d] + accW[q] : accW[q];
                    }
                }
            }
            op_named_barrier(15, nc);
        }
        float* out = a.partials + (long long)(i + b) * 3 * d;
        for (int c = threadIdx.x; c < 3 * d; c += nc) out[c] = fac[c];
    }
}

// Adds up the partial column sums of replica blockIdx.y (CTA after CTA) and forms the gradients of
// the four vectors.  G == 0: there were no rows.
template <typename T>
__global__ void __launch_bounds__(256) k_norm_columns(const __grid_constant__ NormArgs a, Mat d_w_post, Mat d_gate, Mat d_scale,
                                                      Mat d_w_pre, int G) {
    __shared__ float s_sum[8][3][33];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32, i = blockIdx.y, d = a.d;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float sum[3] = {0.f, 0.f, 0.f};
    if (G > 0 && c < d) {
        const long long W = (long long)a.P * a.rows, first = (long long)i * a.rows, last = first + a.rows - 1;
        int b0 = (int)(first * G / W), b1 = (int)(last * G / W);
        while (cut(W, b0 + 1, G) <= first) ++b0;              // the quotients are off by one at most
        while (b0 > 0 && cut(W, b0, G) > first) --b0;
        while (cut(W, b1 + 1, G) <= last) ++b1;
        while (b1 > 0 && cut(W, b1, G) > last) --b1;
#pragma unroll 4
        for (int b = b0 + part; b <= b1; b += 8) {
            const float* p = a.partials + (long long)(i + b) * 3 * d + c;
#pragma unroll
            for (int k = 0; k < 3; ++k) sum[k] += p[(long long)k * d];
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) s_sum[part][k][threadIdx.x % 32] = sum[k];
    __syncthreads();
    if (part != 0 || c >= d) return;
#pragma unroll
    for (int k = 0; k < 3; ++k)
        for (int q = 1; q < 8; ++q) sum[k] += s_sum[q][k][threadIdx.x];
    const float sg = a.gate.p ? sigmoid_f(to_f32(row_of<T>(a.gate, i, 0)[c])) : 1.f;
    const float wp = a.w_post.p ? to_f32(row_of<T>(a.w_post, i, 0)[c]) : 1.f;
    if (d_w_post.p) row_of<T>(d_w_post, i, 0)[c] = from_f32<T>(sg * sum[0]);
    if (d_gate.p) row_of<T>(d_gate, i, 0)[c] = from_f32<T>(wp * sg * (1.f - sg) * sum[0]);
    if (d_scale.p) row_of<T>(d_scale, i, 0)[c] = from_f32<T>(sum[1]);
    if (d_w_pre.p) row_of<T>(d_w_pre, i, 0)[c] = from_f32<T>(sum[2]);
}

// ----------------------------------------------------------------------------------- host
Mat mat(const eg_matrix& m) { return Mat{m.data, (long long)m.replica_stride, (long long)m.row_stride}; }

bool whole_vectors(const Mat& m, size_t size, bool vector) {
    return !m.p || (aligned16(m.p) && m.rep * (long long)size % 16 == 0 && (vector || m.row * (long long)size % 16 == 0));
}

eg_status check(const eg_residual_norm_args* q, NormArgs* a, bool* aligned) {
    if (!q) return EG_ERR_INVALID;
    if (q->dtype != EG_F32 && q->dtype != EG_BF16 && q->dtype != EG_F16) return EG_ERR_INVALID;
    if (q->P < 1 || q->P > 65535 || q->rows < 0 || q->rows > (1ll << 40) || q->width < 1 || q->width > kMaxWidth)
        return EG_ERR_INVALID;
    if (!(q->eps >= 0.0) || q->eps > 3e38) return EG_ERR_INVALID;
    if (!q->residual.data) return EG_ERR_INVALID;
    if (!q->y.data && (q->w_post.data || q->gate.data)) return EG_ERR_INVALID;    // nothing to act on
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    const eg_matrix* rows[] = {&q->y, &q->residual, &q->residual_out, &q->out, &q->d_residual_out, &q->d_out, &q->dy, &q->d_residual};
    for (const eg_matrix* m : rows)
        if (m->data && (((uintptr_t)m->data % size) || m->row_stride < 0 || m->replica_stride < 0)) return EG_ERR_INVALID;
    const eg_matrix* vectors[] = {&q->w_post, &q->gate, &q->scale, &q->w_pre, &q->d_w_post, &q->d_gate, &q->d_scale, &q->d_w_pre};
    for (const eg_matrix* m : vectors)
        if (m->data && (((uintptr_t)m->data % size) || m->replica_stride < 0)) return EG_ERR_INVALID;
    // outputs are written once: rows and replicas of an output must not fall on one another
    const eg_matrix* written[] = {&q->residual_out, &q->out, &q->dy, &q->d_residual};
    for (const eg_matrix* m : written)
        if (m->data && ((q->rows > 1 && m->row_stride < q->width) || (q->P > 1 && m->replica_stride < q->width))) return EG_ERR_INVALID;
    const eg_matrix* sums[] = {&q->d_w_post, &q->d_gate, &q->d_scale, &q->d_w_pre};
    for (const eg_matrix* m : sums)
        if (m->data && q->P > 1 && m->replica_stride < q->width) return EG_ERR_INVALID;
    *a = NormArgs{};
    a->P = (int)q->P; a->rows = q->rows; a->d = (int)q->width;
    a->eps = (float)q->eps; a->inv_d = 1.0f / (float)q->width;
    a->in[0] = mat(q->y); a->in[1] = mat(q->residual); a->w_post = mat(q->w_post); a->gate = mat(q->gate);
    a->scale = mat(q->scale); a->w_pre = mat(q->w_pre); a->r_out = mat(q->residual_out); a->o = mat(q->out);
    a->in[2] = mat(q->d_residual_out); a->in[3] = mat(q->d_out); a->dy = mat(q->dy); a->dr = mat(q->d_residual);
    *aligned = q->width * size % 16 == 0;
    for (const Mat* m : {&a->in[0], &a->in[1], &a->r_out, &a->o, &a->in[2], &a->in[3], &a->dy, &a->dr}) *aligned &= whole_vectors(*m, size, false);
    for (const Mat* m : {&a->w_post, &a->gate, &a->scale, &a->w_pre}) *aligned &= whole_vectors(*m, size, true);
    return EG_OK;
}

template <typename T, int VEC, int E>
cudaError_t forward(const NormArgs& a, cudaStream_t stream) {
    const int tpr = threads_per_row(a.d, E), threads = tpr > kFwdThreads ? tpr : kFwdThreads / tpr * tpr;
    const int groups = threads / tpr;
    const long long W = (long long)a.P * a.rows, slots = (long long)sm_count() * (threads > 256 ? 2 : 4);
    if (slots < 1) return cudaErrorInvalidDevice;
    long long per = (W + slots - 1) / slots;
    per = (per + groups - 1) / groups * groups;
    k_norm_forward<T, VEC, E><<<(unsigned)((W + per - 1) / per), threads, 0, stream>>>(a, tpr, per);
    return cudaGetLastError();
}

template <typename T, int VEC, int E>
cudaError_t backward(NormArgs a, const eg_residual_norm_args* q, cudaStream_t stream) {
    const long long W = (long long)a.P * a.rows;
    int G = 0;
    if (W > 0) {
        const int tpr = threads_per_row(a.d, E), sms = sm_count();
        if (sms < 1) return cudaErrorInvalidDevice;
        a.slot_bytes = VEC > 1 ? a.d * (int)sizeof(T) : (a.d * (int)sizeof(T) + 30) / 16 * 16;
        const int factors = (3 * a.d * (int)sizeof(float) + 127) & ~127, room = kSmemMax - 2048 - factors;
        int R = kBwdThreads / tpr;
        while (R > 1 && 2 * 4 * R * a.slot_bytes > room) --R;      // two stages at least, while rows can be given up
        a.group_rows = R;
        a.stages = room / (4 * R * a.slot_bytes);
        a.stages = a.stages > 4 ? 4 : a.stages;
        if (a.stages < 1) return cudaErrorInvalidValue;
        const int smem = factors + a.stages * 4 * R * a.slot_bytes;
        G = (int)(W < sms ? W : sms);
        G = G > kBwdMaxCtas ? kBwdMaxCtas : G;
        cudaError_t e = cudaFuncSetAttribute(k_norm_backward<T, VEC, E>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        const int threads = ((R * tpr + 31) & ~31) + 32;
        k_norm_backward<T, VEC, E><<<G, threads, smem, stream>>>(a, tpr);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (!q->d_w_post.data && !q->d_gate.data && !q->d_scale.data && !q->d_w_pre.data) return cudaSuccess;
    return launch_after(k_norm_columns<T>, dim3((a.d + 31) / 32, a.P), dim3(256), 0, stream, a, mat(q->d_w_post), mat(q->d_gate),
                        mat(q->d_scale), mat(q->d_w_pre), G);
}

// 16-byte accesses where every row allows them; eight elements a thread up to 2048 columns, so that
// a CTA works on two rows or more at a time, sixteen above.
template <typename T, bool BACKWARD>
cudaError_t dispatch(const NormArgs& a, bool aligned, const eg_residual_norm_args* q, cudaStream_t stream) {
    constexpr int V = 16 / (int)sizeof(T);
    if constexpr (BACKWARD) {
        if (aligned) return a.d <= 2048 ? backward<T, V, 8>(a, q, stream) : backward<T, V, 16>(a, q, stream);
        return a.d <= 2048 ? backward<T, 1, 8>(a, q, stream) : backward<T, 1, 16>(a, q, stream);
    } else {
        if (aligned) return a.d <= 2048 ? forward<T, V, 8>(a, stream) : forward<T, V, 16>(a, stream);
        return a.d <= 2048 ? forward<T, 1, 8>(a, stream) : forward<T, 1, 16>(a, stream);
    }
}

__device__ unsigned int g_operator_error;

}  // namespace

unsigned int* operator_error_word() {
    static unsigned int* known[64] = {nullptr};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    if (!known[dev]) {
        void* p = nullptr;
        if (cudaGetSymbolAddress(&p, g_operator_error) != cudaSuccess) return nullptr;
        known[dev] = static_cast<unsigned int*>(p);
    }
    return known[dev];
}

}  // namespace eg

using namespace eg;

extern "C" {

eg_status eg_operator_status(void* stream_v) {
    unsigned int* w = operator_error_word();
    if (!w) return EG_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    unsigned int e = 0;
    const unsigned int zero = 0;
    if (cudaMemcpyAsync(&e, w, sizeof(e), cudaMemcpyDeviceToHost, stream) != cudaSuccess ||
        cudaStreamSynchronize(stream) != cudaSuccess)
        return EG_ERR_CUDA;
    if (e && cudaMemcpyAsync(w, &zero, sizeof(zero), cudaMemcpyHostToDevice, stream) != cudaSuccess) return EG_ERR_CUDA;
    if (e && cudaStreamSynchronize(stream) != cudaSuccess) return EG_ERR_CUDA;
    return eg_status_of_error_word(e);
}

int64_t eg_residual_norm_workspace(int64_t P, int64_t width) {
    if (P < 1 || P > 65535 || width < 1 || width > kMaxWidth) return 0;
    return (P + kBwdMaxCtas) * 3 * width * (int64_t)sizeof(float);
}

eg_status eg_residual_norm(const eg_residual_norm_args* q, void* stream_v) {
    NormArgs a;
    bool aligned = false;
    const eg_status s = check(q, &a, &aligned);
    if (s != EG_OK) return s;
    if ((q->w_pre.data == nullptr) != (q->out.data == nullptr)) return EG_ERR_INVALID;
    if (!q->residual_out.data && (q->y.data || !q->out.data)) return EG_ERR_INVALID;
    if (a.rows == 0) return EG_OK;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    const cudaError_t e = q->dtype == EG_F32    ? dispatch<float, false>(a, aligned, q, stream)
                          : q->dtype == EG_BF16 ? dispatch<__nv_bfloat16, false>(a, aligned, q, stream)
                                                : dispatch<__half, false>(a, aligned, q, stream);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

eg_status eg_residual_norm_backward(const eg_residual_norm_args* q, void* stream_v) {
    NormArgs a;
    bool aligned = false;
    const eg_status s = check(q, &a, &aligned);
    if (s != EG_OK) return s;
    if (q->d_out.data && !q->w_pre.data) return EG_ERR_INVALID;
    if ((q->dy.data && !q->y.data) || (q->d_w_post.data && !q->w_post.data) || (q->d_gate.data && !q->gate.data) ||
        (q->d_scale.data && !q->scale.data) || (q->d_w_pre.data && !q->w_pre.data))
        return EG_ERR_INVALID;
    if (!q->workspace || !aligned16(q->workspace) || q->workspace_bytes < eg_residual_norm_workspace(q->P, q->width))
        return EG_ERR_INVALID;
    a.partials = static_cast<float*>(q->workspace);
    a.err = operator_error_word();
    if (!a.err) return EG_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    const cudaError_t e = q->dtype == EG_F32    ? dispatch<float, true>(a, aligned, q, stream)
                          : q->dtype == EG_BF16 ? dispatch<__nv_bfloat16, true>(a, aligned, q, stream)
                                                : dispatch<__half, true>(a, aligned, q, stream);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

}  // extern "C"
