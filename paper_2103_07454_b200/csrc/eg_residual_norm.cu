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
//
// k_norm_stream does both for many rows: one CTA (cluster) per multiprocessor (group of them), rows
// streamed through shared memory by bulk copies well ahead of their use, everything else in
// registers.  k_norm_few does the forward pass where there are few rows and a row's way through
// shared memory would only add to its latency.
#include <type_traits>

#include "eg_ops.cuh"

namespace eg {
namespace {

constexpr int kMaxWidth = EG_NORM_MAX_WIDTH;
constexpr int kFewThreads = 256;
constexpr int kThreads = 256;             // of a streaming CTA (a ninth warp would cost each thread a third of its registers)
constexpr int kElems = 16;                // elements of a row per thread
constexpr int kCtaWidth = kThreads * kElems;   // columns of one CTA; wider rows are shared by a cluster
constexpr int kMaxCtas = 160;             // one per multiprocessor; bounds the workspace
constexpr int kMaxStages = 4;
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
    // k_norm_stream: threads of a row in one CTA, CTAs of a row, columns of one CTA, shared-memory stages
    int tpr, teams, ctas, cols, stages, slot_bytes;
};

__device__ __forceinline__ float sigmoid_f(float g) { return 1.f / (1.f + expf(-g)); }

template <typename T> __device__ __forceinline__ T* row_of(const Mat& m, int i, long long t) {
    return static_cast<T*>(m.p) + (long long)i * m.rep + t * m.row;
}

// Sum over the tpr threads of a group, valid in all of them.  Groups wider than a warp meet at the named
// barrier 1 + group; `red` (one float per warp of the group) must not be the one of the previous call.
__device__ __forceinline__ float group_sum(float v, int tpr, int t, int group, float* red) {
    for (int o = (tpr < 32 ? tpr : 32) >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (tpr <= 32) return v;
    if ((t & 31) == 0) red[t >> 5] = v;
    op_named_barrier(1 + group, tpr);
    float s = 0.f;
    for (int w = 0; w < tpr >> 5; ++w) s += red[w];
    return s;
}

// Threads that share a row of width d with E elements each: a power of two below a warp, whole
// warps above.
inline int threads_per_row(int d, int E) {
    const int need = (d + E - 1) / E;
    if (need <= 8) return 8;
    if (need <= 16) return 16;
    return (need + 31) / 32 * 32;
}

// ----------------------------------------------------------------------------------- few rows
// A CTA holds blockDim / tpr groups; each takes one row at a time of the CTA's run of rows.
// E elements per thread: vector v of the row's VEC-element vectors v * tpr + t.
template <typename T, int VEC, int E>
__global__ void __launch_bounds__(512) k_norm_few(const __grid_constant__ NormArgs a, int tpr, long long rows_per_cta) {
    constexpr int NV = E / VEC;
    __shared__ float s_red[2][16];
    const int group = threadIdx.x / tpr, t = threadIdx.x % tpr, groups = blockDim.x / tpr;
    const long long W = (long long)a.P * a.rows;
    const long long u0 = blockIdx.x * rows_per_cta, u1 = min(W, u0 + rows_per_cta);
    const bool post = a.w_post.p != nullptr, has_y = a.in[0].p != nullptr, pre = a.o.p != nullptr;
    long long u = u0 + group;
    int i = (int)(u / a.rows);
    long long row = u % a.rows;
    int have = -1;                                   // replica whose factors are held
    float fa[E], fs[E];
    float *red0 = s_red[0] + (group * tpr >> 5), *red1 = s_red[1] + (group * tpr >> 5);
    // every group makes the same number of turns: the groups of a warp shuffle together
    for (long long base = u0; base < u1; base += groups, u += groups, row += groups) {
        while (row >= a.rows) { row -= a.rows; ++i; }
        const bool active = u < u1 && group < groups;
        float y[E], r[E];
        float sum = 0.f;
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
            for (int e = 0; e < E; ++e) sum = fmaf(y[e], y[e], sum);
            inv1 = __frsqrt_rn(fmaf(group_sum(sum, tpr, t, group, red0), a.inv_d, a.eps));
        }
        sum = 0.f;
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
        for (int e = 0; e < E; ++e) sum = fmaf(r[e], r[e], sum);
        const float inv2 = __frsqrt_rn(fmaf(group_sum(sum, tpr, t, group, red1), a.inv_d, a.eps));
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

// ----------------------------------------------------------------------------------- many rows
// First of the W rows (replica after replica) that CTA (cluster) b of G works on.
__host__ __device__ __forceinline__ long long cut(long long W, int b, int G) { return W * b / G; }

// The rows of a CTA, step by step: up to `per` consecutive rows of one replica.
struct Walk {
    long long row, end, left;          // first row of the step and end of the CTA's rows in replica i; rows after that
    long long rows;
    int i, per;

    __device__ __forceinline__ void start(long long u0, long long u1, long long n, int rows_a_step) {
        rows = n;
        per = rows_a_step;
        i = (int)(u0 / n);
        row = u0 - (long long)i * n;
        end = min(n, row + (u1 - u0));
        left = u1 - u0 - (end - row);
    }
    __device__ __forceinline__ bool done() const { return row >= end; }
    __device__ __forceinline__ int count() const { return (int)min((long long)per, end - row); }
    // true: the next step is in another replica (or there is none)
    __device__ __forceinline__ bool next() {
        row += per;
        if (row < end) return false;
        ++i;
        row = 0;
        end = min(rows, left);
        left -= end;
        return true;
    }
};

// A thread's elements of one row, as they are stored (16-bit types: two to a register).
template <typename T> struct Raw {
    static constexpr int N = kElems * (int)sizeof(T) / 4;
    uint32_t w[N];
    __device__ __forceinline__ float2 pair(int p) const {
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * p]), __uint_as_float(w[2 * p + 1]));
        else return unpack2<T>(w[p]);
    }
    // Makes the compiler unpack again after this point instead of carrying unpacked values in registers.
    __device__ __forceinline__ void repack() {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int q = 0; q < N; ++q) asm volatile("" : "+r"(w[q]));
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int q = 0; q < N; ++q) w[q] = 0;
    }
    // vector v of VEC elements is number v * tpr + t of the row; `d` columns
    template <int VEC> __device__ __forceinline__ void load(const T* p, int tpr, int t, int d) {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int v = 0; v < kElems / VEC; ++v) {
                const int c = (v * tpr + t) * VEC;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (c < d) x = *reinterpret_cast<const uint4*>(p + c);
                w[4 * v] = x.x; w[4 * v + 1] = x.y; w[4 * v + 2] = x.z; w[4 * v + 3] = x.w;
            }
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < kElems; ++e) {
                const int c = e * tpr + t;
                w[e] = c < d ? __float_as_uint(p[c]) : 0u;
            }
        } else {
            const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
            for (int e = 0; e < kElems; e += 2) {
                const int c0 = e * tpr + t, c1 = c0 + tpr;
                w[e / 2] = (c0 < d ? (uint32_t)h[c0] : 0u) | (c1 < d ? (uint32_t)h[c1] << 16 : 0u);
            }
        }
    }
    template <int VEC> __device__ __forceinline__ void store(T* p, int tpr, int t, int d) const {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int v = 0; v < kElems / VEC; ++v) {
                const int c = (v * tpr + t) * VEC;
                if (c < d) *reinterpret_cast<uint4*>(p + c) = make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]);
            }
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < kElems; ++e) {
                const int c = e * tpr + t;
                if (c < d) p[c] = __uint_as_float(w[e]);
            }
        } else {
            uint16_t* h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
            for (int e = 0; e < kElems; e += 2) {
                const int c0 = e * tpr + t, c1 = c0 + tpr;
                if (c0 < d) h[c0] = (uint16_t)w[e / 2];
                if (c1 < d) h[c1] = (uint16_t)(w[e / 2] >> 16);
            }
        }
    }
    __device__ __forceinline__ void set(int p, float a, float b) {
        if constexpr (sizeof(T) == 4) { w[2 * p] = __float_as_uint(a); w[2 * p + 1] = __float_as_uint(b); }
        else w[p] = pack2<T>(a, b);
    }
};

// K values (a power of two) summed over the lanes of a warp (`width` lanes, a power of two, K <= width): halves
// are exchanged, so that every step halves the values instead of repeating all of them (16 values: 16
// shuffles, not 80).  Lane l ends up with the sum over its group of value number held(l).
template <int K> __device__ __forceinline__ float warp_sums(float (&v)[K], int lane, int width) {
    int bit = 1;
#pragma unroll
    for (int half = K / 2; half > 0; half >>= 1, bit <<= 1) {
#pragma unroll
        for (int k = 0; k < half; ++k) {
            const float give = lane & bit ? v[k] : v[k + half], keep = lane & bit ? v[k + half] : v[k];
            v[k] = keep + __shfl_xor_sync(0xffffffffu, give, bit);
        }
    }
    for (; bit < width; bit <<= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], bit);
    return v[0];
}
// Value that lane l holds; it is its own inverse, so also the lane (of the first K) that holds value k.
template <int K> __device__ __forceinline__ int held(int l) {
    int r = 0;
#pragma unroll
    for (int b = 1, h = K / 2; h > 0; b <<= 1, h >>= 1) r |= l & b ? h : 0;
    return r;
}
__host__ __device__ constexpr int ceil_pow2(int k) { return k <= 1 ? 1 : 2 * ceil_pow2((k + 1) / 2); }

// A CTA works through its rows in steps of up to teams * ROWS * (rows of a warp) consecutive rows of one
// replica.  The rows of y, r (and d_r', d_o) of the steps ahead come into a ring of stages in
// shared memory, one bulk copy an array and step where the rows lie one after the other; rows off the
// 16-byte boundaries are copied from the boundary below and read from the remainder.  A team is the tpr
// threads of a row, or a warp with 32 / tpr rows below a warp; it takes ROWS rows at a time, so that the
// latencies of one row's sums are covered by the other's arithmetic (one row in fp32, whose rows are twice as
// long to move).  A thread owns the same columns of every row, so the factors a, scale, w_pre of the replica and
// (backward) its three column sums stay in registers; at the end of a replica's rows the teams add up their
// sums in shared memory and leave one partial sum per (replica, CTA) pair that meet; i + b numbers the pairs
// without a gap.  Rows wider than kCtaWidth are shared by a cluster of two CTAs, which exchange the sums of a row.
template <typename T, int VEC, bool BWD>
__global__ void __launch_bounds__(kThreads, 1) k_norm_stream(const __grid_constant__ NormArgs a) {
    constexpr int E = kElems, ROWS = sizeof(T) == 2 ? 2 : 1, ARRAYS = BWD ? 4 : 2;
    constexpr int K1 = ROWS, K2 = ceil_pow2((BWD ? 5 : 1) * ROWS);
    constexpr int kWarps = kThreads / 32;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_peer[2];
    __shared__ float s_red[2][2 * kWarps][16];                 // [parity][CTA of the cluster, warp][value]
    __shared__ volatile int s_abort;
    if (BWD) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tpr = a.tpr, S = a.stages, C = a.ctas, teams = a.teams;
    const int team_threads = tpr < 32 ? 32 : tpr, each = tpr < 32 ? 32 / tpr : 1;
    const int nc = teams * team_threads;                       // consumer threads
    const int rank = C > 1 ? blockIdx.x % C : 0, b = blockIdx.x / C, G = gridDim.x / C;
    const int c0 = rank * a.cols, d = min(a.cols, a.d - c0);   // columns of this CTA
    const bool post = a.w_post.p != nullptr && a.in[0].p != nullptr;
    const long long W = (long long)a.P * a.rows, u0 = cut(W, b, G), u1 = cut(W, b + 1, G);
    const int per = teams * ROWS * each;
    const int array_bytes = per * a.slot_bytes, stage_bytes = ARRAYS * array_bytes;
    float* s_sums = reinterpret_cast<float*>(smem);            // [3][d] where teams meet (BWD, teams > 1)
    unsigned char* ring = smem + (BWD && teams > 1 ? (3 * a.cols * 4 + 127) & ~127 : 0);
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        s_abort = 0;
        int present = 0;
        for (int q = 0; q < ARRAYS; ++q) present += a.in[q].p != nullptr;
        for (int s = 0; s < S; ++s) {
            op_mbar_init(&s_full[s], present);
            op_mbar_init(&s_empty[s], nc / 32);
        }
        for (int q = 0; q < 2; ++q) op_mbar_init(&s_peer[q], 2 * nc / 32);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (C > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    Walk w;
    w.start(u0, u1, a.rows, per);

    // the rows of array q come in by lane 0 of warp q (few warps: of the last one, q after q)
    Walk ahead = w;
    const int fetcher = threadIdx.x >> 5;
    int as = 0, around = 0;
    auto fetch = [&]() {
        if (ahead.done()) return;
        if (lane == 0 && fetcher < ARRAYS) {
            for (int q = fetcher; q < ARRAYS; q += nc / 32) {
                const Mat& m = a.in[q];
                if (!m.p) continue;
                const bool together = m.row == a.d && C == 1;      // rows one after the other
                const int n = ahead.count();
                if (around > 0 && !op_mbar_wait(&s_empty[as], (around - 1) & 1, &s_abort, a.err)) break;
                unsigned char* dst = ring + as * stage_bytes + q * array_bytes;
                const uintptr_t p = (uintptr_t)(row_of<T>(m, ahead.i, ahead.row) + c0);
                if (VEC > 1 && together) {
                    const uint32_t bytes = (uint32_t)(d * sizeof(T)) * n;
                    op_mbar_expect(&s_full[as], bytes);
                    op_bulk_load(dst, (const void*)p, bytes, &s_full[as]);
                    continue;
                }
                const int copies = together ? 1 : n;
                const uint32_t len = (uint32_t)(d * sizeof(T)) * (together ? n : 1);
                const uintptr_t step = (uintptr_t)m.row * sizeof(T);
                uint32_t bytes = 0;
                for (int z = 0; z < copies; ++z)
                    bytes += (uint32_t)(((p + z * step + len + 15) & ~(uintptr_t)15) - ((p + z * step) & ~(uintptr_t)15));
                op_mbar_expect(&s_full[as], bytes);
                for (int z = 0; z < copies; ++z) {
                    const uintptr_t x = p + z * step, from = x & ~(uintptr_t)15;
                    op_bulk_load(dst + z * a.slot_bytes, (const void*)from, (uint32_t)(((x + len + 15) & ~(uintptr_t)15) - from), &s_full[as]);
                }
            }
        }
        __syncwarp();
        ahead.next();
        if (++as == S) { as = 0; ++around; }
    };
    // a stage is refilled one step after its last use, when no other team should still be reading it
    for (int q = 0; q < S - 1; ++q) fetch();
    if (S == 1) fetch();
    {
        const int team = threadIdx.x / team_threads, tt = threadIdx.x % team_threads;
        const int warps = team_threads >> 5, warp = tt >> 5;
        const int sub = tpr < 32 ? lane / tpr : 0, t = tpr < 32 ? lane % tpr : tt;
        int parity = 0, meets = 0;
        // `used` of KP values of the team's rows, summed over their threads (and CTAs): v[k] in every thread
        auto row_sums = [&](auto& v, int used) {
            constexpr int KP = sizeof(v) / sizeof(float);
            const int width = tpr < 32 ? tpr : 32;
            float sum = warp_sums<KP>(v, lane, width);
            const int first = lane & ~(width - 1);
            if (tpr <= 32 && C == 1) {
#pragma unroll
                for (int k = 0; k < KP; ++k)
                    if (k < used) v[k] = __shfl_sync(0xffffffffu, sum, first + held<KP>(k));
                return;
            }
            if (lane < KP) {
                float* to = &s_red[parity][rank * kWarps + team * warps + warp][held<KP>(lane)];
                *to = sum;
                if (C > 1) {
                    uint32_t other;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(other) : "r"(op_smem(to)), "r"(rank ^ 1));
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(other), "f"(sum) : "memory");
                }
            }
            if (C > 1) {
                // every consumer warp of both CTAs tells both CTAs that its sums are there
                __syncwarp();
                if (lane < 2) {
                    uint32_t bar;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(op_smem(&s_peer[parity])), "r"(lane));
                    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
                }
                (void)op_mbar_wait_cluster(&s_peer[parity], meets >> 1 & 1, &s_abort, a.err);
                ++meets;
            } else {
                op_named_barrier(1 + team, team_threads);
            }
            // lane l adds value l % KP of every (32 / KP)-th warp
            constexpr int L = 32 / KP;
            const int from = C > 1 ? 0 : team * warps, count = C > 1 ? kWarps + warps : warps;
            sum = 0.f;
            for (int x = lane / KP; x < count; x += L)
                if (C == 1 || x % kWarps < warps) sum += s_red[parity][from + x][lane % KP];
#pragma unroll
            for (int o = KP; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
            for (int k = 0; k < KP; ++k)
                if (k < used) v[k] = __shfl_sync(0xffffffffu, sum, k);
            parity ^= 1;
        };

        int s = 0, round = 0;
        while (!w.done()) {
            const int i = w.i;
            Raw<T> fs, fw;
            float fa[E];
            float accC[BWD ? E : 1], accD[BWD ? E : 1], accW[BWD ? E : 1];
            {
                Raw<T> x;
                if (a.w_post.p) x.template load<VEC>(row_of<T>(a.w_post, i, 0) + c0, tpr, t, d);
#pragma unroll
                for (int p = 0; p < E / 2; ++p) {
                    const float2 f = a.w_post.p ? x.pair(p) : make_float2(1.f, 1.f);
                    fa[2 * p] = a.in[0].p ? f.x : 0.f;
                    fa[2 * p + 1] = a.in[0].p ? f.y : 0.f;
                }
                if (a.gate.p) {
                    x.template load<VEC>(row_of<T>(a.gate, i, 0) + c0, tpr, t, d);
#pragma unroll
                    for (int p = 0; p < E / 2; ++p) {
                        const float2 f = x.pair(p);
                        fa[2 * p] *= sigmoid_f(f.x);
                        fa[2 * p + 1] *= sigmoid_f(f.y);
                    }
                }
            }
#pragma unroll
            for (int p = 0; p < E / 2; ++p) fs.set(p, 1.f, 1.f);
            fw.clear();
            if (a.scale.p) fs.template load<VEC>(row_of<T>(a.scale, i, 0) + c0, tpr, t, d);
            if (BWD ? a.in[3].p != nullptr : a.o.p != nullptr) fw.template load<VEC>(row_of<T>(a.w_pre, i, 0) + c0, tpr, t, d);
            if constexpr (BWD) {
#pragma unroll
                for (int e = 0; e < E; ++e) accC[e] = accD[e] = accW[e] = 0.f;
            }
            bool last = false;
            while (!last) {
                const int n = w.count(), mine = team * ROWS * each + sub;      // this thread's rows: mine + z * each
                const unsigned char* stage = ring + s * stage_bytes;
                (void)op_mbar_wait(&s_full[s], round & 1, &s_abort, a.err);    // after a time-out the walk just goes on
                Raw<T> in[ARRAYS][ROWS];
#pragma unroll
                for (int q = 0; q < ARRAYS; ++q) {
                    if (!a.in[q].p) {
#pragma unroll
                        for (int z = 0; z < ROWS; ++z) in[q][z].clear();
                        continue;
                    }
                    const bool together = a.in[q].row == a.d && C == 1;
                    const T* first = row_of<T>(a.in[q], i, w.row) + c0;
#pragma unroll
                    for (int z = 0; z < ROWS; ++z) {
                        const int j = mine + z * each;
                        const T* at;
                        if (VEC > 1) at = reinterpret_cast<const T*>(stage + q * array_bytes + j * a.slot_bytes);
                        else if (together) at = reinterpret_cast<const T*>(stage + q * array_bytes + ((uintptr_t)first & 15)) + j * d;
                        else at = reinterpret_cast<const T*>(stage + q * array_bytes + j * a.slot_bytes + ((uintptr_t)(first + (long long)j * a.in[q].row) & 15));
                        if (j < n) in[q][z].template load<VEC>(at, tpr, t, d);
                        else in[q][z].clear();
                    }
                }
                __syncwarp();
                if (lane == 0) op_mbar_arrive(&s_empty[s]);
                if (++s == S) { s = 0; ++round; }
                if (S > 1) fetch();
                float inv1[ROWS];
#pragma unroll
                for (int z = 0; z < ROWS; ++z) inv1[z] = 1.f;
                if (post) {
                    float v[K1];
#pragma unroll
                    for (int z = 0; z < ROWS; ++z) {
                        float p0 = 0.f, p1 = 0.f;
#pragma unroll
                        for (int p = 0; p < E / 2; ++p) {
                            const float2 y = in[0][z].pair(p);
                            p0 = fmaf(y.x, y.x, p0);
                            p1 = fmaf(y.y, y.y, p1);
                        }
                        v[z] = p0 + p1;
                    }
                    row_sums(v, ROWS);
                    in[0][0].repack();
                    in[0][ROWS - 1].repack();
#pragma unroll
                    for (int z = 0; z < ROWS; ++z) inv1[z] = __frsqrt_rn(fmaf(v[z], a.inv_d, a.eps));
                }
                float v[K2];
#pragma unroll
                for (int k = 0; k < K2; ++k) v[k] = 0.f;
                if constexpr (!BWD) {
                    float rn[ROWS][E];
#pragma unroll
                    for (int z = 0; z < ROWS; ++z) {
                        float p0 = 0.f, p1 = 0.f;
#pragma unroll
                        for (int p = 0; p < E / 2; ++p) {
                            const float2 y = in[0][z].pair(p), r = in[1][z].pair(p), f = fs.pair(p);
                            rn[z][2 * p] = fmaf(fa[2 * p], y.x * inv1[z], f.x * r.x);
                            rn[z][2 * p + 1] = fmaf(fa[2 * p + 1], y.y * inv1[z], f.y * r.y);
                            p0 = fmaf(rn[z][2 * p], rn[z][2 * p], p0);
                            p1 = fmaf(rn[z][2 * p + 1], rn[z][2 * p + 1], p1);
                        }
                        v[z] = p0 + p1;
                        const int j = mine + z * each;
                        if (a.r_out.p && j < n) {
                            Raw<T> x;
#pragma unroll
                            for (int p = 0; p < E / 2; ++p) x.set(p, rn[z][2 * p], rn[z][2 * p + 1]);
                            x.template store<VEC>(row_of<T>(a.r_out, i, w.row + j) + c0, tpr, t, d);
                        }
                    }
                    if (a.o.p) {
                        row_sums(v, ROWS);
#pragma unroll
                        for (int z = 0; z < ROWS; ++z) {
                            const float inv2 = __frsqrt_rn(fmaf(v[z], a.inv_d, a.eps));
                            const int j = mine + z * each;
                            Raw<T> x;
#pragma unroll
                            for (int p = 0; p < E / 2; ++p) {
                                const float2 f = fw.pair(p);
                                x.set(p, rn[z][2 * p] * inv2 * f.x, rn[z][2 * p + 1] * inv2 * f.y);
                            }
                            if (j < n) x.template store<VEC>(row_of<T>(a.o, i, w.row + j) + c0, tpr, t, d);
                        }
                    }
                } else {
                    // sums of rn^2, dn*rn, a*yh*d_r, a*yh*dn, a*yh*rn: c3 and c4 follow from them
#pragma unroll
                    for (int z = 0; z < ROWS; ++z) {
#pragma unroll
                        for (int p = 0; p < E / 2; ++p) {
                            const float2 y2 = in[0][z].pair(p), r2 = in[1][z].pair(p), g2 = in[2][z].pair(p), o2 = in[3][z].pair(p);
                            const float2 f2 = fs.pair(p), q2 = fw.pair(p);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float y = h ? y2.y : y2.x, r = h ? r2.y : r2.x, g = h ? g2.y : g2.x, o = h ? o2.y : o2.x;
                                const float ay = fa[2 * p + h] * (y * inv1[z]), rn = fmaf(h ? f2.y : f2.x, r, ay), dn = (h ? q2.y : q2.x) * o;
                                v[5 * z] = fmaf(rn, rn, v[5 * z]);
                                v[5 * z + 1] = fmaf(dn, rn, v[5 * z + 1]);
                                v[5 * z + 2] = fmaf(ay, g, v[5 * z + 2]);
                                v[5 * z + 3] = fmaf(ay, dn, v[5 * z + 3]);
                                v[5 * z + 4] = fmaf(ay, rn, v[5 * z + 4]);
                            }
                        }
                    }
                    row_sums(v, 5 * ROWS);
#pragma unroll
                    for (int z = 0; z < ROWS; ++z)
#pragma unroll
                        for (int q = 0; q < ARRAYS; ++q) in[q][z].repack();
                    fs.repack();
                    fw.repack();
                    const bool has_do = a.in[3].p != nullptr;
#pragma unroll
                    for (int z = 0; z < ROWS; ++z) {
                        const float inv2 = has_do ? __frsqrt_rn(fmaf(v[5 * z], a.inv_d, a.eps)) : 0.f;
                        const float c3 = inv2 * inv2 * v[5 * z + 1] * a.inv_d;                     // inv2 * mean(dn * rh)
                        const float c4 = post ? (v[5 * z + 2] + inv2 * (v[5 * z + 3] - c3 * v[5 * z + 4])) * a.inv_d : 0.f;
                        Raw<T> xr, xy;
#pragma unroll
                        for (int p = 0; p < E / 2; ++p) {
                            const float2 y2 = in[0][z].pair(p), r2 = in[1][z].pair(p), g2 = in[2][z].pair(p), o2 = in[3][z].pair(p);
                            const float2 f2 = fs.pair(p), q2 = fw.pair(p);
                            float dr[2], dy[2];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const int e = 2 * p + h;
                                const float y = (h ? y2.y : y2.x) * inv1[z], r = h ? r2.y : r2.x, g = h ? g2.y : g2.x, o = h ? o2.y : o2.x;
                                const float f = h ? f2.y : f2.x;
                                const float rn = fmaf(f, r, fa[e] * y);
                                const float dR = has_do ? fmaf(inv2, fmaf(h ? q2.y : q2.x, o, -rn * c3), g) : g;
                                accC[e] = fmaf(dR, y, accC[e]);
                                accD[e] = fmaf(dR, r, accD[e]);
                                accW[e] = fmaf(o * inv2, rn, accW[e]);
                                dr[h] = f * dR;
                                dy[h] = inv1[z] * fmaf(fa[e], dR, -y * c4);
                            }
                            xr.set(p, dr[0], dr[1]);
                            xy.set(p, dy[0], dy[1]);
                        }
                        const int j = mine + z * each;
                        if (j < n) {
                            if (a.dr.p) xr.template store<VEC>(row_of<T>(a.dr, i, w.row + j) + c0, tpr, t, d);
                            if (a.dy.p) xy.template store<VEC>(row_of<T>(a.dy, i, w.row + j) + c0, tpr, t, d);
                        }
                    }
                }
                last = w.next();
                if (S == 1) fetch();
            }
            if constexpr (BWD) {
                // column sums of this replica: first the rows of a warp, then team after team
                for (int x = tpr; x < 32; x <<= 1) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        accC[e] += __shfl_xor_sync(0xffffffffu, accC[e], x);
                        accD[e] += __shfl_xor_sync(0xffffffffu, accD[e], x);
                        accW[e] += __shfl_xor_sync(0xffffffffu, accW[e], x);
                    }
                }
                float* out = a.partials + (long long)(i + b) * 3 * a.d + c0;
                for (int turn = 0; turn < teams; ++turn) {
                    if (turn == team && sub == 0) {
                        float* to = turn == teams - 1 ? out : s_sums;
                        const int step = turn == teams - 1 ? a.d : d;
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const int c = VEC > 1 ? (e / VEC * tpr + t) * VEC + e % VEC : e * tpr + t;
                            if (c >= d) continue;
                            to[c] = accC[e] + (turn ? s_sums[c] : 0.f);
                            to[step + c] = accD[e] + (turn ? s_sums[d + c] : 0.f);
                            to[2 * step + c] = accW[e] + (turn ? s_sums[2 * d + c] : 0.f);
                        }
                    }
                    if (teams > 1) op_named_barrier(15, nc);
                }
            }
        }
    }
    if (s_abort) {            // a wait ran out: the copies in flight get a millisecond to land
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) {}
    }
    // no CTA of a cluster ends while the other may still write to its shared memory
    if (C > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
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
cudaError_t few(const NormArgs& a, cudaStream_t stream) {
    const int tpr = threads_per_row(a.d, E), threads = tpr > kFewThreads ? tpr : kFewThreads / tpr * tpr;
    const int groups = threads / tpr;
    const long long W = (long long)a.P * a.rows, slots = (long long)sm_count() * (threads > 256 ? 2 : 4);
    if (slots < 1) return cudaErrorInvalidDevice;
    long long per = (W + slots - 1) / slots;
    per = (per + groups - 1) / groups * groups;
    k_norm_few<T, VEC, E><<<(unsigned)((W + per - 1) / per), threads, 0, stream>>>(a, tpr, per);
    return cudaGetLastError();
}

// Launches k_norm_stream; *G: its CTAs (clusters).
template <typename T, int VEC, bool BWD>
cudaError_t stream_rows(NormArgs a, int* G, cudaStream_t stream) {
    const long long W = (long long)a.P * a.rows;
    int sms = sm_count();
    if (sms < 1) return cudaErrorInvalidDevice;
    sms = sms > kMaxCtas ? kMaxCtas : sms;
    constexpr int ARRAYS = BWD ? 4 : 2;
    a.ctas = a.d <= kCtaWidth ? 1 : 2;
    a.cols = a.ctas == 1 ? a.d : ((a.d + 1) / 2 + 7) / 8 * 8;
    a.tpr = threads_per_row(a.cols, kElems);
    a.tpr = a.tpr < 16 ? 16 : a.tpr;                      // the ten sums of two rows are spread over sixteen lanes
    constexpr int ROWS = sizeof(T) == 2 ? 2 : 1;
    const int team = a.tpr < 32 ? 32 : a.tpr, rows = ROWS * (a.tpr < 32 ? 32 / a.tpr : 1), spots = sms / a.ctas;
    a.teams = kThreads / team;
    const long long need = (W + (long long)spots * rows - 1) / ((long long)spots * rows);
    if (a.teams > need) a.teams = (int)need;              // few rows: spread over the multiprocessors first
    a.slot_bytes = VEC > 1 ? a.cols * (int)sizeof(T) : (a.cols * (int)sizeof(T) + 30) / 16 * 16;
    const int sums = BWD && a.teams > 1 ? (3 * a.cols * 4 + 127) & ~127 : 0;
    const int stage = ARRAYS * a.teams * rows * a.slot_bytes;
    a.stages = (kSmemMax - 8192 - sums) / stage;
    a.stages = a.stages > kMaxStages ? kMaxStages : a.stages;
    if (a.stages < 1) return cudaErrorInvalidValue;
    const int smem = sums + a.stages * stage;
    const long long steps = (W + (long long)a.teams * rows - 1) / ((long long)a.teams * rows);
    *G = (int)(steps < spots ? steps : spots);
    const void* kernel = (const void*)k_norm_stream<T, VEC, BWD>;
    static bool raised[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !raised[dev]) {
        if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax - 8192)) != cudaSuccess) return e;
        if (dev < 64) raised[dev] = true;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(*G * a.ctas);
    cfg.blockDim = dim3(a.teams * team);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_norm_stream<T, VEC, BWD>, a);
}

// 16-byte accesses where every row allows them.
template <typename T> cudaError_t forward(const NormArgs& a, bool aligned, cudaStream_t stream) {
    constexpr int V = 16 / (int)sizeof(T);
    int G = 0;
    // few rows: below eight for every warp of the streaming kernel its ring hardly fills
    if ((long long)a.P * a.rows * ((a.d + 511) / 512) > 8ll * (kThreads / 32) * sm_count())
        return aligned ? stream_rows<T, V, false>(a, &G, stream) : stream_rows<T, 1, false>(a, &G, stream);
    if (a.d <= 2048) return aligned ? few<T, V, 8>(a, stream) : few<T, 1, 8>(a, stream);
    return aligned ? few<T, V, 16>(a, stream) : few<T, 1, 16>(a, stream);
}

template <typename T> cudaError_t backward(const NormArgs& a, bool aligned, const eg_residual_norm_args* q, cudaStream_t stream) {
    constexpr int V = 16 / (int)sizeof(T);
    int G = 0;
    if (a.rows > 0) {
        const cudaError_t e = aligned ? stream_rows<T, V, true>(a, &G, stream) : stream_rows<T, 1, true>(a, &G, stream);
        if (e != cudaSuccess) return e;
    }
    if (!q->d_w_post.data && !q->d_gate.data && !q->d_scale.data && !q->d_w_pre.data) return cudaSuccess;
    return launch_after(k_norm_columns<T>, dim3((a.d + 31) / 32, a.P), dim3(256), 0, stream, a, mat(q->d_w_post), mat(q->d_gate),
                        mat(q->d_scale), mat(q->d_w_pre), G);
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
    return (P + kMaxCtas) * 3 * width * (int64_t)sizeof(float);
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
    a.err = operator_error_word();
    if (!a.err) return EG_ERR_CUDA;
    const cudaError_t e = q->dtype == EG_F32    ? forward<float>(a, aligned, stream)
                          : q->dtype == EG_BF16 ? forward<__nv_bfloat16>(a, aligned, stream)
                                                : forward<__half>(a, aligned, stream);
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
    const cudaError_t e = q->dtype == EG_F32    ? backward<float>(a, aligned, q, stream)
                          : q->dtype == EG_BF16 ? backward<__nv_bfloat16>(a, aligned, q, stream)
                                                : backward<__half>(a, aligned, q, stream);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

}  // extern "C"
