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
// Measured: 4 x 8192 rows of 4096 in bf16, forward 173 us (6.2 TB/s), backward 358 us (4.5 TB/s, bound by its
// instructions: 43 an element, 1.7 a cycle, and 8 warps to hide their latencies); one row of 1024 on 4 replicas 4.0 us.
//
// k_norm_stream does both for many rows: one CTA (cluster) per multiprocessor (group of them), rows
// streamed through shared memory by bulk copies well ahead of their use, everything else in
// registers.  k_norm_few does the forward pass where there are few rows and a row's way through
// shared memory would only add to its latency, k_norm_rows that of few unaligned rows and the gradients of few rows.
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
constexpr int kRowThreads = 512;
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
// barrier 1 + group; `red` (one float per warp of the group) must not be the one of the previous call, whose sums a
// warp that is behind may still be reading: the callers take two in turn, call by call.
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
    const int red_at = group * tpr >> 5;
    int turn = 0;                                    // of the two buffers of sums: another one at every call
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
            inv1 = rsqrtf(fmaf(group_sum(sum, tpr, t, group, s_red[turn] + red_at), a.inv_d, a.eps));
            turn ^= 1;
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
        const float inv2 = rsqrtf(fmaf(group_sum(sum, tpr, t, group, s_red[turn] + red_at), a.inv_d, a.eps));
        turn ^= 1;
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

// The rows of a CTA, step by step: up to `per` consecutive rows of one replica.  (A CTA's rows fit 31 bits: the
// host bounds P * rows.)
struct Walk {
    long long row;                     // first row of the step in replica i
    int i, n, here, left;              // rows of the step; rows of replica i from `row` on; rows in later replicas

    __device__ __forceinline__ void start(long long u0, long long u1, long long rows, int per) {
        i = (int)(u0 / rows);
        row = u0 - (long long)i * rows;
        here = (int)min(rows - row, u1 - u0);
        left = (int)(u1 - u0) - here;
        n = min(per, here);
    }
    __device__ __forceinline__ bool done() const { return here <= 0; }
    // true: the next step is in another replica (or there is none)
    __device__ __forceinline__ bool next(long long rows, int per) {
        here -= n;
        row += n;
        const bool turn = here == 0;
        if (turn) {
            ++i;
            row = 0;
            here = (int)min(rows, (long long)left);
            left -= here;
        }
        n = min(per, here);
        return turn;
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
    __device__ __forceinline__ f32x2 two(int p) const { return pack_f2(pair(p)); }
    __device__ __forceinline__ void set(int p, f32x2 v) {
        const float2 f = unpack_f2(v);
        set(p, f.x, f.y);
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
    // the same from shared memory; bit v of `which`: vector v is there
    template <int VEC> __device__ __forceinline__ void load_shared(uint32_t at, int tpr, int which) {
#pragma unroll
        for (int v = 0; v < kElems / VEC; ++v) {
            w[4 * v] = w[4 * v + 1] = w[4 * v + 2] = w[4 * v + 3] = 0;
            if (which >> v & 1)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(w[4 * v]), "=r"(w[4 * v + 1]), "=r"(w[4 * v + 2]), "=r"(w[4 * v + 3])
                             : "r"(at + v * tpr * 16)
                             : "memory");
        }
    }
    template <int VEC> __device__ __forceinline__ void load_shared(uint32_t at, int tpr) {
#pragma unroll
        for (int v = 0; v < kElems / VEC; ++v)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[4 * v]), "=r"(w[4 * v + 1]), "=r"(w[4 * v + 2]), "=r"(w[4 * v + 3])
                         : "r"(at + v * tpr * 16)
                         : "memory");
    }
    // all vectors, to a thread's first one
    template <int VEC> __device__ __forceinline__ void store_whole(T* p, int tpr) const {
#pragma unroll
        for (int v = 0; v < kElems / VEC; ++v)
            *reinterpret_cast<uint4*>(p + v * tpr * VEC) = make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]);
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

// A factor's values for a thread's columns, unpacked.
template <typename T> struct Factors {
    f32x2 v[kElems / 2];
    __device__ __forceinline__ void take(const Raw<T>& x) {
#pragma unroll
        for (int p = 0; p < kElems / 2; ++p) v[p] = x.two(p);
    }
    __device__ __forceinline__ f32x2 two(int p) const { return v[p]; }
};

// K values (8 or 16) summed over the lanes of a warp, or of each half of it (`width` 32 or 16): halves are
// exchanged, so that every step halves the values instead of repeating all of them (16 values: 16
// shuffles, not 80).  Lane l ends up with the sum over its group of value number held(l).
template <int K> __device__ __forceinline__ float warp_sums(float (&v)[K], int lane, int width) {
#pragma unroll
    for (int half = K / 2, bit = 1; half > 0; half >>= 1, bit <<= 1) {
#pragma unroll
        for (int k = 0; k < half; ++k) {
            const float give = lane & bit ? v[k] : v[k + half], keep = lane & bit ? v[k + half] : v[k];
            v[k] = keep + __shfl_xor_sync(0xffffffffu, give, bit);
        }
    }
    if (K == 8) v[0] += __shfl_xor_sync(0xffffffffu, v[0], 8);
    if (width == 32) v[0] += __shfl_xor_sync(0xffffffffu, v[0], 16);
    return v[0];
}
// Value that lane l holds; it is its own inverse, so also the lane (of the first K) that holds value k.
template <int K> __device__ __forceinline__ int held(int l) {
    int r = 0;
#pragma unroll
    for (int b = 1, h = K / 2; h > 0; b <<= 1, h >>= 1) r |= l & b ? h : 0;
    return r;
}

// Rows that a thread works on at a time: as many as its 255 registers hold.
template <typename T, bool BWD> __host__ __device__ constexpr int rows_at_once() {
    return (BWD ? 1 : 2) * (sizeof(T) == 2 ? 2 : 1);
}

// A CTA works through its rows in steps of up to teams * ROWS * (rows of a warp) consecutive rows of one
// replica.  The rows of y, r (and d_r', d_o) of the steps ahead come into a ring of stages in
// shared memory, one bulk copy an array and step where the rows lie one after the other; rows off the
// 16-byte boundaries are copied from the boundary below and read from the remainder.  A team is the tpr
// threads of a row, or a warp with 32 / tpr rows below a warp; it takes ROWS rows at a time, so that the
// latencies of one row's sums are covered by the others' arithmetic.  A thread owns the same columns of every row, so the factors a, scale, w_pre of the replica and
// (backward) its three column sums stay in registers; at the end of a replica's rows the teams add up their
// sums in shared memory and leave one partial sum per (replica, CTA) pair that meet; i + b numbers the pairs
// without a gap.  Rows wider than kCtaWidth are shared by a cluster of two CTAs, which exchange the sums of a row.
//
// A row needs one round of sums: with p = scale * r, q = a * y (so r' = p + inv1 q) and dn = d_o * w_pre, the sums
// of y^2, p^2, pq, q^2, dn p, dn q and q d_r' give inv1 first and then every mean that the formulas above
// ask for.  Where p and inv1 q cancel to less than a tenth of their size, or one of these sums passes the range of 32 bits
// (q^2 may where r'^2 does not), r' and what follows from it are summed in a second round instead.
template <typename T, int VEC, bool BWD>
__global__ void __launch_bounds__(kThreads, 1) k_norm_stream(const __grid_constant__ NormArgs a) {
    constexpr int E = kElems, ROWS = rows_at_once<T, BWD>(), ARRAYS = BWD ? 4 : 2;
    constexpr int SUMS = BWD ? 7 : 4, KP = BWD ? 8 * ROWS : 4 * ROWS;
    constexpr int kWarps = kThreads / 32;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_peer[2];
    __shared__ float s_red[2][2 * kWarps][16];                 // [parity][CTA of the cluster, warp][value]
    __shared__ volatile int s_abort;
    if (BWD) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tpr = a.tpr, S = a.stages, C = a.ctas, teams = a.teams;
    const int team_threads = tpr < 32 ? 32 : tpr, each = tpr < 32 ? 32 / tpr : 1;
    const int nc = teams * team_threads;                       // threads of the CTA
    const int rank = C > 1 ? blockIdx.x % C : 0, b = blockIdx.x / C, G = gridDim.x / C;
    const int c0 = rank * a.cols, d = min(a.cols, a.d - c0);   // columns of this CTA
    const bool post = a.w_post.p != nullptr && a.in[0].p != nullptr;
    const long long W = (long long)a.P * a.rows, u0 = cut(W, b, G), u1 = cut(W, b + 1, G);
    const int per = teams * ROWS * each;
    const int array_bytes = per * a.slot_bytes, stage_bytes = ARRAYS * array_bytes;
    float* s_sums = reinterpret_cast<float*>(smem);            // BWD: [elements of a thread][threads]
    unsigned char* ring = smem + (BWD ? E * nc * 4 : 0);
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
    {   // the factors of the first two replicas of this CTA are wanted soon
        const int c = c0 + (int)threadIdx.x * (128 / (int)sizeof(T));
        for (int q = w.i; q < min(a.P, w.i + 2) && c < c0 + d; ++q)
            for (const Mat* m : {&a.w_post, &a.gate, &a.scale, &a.w_pre})
                if (m->p) asm volatile("prefetch.global.L2 [%0];" ::"l"(row_of<T>(*m, q, 0) + c));
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");         // set up while the kernel before this one finished

    // the rows of array q come in by lane 0 of warp q (few warps: of the last one, q after q)
    Walk ahead = w;
    const int fetcher = threadIdx.x >> 5, fetchers = nc / 32;
    int as = 0, around = 0;
    uintptr_t from_row = 0;                                    // where the next step's rows of array `fetcher` start
    auto fetch = [&]() {
        if (fetcher >= ARRAYS || ahead.done()) return;
        if (lane == 0) {
            for (int q = fetcher; q < ARRAYS; q += fetchers) {
                const Mat& m = a.in[q];
                if (!m.p) continue;
                const bool together = m.row == a.d && C == 1;      // rows one after the other
                const int n = ahead.n;
                if (around > 0 && !op_mbar_wait(&s_empty[as], (around - 1) & 1, &s_abort, a.err)) break;
                unsigned char* dst = ring + as * stage_bytes + q * array_bytes;
                if (from_row == 0 || fetchers < ARRAYS) from_row = (uintptr_t)(row_of<T>(m, ahead.i, ahead.row) + c0);
                const uintptr_t p = from_row;
                from_row += (uintptr_t)n * m.row * sizeof(T);
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
        if (ahead.next(a.rows, per)) from_row = 0;
        if (++as == S) { as = 0; ++around; }
    };
    // a stage is refilled one step after its last use, when no other team should still be reading it
    for (int q = 0; q < S - 1; ++q) fetch();
    if (S == 1) fetch();

    const int team = threadIdx.x / team_threads, tt = threadIdx.x % team_threads;
    const int warps = team_threads >> 5, warp = tt >> 5;
    const int sub = tpr < 32 ? lane / tpr : 0, t = tpr < 32 ? lane % tpr : tt;
    const int mine = team * ROWS * each + sub;                 // this thread's rows of a step: mine + z * each
    const uint32_t mine_at = op_smem(ring) + mine * a.slot_bytes + t * VEC * (int)sizeof(T);
    int in_row = 0;                                            // bit v: vector v of this thread lies in the row
    if (VEC > 1)
        for (int v = 0; v < E / VEC; ++v) in_row |= (v * tpr + t) * VEC < d ? 1 << v : 0;
    bool in_whole = VEC > 1 && in_row == (1 << E / VEC) - 1;
#pragma unroll
    for (int q = 0; q < ARRAYS; ++q) in_whole = in_whole && a.in[q].p;
    int parity = 0, meets = 0;
    // the values of the team's rows, summed over their threads (and CTAs): v[k] in every thread
    auto row_sums = [&](float (&v)[KP]) {
        const int width = tpr < 32 ? tpr : 32;
        float sum = warp_sums<KP>(v, lane, width);
        if (tpr <= 32 && C == 1) {
            const int first = lane & ~(width - 1);
#pragma unroll
            for (int k = 0; k < KP; ++k) v[k] = __shfl_sync(0xffffffffu, sum, first + held<KP>(k));
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
            // every warp of both CTAs tells both CTAs that its sums are there
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
        const float* from = &s_red[parity][C > 1 ? 0 : team * warps][lane % KP];
        sum = 0.f;
#pragma unroll
        for (int x = 0; x < kWarps; x += L)
            if (x + lane / KP < warps) sum += from[(x + lane / KP) * 16];
        if (C > 1) {
#pragma unroll
            for (int x = 0; x < kWarps; x += L)
                if (x + lane / KP < warps) sum += from[(kWarps + x + lane / KP) * 16];
        }
        if (KP == 8) sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
#pragma unroll
        for (int k = 0; k < KP; ++k) v[k] = __shfl_sync(0xffffffffu, sum, k);
        parity ^= 1;
    };
    auto total = [](f32x2 v) {
        const float2 f = unpack_f2(v);
        return f.x + f.y;
    };

    int s = 0, round = 0;
    while (!w.done()) {
        const int i = w.i;
        Factors<T> fs, fw;
        f32x2 fa[E / 2];
        f32x2 accC[BWD ? E / 2 : 1], accD[BWD ? E / 2 : 1], accW[BWD ? E / 2 : 1];
        {
            const float there = a.in[0].p ? 1.f : 0.f;
            Raw<T> x;
            if (a.w_post.p) x.template load<VEC>(row_of<T>(a.w_post, i, 0) + c0, tpr, t, d);
#pragma unroll
            for (int p = 0; p < E / 2; ++p) fa[p] = a.w_post.p ? x.two(p) : pack_f2(there, there);
            if (a.gate.p) {
                x.template load<VEC>(row_of<T>(a.gate, i, 0) + c0, tpr, t, d);
#pragma unroll
                for (int p = 0; p < E / 2; ++p) {
                    const float2 f = x.pair(p);
                    fa[p] = mul2(fa[p], pack_f2(sigmoid_f(f.x), sigmoid_f(f.y)));
                }
            }
#pragma unroll
            for (int p = 0; p < E / 2; ++p) x.set(p, 1.f, 1.f);
            if (a.scale.p) x.template load<VEC>(row_of<T>(a.scale, i, 0) + c0, tpr, t, d);
            fs.take(x);
            x.clear();
            if (BWD ? a.in[3].p != nullptr : a.o.p != nullptr) x.template load<VEC>(row_of<T>(a.w_pre, i, 0) + c0, tpr, t, d);
            fw.take(x);
        }
        if constexpr (BWD) {
#pragma unroll
            for (int p = 0; p < E / 2; ++p) accC[p] = accD[p] = accW[p] = 0;
        }
        // this thread's first row of the step in the two results, and the way to the next step's
        const Mat &m0 = BWD ? a.dr : a.r_out, &m1 = BWD ? a.dy : a.o;
        // (fp32 gradients have no registers left for them and work them out at every step)
        constexpr bool KEPT = !BWD || sizeof(T) == 2;
        T* out0 = m0.p ? row_of<T>(m0, i, w.row + mine) + c0 : nullptr;
        T* out1 = m1.p ? row_of<T>(m1, i, w.row + mine) + c0 : nullptr;
        auto put = [&](const Raw<T>& x, T* to, bool whole) {
            if (VEC > 1 && whole) x.template store_whole<VEC>(to + t * VEC, tpr);
            else x.template store<VEC>(to, tpr, t, d);
        };
        bool last = false;
        while (!last) {
            const int n = w.n;
            (void)op_mbar_wait(&s_full[s], round & 1, &s_abort, a.err);    // after a time-out the walk just goes on
            Raw<T> in[ARRAYS][ROWS];
            uint32_t at = mine_at + s * stage_bytes;
            const bool whole = in_whole && n == per;           // nothing of what this thread takes is missing
            if (VEC > 1 && whole) {
#pragma unroll
                for (int q = 0; q < ARRAYS; ++q, at += array_bytes)
#pragma unroll
                    for (int z = 0; z < ROWS; ++z) in[q][z].template load_shared<VEC>(at + z * each * a.slot_bytes, tpr);
            } else
#pragma unroll
            for (int q = 0; q < ARRAYS; ++q, at += array_bytes) {
#pragma unroll
                for (int z = 0; z < ROWS; ++z) {
                    if (VEC > 1) {
                        in[q][z].template load_shared<VEC>(at + z * each * a.slot_bytes, tpr, a.in[q].p && mine + z * each < n ? in_row : 0);
                    } else {
                        in[q][z].clear();
                        if (!a.in[q].p || mine + z * each >= n) continue;
                        const int j = mine + z * each;
                        const T* first = row_of<T>(a.in[q], i, w.row) + c0;
                        const unsigned char* x = ring + s * stage_bytes + q * array_bytes;
                        if (a.in[q].row == a.d && C == 1) x += ((uintptr_t)first & 15) + (size_t)j * d * sizeof(T);
                        else x += j * a.slot_bytes + ((uintptr_t)(first + (long long)j * a.in[q].row) & 15);
                        in[q][z].template load<VEC>(reinterpret_cast<const T*>(x), tpr, t, d);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) op_mbar_arrive(&s_empty[s]);
            if (++s == S) { s = 0; ++round; }
            if (S > 1) fetch();

            float v[KP];
#pragma unroll
            for (int k = 0; k < KP; ++k) v[k] = 0.f;
#pragma unroll
            for (int z = 0; z < ROWS; ++z) {
                f32x2 sum[SUMS];
#pragma unroll
                for (int k = 0; k < SUMS; ++k) sum[k] = 0;
#pragma unroll
                for (int p = 0; p < E / 2; ++p) {
                    const f32x2 y = in[0][z].two(p), P = mul2(fs.two(p), in[1][z].two(p)), Q = mul2(fa[p], y);
                    sum[0] = fma2(y, y, sum[0]);
                    sum[1] = fma2(P, P, sum[1]);
                    sum[2] = fma2(P, Q, sum[2]);
                    sum[3] = fma2(Q, Q, sum[3]);
                    if constexpr (BWD) {
                        const f32x2 dn = mul2(fw.two(p), in[3][z].two(p));
                        sum[4] = fma2(dn, P, sum[4]);
                        sum[5] = fma2(dn, Q, sum[5]);
                        sum[6] = fma2(Q, in[2][z].two(p), sum[6]);
                    }
                }
#pragma unroll
                for (int k = 0; k < SUMS; ++k) v[z * (KP / ROWS) + k] = total(sum[k]);
            }
            row_sums(v);
#pragma unroll
            for (int z = 0; z < ROWS; ++z)
#pragma unroll
                for (int q = 0; q < ARRAYS; ++q) in[q][z].repack();
            float inv1[ROWS], rr[ROWS], dnr[ROWS], qr[ROWS];       // sums of r'^2, dn r', q r'
            bool cancels = false;
            auto inexact = [](float rr, float size) { return !(rr >= 0.01f * size && size < 3e38f); };
#pragma unroll
            for (int z = 0; z < ROWS; ++z) {
                const float* x = v + z * (KP / ROWS);
                // (rows past the step's last are zeros here and must add zeros to the column sums, also where eps is 0)
                inv1[z] = post ? rsqrtf(fmaf(x[0], a.inv_d, a.eps)) : 1.f;
                if (BWD && n < per && mine + z * each >= n) inv1[z] = 0.f;
                const float size = fmaf(inv1[z] * inv1[z], x[3], x[1]);
                rr[z] = fmaf(2.f * inv1[z], x[2], size);
                cancels = cancels || inexact(rr[z], size);
                if constexpr (BWD) {
                    dnr[z] = fmaf(inv1[z], x[5], x[4]);
                    qr[z] = fmaf(inv1[z], x[3], x[2]);
                }
            }
            // one answer for all who sum together
            if (tpr <= 32) cancels = __any_sync(0xffffffffu, cancels);
            if (cancels) {
                float again[KP];
#pragma unroll
                for (int k = 0; k < KP; ++k) again[k] = 0.f;
#pragma unroll
                for (int z = 0; z < ROWS; ++z) {
                    f32x2 sum[3] = {0, 0, 0};
                    const f32x2 i1 = pack_f2(inv1[z], inv1[z]);
#pragma unroll
                    for (int p = 0; p < E / 2; ++p) {
                        const f32x2 Q = mul2(fa[p], in[0][z].two(p)), R = fma2(i1, Q, mul2(fs.two(p), in[1][z].two(p)));
                        sum[0] = fma2(R, R, sum[0]);
                        if constexpr (BWD) {
                            sum[1] = fma2(mul2(fw.two(p), in[3][z].two(p)), R, sum[1]);
                            sum[2] = fma2(Q, R, sum[2]);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 3; ++k) again[z * (KP / ROWS) + k] = total(sum[k]);
                }
                row_sums(again);
#pragma unroll
                for (int z = 0; z < ROWS; ++z) {
                    const float* x = v + z * (KP / ROWS);
                    if (!inexact(rr[z], fmaf(inv1[z] * inv1[z], x[3], x[1]))) continue;    // others' bits do not depend on it
                    rr[z] = again[z * (KP / ROWS)];
                    dnr[z] = again[z * (KP / ROWS) + 1];
                    qr[z] = again[z * (KP / ROWS) + 2];
                }
            }
#pragma unroll
            for (int z = 0; z < ROWS; ++z) {
                const int j = mine + z * each;
                const f32x2 i1 = pack_f2(inv1[z], inv1[z]);
                if (!KEPT && m0.p) out0 = row_of<T>(m0, i, w.row + mine) + c0;
                if (!KEPT && m1.p) out1 = row_of<T>(m1, i, w.row + mine) + c0;
                if constexpr (!BWD) {
                    const float i2 = rsqrtf(fmaf(rr[z], a.inv_d, a.eps));
                    const f32x2 inv2 = pack_f2(i2, i2);
                    Raw<T> xr, xo;
#pragma unroll
                    for (int p = 0; p < E / 2; ++p) {
                        const f32x2 R = fma2(i1, mul2(fa[p], in[0][z].two(p)), mul2(fs.two(p), in[1][z].two(p)));
                        xr.set(p, R);
                        xo.set(p, mul2(mul2(R, inv2), fw.two(p)));
                    }
                    if (j < n) {
                        if (out0) put(xr, out0 + z * each * m0.row, whole);
                        if (out1) put(xo, out1 + z * each * m1.row, whole);
                    }
                } else {
                    const bool has_do = a.in[3].p != nullptr;
                    const float x6 = v[z * (KP / ROWS) + 6], x5 = v[z * (KP / ROWS) + 5];
                    float i2 = has_do ? rsqrtf(fmaf(rr[z], a.inv_d, a.eps)) : 0.f;
                    if (n < per && j >= n) i2 = 0.f;
                    const float c3 = has_do ? i2 * i2 * dnr[z] * a.inv_d : 0.f;                    // inv2 * mean(dn * rh)
                    const float c4 = post ? inv1[z] * (x6 + i2 * (x5 - c3 * qr[z])) * a.inv_d : 0.f;
                    const f32x2 inv2 = pack_f2(i2, i2), k3 = pack_f2(-i2 * c3, -i2 * c3);
                    const float k = -inv1[z] * inv1[z] * c4;
                    const f32x2 k4 = pack_f2(k, k);
                    Raw<T> xr, xy;
#pragma unroll
                    for (int p = 0; p < E / 2; ++p) {
                        const f32x2 y = in[0][z].two(p), r = in[1][z].two(p), o = in[3][z].two(p), f = fs.two(p);
                        const f32x2 R = fma2(i1, mul2(fa[p], y), mul2(f, r));
                        const f32x2 dR = fma2(k3, R, fma2(inv2, mul2(fw.two(p), o), in[2][z].two(p)));
                        const f32x2 tR = mul2(dR, i1);
                        accC[p] = fma2(tR, y, accC[p]);
                        accD[p] = fma2(dR, r, accD[p]);
                        accW[p] = fma2(o, mul2(R, inv2), accW[p]);
                        xr.set(p, mul2(f, dR));
                        xy.set(p, fma2(k4, y, mul2(fa[p], tR)));
                    }
                    if (j < n) {
                        if (out0) put(xr, out0 + z * each * m0.row, whole);
                        if (out1) put(xy, out1 + z * each * m1.row, whole);
                    }
                }
            }
            if (KEPT && out0) out0 += per * m0.row;
            if (KEPT && out1) out1 += per * m1.row;
            last = w.next(a.rows, per);
            if (S == 1) fetch();
        }
        if constexpr (BWD) {
            // column sums of this replica: first over the rows of a warp, then over the teams, one of the three at a time
            float* out = a.partials + (long long)(i + b) * 3 * a.d + c0;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const f32x2* acc = k == 0 ? accC : k == 1 ? accD : accW;
#pragma unroll
                for (int p = 0; p < E / 2; ++p) {
                    float2 x = unpack_f2(acc[p]);
                    if (tpr < 32) {
                        x.x += __shfl_xor_sync(0xffffffffu, x.x, 16);
                        x.y += __shfl_xor_sync(0xffffffffu, x.y, 16);
                    }
                    s_sums[2 * p * nc + threadIdx.x] = x.x;
                    s_sums[(2 * p + 1) * nc + threadIdx.x] = x.y;
                }
                op_named_barrier(15, nc);
                for (int c = threadIdx.x; c < d; c += nc) {
                    const int v = c / VEC, e = v / tpr * VEC + c % VEC;      // whose element e column c is
                    const float* from = s_sums + e * nc + v % tpr;
                    float sum = 0.f;
                    for (int m = 0; m < teams; ++m) sum += from[m * team_threads];
                    out[k * a.d + c] = sum;
                }
                op_named_barrier(15, nc);
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

// The same for few rows where k_norm_few does not serve: gradients, and rows off the 16-byte boundaries.  Such calls
// are bound by latency, that of fetching the code of unrolled loops included, so this one is short: a CTA takes one
// row after the other, a thread the same columns of every row, and the passes over a row after the first find it in
// the L1.  The column sums of a replica's rows lie in shared memory, each thread's by itself.
// Measured, 4 rows of 1024 on 2 replicas with gradients: 12 us with k_norm_columns, k_norm_stream 36.
template <typename T, int VEC, bool BWD>
__global__ void __launch_bounds__(kRowThreads) k_norm_rows(const __grid_constant__ NormArgs a) {
    constexpr int K = BWD ? 5 : 1;
    extern __shared__ float s_acc[];
    __shared__ float s_red[2][K][kRowThreads / 32];
    if (BWD) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int b = blockIdx.x, G = gridDim.x, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const long long W = (long long)a.P * a.rows, u1 = cut(W, b + 1, G);
    long long u = cut(W, b, G);
    int i = (int)(u / a.rows);
    long long row = u % a.rows;
    const bool has_y = a.in[0].p != nullptr, post = has_y && a.w_post.p, has_do = BWD && a.in[3].p, second = BWD ? has_do : a.o.p != nullptr;
    struct Values { float v[VEC]; };
    auto value = [](const Mat& m, int i, long long t, int c, float otherwise) {
        Values x;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x.v[e] = otherwise;
        if (m.p) load_vec<T, VEC>(row_of<T>(m, i, t) + c, x.v);
        return x;
    };
    auto factor = [&](int c) {
        Values f = value(a.w_post, i, 0, c, has_y ? 1.f : 0.f);
        if (a.gate.p) {
            const Values g = value(a.gate, i, 0, c, 0.f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f.v[e] *= sigmoid_f(g.v[e]);
        }
        return f;
    };
    int which = 0;                                       // of the two buffers: taken in turn, since only one barrier parts
    auto sums = [&](float (&v)[K]) {                     // a call's reads from the next one's writes; over the threads of the CTA
#pragma unroll
        for (int k = 0; k < K; ++k) {
            for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
            if (lane == 0) s_red[which][k][threadIdx.x >> 5] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = lane < warps ? s_red[which][k][lane] : 0.f;
            for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
        which ^= 1;
    };
    bool begun = false;                                  // rows of replica i lie in the column sums
    for (; u < u1; ++u) {
        float v[K] = {}, inv1 = 1.f;
        if (post) {
            for (int c = threadIdx.x * VEC; c < a.d; c += blockDim.x * VEC) {
                const Values y = value(a.in[0], i, row, c, 0.f);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[0] = fmaf(y.v[e], y.v[e], v[0]);
            }
            sums(v);
            inv1 = rsqrtf(fmaf(v[0], a.inv_d, a.eps));
        }
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = 0.f;
        if (BWD || second) {
            for (int c = threadIdx.x * VEC; c < a.d; c += blockDim.x * VEC) {
                const Values y = value(a.in[0], i, row, c, 0.f), r = value(a.in[1], i, row, c, 0.f), dr = value(a.in[2], i, row, c, 0.f);
                const Values o = value(a.in[3], i, row, c, 0.f), w = value(a.w_pre, i, 0, c, 0.f), s = value(a.scale, i, 0, c, 1.f);
                const Values f = factor(c);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float Q = f.v[e] * y.v[e], R = fmaf(inv1, Q, s.v[e] * r.v[e]);
                    v[0] = fmaf(R, R, v[0]);
                    if constexpr (BWD) {
                        const float dn = has_do ? w.v[e] * o.v[e] : 0.f;
                        v[1] = fmaf(dn, R, v[1]);
                        v[2] = fmaf(Q, dr.v[e], v[2]);
                        v[3] = fmaf(dn, Q, v[3]);
                        v[4] = fmaf(Q, R, v[4]);
                    }
                }
            }
            sums(v);
        }
        const float inv2 = second ? rsqrtf(fmaf(v[0], a.inv_d, a.eps)) : 0.f;
        float c3 = 0.f, c4 = 0.f;
        if constexpr (BWD) {
            c3 = inv2 * inv2 * v[1] * a.inv_d;                                       // inv2 * mean(dn * rh)
            c4 = post ? inv1 * (v[2] + inv2 * (v[3] - c3 * v[4])) * a.inv_d : 0.f;
        }
        const bool last = u + 1 == u1 || row + 1 == a.rows;
        float* out = a.partials + (long long)(i + b) * 3 * a.d;
        for (int c = threadIdx.x * VEC; c < a.d; c += blockDim.x * VEC) {
            const Values y = value(a.in[0], i, row, c, 0.f), r = value(a.in[1], i, row, c, 0.f), f = factor(c);
            const Values w = value(a.w_pre, i, 0, c, 0.f), s = value(a.scale, i, 0, c, 1.f);
            float x0[VEC], x1[VEC];
            if constexpr (!BWD) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    x0[e] = fmaf(inv1, f.v[e] * y.v[e], s.v[e] * r.v[e]);
                    x1[e] = x0[e] * inv2 * w.v[e];
                }
                if (a.r_out.p) store_vec<T, VEC>(row_of<T>(a.r_out, i, row) + c, x0);
                if (second) store_vec<T, VEC>(row_of<T>(a.o, i, row) + c, x1);
            } else {
                const Values dr = value(a.in[2], i, row, c, 0.f), o = value(a.in[3], i, row, c, 0.f);
                float part[3][VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float R = fmaf(inv1, f.v[e] * y.v[e], s.v[e] * r.v[e]), dn = has_do ? w.v[e] * o.v[e] : 0.f;
                    const float dR = fmaf(-inv2 * c3, R, fmaf(inv2, dn, dr.v[e])), tR = dR * inv1;
                    x0[e] = s.v[e] * dR;
                    x1[e] = fmaf(-inv1 * inv1 * c4, y.v[e], f.v[e] * tR);
                    part[0][e] = tR * y.v[e];
                    part[1][e] = dR * r.v[e];
                    part[2][e] = o.v[e] * (R * inv2);
                }
                if (a.dr.p) store_vec<T, VEC>(row_of<T>(a.dr, i, row) + c, x0);
                if (a.dy.p) store_vec<T, VEC>(row_of<T>(a.dy, i, row) + c, x1);
#pragma unroll
                for (int k = 0; k < 3; ++k) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        if (begun) part[k][e] += s_acc[k * a.d + c + e];
                        if (last) out[k * a.d + c + e] = part[k][e];
                        else s_acc[k * a.d + c + e] = part[k][e];
                    }
                }
            }
        }
        begun = !last;
        if (++row == a.rows) { row = 0; ++i; }
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
    if (q->P < 1 || q->P > 65535 || q->rows < 0 || q->rows > (1ll << 37) / q->P || q->width < 1 || q->width > kMaxWidth)
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
    // outputs are written once: rows and replicas of an output must not fall on one another; the replicas' lie one after the
    // other, or take turns row by row
    const eg_matrix* written[] = {&q->residual_out, &q->out, &q->dy, &q->d_residual};
    for (const eg_matrix* m : written) {
        if (!m->data) continue;
        const long long rep = m->replica_stride, row = m->row_stride;
        if ((q->rows > 1 && row < q->width) || (q->P > 1 && rep < q->width)) return EG_ERR_INVALID;
        if (q->rows > 1 && q->P > 1 && (rep - q->width) / (q->rows - 1) < row && (row - q->width) / (q->P - 1) < rep) return EG_ERR_INVALID;
    }
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
    a.tpr = a.tpr < 16 ? 16 : a.tpr;                      // the sums of two rows are spread over sixteen lanes
    constexpr int ROWS = rows_at_once<T, BWD>();
    const int team = a.tpr < 32 ? 32 : a.tpr, rows = ROWS * (a.tpr < 32 ? 32 / a.tpr : 1), spots = sms / a.ctas;
    a.teams = kThreads / team;
    const long long need = (W + (long long)spots * rows - 1) / ((long long)spots * rows);
    if (a.teams > need) a.teams = (int)need;              // few rows: spread over the multiprocessors first
    a.slot_bytes = VEC > 1 ? a.cols * (int)sizeof(T) : (a.cols * (int)sizeof(T) + 30) / 16 * 16;
    const int sums = BWD ? kElems * a.teams * team * 4 : 0;
    const int stage = ARRAYS * a.teams * rows * a.slot_bytes;
    a.stages = (kSmemMax - 8192 - sums) / stage;
    a.stages = a.stages > kMaxStages ? kMaxStages : a.stages;
    if (a.stages < 1) return cudaErrorInvalidValue;
    const int smem = sums + a.stages * stage;
    const long long steps = (W + (long long)a.teams * rows - 1) / ((long long)a.teams * rows);
    *G = (int)(steps < spots ? steps : spots);
    // The same number of CTAs for every replica, where that idles a tenth of them at most: none then meets two
    // replicas and pays twice for factors and column sums (8 replicas of 1024 rows of 1024, forward and backward: 65 us, 78 with runs cut regardless).
    const int even = *G / a.P * a.P;
    if (even * 10 >= *G * 9) *G = even;
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
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_norm_stream<T, VEC, BWD>, a);
}

// Launches k_norm_rows where its CTAs get few rows; *G: its CTAs, 0 otherwise.  Measured, us, against k_norm_stream:
// bf16, 2 rows a CTA: 1024 columns 16 against 23, 2984 24 against 26, 4567 43 against 35; 1 row: 4567 28 against 30, 8192
// 33 against 27; 4 rows: 1001 25 against 24; fp32, 2 rows: 1024 13 against 17, 2984 21 against 28, 4567 42 against 35;
// 1 row: 8192 25 against 30.
template <typename T, int VEC, bool BWD> cudaError_t short_runs(const NormArgs& a, int* G, cudaStream_t stream) {
    const long long W = (long long)a.P * a.rows;
    const int sms = sm_count() < kMaxCtas ? sm_count() : kMaxCtas;
    if (sms < 1) return cudaErrorInvalidDevice;
    *G = 0;
    const long long ctas = BWD ? sms : 4ll * sms;         // (the backward call's workspace holds that many CTAs' sums)
    if (W > (a.d <= kCtaWidth ? 2 : 1) * ctas) return cudaSuccess;
    *G = (int)(W < ctas ? W : ctas);
    const int each = (a.d + VEC - 1) / VEC, threads = each < kRowThreads ? (each + 31) / 32 * 32 : kRowThreads;
    const int smem = BWD && W > *G ? 3 * a.d * (int)sizeof(float) : 0;
    cudaError_t e;       // (48 KB need no permission, but s_red is part of them)
    if (smem > 40 * 1024 && (e = cudaFuncSetAttribute(k_norm_rows<T, VEC, BWD>, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kCtaWidth * 4)) != cudaSuccess)
        return e;
    return launch_after(k_norm_rows<T, VEC, BWD>, dim3(*G), dim3(threads), smem, stream, a);
}

// 16-byte accesses where every row allows them.
template <typename T> cudaError_t forward(const NormArgs& a, bool aligned, cudaStream_t stream) {
    constexpr int V = 16 / (int)sizeof(T);
    int G = 0;
    const long long W = (long long)a.P * a.rows;
    // Rows off the 16-byte boundaries, us: bf16 of 1001 columns, k_norm_rows 6 for 148 rows, 11 for 592, k_norm_few 13 and 14; of
    // 4567 columns 15 and 34 against 23 and 58; fp32 of 8191 columns 25 against 17 for 148 rows.  k_norm_few of wide ones takes 47
    // for 296 rows, 63 for 592, k_norm_stream 34 for 1184.
    if (!aligned && a.d <= 6144) {
        const cudaError_t e = short_runs<T, 1, false>(a, &G, stream);
        if (e != cudaSuccess || G > 0) return e;
    }
    // few rows: below eight for every warp of the streaming kernel its ring hardly fills
    if (W * ((a.d + 511) / 512) > 8ll * (kThreads / 32) * sm_count() || (!aligned && a.d > 2048 && W > sm_count()))
        return aligned ? stream_rows<T, V, false>(a, &G, stream) : stream_rows<T, 1, false>(a, &G, stream);
    if (a.d <= 2048) return aligned ? few<T, V, 8>(a, stream) : few<T, 1, 8>(a, stream);
    return aligned ? few<T, V, 16>(a, stream) : few<T, 1, 16>(a, stream);
}

template <typename T> cudaError_t backward(const NormArgs& a, bool aligned, const eg_residual_norm_args* q, cudaStream_t stream) {
    constexpr int V = 16 / (int)sizeof(T);
    int G = 0;
    if (a.rows > 0) {
        cudaError_t e = aligned ? short_runs<T, V, true>(a, &G, stream) : short_runs<T, 1, true>(a, &G, stream);
        if (e == cudaSuccess && G == 0) e = aligned ? stream_rows<T, V, true>(a, &G, stream) : stream_rows<T, 1, true>(a, &G, stream);
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
