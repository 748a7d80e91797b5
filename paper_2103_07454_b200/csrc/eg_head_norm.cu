// The norm of every head of the queries and keys with the rotation by position (eg_head_norm) and its gradients.
//
//   forward   xh = x * inv,  inv = 1 / sqrt(mean(x^2) + eps);   z = xh * w;   o = R z
//             R turns the pair (z_a, z_b) of pair j by position * base^(-2 j / rotary):
//             o_a = z_a cos - z_b sin,  o_b = z_a sin + z_b cos
//   backward  dz = R^T do;   dw = sum dz * xh;   dx = inv * (dz * w - xh * mean(dz * w * xh))
//
// Bound by memory: forward moves a value in and out, backward two in and one out (nothing is saved between them).
//
// A head's row is small, so a few threads share it, each with whole pairs: a "slot" is two vectors of VEC values whose
// elements are partners (halves: j and j + rotary / 2; neighbours: inside either vector).  A CTA takes a few places of one replica
// at a time and forms their cosines and sines once, in shared memory, for all heads of the queries and keys: a sine costs
// some forty instructions, a value of a row about four.  An angle is reduced in 64 bits, where positions of any
// size keep their fraction of a turn, and only the fraction goes on in 32.
#include <type_traits>

#include "eg_ops.cuh"

namespace eg {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxWidth = EG_HEAD_MAX_WIDTH, kMaxPairs = kMaxWidth / 2;
constexpr int kMaxTile = 16;                // places whose angles a CTA holds
constexpr int kTableMax = 2048;             // cosines and sines that it holds
constexpr int kCtasPerSm = 4;

struct Heads {
    void* p;
    long long rep, row, head;               // strides in elements
};
struct Vec {
    void* p;
    long long rep;
};

struct HeadArgs {
    int P;
    long long n;
    int d, rotary, half;                    // half: pairs that turn
    int interleaved;
    float eps, inv_d;
    const void* positions;                  // nullptr: 0, 1, ...
    long long pos_rep, pos_step;
    int wide;
    int tile;                               // places at a time
    int table;                              // pairs of the table (neighbours: all of a row's, those that stay with cosine 1)
    int slots, team, ctas;                  // of a row; threads of a row; CTAs of a replica
    int heads[2];                           // of the queries, of the keys
    Heads x[2], out[2], d_out[2];           // forward: x, out; backward: x, d_out and in out the gradient of x
    Vec w[2];
    float* partial;                         // [P][ctas][2][d] sums of dz * xh
    double turns[kMaxPairs];                // turns of pair j per place
};

template <typename T> __device__ __forceinline__ T* head_at(const Heads& m, int i, long long t, int h) {
    return static_cast<T*>(m.p) + (long long)i * m.rep + t * m.row + (long long)h * m.head;
}

// Where the two vectors of slot s begin, and whether they are there.
template <int VEC> __device__ __forceinline__ void slot_place(const HeadArgs& a, int s, int& first, int& second, bool& turned) {
    if (a.interleaved) {
        first = 2 * s * VEC;
        second = first + VEC;
        turned = true;
    } else {
        const int lead = a.half / VEC;                       // slots that turn
        turned = s < lead;
        first = turned ? s * VEC : a.rotary + 2 * (s - lead) * VEC;
        second = turned ? a.half + s * VEC : first + VEC;
    }
}

// (a, b) by the angle (c, s); BACK: by its opposite.
template <bool BACK> __device__ __forceinline__ void turn(float& a, float& b, float2 cs) {
    const float s = BACK ? -cs.y : cs.y, x = a;
    a = fmaf(-s, b, cs.x * x);
    b = fmaf(s, x, cs.x * b);
}
template <int VEC, bool BACK> __device__ __forceinline__ void turn_slot(const HeadArgs& a, int s, bool turned, bool second, const float2* table,
                                                                       float (&x)[2][VEC]) {
    if (!turned) return;
    if constexpr (VEC > 1) {
        if (a.interleaved) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (k == 1 && !second) return;               // (the table ends with the row)
#pragma unroll
                for (int e = 0; e < VEC; e += 2) turn<BACK>(x[k][e], x[k][e + 1], table[((2 * s + k) * VEC + e) / 2]);
            }
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) turn<BACK>(x[0][e], x[1][e], table[s * VEC + e]);
}

// Sums over the `team` threads of a row (a power of two, at most a warp).
__device__ __forceinline__ float team_sum(float v, int team) {
    for (int o = team >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// NS: slots of a thread.
template <typename T, int VEC, int NS, bool BWD>
__global__ void __launch_bounds__(kThreads) k_head_norm(const __grid_constant__ HeadArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float2 s_table[kTableMax];
    __shared__ float s_sum[BWD ? kThreads / 32 : 1][BWD ? kMaxWidth : 1];
    const int i = blockIdx.y, b = blockIdx.x;
    const long long t0 = a.n * b / a.ctas, t1 = a.n * (b + 1) / a.ctas;
    const int lane = threadIdx.x % a.team, group = threadIdx.x / a.team, groups = kThreads / a.team;
    float w[2][NS][2][VEC], dw[BWD ? 2 : 1][NS][2][VEC];
    int at[NS][2];
    bool turned[NS], here[NS][2];
#pragma unroll
    for (int z = 0; z < NS; ++z) {
        const int s = z * a.team + lane;
        slot_place<VEC>(a, s, at[z][0], at[z][1], turned[z]);
#pragma unroll
        for (int k = 0; k < 2; ++k) here[z][k] = s < a.slots && at[z][k] < a.d;
        turned[z] = turned[z] && here[z][0];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    w[m][z][k][e] = a.w[m].p && here[z][k] ? to_f32(static_cast<const T*>(a.w[m].p)[i * a.w[m].rep + at[z][k] + e]) : 1.f;
                    if (BWD) dw[m][z][k][e] = 0.f;
                }
            }
    }
    for (long long t = t0; t < t1; t += a.tile) {
        const int places = (int)(t1 - t < a.tile ? t1 - t : a.tile);
        if (t > t0) __syncthreads();
        for (int q = threadIdx.x; q < places * a.table; q += kThreads) {
            const int place = q / a.table, j = q - place * a.table;
            float2 cs = make_float2(1.f, 0.f);
            if (j < a.half) {
                const long long u = i * a.pos_rep + (t + place) * a.pos_step;
                const double pos = !a.positions ? (double)(t + place)
                                   : a.wide     ? (double)__ldg(static_cast<const long long*>(a.positions) + u)
                                                : (double)__ldg(static_cast<const int*>(a.positions) + u);
                double x = pos * a.turns[j];
                x -= rint(x);
                const float hi = (float)x, lo = (float)(x - (double)hi) * 6.283185307179586f;
                float s, c;
                sincospif(2.f * hi, &s, &c);
                cs = make_float2(fmaf(-lo, s, c), fmaf(lo, c, s));
            }
            s_table[q] = cs;
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int H = a.heads[m], rows = places * H;
            const bool normed = a.w[m].p != nullptr;
            // every group makes the same number of turns: the groups of a warp shuffle together
#pragma unroll 2
            for (int base = 0; base < rows; base += groups) {
                const int r = base + group;
                const bool active = r < rows;
                const int place = active ? r / H : 0, h = active ? r - place * H : 0;
                const float2* table = s_table + place * a.table;
                float x[NS][2][VEC], g[BWD ? NS : 1][2][VEC];
                const T* from = head_at<T>(a.x[m], i, t + place, h);
                const T* grad = BWD ? head_at<T>(a.d_out[m], i, t + place, h) : nullptr;
#pragma unroll
                for (int z = 0; z < NS; ++z)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            x[z][k][e] = 0.f;
                            if (BWD) g[z][k][e] = 0.f;
                        }
                        if (active && here[z][k]) {
                            load_vec<T, VEC>(from + at[z][k], x[z][k]);
                            if (BWD) load_vec<T, VEC>(grad + at[z][k], g[z][k]);
                        }
                    }
                float square = 0.f, along = 0.f;
#pragma unroll
                for (int z = 0; z < NS; ++z) {
                    if (BWD) turn_slot<VEC, true>(a, z * a.team + lane, turned[z], here[z][1], table, g[z]);
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            square = fmaf(x[z][k][e], x[z][k][e], square);
                            if (BWD) along = fmaf(g[z][k][e] * w[m][z][k][e], x[z][k][e], along);
                        }
                }
                float inv = 1.f;
                if (normed) inv = 1.f / sqrtf(fmaf(team_sum(square, a.team), a.inv_d, a.eps));
                if (!active) inv = 0.f;                      // (eps may be 0: no infinity times the zeros of a missing row)
                if constexpr (!BWD) {
                    T* to = head_at<T>(a.out[m], i, t + place, h);
#pragma unroll
                    for (int z = 0; z < NS; ++z) {
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int e = 0; e < VEC; ++e) x[z][k][e] *= inv * w[m][z][k][e];
                        turn_slot<VEC, false>(a, z * a.team + lane, turned[z], here[z][1], table, x[z]);
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            if (active && here[z][k]) store_vec<T, VEC>(to + at[z][k], x[z][k]);
                    }
                } else {
                    float back = 0.f;
                    if (normed) back = team_sum(along, a.team) * a.inv_d * inv * inv;
                    T* to = a.out[m].p ? head_at<T>(a.out[m], i, t + place, h) : nullptr;
#pragma unroll
                    for (int z = 0; z < NS; ++z)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float dx[VEC];
#pragma unroll
                            for (int e = 0; e < VEC; ++e) {
                                dw[m][z][k][e] = fmaf(g[z][k][e], x[z][k][e] * inv, dw[m][z][k][e]);
                                dx[e] = inv * fmaf(-back, x[z][k][e], g[z][k][e] * w[m][z][k][e]);
                            }
                            if (to && active && here[z][k]) store_vec<T, VEC>(to + at[z][k], dx);
                        }
                }
            }
        }
    }
    if constexpr (BWD) {
        // sums of the CTA: over the groups of a warp, then over the warps
        if (!a.partial) return;
        for (int m = 0; m < 2; ++m) {
            __syncthreads();
#pragma unroll
            for (int z = 0; z < NS; ++z)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        float v = m == 0 ? dw[0][z][k][e] : dw[1][z][k][e];
                        for (int o = a.team; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                        if ((threadIdx.x & 31) < a.team && here[z][k]) s_sum[threadIdx.x >> 5][at[z][k] + e] = v;
                    }
            __syncthreads();
            float* to = a.partial + (((long long)i * a.ctas + b) * 2 + m) * a.d;
            for (int c = threadIdx.x; c < a.d; c += kThreads) {
                float v = 0.f;
#pragma unroll
                for (int q = 0; q < kThreads / 32; ++q) v += s_sum[q][c];
                to[c] = v;
            }
        }
    }
}

// Adds up the CTAs' sums of one replica (blockIdx.y) and vector (blockIdx.z), in order.
template <typename T> __global__ void __launch_bounds__(256) k_head_sums(const __grid_constant__ HeadArgs a, Vec d_q, Vec d_k) {
    __shared__ float s_part[8][33];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32, i = blockIdx.y, m = blockIdx.z;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float v = 0.f;
    if (c < a.d && a.n > 0) {
        const float* p = a.partial + ((long long)i * a.ctas * 2 + m) * a.d + c;
#pragma unroll 8
        for (int b = part; b < a.ctas; b += 8) v += p[(long long)b * 2 * a.d];
    }
    s_part[part][threadIdx.x % 32] = v;
    __syncthreads();
    if (part != 0 || c >= a.d) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) v += s_part[q][threadIdx.x];
    const Vec to = m ? d_k : d_q;
    if (to.p) static_cast<T*>(to.p)[i * to.rep + c] = from_f32<T>(v);
}

// ----------------------------------------------------------------------------------- host
Heads heads(const eg_heads& m) { return Heads{m.data, (long long)m.replica_stride, (long long)m.row_stride, (long long)m.head_stride}; }

struct Axis {
    int64_t size, stride;
};
// Whether the elements of [P][rows][heads][width] with these strides all lie apart: taken from the shortest stride on, every
// axis steps over what the ones before it span.
bool apart(const eg_heads& m, int64_t P, int64_t rows, int64_t H, int64_t width) {
    Axis x[3] = {{P, m.replica_stride}, {rows, m.row_stride}, {H, m.head_stride}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (x[j].stride < x[i].stride) {
                const Axis y = x[i];
                x[i] = x[j];
                x[j] = y;
            }
    __int128 span = width;
    for (const Axis& y : x) {
        if (y.size <= 1) continue;
        if (y.stride < span) return false;
        span += (__int128)(y.size - 1) * y.stride;
    }
    return true;
}
bool usable(const eg_heads& m, int64_t P, int64_t rows, int64_t H, int64_t width, size_t size, bool written) {
    if (!m.data || (uintptr_t)m.data % size) return false;
    for (int64_t s : {m.replica_stride, m.row_stride, m.head_stride})
        if (s < 0 || s >= (1ll << 42)) return false;
    return !written || apart(m, P, rows, H, width);
}
bool whole_vectors(const eg_heads& m, int64_t P, int64_t rows, int64_t H, size_t size) {
    return !m.data || (aligned16(m.data) && (P <= 1 || m.replica_stride * (int64_t)size % 16 == 0) &&
                       (rows <= 1 || m.row_stride * (int64_t)size % 16 == 0) && (H <= 1 || m.head_stride * (int64_t)size % 16 == 0));
}

bool valid(const eg_head_norm_args* q, bool backward) {
    if (!q) return false;
    if (q->dtype != EG_F32 && q->dtype != EG_BF16 && q->dtype != EG_F16) return false;
    if (q->P < 1 || q->P > 65535 || q->rows < 0 || q->rows > (1ll << 30) || q->width < 1 || q->width > kMaxWidth) return false;
    if (q->q_heads < 1 || q->q_heads > 65535 || q->k_heads < 0 || q->k_heads > 65535) return false;
    if (q->rotary < 0 || q->rotary > q->width || q->rotary % 2) return false;
    if (!(q->eps >= 0.0) || q->eps > 3e38 || !(q->base >= 1e-30) || q->base > 1e30) return false;
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    if (q->positions && ((q->position_bytes != 4 && q->position_bytes != 8) || (uintptr_t)q->positions % (size_t)q->position_bytes ||
                         q->position_replica_stride < 0 || q->position_stride < 0 || q->position_replica_stride >= (1ll << 40) ||
                         q->position_stride >= (1ll << 30)))
        return false;
    if ((q->d_w_q.data && !q->w_q.data) || (q->d_w_k.data && !q->w_k.data) || (!q->k_heads && (q->w_k.data || q->d_w_k.data))) return false;
    for (const eg_matrix* m : {&q->w_q, &q->w_k, &q->d_w_q, &q->d_w_k})
        if (m->data && ((uintptr_t)m->data % size || m->replica_stride < 0 || m->replica_stride >= (1ll << 40))) return false;
    for (const eg_matrix* m : {&q->d_w_q, &q->d_w_k})
        if (m->data && q->P > 1 && m->replica_stride < q->width) return false;
    if (q->rows == 0) return true;
    const struct { const eg_heads *x, *out, *d_out, *dx; int64_t H; } both[] = {{&q->q, &q->q_out, &q->dq_out, &q->dq, q->q_heads},
                                                                               {&q->k, &q->k_out, &q->dk_out, &q->dk, q->k_heads}};
    for (const auto& b : both) {
        if (b.H == 0) continue;
        if (!usable(*b.x, q->P, q->rows, b.H, q->width, size, false)) return false;
        if (!backward && !usable(*b.out, q->P, q->rows, b.H, q->width, size, true)) return false;
        if (backward && !usable(*b.d_out, q->P, q->rows, b.H, q->width, size, false)) return false;
        if (backward && b.dx->data && !usable(*b.dx, q->P, q->rows, b.H, q->width, size, true)) return false;
    }
    return true;
}

// CTAs of a replica; bounds the workspace too.
int ctas_of(int64_t P, int64_t rows) {
    const int64_t all = (int64_t)sm_count() * kCtasPerSm;
    int64_t each = all / P > 1 ? all / P : 1;
    if (each > rows) each = rows > 0 ? rows : 1;
    return (int)each;
}

// Fills the arguments; returns whether 16-byte vectors serve every row.
bool fill(HeadArgs* a, const eg_head_norm_args* q, bool backward) {
    *a = HeadArgs{};
    a->P = (int)q->P; a->n = q->rows; a->d = (int)q->width; a->rotary = (int)q->rotary; a->half = a->rotary / 2;
    a->interleaved = q->interleaved != 0;
    a->eps = (float)q->eps; a->inv_d = 1.f / (float)q->width;
    a->positions = q->positions; a->pos_rep = q->position_replica_stride; a->pos_step = q->position_stride;
    a->wide = q->position_bytes == 8;
    a->heads[0] = (int)q->q_heads; a->heads[1] = (int)q->k_heads;
    a->x[0] = heads(q->q); a->x[1] = heads(q->k);
    a->out[0] = heads(backward ? q->dq : q->q_out); a->out[1] = heads(backward ? q->dk : q->k_out);
    a->d_out[0] = heads(q->dq_out); a->d_out[1] = heads(q->dk_out);
    a->w[0] = Vec{q->w_q.data, (long long)q->w_q.replica_stride};
    a->w[1] = Vec{q->w_k.data, (long long)q->w_k.replica_stride};
    const double full = 6.283185307179586476925;
    const double step = a->rotary > 0 ? -2.0 * log(q->base) / a->rotary : 0.0;
    for (int j = 0; j < a->half; ++j) a->turns[j] = exp(step * j) / full;
    a->ctas = ctas_of(q->P, q->rows);
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    const int V = 16 / (int)size;
    bool vec = a->d % V == 0 && (a->interleaved || (a->half % V == 0 && a->rotary % V == 0));
    const struct { const eg_heads *x, *out, *d_out; int64_t H; } both[] = {{&q->q, backward ? &q->dq : &q->q_out, &q->dq_out, q->q_heads},
                                                                          {&q->k, backward ? &q->dk : &q->k_out, &q->dk_out, q->k_heads}};
    for (const auto& b : both) {
        if (b.H == 0) continue;
        vec = vec && whole_vectors(*b.x, q->P, q->rows, b.H, size) && whole_vectors(*b.out, q->P, q->rows, b.H, size) &&
              (!backward || whole_vectors(*b.d_out, q->P, q->rows, b.H, size));
    }
    const int v = vec ? V : 1;
    if (a->interleaved) {
        // single values: the slot's two are neighbours, (2 s, 2 s + 1)
        a->slots = (a->d + 2 * v - 1) / (2 * v);
        a->table = (a->d + 1) / 2;
    } else {
        a->slots = a->half / v + (a->d - a->rotary + 2 * v - 1) / (2 * v);
        a->table = a->half;
    }
    a->team = 1;
    while (a->team < 32 && a->team < a->slots) a->team *= 2;
    a->tile = kMaxTile;
    while (a->tile > 1 && a->tile * a->table > kTableMax) a->tile /= 2;
    return vec;
}

template <typename T, bool BWD> cudaError_t launch(const HeadArgs& a, bool vec, cudaStream_t stream) {
    constexpr int V = 16 / (int)sizeof(T);
    const dim3 grid(a.ctas, a.P);
    static_assert(kMaxWidth / (2 * V) <= 32 && kMaxWidth / 2 <= 4 * 32, "slots of a row");
    if (vec) return launch_after(k_head_norm<T, V, 1, BWD>, grid, dim3(kThreads), 0, stream, a);
    if (a.slots <= 32) return launch_after(k_head_norm<T, 1, 1, BWD>, grid, dim3(kThreads), 0, stream, a);
    if (a.slots <= 64) return launch_after(k_head_norm<T, 1, 2, BWD>, grid, dim3(kThreads), 0, stream, a);
    return launch_after(k_head_norm<T, 1, 4, BWD>, grid, dim3(kThreads), 0, stream, a);
}

template <typename T> cudaError_t backward(HeadArgs a, bool vec, const eg_head_norm_args* q, cudaStream_t stream) {
    if (!q->d_w_q.data && !q->d_w_k.data) a.partial = nullptr;
    if (a.n > 0) {
        const cudaError_t e = launch<T, true>(a, vec, stream);
        if (e != cudaSuccess) return e;
    }
    if (!q->d_w_q.data && !q->d_w_k.data) return cudaSuccess;
    return launch_after(k_head_sums<T>, dim3((a.d + 31) / 32, a.P, 2), dim3(256), 0, stream, a,
                        Vec{q->d_w_q.data, (long long)q->d_w_q.replica_stride}, Vec{q->d_w_k.data, (long long)q->d_w_k.replica_stride});
}

}  // namespace
}  // namespace eg

using namespace eg;

extern "C" {

eg_status eg_head_norm(const eg_head_norm_args* q, void* stream_v) {
    if (!valid(q, false)) return EG_ERR_INVALID;
    if (q->rows == 0) return EG_OK;
    if (sm_count() < 1) return EG_ERR_CUDA;
    HeadArgs a;
    const bool vec = fill(&a, q, false);
    cudaStream_t s = static_cast<cudaStream_t>(stream_v);
    const cudaError_t e = q->dtype == EG_F32    ? launch<float, false>(a, vec, s)
                          : q->dtype == EG_BF16 ? launch<__nv_bfloat16, false>(a, vec, s)
                                                : launch<__half, false>(a, vec, s);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

int64_t eg_head_norm_workspace(const eg_head_norm_args* q) {
    if (!valid(q, true) || sm_count() < 1) return 0;
    return q->P * (int64_t)ctas_of(q->P, q->rows) * 2 * q->width * 4;
}

eg_status eg_head_norm_backward(const eg_head_norm_args* q, void* workspace, int64_t workspace_bytes, void* stream_v) {
    if (!valid(q, true)) return EG_ERR_INVALID;
    if (sm_count() < 1) return EG_ERR_CUDA;
    if (!workspace || !aligned16(workspace) || workspace_bytes < eg_head_norm_workspace(q)) return EG_ERR_INVALID;
    HeadArgs a;
    const bool vec = fill(&a, q, true);
    a.partial = static_cast<float*>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream_v);
    const cudaError_t e = q->dtype == EG_F32    ? backward<float>(a, vec, q, s)
                          : q->dtype == EG_BF16 ? backward<__nv_bfloat16>(a, vec, q, s)
                                                : backward<__half>(a, vec, q, s);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

}  // extern "C"
