// The norm of every head of the queries and keys with the rotation by position (eg_head_norm) and its gradients.
//
//   forward   xh = x * inv,  inv = 1 / sqrt(mean(x^2) + eps);   z = xh * w;   o = R z
//             R turns the pair (z_a, z_b) of pair j by position * base^(-2 j / rotary):
//             o_a = z_a cos - z_b sin,  o_b = z_a sin + z_b cos
//   backward  dz = R^T do;   dw = sum dz * xh;   dx = inv * (dz * w - xh * mean(dz * w * xh))
//
// Bound by memory: forward moves a value in and out, backward two in and one out (nothing is saved between them).  4 x 8192 places of 16
// + 4 heads of 128 in bf16: forward 70 us (4.8 TB/s), backward 109 (4.6): the warps that registers leave room for (24 and 16 a
// multiprocessor) have shared memory full of rows on their way, and issue 45 and 63 M instructions.
//
// A head's row is small, so a team of a few threads shares it, each with whole pairs: a "slot" is two vectors of VEC values whose
// elements are partners (halves: j and j + rotary / 2; neighbours: inside either vector).  A warp takes one place after
// another, all heads of the queries or of the keys, a row a team at a time; cosines and sines of the place stay in registers for all
// of them (a sine costs some forty instructions, a value of a row about six), each formed by one team and handed to
// the others.  Angles are whole 64-bit numbers in units of 2^-64 of a turn, which overflow where a turn ends: a product of
// position and frequency keeps its fraction for positions of any size and sign, and is off by what the frequency was rounded by,
// about 2^-64 of a turn for every place: 2^-24 at 2^40, 2^-19 at 2^45.
#include <math.h>

#include <type_traits>

#include "eg_ops.cuh"

namespace eg {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxWidth = EG_HEAD_MAX_WIDTH, kMaxPairs = kMaxWidth / 2;
constexpr int kCtasForward = 3, kCtasBackward = 2;      // of a multiprocessor: all resident at once

struct Heads {
    void* p;
    long long rep, row, head;               // strides in elements
};
struct Vec {
    void* p;
    long long rep;
};

// The queries, or the keys.
struct Side {
    int heads, ctas, split;                 // ctas: of a replica; split: warps that share a place's heads
    Heads x, out, d_out;                    // forward: x, out; backward: x, d_out and in out the gradient of x
    Vec w;
    float* partial;                         // [P][ctas][d] sums of dz * xh
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
    int slots;                              // of a row
    Side side[2];
    unsigned long long turns[kMaxPairs];    // turns of pair j per place, in 2^-64
};

template <typename T> __device__ __forceinline__ T* head_at(const Heads& m, int i, long long t, int h) {
    return static_cast<T*>(m.p) + (long long)i * m.rep + t * m.row + (long long)h * m.head;
}

// VEC values on their way through shared memory: a thread copies what it will itself read, so that nobody waits for anybody.
template <typename T, int VEC> struct Piece {
    static constexpr int kBytes = VEC * (int)sizeof(T) < 4 ? 4 : VEC * (int)sizeof(T);
    static constexpr int kWords = kBytes / 4;
    // A single 16-bit value comes with the other half of its word.
    __device__ __forceinline__ static const void* word(const T* p) { return reinterpret_cast<const void*>((uintptr_t)p & ~(uintptr_t)3); }
    __device__ __forceinline__ static void copy(unsigned char* to, const T* from, bool there) {
        const uint32_t dst = op_smem(to);
        const int bytes = there ? kBytes : 0;                // the rest becomes zero
        const void* src = word(from);
        if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(kBytes), "r"(bytes) : "memory");
    }
    __device__ __forceinline__ static void read(const unsigned char* at, const T* from, uint32_t (&w)[kWords]) {
        if constexpr (kWords == 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(at);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else if constexpr (kWords == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(at);
            w[0] = v.x; w[1] = v.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(at);
            if (VEC * sizeof(T) == 2 && ((uintptr_t)from & 2)) w[0] >>= 16;
        }
    }
};

// The two vectors of a slot as VEC pairs of registers, for packed arithmetic: neighbours of one vector (VEC == 1: the two vectors' values).
template <typename T, int VEC> __device__ __forceinline__ void widen(const uint32_t (&w)[2][Piece<T, VEC>::kWords], f32x2 (&v)[VEC]) {
    if constexpr (VEC == 1) {
        if constexpr (sizeof(T) == 4) v[0] = pack_f2(__uint_as_float(w[0][0]), __uint_as_float(w[1][0]));
        else v[0] = pack_f2(unpack2<T>(w[0][0]).x, unpack2<T>(w[1][0]).x);
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) {
                if constexpr (sizeof(T) == 4) v[k * (VEC / 2) + e] = pack_f2(__uint_as_float(w[k][2 * e]), __uint_as_float(w[k][2 * e + 1]));
                else v[k * (VEC / 2) + e] = pack_f2(unpack2<T>(w[k][e]));
            }
    }
}
// The values of vector k.
template <int VEC> __device__ __forceinline__ void values_of(const f32x2 (&v)[VEC], int k, float (&x)[VEC]) {
    if constexpr (VEC == 1) {
        const float2 f = unpack_f2(v[0]);
        x[0] = k ? f.y : f.x;
    } else {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) {
            const float2 f = unpack_f2(v[k * (VEC / 2) + e]);
            x[2 * e] = f.x;
            x[2 * e + 1] = f.y;
        }
    }
}
template <typename T, int VEC> __device__ __forceinline__ void store_some(T* p, const float (&v)[VEC]) {
    if constexpr (VEC == 1 || VEC * sizeof(T) == 16) store_vec<T, VEC>(p, v);
    else if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
    else *reinterpret_cast<uint32_t*>(p) = pack2<T>(v[0], v[1]);
}

// A slot's VEC pairs by their angles (cosine, sine); pairs that stay have cosine 1.
//   halves: partners in the two vectors;  neighbours (and single values): partners in one pair of registers
template <int VEC> __device__ __forceinline__ void turn_slot(bool interleaved, const float2* cs, f32x2 (&x)[VEC]) {
    if (VEC == 1 || interleaved) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float2 f = unpack_f2(x[e]);
            x[e] = fma2(x[e], pack_f2(cs[e].x, cs[e].x), mul2(pack_f2(f.y, f.x), pack_f2(-cs[e].y, cs[e].y)));
        }
        return;
    }
    if constexpr (VEC > 1) {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) {
            const f32x2 a = x[e], b = x[e + VEC / 2], c = pack_f2(cs[2 * e].x, cs[2 * e + 1].x), s = pack_f2(cs[2 * e].y, cs[2 * e + 1].y);
            x[e] = fma2(c, a, mul2(pack_f2(-cs[2 * e].y, -cs[2 * e + 1].y), b));
            x[e + VEC / 2] = fma2(c, b, mul2(s, a));
        }
    }
}

// Cosine and sine of an angle in 2^-64 of a turn.  16-bit results take the hardware's (2^-21, after the reduction).
template <typename T> __device__ __forceinline__ float2 cos_sin(unsigned long long angle) {
    const int top = (int)(angle >> 32);                      // -1/2 to 1/2 of a turn
    const float hi = (float)top;
    float s, c;
    if constexpr (sizeof(T) == 2) {
        const float x = hi * 1.4629180792671596e-9f;         // 2 pi / 2^32
        s = __sinf(x);
        c = __cosf(x);
        return make_float2(c, s);
    } else {
        const float lo = (float)(int)((long long)top - (long long)hi) * 1.4629180792671596e-9f;   // what 24 bits left over
        sincospif(hi * 4.656612873077393e-10f, &s, &c);      // 2 / 2^32
        return make_float2(fmaf(-lo, s, c), fmaf(lo, c, s));
    }
}

// Sums over the TEAM threads of a row.
template <int TEAM> __device__ __forceinline__ float team_sum(float v) {
#pragma unroll
    for (int o = TEAM >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Shared memory of a thread for one unit (a row's slots, their gradients, the place): as many units as DEPTH are on their way.
template <typename T, int VEC, int NS, bool BWD> struct Ring {
    static constexpr int kPieces = NS * 2 * (BWD ? 2 : 1);
    static constexpr int kUnit = kPieces * Piece<T, VEC>::kBytes + 8;
    static constexpr int kDepth = 3 + (kUnit < 40) + (kUnit < 24);
    static constexpr int kBytes = kDepth * kUnit * kThreads;
};

// NS: slots of a thread; TEAM: threads of a row.
template <typename T, int VEC, int NS, int TEAM, bool BWD>
__global__ void __launch_bounds__(kThreads, BWD ? kCtasBackward : kCtasForward) k_head_norm(const __grid_constant__ HeadArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int GROUPS = 32 / TEAM, PAIRS = NS * VEC;
    __shared__ float s_sum[BWD ? kWarps : 1][BWD ? kMaxWidth : 1];
    const int m = (int)blockIdx.x >= a.side[0].ctas, i = blockIdx.y;
    const Side& side = a.side[m];
    const int b = blockIdx.x - (m ? a.side[0].ctas : 0);
    const long long t0 = a.n * b / side.ctas, t1 = a.n * (b + 1) / side.ctas;
    const int lane = threadIdx.x % TEAM, group = threadIdx.x % 32 / TEAM, warp = threadIdx.x >> 5;
    const bool normed = side.w.p != nullptr;
    f32x2 w[NS][VEC], dw[BWD ? NS : 1][VEC];
    int at[NS][2];
    bool here[NS][2];
#pragma unroll
    for (int z = 0; z < NS; ++z) {
        const int s = z * TEAM + lane;
        if (a.interleaved) {
            at[z][0] = 2 * s * VEC;
            at[z][1] = at[z][0] + VEC;
        } else {
            const int lead = a.half / VEC;                   // slots that turn
            at[z][0] = s < lead ? s * VEC : a.rotary + 2 * (s - lead) * VEC;
            at[z][1] = s < lead ? a.half + s * VEC : at[z][0] + VEC;
        }
        float f[2][VEC];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            here[z][k] = s < a.slots && at[z][k] < a.d;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                f[k][e] = normed && here[z][k] ? to_f32(static_cast<const T*>(side.w.p)[i * side.w.rep + at[z][k] + e]) : 1.f;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            w[z][e] = VEC == 1 ? pack_f2(f[0][0], f[1][0]) : pack_f2(f[2 * e / VEC][2 * e % VEC], f[2 * e / VEC][(2 * e + 1) % VEC]);
            if (BWD) dw[z][e] = 0;
        }
    }
    // pair q of a thread is formed by team q % GROUPS; the turns of those that this one forms
    constexpr int OWN = (PAIRS + GROUPS - 1) / GROUPS;
    unsigned long long turns_of[OWN];
#pragma unroll
    for (int q = 0; q < OWN; ++q) {
        const int pair = q * GROUPS + group, j = (pair / VEC * TEAM + lane) * VEC + pair % VEC;
        turns_of[q] = pair < PAIRS && j < a.half ? a.turns[j] : 0;
    }
    const int part = warp % side.split, H = side.heads;
    // A unit: the rows that the teams take at one turn, of one place.  Its values come by way of shared memory, DEPTH - 1 units ahead:
    // in registers a multiprocessor held too few bytes on their way (8192 places of 16 + 4 heads of 128 on 4 replicas: 79 and 153 us).
    using R = Ring<T, VEC, NS, BWD>;
    using P = Piece<T, VEC>;
    constexpr int DEPTH = R::kDepth;
    extern __shared__ __align__(16) unsigned char s_ring[];
    const int turns = (H - part * GROUPS + side.split * GROUPS - 1) / (side.split * GROUPS), stride = kWarps / side.split;
    auto piece = [&](int slot, int n) { return s_ring + ((slot * R::kPieces + n) * kThreads + threadIdx.x) * P::kBytes; };
    auto place_at = [&](int slot) { return s_ring + DEPTH * R::kPieces * kThreads * P::kBytes + (slot * kThreads + threadIdx.x) * 8; };
    long long t = t0 + warp / side.split, ta = t;            // the unit worked on, and the one to fetch
    int q = 0, qa = 0, slot = 0, slot_a = 0;
    auto fetch = [&]() {
        if (ta < t1 && turns > 0) {
            const int h = (part + qa * side.split) * GROUPS + group;
            const bool active = h < H;
            const T* const x0 = head_at<T>(side.x, i, ta, active ? h : 0);
            const T* const g0 = BWD ? head_at<T>(side.d_out, i, ta, active ? h : 0) : nullptr;
#pragma unroll
            for (int z = 0; z < NS; ++z)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bool there = active && here[z][k];
                    P::copy(piece(slot_a, z * 2 + k), x0 + (there ? at[z][k] : 0), there);
                    if (BWD) P::copy(piece(slot_a, NS * 2 + z * 2 + k), g0 + (there ? at[z][k] : 0), there);
                }
            if (qa == 0 && a.positions) {
                const char* p = static_cast<const char*>(a.positions) + (i * a.pos_rep + ta * a.pos_step) * (a.wide ? 8 : 4);
                if (a.wide) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(op_smem(place_at(slot_a))), "l"(p) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(op_smem(place_at(slot_a))), "l"(p) : "memory");
            }
            if (++qa == turns) { qa = 0; ta += stride; }
            if (++slot_a == DEPTH) slot_a = 0;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    float2 cs[PAIRS];
#pragma unroll
    for (int n = 0; n < DEPTH - 1; ++n) fetch();
    while (t < t1 && turns > 0) {
        fetch();
        asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
        if (q == 0) {
            // this place's cosines and sines (no turns: cosine 1)
            float2 own[OWN];
            const unsigned long long pos = (unsigned long long)(!a.positions ? t
                                                                : a.wide     ? *reinterpret_cast<const long long*>(place_at(slot))
                                                                             : (long long)*reinterpret_cast<const int*>(place_at(slot)));
#pragma unroll
            for (int z = 0; z < OWN; ++z) {
                own[z] = cos_sin<T>(pos * turns_of[z]);
                if (BWD) own[z].y = -own[z].y;               // back
            }
#pragma unroll
            for (int z = 0; z < PAIRS; ++z) {
                if constexpr (GROUPS == 1) {
                    cs[z] = own[z];
                } else {
                    const int from = z % GROUPS * TEAM + lane;
                    cs[z] = make_float2(__shfl_sync(0xffffffffu, own[z / GROUPS].x, from), __shfl_sync(0xffffffffu, own[z / GROUPS].y, from));
                }
            }
        }
        {
            const int h = (part + q * side.split) * GROUPS + group;
            const bool active = h < H;
            T* const o0 = side.out.p ? head_at<T>(side.out, i, t, h) : nullptr;
            const T* const x0 = head_at<T>(side.x, i, t, h);         // (single 16-bit values: which half of their word)
            const T* const g0 = BWD ? head_at<T>(side.d_out, i, t, h) : nullptr;
            f32x2 x[NS][VEC], g[BWD ? NS : 1][VEC], squares = 0, along2 = 0;
#pragma unroll
            for (int z = 0; z < NS; ++z) {
                uint32_t raw[2][P::kWords];
#pragma unroll
                for (int k = 0; k < 2; ++k) P::read(piece(slot, z * 2 + k), x0 + at[z][k], raw[k]);
                widen<T, VEC>(raw, x[z]);
                if constexpr (BWD) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) P::read(piece(slot, NS * 2 + z * 2 + k), g0 + at[z][k], raw[k]);
                    widen<T, VEC>(raw, g[z]);
                    turn_slot<VEC>(a.interleaved, cs + z * VEC, g[z]);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    squares = fma2(x[z][e], x[z][e], squares);
                    if (BWD) along2 = fma2(mul2(g[z][e], w[z][e]), x[z][e], along2);
                }
            }
            float inv = 1.f;
            if (normed) {
                const float2 f = unpack_f2(squares);
                inv = rsqrtf(fmaf(team_sum<TEAM>(f.x + f.y), a.inv_d, a.eps));
            }
            if (!active) inv = 0.f;                          // (eps may be 0: no infinity times the zeros of a missing row)
            const f32x2 inv2 = pack_f2(inv, inv);
            if constexpr (!BWD) {
#pragma unroll
                for (int z = 0; z < NS; ++z) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[z][e] = mul2(x[z][e], mul2(inv2, w[z][e]));
                    turn_slot<VEC>(a.interleaved, cs + z * VEC, x[z]);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float f[VEC];
                        values_of<VEC>(x[z], k, f);
                        if (active && here[z][k]) store_some<T, VEC>(o0 + at[z][k], f);
                    }
                }
            } else {
                float back = 0.f;
                if (normed) {
                    const float2 f = unpack_f2(along2);
                    back = -team_sum<TEAM>(f.x + f.y) * a.inv_d * inv * inv;
                }
                const f32x2 back2 = pack_f2(back, back);
#pragma unroll
                for (int z = 0; z < NS; ++z) {
                    f32x2 dx[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        dw[z][e] = fma2(g[z][e], mul2(x[z][e], inv2), dw[z][e]);
                        dx[e] = mul2(inv2, fma2(back2, x[z][e], mul2(g[z][e], w[z][e])));
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float f[VEC];
                        values_of<VEC>(dx, k, f);
                        if (o0 && active && here[z][k]) store_some<T, VEC>(o0 + at[z][k], f);
                    }
                }
            }
        }
        if (++q == turns) { q = 0; t += stride; }
        if (++slot == DEPTH) slot = 0;
    }
    if constexpr (BWD) {
        // sums of the CTA: over the teams of a warp, then over the warps
        if (!side.partial) return;
#pragma unroll
        for (int z = 0; z < NS; ++z)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float f[VEC];
                values_of<VEC>(dw[z], k, f);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float v = f[e];
#pragma unroll
                    for (int o = TEAM; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                    if (group == 0 && here[z][k]) s_sum[warp][at[z][k] + e] = v;
                }
            }
        __syncthreads();
        float* to = side.partial + ((long long)i * side.ctas + b) * a.d;
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            float v = 0.f;
#pragma unroll
            for (int q = 0; q < kWarps; ++q) v += s_sum[q][c];
            to[c] = v;
        }
    }
}

// Adds up the CTAs' sums of one replica (blockIdx.y) and vector (blockIdx.z), in order.
template <typename T> __global__ void __launch_bounds__(256) k_head_sums(const __grid_constant__ HeadArgs a, Vec d_q, Vec d_k) {
    __shared__ float s_part[8][33];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32, i = blockIdx.y, m = blockIdx.z;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float v = 0.f;
    const Vec to = m ? d_k : d_q;
    if (!to.p) return;
    if (c < a.d && a.n > 0) {
        const float* p = a.side[m].partial + (long long)i * a.side[m].ctas * a.d + c;
#pragma unroll 8
        for (int b = part; b < a.side[m].ctas; b += 8) v += p[(long long)b * a.d];
    }
    s_part[part][threadIdx.x % 32] = v;
    __syncthreads();
    if (part != 0 || c >= a.d) return;
#pragma unroll
    for (int q = 1; q < 8; ++q) v += s_part[q][threadIdx.x];
    static_cast<T*>(to.p)[i * to.rep + c] = from_f32<T>(v);
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
// Whether every row begins on a multiple of so many bytes.
bool begins_on(const eg_heads& m, int64_t P, int64_t rows, int64_t H, size_t size, size_t bytes) {
    return !m.data || ((uintptr_t)m.data % bytes == 0 && (P <= 1 || m.replica_stride * size % bytes == 0) &&
                       (rows <= 1 || m.row_stride * size % bytes == 0) && (H <= 1 || m.head_stride * size % bytes == 0));
}

bool valid(const eg_head_norm_args* q, bool backward) {
    if (!q) return false;
    if (q->dtype != EG_F32 && q->dtype != EG_BF16 && q->dtype != EG_F16) return false;
    if (q->P < 1 || q->P > 65535 || q->rows < 0 || q->rows > (1ll << 30) || q->width < 1 || q->width > kMaxWidth) return false;
    if (q->q_heads < 1 || q->q_heads > 65535 || q->k_heads < 0 || q->k_heads > 65535) return false;
    if (q->rotary < 0 || q->rotary > q->width || q->rotary % 2) return false;
    if (!(q->eps >= 0.0) || q->eps > 3e38 || !(q->base >= 1.0) || q->base > 1e30) return false;
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

// CTAs of a replica for one side; bounds the workspace too.
int ctas_of(int64_t P, int64_t rows, int64_t mine, int64_t other, int per_sm) {
    if (mine == 0) return 0;
    // both sides' warps take as long: their heads, and a place's sines (as long as about four)
    const double share = (double)(mine + 4) / (double)(mine + 4 + (other ? other + 4 : 0));
    int64_t each = (int64_t)((double)(sm_count() * per_sm) * share / (double)P);
    if (each > (rows + 1) / 2) each = (rows + 1) / 2;
    return (int)(each > 1 ? each : 1);
}

struct Sizes {
    int ctas[2];
    int64_t bytes;
};
Sizes sizes_of(const eg_head_norm_args* q, bool backward) {
    Sizes s;
    s.ctas[0] = ctas_of(q->P, q->rows, q->q_heads, q->k_heads, backward ? kCtasBackward : kCtasForward);
    s.ctas[1] = ctas_of(q->P, q->rows, q->k_heads, q->q_heads, backward ? kCtasBackward : kCtasForward);
    s.bytes = q->P * (int64_t)(s.ctas[0] + s.ctas[1]) * q->width * 4;
    return s;
}

// Fills the arguments; returns how many values an access takes: 16 bytes, 2 values, 1.
int fill(HeadArgs* a, const eg_head_norm_args* q, bool backward, float* partial) {
    *a = HeadArgs{};
    a->P = (int)q->P; a->n = q->rows; a->d = (int)q->width; a->rotary = (int)q->rotary; a->half = a->rotary / 2;
    a->interleaved = q->interleaved != 0;
    a->eps = (float)q->eps; a->inv_d = 1.f / (float)q->width;
    a->positions = q->positions; a->pos_rep = q->position_replica_stride; a->pos_step = q->position_stride;
    a->wide = q->position_bytes == 8;
    const Sizes n = sizes_of(q, backward);
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    const struct { const eg_heads *x, *out, *d_out; const eg_matrix *w, *dw; int64_t H; } both[] = {
        {&q->q, backward ? &q->dq : &q->q_out, &q->dq_out, &q->w_q, &q->d_w_q, q->q_heads},
        {&q->k, backward ? &q->dk : &q->k_out, &q->dk_out, &q->w_k, &q->d_w_k, q->k_heads}};
    auto serves = [&](int v) {
        if (a->d % v || (!a->interleaved && a->half % v)) return false;
        for (const auto& b : both) {
            if (b.H == 0) continue;
            for (const eg_heads* m : {b.x, b.out, b.d_out})
                if ((m != b.d_out || backward) && !begins_on(*m, q->P, q->rows, b.H, size, v * size)) return false;
        }
        return true;
    };
    const int v = serves(16 / (int)size) ? 16 / (int)size : serves(2) ? 2 : 1;
    a->slots = a->interleaved ? (a->d + 2 * v - 1) / (2 * v) : a->half / v + (a->d - a->rotary + 2 * v - 1) / (2 * v);
    for (int m = 0; m < 2; ++m) {
        Side* s = &a->side[m];
        s->heads = (int)both[m].H;
        s->ctas = n.ctas[m];
        // few places of a CTA: warps share their heads.  A warp's places times its turns for each, and about one for the sines.  (us, forward and
        // backward, and with a warp a place: 1 place of 32 + 8 heads of 128 in bf16 8 + 10, 10 + 13; 100 of them 8 + 12, 10 + 14; 300 in fp32 10 + 14,
        // 14 + 21; 1 of 64 + 64 heads of 90 in fp32 10 + 12, 31 + 41; 8 x 1024 of 16 + 4 of 64 in bf16, where the rule shares nothing, 18 + 27)
        const int64_t places = s->ctas ? (q->rows + s->ctas - 1) / s->ctas : 1;
        int team = v * (int)size == 16 ? 2 : 32;
        while (team < 32 && team < a->slots) team *= 2;
        const int64_t turns = (s->heads * team + 31) / 32;
        int64_t least = 0;
        for (int split = 1; split <= kWarps; split *= 2) {
            const int64_t time = (places * split + kWarps - 1) / kWarps * ((turns + split - 1) / split + 1);
            if (split == 1 || time < least) {
                least = time;
                s->split = split;
            }
        }
        s->x = heads(*both[m].x); s->out = heads(*both[m].out); s->d_out = heads(*both[m].d_out);
        s->w = Vec{both[m].w->data, (long long)both[m].w->replica_stride};
        s->partial = backward && both[m].dw->data ? partial + (m ? q->P * (int64_t)n.ctas[0] * q->width : 0) : nullptr;
    }
    // Turns of the pairs per place to about the last of 64 bits, in the host's 64-bit significands (53 bits left a position of 2^45 off by 2^-10
    // of a turn).  Pair 16 c + 4 b + a is a product of three powers, so that few exponentials are formed: a call for one token waits for
    // them (32 pairs with 7 of them 6.4 us, with 12 6.9; 32 of 53 bits 6.1).
    const long double step = a->rotary > 0 ? -2.0L * logl((long double)q->base) / a->rotary : 0.0L;
    long double power[3][8];
    for (int z = 0, stride = 1; z < 3; ++z, stride *= 4)
        for (int j = 0; j < (z < 2 ? 4 : 8) && j * stride < a->half; ++j) power[z][j] = j ? expl(step * (j * stride)) : 1.0L;
    for (int j = 0; j < a->half; j += 4) {
        const long double coarse = power[1][j / 4 % 4] * power[2][j / 16] * (0x1p64L / 6.283185307179586476925286766559L);
        for (int z = 0; z < 4 && j + z < a->half; ++z) a->turns[j + z] = (unsigned long long)(long long)(coarse * power[0][z] + 0.5L);    // (below 0.16 of a turn)
    }
    return v;
}

template <typename T, bool BWD> cudaError_t launch(const HeadArgs& a, int v, cudaStream_t stream) {
    constexpr int V = 16 / (int)sizeof(T);
    const dim3 grid(a.side[0].ctas + a.side[1].ctas, a.P);
    auto run = [&](auto kernel, int smem) {
        cudaError_t e = cudaSuccess;                         // (48 KB need no permission, but the sums are part of them)
        if (smem > 40 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        return e != cudaSuccess ? e : launch_after(kernel, grid, dim3(kThreads), smem, stream, a);
    };
    static_assert(kMaxWidth / (2 * V) <= 32 && kMaxWidth / 4 <= 2 * 32 && kMaxWidth / 2 <= 4 * 32, "slots of a row");
    if (v == V) {
        if (a.slots <= 2) return run(k_head_norm<T, V, 1, 2, BWD>, Ring<T, V, 1, BWD>::kBytes);
        if (a.slots <= 4) return run(k_head_norm<T, V, 1, 4, BWD>, Ring<T, V, 1, BWD>::kBytes);
        if (a.slots <= 8) return run(k_head_norm<T, V, 1, 8, BWD>, Ring<T, V, 1, BWD>::kBytes);
        if (a.slots <= 16) return run(k_head_norm<T, V, 1, 16, BWD>, Ring<T, V, 1, BWD>::kBytes);
        return run(k_head_norm<T, V, 1, 32, BWD>, Ring<T, V, 1, BWD>::kBytes);
    }
    if (v == 2) return a.slots <= 32 ? run(k_head_norm<T, 2, 1, 32, BWD>, Ring<T, 2, 1, BWD>::kBytes) : run(k_head_norm<T, 2, 2, 32, BWD>, Ring<T, 2, 2, BWD>::kBytes);
    if (a.slots <= 32) return run(k_head_norm<T, 1, 1, 32, BWD>, Ring<T, 1, 1, BWD>::kBytes);
    return a.slots <= 64 ? run(k_head_norm<T, 1, 2, 32, BWD>, Ring<T, 1, 2, BWD>::kBytes) : run(k_head_norm<T, 1, 4, 32, BWD>, Ring<T, 1, 4, BWD>::kBytes);
}

template <typename T> cudaError_t backward(const HeadArgs& a, int v, const eg_head_norm_args* q, cudaStream_t stream) {
    if (a.n > 0) {
        const cudaError_t e = launch<T, true>(a, v, stream);
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
    const int v = fill(&a, q, false, nullptr);
    cudaStream_t s = static_cast<cudaStream_t>(stream_v);
    const cudaError_t e = q->dtype == EG_F32    ? launch<float, false>(a, v, s)
                          : q->dtype == EG_BF16 ? launch<__nv_bfloat16, false>(a, v, s)
                                                : launch<__half, false>(a, v, s);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

int64_t eg_head_norm_workspace(const eg_head_norm_args* q) {
    if (!valid(q, true) || sm_count() < 1) return 0;
    return sizes_of(q, true).bytes;
}

eg_status eg_head_norm_backward(const eg_head_norm_args* q, void* workspace, int64_t workspace_bytes, void* stream_v) {
    if (!valid(q, true)) return EG_ERR_INVALID;
    if (sm_count() < 1) return EG_ERR_CUDA;
    if (!workspace || !aligned16(workspace) || workspace_bytes < eg_head_norm_workspace(q)) return EG_ERR_INVALID;
    HeadArgs a;
    const int v = fill(&a, q, true, static_cast<float*>(workspace));
    cudaStream_t s = static_cast<cudaStream_t>(stream_v);
    const cudaError_t e = q->dtype == EG_F32    ? backward<float>(a, v, q, s)
                          : q->dtype == EG_BF16 ? backward<__nv_bfloat16>(a, v, q, s)
                                                : backward<__half>(a, v, q, s);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

}  // extern "C"
