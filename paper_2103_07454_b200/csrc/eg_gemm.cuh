// Batched matrix products on the tensor cores for the feed-forward block (sm_100a).
//
// One launch works through the tiles of up to four products ("problems"), each of which is, for
// every replica, D[M, N] = sum over segments of A[M, K] * B[N, K]^T with 16-bit operands and fp32
// accumulators.  A segment is one pair of operand matrices; several segments add into one result
// (dX = dG Wg + dU Wu; the parts of fp32 operands).
//
// fp32 operands come in kParts = 3 bf16 parts, each the nearest to what the ones before leave, whose sum is the value
// (down to 2^-109, where the last parts leave bf16's range).  The second part is at most 2^-8 of the value, the third 2^-17,
// and their signs are as often one as the other.  The six products of parts that matter (part i of A with part j of B,
// i + j <= 2) are formed from one copy of the parts in shared memory.  What is left out is at most 2^-24 of |a||b|.
//
// Two CTAs of a cluster share a tile of 256 x BN (tcgen05.mma, cta_group::2): each stages its 128
// rows of A and its half of B with TMA (128-byte swizzle, 64 elements of K a stage), the even CTA
// issues the products, and each CTA keeps its 128 rows of D in its own tensor memory -- twice, so
// that the epilogue of one tile runs under the products of the next.  An operand whose K runs
// along its rows ("MN-major": the transposed uses of the backward pass) is staged in boxes of 64
// columns and read by the tensor cores in that order; nothing is ever transposed in memory.
//
// Measured, 4 replicas x 4096 tokens, 2048 x 5504, bf16: gate/up with activation 470 us (1.57 PFLOP/s), down 214-228
// us (1.62-1.73), activation gradient 290-300 us (1.23-1.27: its epilogue moves four more matrices), the four
// gradients 1236 us (1.49); a stage of 64 of K takes 540-580 cycles of 512 on the tensor cores; fp32, 8 x 1021 tokens, 1280 x
// 4992: forward 1.51 ms, forward and backward with the copies of both 4.6-4.8 ms (1.2 PFLOP/s of products of parts).  8 x 512
// tokens, 1024 x 2816: 45 + 23 + 35 + 95 us, 750-850 cycles a stage, with the tensor cores 30-56 % and the memory 33-39 %
// busy: why a stage takes so long there is not known (160-190 KB of stages look some 3000 cycles ahead, which covers the
// memory's latency; asking for the weights earlier into the L2 was slower).
//
// Warps: 0 and 3 TMA producers (A, B), 1 tensor-core issue, 2 tensor memory, 4..11 epilogue (warp w reads the
// 32 lanes w % 4 of tensor memory; warps 4..7 take the first half of the columns, 8..11 the other).
#pragma once
#include <cuda.h>

#include <type_traits>

#include "eg_ops.cuh"

namespace eg {

constexpr int kGemmThreads = 384;
constexpr int kGemmEpiWarps = 8;
constexpr int kGemmK = 64;                        // elements of K per stage: 128 bytes, one swizzle row
constexpr int kGemmM = 256;                       // rows of a tile (two CTAs)
constexpr int kGemmMaxStages = 24;
constexpr int kGemmMaxMaps = 40, kGemmMaxSegs = 2, kGemmMaxProblems = 4;

struct GemmSeg {
    int a, b0, b1;                                // maps (fp32: of the first part); b0 / b1: B of the even / odd CTA
    int ksteps;
};

// Adding into the accumulator truncates: about 3e-8 of it per instruction, always towards zero, so that the
// error of a sum grows with K (5e-6 after 2816).  In fp32 the accumulator is therefore moved to registers,
// where an addition rounds, every kChunk steps of the products of first parts (16 instructions: 5e-7 at most).
// The products of smaller parts have an accumulator of their own for all of a tile.  It holds at most 2^-7 of the sum of
// |a||b| and meets five instructions for every 16 of K: 4e-11 K of that sum at most (3e-7 for K = 8192), and only
// where all these products have one sign.
constexpr int kChunk = 4;
constexpr int kParts = 3;
enum { kEpiStore = 0, kEpiGateUp = 1, kEpiDact = 2 };

struct GemmProblem {
    int tiles, mt, nt;                            // all tiles; tiles of one replica
    int nseg;
    GemmSeg seg[kGemmMaxSegs];
    int a_mn, b_mn;                               // the operand's K runs along its rows
    int a_box;                                    // rows of a box of A (K along the columns): 128, fewer where M is smaller
    int b_pair;                                   // B of the two CTAs are two matrices, same rows
    int M, N;                                     // of the result
    int out;                                      // map of the result, -1: `ptr` (no 16-byte rows)
    void* ptr;
    long long rep, row;
};

struct GemmArgs {
    CUtensorMap maps[kGemmMaxMaps];
    GemmProblem p[kGemmMaxProblems];
    int problems, tiles;
    // The first `heavy` tiles take much longer than the others: see tile_of.
    int heavy, extra;
    // Stages, and bytes of A from one to the next.  A tile with few rows fetches only those; the tensor cores then
    // read on into the next stage, for rows of D that nobody stores.
    int stages, a_pitch;
    int n_maps;
    uint32_t idesc;                               // instruction descriptor without the majors
    unsigned int* err;
    // gate/up and activation-gradient epilogues: maps of 32 x 32 boxes
    int act;
    int map_a, map_b, map_h;                      // act(G), U act'(G) (-1: not wanted), H; of H, dG and dU the parts
    int map_dg, map_du;                           // follow one another where the values are fp32
};

// ------------------------------------------------------------------------------- PTX
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// One thread of a converged warp.  The single-thread instructions (TMA, tcgen05.mma, commits) are issued
// behind this test and not behind `lane == 0`: only here does the compiler know that one thread is active
// and keeps their operands in uniform registers (measured: the four products of a stage 310 -> 58 cycles, a stage's copies 475 -> 250).
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool mbar_test_now(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(op_smem(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded; after a time-out anywhere in the CTA every wait returns at once and the walk goes on.
__device__ __forceinline__ void mbar_wait(uint64_t* bar, uint32_t parity, volatile int* s_abort, unsigned int* err,
                                          long long cycles = kOpWaitCycles) {
    if (mbar_test_now(bar, parity)) return;
    const long long t0 = clock64();
    unsigned spins = 0;
    while (!mbar_test_now(bar, parity)) {
        if ((++spins & 63u) != 0) continue;
        if (*s_abort) return;
        if (clock64() - t0 > cycles) {
            *s_abort = 1;
            atomicOr(err, kOpErrWaitTimeout);
            return;
        }
    }
}
// This CTA's box of a tensor; completion on the even CTA's barrier (cluster address).
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            op_smem(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_load(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                     op_smem(dst)),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(op_smem(bar))
                 : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, const void* src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z),
                 "r"(op_smem(src))
                 : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}
// Arrives on the barrier at this address in both CTAs once the products issued so far are done.
__device__ __forceinline__ void tc_commit_pair(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     op_smem(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}

#define EG_R8(a, o) "=r"(a[o]), "=r"(a[o + 1]), "=r"(a[o + 2]), "=r"(a[o + 3]), "=r"(a[o + 4]), "=r"(a[o + 5]), "=r"(a[o + 6]), "=r"(a[o + 7])
// 32 (16, 8) columns of this warp's 32 lanes of tensor memory: thread <-> row.
__device__ __forceinline__ void tc_load(uint32_t (&v)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : EG_R8(v, 0), EG_R8(v, 8), EG_R8(v, 16), EG_R8(v, 24)
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_load(uint32_t (&v)[16], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : EG_R8(v, 0), EG_R8(v, 8)
        : "r"(addr)
        : "memory");
}
#undef EG_R8

// Descriptor of a shared-memory operand, 128-byte swizzle.  K-major: groups of 8 rows are 1024 bytes
// apart.  MN-major: groups of 8 rows of K are 1024 bytes apart, the next 64 columns of M or N 8192.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn) {
    uint64_t d = (uint64_t)((addr & 0x3ffff) >> 4);
    d |= (uint64_t)(mn ? (8192 >> 4) : 1) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= 1ull << 46;
    d |= 2ull << 61;
    return d;
}
__device__ __forceinline__ uint32_t swz128(uint32_t off) { return off ^ ((off >> 3) & 0x70u); }
__device__ __forceinline__ uint32_t swz64(uint32_t off) { return off ^ ((off >> 3) & 0x30u); }

// act(g) and its derivative.  The hardware's exponential and reciprocal (errors of a few 2^-23) serve results
// that are rounded to 16 bits; fp32 results take the library's.
__device__ __forceinline__ float rcp_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <typename T> __device__ __forceinline__ float exp_of(float x) {
    if constexpr (sizeof(T) == 4) return expf(x);
    else return __expf(x);
}
template <typename T> __device__ __forceinline__ float sigmoid_of(float x) {
    if constexpr (sizeof(T) == 4) return 1.f / (1.f + expf(-x));
    else return rcp_fast(1.f + __expf(-x));
}
template <typename T, int ACT> __device__ __forceinline__ float act_value(float g) {
    if constexpr (ACT == EG_ACT_SILU) return g * sigmoid_of<T>(g);
    else if constexpr (ACT == EG_ACT_RELU) return g > 0.f ? g : g != g ? g : 0.f;
    else return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
}
template <typename T, int ACT> __device__ __forceinline__ void act_both(float g, float& v, float& dv) {
    if constexpr (ACT == EG_ACT_SILU) {
        const float s = sigmoid_of<T>(g);
        v = g * s;
        dv = fmaf(v, 1.f - s, s);
    } else if constexpr (ACT == EG_ACT_RELU) {
        v = g > 0.f ? g : g != g ? g : 0.f;
        dv = g > 0.f ? 1.f : 0.f;
    } else {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        v = g * cdf;
        dv = fmaf(g * exp_of<T>(-0.5f * g * g), 0.39894228040143268f, cdf);
    }
}
// The activation is chosen once per box of columns, not per element.
template <typename F> __device__ __forceinline__ void with_act(int act, F&& f) {
    if (act == EG_ACT_SILU) f(std::integral_constant<int, EG_ACT_SILU>{});
    else if (act == EG_ACT_GELU) f(std::integral_constant<int, EG_ACT_GELU>{});
    else f(std::integral_constant<int, EG_ACT_RELU>{});
}

// The three bf16 parts of two fp32 values, packed.  Each is rounded to nearest: truncated ones have the value's sign, and
// what the products leave out (2^-21 then) would make every sum too small.  A value that rounds to infinity keeps its leading
// 8 bits as its first part; one that is not finite is its own first part.
__device__ __forceinline__ void split2(float a, float b, uint32_t (&w)[kParts]) {
    constexpr float kTop = 3.3961775e38f;                          // half way from the largest bf16 to infinity
    w[0] = pack2<__nv_bfloat16>(a, b);
    float ra = a - __uint_as_float(w[0] << 16), rb = b - __uint_as_float(w[0] & 0xffff0000u);
    if (!(fabsf(a) < kTop && fabsf(b) < kTop)) {
        if (fabsf(a) >= kTop) {
            w[0] = (w[0] & 0xffff0000u) | __float_as_uint(a) >> 16;
            ra = a - __uint_as_float(w[0] << 16);
        }
        if (fabsf(b) >= kTop) {
            w[0] = (w[0] & 0xffffu) | (__float_as_uint(b) & 0xffff0000u);
            rb = b - __uint_as_float(w[0] & 0xffff0000u);
        }
        if (!isfinite(a)) ra = 0.f;
        if (!isfinite(b)) rb = 0.f;
    }
#pragma unroll
    for (int k = 1; k < kParts; ++k) {
        w[k] = pack2<__nv_bfloat16>(ra, rb);
        ra -= __uint_as_float(w[k] << 16);
        rb -= __uint_as_float(w[k] & 0xffff0000u);
    }
}
// 32 columns of one row (fp32, in registers) as the parts' boxes of 2048 bytes.
__device__ __forceinline__ void write_parts(unsigned char* boxes, int lane, const float (&v)[32]) {
#pragma unroll
    for (int e = 0; e < 32; e += 8) {
        uint32_t w[4][kParts];
#pragma unroll
        for (int z = 0; z < 4; ++z) split2(v[e + 2 * z], v[e + 2 * z + 1], w[z]);
        const uint32_t off = swz64(lane * 64 + e * 2);
#pragma unroll
        for (int k = 0; k < kParts; ++k)
            *reinterpret_cast<uint4*>(boxes + k * 2048 + off) = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
    }
}
__device__ __forceinline__ void write_f32(unsigned char* box, int lane, const float (&v)[32]) {
#pragma unroll
    for (int e = 0; e < 32; e += 4)
        *reinterpret_cast<float4*>(box + swz128(lane * 128 + e * 4)) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
}

// The i-th tile of a pair of CTAs, -1 after its last.  Pairs take turns.  Where the first problem's tiles are longer
// than the others' and do not come out even, the pairs that have one less of them (all from `r` on) first take
// `extra` rounds of the others among themselves; the turns after that run backwards, so that a last, broken one
// falls to those pairs too.
__device__ __forceinline__ int tile_of(const GemmArgs& a, int pair, int pairs, int i) {
    if (a.heavy == 0) {
        const int t = pair + i * pairs;
        return t < a.tiles ? t : -1;
    }
    const int r = a.heavy % pairs, mine = a.heavy / pairs + (pair < r);
    if (i < mine) return pair + i * pairs;
    int j = i - mine;
    int t = a.heavy;
    if (pair >= r && j < a.extra) {
        t += j * (pairs - r) + pair - r;
    } else {
        if (pair >= r) j -= a.extra;
        t += a.extra * (pairs - r) + j * pairs + pairs - 1 - pair;
    }
    return t < a.tiles ? t : -1;
}

struct TilePos {
    int problem, p, m, n;
};
__device__ __forceinline__ TilePos tile_pos(const GemmArgs& a, int t) {
    TilePos q;
    q.problem = 0;
    while (t >= a.p[q.problem].tiles) t -= a.p[q.problem++].tiles;
    const GemmProblem& g = a.p[q.problem];
    const int per = g.mt * g.nt;
    q.p = t / per;
    t -= q.p * per;
    q.n = t / g.mt;                 // neighbouring pairs of CTAs share their rows of B
    q.m = t - q.n * g.mt;
    return q;
}

// `rows` (of 32) rows x `n` columns out of staged boxes of CW columns (WC in all, box after box `next` bytes apart) to
// rows of any alignment; eight rows are read before the first of them is written, since the compiler cannot see that
// the two do not overlap.  16-bit values go out in whole words, one of each row's WC / 2 a lane: rows that start in the
// middle of a word take half of it from the lane before, and their first and last value go by themselves.
template <typename T, int CW, int WC>
__device__ __forceinline__ void write_rows(T* out, long long row, int rows, int n, int lane, const unsigned char* boxes, int next) {
    constexpr int ROW = CW * (int)sizeof(T);
    const bool whole = rows == 32 && n == WC;
    if constexpr (sizeof(T) == 4) {
        constexpr int X = (WC + 31) / 32;
        float* to = out + lane;
#pragma unroll 1
        for (int k = 0; k < 32; k += 8) {
            float v[8][X];
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int x = 0; x < X; ++x)
                    v[u][x] = *reinterpret_cast<const float*>(
                        boxes + x * next + (k + u) * ROW + ((lane % CW * 4) ^ (ROW == 128 ? u << 4 : ROW == 64 ? (u >> 1 & 3) << 4 : 0)));
#pragma unroll
            for (int u = 0; u < 8; ++u, to += row)
#pragma unroll
                for (int x = 0; x < X; ++x)
                    if (whole ? WC >= 32 || lane < WC : k + u < rows && x * 32 + lane < n) to[x * 32] = v[u][x];
        }
    } else {
        constexpr int LANES = WC / 2, EACH = 32 / LANES;        // lanes of a row, rows at a time
        const int j = lane % LANES, sub = lane / LANES;
        uintptr_t at = reinterpret_cast<uintptr_t>(out + sub * row) + 4 * j;
        const unsigned char* from = boxes + 2 * j / CW * next + sub * ROW;
#pragma unroll 1
        for (int k = 0; k < 32; k += 8 * EACH) {
            uint32_t v[8], before[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = *reinterpret_cast<const uint32_t*>(
                    from + (k + u * EACH) * ROW + ((2 * j % CW * 2) ^ (ROW == 64 ? (u * EACH >> 1 & 3) << 4 : 0)));
#pragma unroll
            for (int u = 0; u < 8; ++u) before[u] = __shfl_sync(0xffffffffu, v[u], (j - 1) & (LANES - 1), LANES);
#pragma unroll
            for (int u = 0; u < 8; ++u, at += EACH * row * 2) {
                const bool odd = at & 2;
                const uint32_t word = odd ? __byte_perm(before[u], v[u], 0x5432) : v[u];
                uint32_t* to = reinterpret_cast<uint32_t*>(at & ~(uintptr_t)3);
                uint16_t* first = reinterpret_cast<uint16_t*>(at);
                if (whole) {
                    if (!odd || j > 0) {
                        *to = word;
                    } else {
                        first[0] = (uint16_t)v[u];
                        first[WC - 1] = (uint16_t)(before[u] >> 16);
                    }
                } else if (k + u * EACH + sub < rows) {
                    const int x = 2 * j - odd;
                    if (x < 0) {
                        if (n > 0) first[0] = (uint16_t)v[u];
                        if (n == WC) first[WC - 1] = (uint16_t)(before[u] >> 16);
                    } else if (x + 1 < n) {
                        *to = word;
                    } else if (x < n) {
                        *reinterpret_cast<uint16_t*>(to) = (uint16_t)word;
                    }
                }
            }
        }
    }
}

template <typename T, int EPI, int BN> struct GemmShape {
    static constexpr int kBBytes = BN / 2 * kGemmK * 2;         // of a stage
    // Staging of an epilogue warp, as small as it gets: what it takes is missing for stages.  Two boxes of 64 bytes a
    // row; the gradients' epilogue fetches its factors a box ahead, the fp32 ones stage values of 4 bytes.
    static constexpr int kBoxCols = BN / 2 < 32 ? BN / 2 : 32;
    static constexpr int kEpiBytes = EPI == kEpiStore ? 2 * 32 * kBoxCols * (int)sizeof(T) : EPI == kEpiGateUp && sizeof(T) == 2 ? 4096 : 8192;
    static constexpr int kEpi = kGemmEpiWarps * kEpiBytes;
    static constexpr int kBarBytes = 1024;
    static constexpr int kRing = 227 * 1024 - 1024 - kEpi - kBarBytes;   // both rings of stages
    static constexpr int kBars = kRing / 1024 * 1024 + kEpi;
    static constexpr int kSmem = 1024 + kBars + kBarBytes;
    static constexpr int kCols = BN < 32 ? 32 : BN;             // tensor memory columns of one accumulator
    static constexpr int kTmem = (sizeof(T) == 4 ? 4 : 2) * kCols;      // fp32: two more for the smaller products
    // stages for A boxes of a_pitch bytes
    static int stages(int a_pitch) {
        const int n = kRing / 1024 * 1024 / (a_pitch + kBBytes);
        return n < kGemmMaxStages ? n : kGemmMaxStages;
    }
};

// What one CTA fetches per stage for rows m0.. of A, rows n0.. of B.  Boxes wholly outside the operands stay away (rows and columns of
// D that nobody stores), but one box at least is fetched, so that every fetching thread has a part in every stage: one without could
// fall two rounds behind, take the phase of `empty` for the one before, and wait for good.
__host__ __device__ __forceinline__ uint32_t a_bytes(const GemmProblem& g, int m0) {
    if (g.a_mn) return m0 + 64 < g.M ? 16384u : 8192u;
    return (uint32_t)g.a_box * 128u;
}
template <int BN> __host__ __device__ __forceinline__ uint32_t b_bytes(const GemmProblem& g, int n0) {
    if (!g.b_mn) return (uint32_t)(BN / 2) * 128u;
    uint32_t bytes = 8192u;
#pragma unroll
    for (int h = 64; h < BN / 2; h += 64) bytes += n0 + h < g.N ? 8192u : 0u;
    return bytes;
}
// Where a CTA's first box of an operand begins: at its first row, or where it has none, over the operand's end (a box that is
// nearly all zeros; 16-byte boundaries where the rows run along it).
__host__ __device__ __forceinline__ int first_row(int row, int rows, bool mn) {
    return row < rows ? row : mn ? (rows - 1) / 8 * 8 : rows - 1;
}

// T: type of the operands and of 16-bit results; EPI: what becomes of D; BN: columns of a tile; G: stages under one
// barrier -- where stages are small, one wait serves several.
template <typename T, int EPI, int BN, int G>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1) k_gemm(const __grid_constant__ GemmArgs a) {
    using Shape = GemmShape<T, EPI, BN>;
    const int S = a.stages;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* ring_b = smem + S * G * a.a_pitch;
    unsigned char* epi = smem + Shape::kBars - Shape::kEpi;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Shape::kBars);   // [S] (even CTA's are used)
    uint64_t* empty = full + kGemmMaxStages;                             // [S]
    uint64_t* acc_full = empty + kGemmMaxStages;                                      // [2]
    uint64_t* acc_empty = acc_full + 2;                                  // [2] (even CTA's are used)
    uint64_t* epi_full = acc_empty + 2;                                  // [kGemmEpiWarps][2]
    uint64_t* small_full = epi_full + 2 * kGemmEpiWarps;                 // [2]: fp32, the smaller products' accumulators
    uint64_t* small_empty = small_full + 2;                              // [2] (even CTA's are used)
    volatile int* s_abort = reinterpret_cast<volatile int*>(small_empty + 2);
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(const_cast<int*>(s_abort) + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        *s_abort = 0;
        for (int s = 0; s < S; ++s) { op_mbar_init(&full[s], 1); op_mbar_init(&empty[s], 1); }
        for (int q = 0; q < 2; ++q) {
            op_mbar_init(&acc_full[q], 1); op_mbar_init(&acc_empty[q], 2 * kGemmEpiWarps);
            op_mbar_init(&small_full[q], 1); op_mbar_init(&small_empty[q], 2 * kGemmEpiWarps);
        }
        for (int q = 0; q < 2 * kGemmEpiWarps; ++q) op_mbar_init(&epi_full[q], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) {
        for (int m = lane; m < a.n_maps; m += 32) asm volatile("prefetch.tensormap [%0];" ::"l"(&a.maps[m]) : "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(op_smem(s_tmem)), "n"(Shape::kTmem)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    // set up while the kernel before this one finished; from here on its results are read and overwritten
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (warp == 0 || warp == 3) {
        // warp 0 fetches A (and announces a stage's bytes), warp 3 fetches B
        if (elect_one()) {
            int s = 0, round = 0;
            for (int turn = 0, t; (t = tile_of(a, pair, pairs, turn)) >= 0; ++turn) {
                const TilePos q = tile_pos(a, t);
                const GemmProblem& g = a.p[q.problem];
                const int m0 = q.m * kGemmM + (int)rank * 128, n0 = g.b_pair ? q.n * (BN / 2) : q.n * BN + (int)rank * (BN / 2);
                const uint32_t bytes = a_bytes(g, q.m * kGemmM) + a_bytes(g, q.m * kGemmM + 128) +
                                       b_bytes<BN>(g, g.b_pair ? n0 : q.n * BN) + b_bytes<BN>(g, g.b_pair ? n0 : q.n * BN + BN / 2);
                const bool mn = warp == 0 ? g.a_mn : g.b_mn;
                const int rows = warp == 0 ? g.M : g.N, row = first_row(warp == 0 ? m0 : n0, rows, mn);
                for (int e = 0; e < g.nseg; ++e) {
                    const CUtensorMap* map = &a.maps[warp == 0 ? g.seg[e].a : rank ? g.seg[e].b1 : g.seg[e].b0];
                    const int ksteps = g.seg[e].ksteps;
                    for (int k = 0; k < ksteps; k += G) {
                        // fp32: a step's parts in the order in which their stages become free, 1, 0, 2
#pragma unroll 1
                        for (int part = sizeof(T) == 4 ? 1 : 0, z = 0; z < (sizeof(T) == 4 ? kParts : 1); ++z, part = z == 1 ? 0 : 2) {
                            if (round > 0) mbar_wait(&empty[s], (round - 1) & 1, s_abort, a.err);
                            const int n = G == 1 ? 1 : min(G, ksteps - k), pitch = warp == 0 ? a.a_pitch : Shape::kBBytes;
                            unsigned char* to = (warp == 0 ? smem : ring_b) + s * G * pitch;
                            if (warp == 0 && rank == 0) op_mbar_expect(&full[s], n * bytes);
                            const uint32_t bar = map_to_rank(op_smem(&full[s]), 0);
#pragma unroll
                            for (int h = 0; h < G; ++h, to += pitch) {
                                if (h >= n) break;
                                const int at = (k + h) * kGemmK;
                                tma_load_pair(to, map + part, mn ? row : at, mn ? at : row, q.p, bar);
                                if (mn && (warp == 0 || BN == 256) && row + 64 < rows)
                                    tma_load_pair(to + 8192, map + part, row + 64, at, q.p, bar);
                            }
                            if (++s == S) { s = 0; ++round; }
                        }
                    }
                }
            }
            // the last arrivals on this CTA's barriers, which the even CTA's products send, come in before it ends
            for (int j = max(0, round * S + s - S); j < round * S + s; ++j)
                mbar_wait(&empty[j % S], (j / S) & 1, s_abort, a.err);
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            int s = 0, round = 0, count = 0;                 // count: accumulators handed over
            for (int turn = 0, t; (t = tile_of(a, pair, pairs, turn)) >= 0; ++turn) {
                const TilePos q = tile_pos(a, t);
                const GemmProblem& g = a.p[q.problem];
                const uint32_t idesc = a.idesc | (g.a_mn ? 1u << 15 : 0u) | (g.b_mn ? 1u << 16 : 0u) | ((uint32_t)(BN >> 3) << 17) |
                                       ((uint32_t)(kGemmM >> 4) << 24);
                const uint32_t a_step = g.a_mn ? 2048 >> 4 : 32 >> 4, b_step = g.b_mn ? 2048 >> 4 : 32 >> 4;
                uint32_t add = 0;
                if constexpr (sizeof(T) == 4) {
                    const uint32_t small = tmem + (2 + (turn & 1)) * Shape::kCols;
                    uint32_t add_small = 0;
                    int in_chunk = 0;
                    auto product = [&](uint32_t d, int sa, int sb, uint32_t& add) {
                        const uint64_t da = smem_desc(op_smem(smem + sa * a.a_pitch), g.a_mn);
                        const uint64_t db = smem_desc(op_smem(ring_b + sb * Shape::kBBytes), g.b_mn);
#pragma unroll
                        for (int u = 0; u < kGemmK / 16; ++u) {
                            tc_mma_pair(d, da + u * a_step, db + u * b_step, idesc, add);
                            add = 1;
                        }
                    };
                    int at[kParts];                              // stages of the parts
                    auto next = [&](int part) {
                        mbar_wait(&full[s], round & 1, s_abort, a.err);
                        tc_fence_after();
                        at[part] = s;
                        if (++s == S) { s = 0; ++round; }
                    };
                    if (turn >= 2) {
                        mbar_wait(&small_empty[turn & 1], ((turn >> 1) - 1) & 1, s_abort, a.err);
                        tc_fence_after();
                    }
                    for (int e = 0; e < g.nseg; ++e) {
                        for (int k = 0; k < g.seg[e].ksteps; ++k) {
                            const int buf = count & 1;
                            if (!add) {
                                if (count >= 2) mbar_wait(&acc_empty[buf], ((count >> 1) - 1) & 1, s_abort, a.err);
                                tc_fence_after();
                            }
                            next(1);
                            product(small, at[1], at[1], add_small);
                            next(0);
                            product(small, at[0], at[1], add_small);
                            product(small, at[1], at[0], add_small);
                            tc_commit_pair(&empty[at[1]]);
                            product(tmem + buf * Shape::kCols, at[0], at[0], add);
                            next(2);
                            product(small, at[0], at[2], add_small);
                            product(small, at[2], at[0], add_small);
                            tc_commit_pair(&empty[at[0]]);
                            tc_commit_pair(&empty[at[2]]);
                            if (++in_chunk == kChunk) {
                                tc_commit_pair(&acc_full[buf]);
                                ++count;
                                add = in_chunk = 0;
                            }
                        }
                    }
                    if (add) {
                        tc_commit_pair(&acc_full[count & 1]);
                        ++count;
                    }
                    tc_commit_pair(&small_full[turn & 1]);
                } else {
                    const int buf = count & 1;
                    const uint32_t d = tmem + buf * Shape::kCols;
                    if (count >= 2) mbar_wait(&acc_empty[buf], ((count >> 1) - 1) & 1, s_abort, a.err);
                    tc_fence_after();
                    for (int e = 0; e < g.nseg; ++e) {
                        const int ksteps = g.seg[e].ksteps;
                        for (int k = 0; k < ksteps; k += G) {
                            mbar_wait(&full[s], round & 1, s_abort, a.err);
                            tc_fence_after();
                            const int n = G == 1 ? 1 : min(G, ksteps - k);
                            uint64_t da = smem_desc(op_smem(smem + s * G * a.a_pitch), g.a_mn);
                            uint64_t db = smem_desc(op_smem(ring_b + s * G * Shape::kBBytes), g.b_mn);
#pragma unroll
                            for (int h = 0; h < G; ++h, da += a.a_pitch >> 4, db += Shape::kBBytes >> 4) {
                                if (h >= n) break;
#pragma unroll
                                for (int u = 0; u < kGemmK / 16; ++u) {
                                    tc_mma_pair(d, da + u * a_step, db + u * b_step, idesc, add);
                                    add = 1;
                                }
                            }
                            tc_commit_pair(&empty[s]);
                            if (++s == S) { s = 0; ++round; }
                        }
                    }
                    tc_commit_pair(&acc_full[buf]);
                    ++count;
                }
            }
        }
    } else if (warp >= 4) {
        const int w = warp - 4, half = w >> 2;
        unsigned char* buf_mem = epi + w * Shape::kEpiBytes;
        const uint32_t lanes = (uint32_t)((w & 3) * 32) << 16;
        int count = 0, uses = 0;
        (void)uses;
        for (int turn = 0, t; (t = tile_of(a, pair, pairs, turn)) >= 0; ++turn) {
            const TilePos q = tile_pos(a, t);
            const GemmProblem& g = a.p[q.problem];
            const int buf = count & 1;
            const int row0 = q.m * kGemmM + (int)rank * 128 + (w & 3) * 32;
            const uint32_t acc = tmem + buf * Shape::kCols + lanes;
            // first column of D that this warp's x-th one is (gate/up: half of the gate's, half of the other's)
            auto column = [&](int x) {
                if (EPI == kEpiGateUp) return half * (BN / 4) + (x < BN / 4 ? x : BN / 4 + x);
                return half * (BN / 2) + x;
            };
            float sum[sizeof(T) == 4 ? BN / 2 : 1];          // fp32: this row's BN / 2 columns, added up over the chunks
            if constexpr (sizeof(T) == 4) {
                int ksteps = 0;
                for (int e = 0; e < g.nseg; ++e) ksteps += g.seg[e].ksteps;
                const int chunks = (ksteps + kChunk - 1) / kChunk;
#pragma unroll
                for (int x = 0; x < BN / 2; ++x) sum[x] = 0.f;
                // (what is left of a sum that is not finite is infinity times the zeros of the other's smaller parts)
                auto take = [&](uint32_t from, auto smaller) {
                    constexpr int LW = BN / 2 < 32 ? 16 : 32;
                    tc_fence_after();
#pragma unroll
                    for (int x = 0; x < BN / 2; x += LW) {
                        uint32_t v[LW];
                        tc_load(v, from + lanes + column(x));
#pragma unroll
                        for (int e = 0; e < LW; ++e)
                            if (!decltype(smaller)::value || isfinite(sum[x + e])) sum[x + e] += __uint_as_float(v[e]);
                    }
                    tc_fence_before();
                    __syncwarp();
                };
                for (int z = 0; z < chunks; ++z, ++count) {
                    const int from = count & 1;
                    mbar_wait(&acc_full[from], (count >> 1) & 1, s_abort, a.err);
                    take(tmem + from * Shape::kCols, std::false_type{});
                    if (lane == 0) mbar_arrive_cluster(map_to_rank(op_smem(&acc_empty[from]), 0));
                }
                mbar_wait(&small_full[turn & 1], (turn >> 1) & 1, s_abort, a.err);
                take(tmem + (2 + (turn & 1)) * Shape::kCols, std::true_type{});
                if (lane == 0) mbar_arrive_cluster(map_to_rank(op_smem(&small_empty[turn & 1]), 0));
            }
            if constexpr (EPI == kEpiStore) {
                constexpr int CW = Shape::kBoxCols;                  // columns of one staged box
                constexpr int ROW = CW * (int)sizeof(T);
                auto swz = [](uint32_t off) { return ROW == 128 ? swz128(off) : ROW == 64 ? swz64(off) : off; };
                if constexpr (sizeof(T) == 2) {
                    mbar_wait(&acc_full[buf], (count >> 1) & 1, s_abort, a.err);
                    tc_fence_after();
                }
#pragma unroll
                for (int c = 0; c < BN / 2; c += CW) {
                    const int col0 = q.n * BN + half * (BN / 2) + c;
                    unsigned char* box = buf_mem + (uses & 1) * (Shape::kEpiBytes / 2);
                    store_wait_read<1>();
                    __syncwarp();
                    constexpr int LW = CW < 32 ? 16 : 32;
#pragma unroll
                    for (int x = 0; x < CW; x += LW) {
                        if constexpr (sizeof(T) == 4) {
#pragma unroll
                            for (int e = x; e < x + LW; e += 4)
                                *reinterpret_cast<float4*>(box + swz(lane * ROW + e * 4)) =
                                    make_float4(sum[c + e], sum[c + e + 1], sum[c + e + 2], sum[c + e + 3]);
                        } else {
                            uint32_t v[LW];
                            tc_load(v, acc + half * (BN / 2) + c + x);
#pragma unroll
                            for (int e = 0; e < LW; e += 8) {
                                uint32_t o[4];
#pragma unroll
                                for (int z = 0; z < 4; ++z) o[z] = pack2<T>(__uint_as_float(v[e + 2 * z]), __uint_as_float(v[e + 2 * z + 1]));
                                *reinterpret_cast<uint4*>(box + swz(lane * ROW + (x + e) * 2)) = make_uint4(o[0], o[1], o[2], o[3]);
                            }
                        }
                    }
                    if (g.out >= 0) {
                        fence_async_shared();
                        __syncwarp();
                        if (elect_one()) {
                            if (row0 < g.M && col0 < g.N) tma_store(&a.maps[g.out], box, col0, row0, q.p);
                            store_commit();
                        }
                    } else {
                        if (elect_one()) store_commit();     // an empty group: the wait above counts one a box
                        // two boxes at a time where there are two: longer runs of each row
                        constexpr int WC = BN / 2 < 2 * CW ? BN / 2 : 2 * CW;
                        if ((c + CW) % WC == 0) {
                            __syncwarp();
                            T* out = static_cast<T*>(g.ptr) + (long long)q.p * g.rep + (long long)row0 * g.row + (col0 + CW - WC);
                            write_rows<T, CW, WC>(out, g.row, min(32, g.M - row0), min(WC, g.N - (col0 + CW - WC)), lane,
                                                  WC == CW ? box : buf_mem, Shape::kEpiBytes / 2);
                            __syncwarp();
                        }
                    }
                    ++uses;
                }
            } else if constexpr (EPI == kEpiGateUp) {
                // columns [0, BN/2) of D are the gate's, [BN/2, BN) the other projection's
                constexpr int HW = BN / 4, CW = HW < 32 ? HW : 32;
                if constexpr (sizeof(T) == 2) {
                    mbar_wait(&acc_full[buf], (count >> 1) & 1, s_abort, a.err);
                    tc_fence_after();
                }
#pragma unroll
                for (int c = 0; c < HW; c += CW) {
                    const int col0 = q.n * (BN / 2) + half * HW + c;
                    uint32_t gv[sizeof(T) == 2 ? CW : 1], uv[sizeof(T) == 2 ? CW : 1];
                    if constexpr (sizeof(T) == 2) {
                        tc_load(gv, acc + half * HW + c);
                        tc_load(uv, acc + BN / 2 + half * HW + c);
                    }
                    store_wait_read<0>();
                    __syncwarp();
                    if constexpr (sizeof(T) == 4) {
                        static_assert(CW == 32, "boxes of 32 columns");
                        const float *gs = sum + c, *us = sum + HW + c;
                        float x[32], y[32], z[32];
                        const bool in = row0 < g.M && col0 < g.N;
                        with_act(a.act, [&](auto act) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                act_both<T, decltype(act)::value>(gs[e], y[e], z[e]);
                                x[e] = y[e] * us[e];
                                z[e] *= us[e];
                            }
                        });
                        if (a.map_a >= 0) {
                            write_f32(buf_mem, lane, y);
                            write_f32(buf_mem + 4096, lane, z);
                            fence_async_shared();
                            __syncwarp();
                            if (elect_one()) {
                                if (in) {
                                    tma_store(&a.maps[a.map_a], buf_mem, col0, row0, q.p);
                                    tma_store(&a.maps[a.map_b], buf_mem + 4096, col0, row0, q.p);
                                }
                                store_commit();
                            }
                        }
                        store_wait_read<0>();
                        __syncwarp();
                        write_parts(buf_mem, lane, x);
                        fence_async_shared();
                        __syncwarp();
                        if (elect_one()) {
                            if (in) {
#pragma unroll
                                for (int k = 0; k < kParts; ++k) tma_store(&a.maps[a.map_h + k], buf_mem + k * 2048, col0, row0, q.p);
                            }
                            store_commit();
                        }
                    } else {
                        uint32_t oh[CW / 2], oa[CW / 2], ob[CW / 2];
                        with_act(a.act, [&](auto act) {
#pragma unroll
                            for (int z = 0; z < CW / 2; ++z) {
                                const float u0 = __uint_as_float(uv[2 * z]), u1 = __uint_as_float(uv[2 * z + 1]);
                                float a0, d0, a1, d1;
                                act_both<T, decltype(act)::value>(__uint_as_float(gv[2 * z]), a0, d0);
                                act_both<T, decltype(act)::value>(__uint_as_float(gv[2 * z + 1]), a1, d1);
                                oh[z] = pack2<T>(a0 * u0, a1 * u1);
                                oa[z] = pack2<T>(a0, a1);
                                ob[z] = pack2<T>(d0 * u0, d1 * u1);
                            }
                        });
                        auto send = [&](const uint32_t (&v)[CW / 2], unsigned char* box, int map) {
#pragma unroll
                            for (int z = 0; z < CW / 2; z += 4) {
                                const uint32_t off = lane * (CW * 2) + z * 4;
                                *reinterpret_cast<uint4*>(box + (CW == 32 ? swz64(off) : off)) = make_uint4(v[z], v[z + 1], v[z + 2], v[z + 3]);
                            }
                            fence_async_shared();
                            __syncwarp();
                            if (elect_one()) {
                                if (row0 < g.M && col0 < g.N) tma_store(&a.maps[map], box, col0, row0, q.p);
                                store_commit();
                            }
                        };
                        send(oh, buf_mem, a.map_h);
                        if (a.map_a >= 0) {
                            send(oa, buf_mem + 2048, a.map_a);
                            store_wait_read<1>();
                            __syncwarp();
                            send(ob, buf_mem, a.map_b);
                        }
                    }
                }
            } else if constexpr (sizeof(T) == 4) {
                // D = dH in fp32.  act(G) and U act'(G) fill the staging memory; the parts of dG, then of dU take their place.
                constexpr int BOXES = BN / 2 / 32;
                uint64_t* bar = epi_full + 2 * w;
#pragma unroll
                for (int c = 0; c < BOXES; ++c, ++uses) {
                    const int col0 = q.n * BN + half * (BN / 2) + c * 32;
                    store_wait_read<0>();
                    __syncwarp();
                    if (elect_one()) {
                        op_mbar_expect(bar, 8192);
                        tma_load(buf_mem, &a.maps[a.map_a], col0, row0, q.p, bar);
                        tma_load(buf_mem + 4096, &a.maps[a.map_b], col0, row0, q.p, bar);
                    }
                    mbar_wait(bar, uses & 1, s_abort, a.err);
                    float xg[32], xu[32];
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const uint32_t off = swz128(lane * 128 + e * 4);
                        const float4 a4 = *reinterpret_cast<const float4*>(buf_mem + off);
                        const float4 b4 = *reinterpret_cast<const float4*>(buf_mem + 4096 + off);
                        const float af[4] = {a4.x, a4.y, a4.z, a4.w}, bf[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            const float dh = sum[c * 32 + e + z];
                            xg[e + z] = dh * bf[z];
                            xu[e + z] = dh * af[z];
                        }
                    }
                    const bool in = row0 < g.M && col0 < g.N;
#pragma unroll
                    for (int half_out = 0; half_out < 2; ++half_out) {
                        if (half_out) store_wait_read<0>();
                        __syncwarp();
                        write_parts(buf_mem, lane, half_out ? xu : xg);
                        fence_async_shared();
                        __syncwarp();
                        if (elect_one()) {
                            if (in) {
#pragma unroll
                                for (int k = 0; k < kParts; ++k)
                                    tma_store(&a.maps[(half_out ? a.map_du : a.map_dg) + k], buf_mem + k * 2048, col0, row0, q.p);
                            }
                            store_commit();
                        }
                    }
                }
            } else {
                // D = dH.  act(G) and U act'(G) come in through the two halves of the staging memory, one box of 32
                // columns ahead; dU and dG go out in their place.
                constexpr int BOXES = BN / 2 / 32;
                uint64_t* bars = epi_full + 2 * w;
                auto fetch = [&](int c) {
                    const int col = q.n * BN + half * (BN / 2) + c * 32, slot = (uses + c) & 1;
                    if (elect_one()) {
                        op_mbar_expect(&bars[slot], 4096);
                        tma_load(buf_mem + slot * 4096, &a.maps[a.map_a], col, row0, q.p, &bars[slot]);
                        tma_load(buf_mem + slot * 4096 + 2048, &a.maps[a.map_b], col, row0, q.p, &bars[slot]);
                    }
                };
                store_wait_read<0>();
                __syncwarp();
                fetch(0);
                mbar_wait(&acc_full[buf], (count >> 1) & 1, s_abort, a.err);
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < BOXES; ++c) {
                    const int col0 = q.n * BN + half * (BN / 2) + c * 32, slot = (uses + c) & 1;
                    if (c + 1 < BOXES) {
                        store_wait_read<0>();
                        __syncwarp();
                        fetch(c + 1);
                    }
                    uint32_t v[32];
                    tc_load(v, acc + half * (BN / 2) + c * 32);
                    mbar_wait(&bars[slot], ((uses + c) >> 1) & 1, s_abort, a.err);
                    unsigned char* bg = buf_mem + slot * 4096;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        const uint32_t off = swz64(lane * 64 + e * 2);
                        const uint4 a4 = *reinterpret_cast<const uint4*>(bg + off), b4 = *reinterpret_cast<const uint4*>(bg + 2048 + off);
                        const uint32_t aw[4] = {a4.x, a4.y, a4.z, a4.w}, bw[4] = {b4.x, b4.y, b4.z, b4.w};
                        uint32_t ou[4], og[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            const float2 af = unpack2<T>(aw[z]), bf = unpack2<T>(bw[z]);
                            const float h0 = __uint_as_float(v[e + 2 * z]), h1 = __uint_as_float(v[e + 2 * z + 1]);
                            ou[z] = pack2<T>(h0 * af.x, h1 * af.y);
                            og[z] = pack2<T>(h0 * bf.x, h1 * bf.y);
                        }
                        *reinterpret_cast<uint4*>(bg + off) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
                        *reinterpret_cast<uint4*>(bg + 2048 + off) = make_uint4(og[0], og[1], og[2], og[3]);
                    }
                    fence_async_shared();
                    __syncwarp();
                    if (elect_one()) {
                        if (row0 < g.M && col0 < g.N) {
                            tma_store(&a.maps[a.map_du], bg, col0, row0, q.p);
                            tma_store(&a.maps[a.map_dg], bg + 2048, col0, row0, q.p);
                        }
                        store_commit();
                    }
                }
                uses += BOXES;
            }
            if constexpr (sizeof(T) == 2) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_rank(op_smem(&acc_empty[buf]), 0));
                ++count;
            }
        }
        store_wait_read<0>();
    }
    if (*s_abort) {           // a wait ran out: copies and products in flight get a millisecond to end
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000) {}
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Shape::kTmem) : "memory");
}

}  // namespace eg
