// The products of eg_orthogonalise on the tensor cores (sm_100a).
//
// One launch forms one product of a step for all matrices of all replicas (instances).  X: m x n, m <= n.
//   gram     A = X X^T
//   sym      f0 E0 + f1 E1 + fd L R          of symmetric m x m matrices that commute (all are polynomials of A)
//   apply    X <- a X + S X                  (the last one: into the caller's matrix)
// One step is gram, B = b A + c A^2, apply with B.  Where products are of full precision, two steps share one gram and one apply, since
// the second step's gram is known from the first one's:  Q0 = a0 + B0,  A1 = Q0 A Q0 = a0^2 A + 2 a0 C + C B0 with C = A B0,
// Q1 Q0 = a0 a1 + (a1 B0 + a0 B1 + B1 B0).  Five symmetric products of m^3 take the place of 3 m^2 n + 2 m^3 (8 ResNet-18s: 3.1 -> 2.35 ms).
// The terms that cancel cost accuracy (2.9e-6, step by step 1.7e-6; with a on the diagonals of Q0 and Q1 6e-6, since the accumulators truncate
// what stands beside it), so that two steps stay two where they save little.  With operands of 11 bits the second step would see three times
// the error: there they always do.
//
// Everything in between lies in the workspace as fp16 boxes of 64 x 64, each 8 KB in one piece and already in the order that the
// tensor cores want in shared memory (128-byte swizzle): one tensor map serves all matrices of any size, a copy is a whole box,
// and nothing has rows to be aligned.  Boxes of a column lie one after another.  Edges are filled up with zeros, which stay zeros.
//
// Values are bounded (a singular value starts at most at 1 and the polynomial keeps it below a bound that the host
// derives), so that fp16 with a power of two in front is as wide as needed and has three bits more than bf16.  A value is held as two
// fp16 parts, hi + lo: 22 bits and a sign, an error of 2^-23 at most.
//   PARTS == 1 (results of 8 bits): the products take hi alone, which costs 2^-12 of a value each, about what the result's own
//     rounding does.  X is nevertheless carried on in both parts: the term a X, which alone carries small singular values
//     (485 times over in five steps), sees no rounding to 11 bits.  (One part throughout: error 15 % for a matrix of rank 1.)
//     The diagonals of A and B, far larger than what stands beside them, keep what they were rounded by, rest_A and rest_B, as a float a
//     row that the epilogues put back: (H + D)^2 = H^2 + D H + H D + D^2, and a + rest_B is what the row of X's first parts is multiplied by.
//     Its lower parts, which no product takes, are multiplied by a + B_ii: by a alone, X's two parts would be treated unlike where B is far from
//     zero (-2.7 where singular values are 1): errors of 1.9e-3 instead of 2.2e-3 there, 1.70e-3 instead of 1.83e-3 for 1024 x 2816, 1.66e-3 being
//     the rounding alone, at the same times.
//     (Errors of 6 steps of 64 x 784, result's rounding included, 3.0e-3 without, 2.2e-3 with; 134 -> 139 us there, 4.95 -> 5.0 ms in large ones.)
//     No product reads the lo parts of X: they lie as the epilogue's threads want them (see lane_place), once, and are updated in place.
//   PARTS == 2 (results of 11 and 24 bits): hi hi + hi lo + lo hi.  lo lo, 2^-22 of a product, is left out.
//
// A and B are symmetric: only tiles of 256 x 256 on and below the diagonal are formed and stored.  An operand above it is read
// from the box on the other side, as its transpose: the tensor cores take either order, step by step of K.
//
// Tiles and barriers are those of eg_gemm.cuh: pairs of CTAs share a tile of 256 x BN, tcgen05.mma by one thread, the
// accumulators of two tiles in tensor memory.  PARTS == 2: BN = 128, an accumulator for hi hi that moves to registers every
// one to four steps (ortho_chunk: adding into it truncates) and one for the smaller products.  Sixteen warps take the results: a result is
// added to what was there, split and written again, which is latency upon latency, and eight warps took 11700 cycles for a tile whose products take
// 8200 (m = 1024).
//
// Measured, six matrices of 1024 x 2816 on 8 replicas, bf16 results: gram 127 us (1.1 PFLOP/s of what a symmetric product needs, 1.4 of
// what the tiles on and below the diagonal are), sym 60 us, apply 252 to 280 us (1.1 PFLOP/s; 0.6 GB read, 0.5 GB written: boxes of X and its
// lo parts: a warp's epilogue has one box, so that load, sums and store of a tile follow one another and then the next tile's; the clock falls to
// 1.5 GHz in long runs, which is not what bounds them, since a library product keeps 1.4 PFLOP/s up at 1.34).  ResNet-18 on 8 replicas, fp32
// results: gram 157 us, symmetric products 42 to 52 us, each with tiles for less than two rounds of the machine, apply 267 us.
#pragma once
#include "eg_gemm.cuh"

namespace eg {

constexpr int kBox = 64, kBoxBytes = 8192;
constexpr int kOrthoMats = 48;                    // matrices of one launch
constexpr int kOrthoEpiWarps = 16, kOrthoThreads = 128 + 32 * kOrthoEpiWarps;
// kSym0, kSym1, kSym2: with so many terms E.
enum { kGram = 0, kSym0 = 1, kSym1 = 2, kSym2 = 3, kApply = 4, kLast = 5 };
// Steps of 64 between two hand-overs.  The products run two hand-overs ahead of the warps that take them: with 2 steps they waited for
// those in every short tile, with 1 in every tile (8 ResNet-18s: all products with 4 2.32 ms, with 2 2.5, with 1 2.98).  Products of symmetric
// matrices are short and few, and what they truncate is what the result is off by (error 5.0e-6 with 4 for all, 2.9e-6 with 2 for these, 2.5e-6
// with 1 for all; one 128 x 1152: 3.0e-6 with 2, 1.9e-6 with 1).
template <int PASS> __device__ __forceinline__ int ortho_chunk(int ksteps) { return PASS == kGram || PASS >= kApply ? 4 : ksteps > 2 ? 2 : 1; }

struct Strided {
    void* p;
    long long rep, row;
};

struct OrthoMat {
    int m, n, rb, cb;                             // sides of X, and in boxes
    int flip;                                     // X is the gradient's transpose
    int tiles[2];                                 // of one replica: of the symmetric products, of X
    int first;                                    // instance of replica 0
    float scale;
    long long x[2], lo[2], s[3];                  // first boxes of replica 0: X before and after a step, its lo parts, symmetric matrices
    long long x_rep, s_rep;                       // boxes from one replica to the next; lo parts of symmetric matrices lie half as far
    long long rest, rest_rep;                     // PARTS == 1: boxes with what A's diagonal was rounded by and with B's, rb * 64 floats each
    Strided grad, out, velocity, velocity_out;
    int items, begin;                             // of k_ortho_norm and k_ortho_in: items of an instance, the first one of replica 0
};

// One launch.
struct OrthoPass {
    int from;                                     // which X is read
    int first;                                    // X is still to be multiplied by `turn`
    int l, r, e0, e1, to;                         // symmetric matrices; apply: l
    float f0, f1, fd;                             // gram: fd;  apply: f0 X + fd S X
    int read_lower;                               // PARTS == 1, apply: whether X has lower parts
};

struct OrthoArgs {
    CUtensorMap map;                              // the workspace as rows of 128 bytes
    unsigned char* ws;
    double* partial;                              // [instances][kMaxItems] sums of squares
    int items;
    float* turn;                                  // [instances] what is left of 1 / |u| after a power of two
    unsigned int* err;
    int P, count, parts;
    int tiles[2];
    float momentum;
    int nesterov;
    float sx, out;                                // power of two before X; X -> result
    OrthoMat mat[kOrthoMats];
};

template <int PARTS> struct OrthoShape {
    static constexpr int kBN = PARTS == 2 ? 128 : 256;
    static constexpr int kA = 2 * kBoxBytes * PARTS, kB = kBN / 128 * kBoxBytes * PARTS;     // of a stage and CTA
    static constexpr int kStages = PARTS == 2 ? 3 : 5;
    static constexpr int kEpi = 8 * kBoxBytes;                  // 32 rows x 64 columns, hi and lo, of two warps; PARTS == 1: hi, of one
    static constexpr int kBars = kStages * (kA + kB) + kEpi;
    static constexpr int kSmem = 1024 + kBars + 1024;
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

// The tiles in order, one pair's at a time: t only grows.
struct OrthoWalk {
    int k = 0;
    int base = 0;
};
struct OrthoPos {
    int k = 0, p = 0, i = 0, j = 0;               // matrix, replica, tile row and column
};
template <int PARTS, int PASS> __device__ __forceinline__ OrthoPos ortho_pos(const OrthoArgs& a, OrthoWalk& w, int t) {
    constexpr int S = PASS >= kApply ? 1 : 0, BOXES = OrthoShape<PARTS>::kBN / kBox;
    while (t - w.base >= a.mat[w.k].tiles[S] * a.P) w.base += a.mat[w.k++].tiles[S] * a.P;
    const OrthoMat& m = a.mat[w.k];
    OrthoPos q;
    q.k = w.k;
    int r = t - w.base;
    q.p = r / m.tiles[S];
    r -= q.p * m.tiles[S];
    if (S == 1) {
        const int rows = (m.rb + 3) / 4;
        q.j = r / rows;                           // neighbouring pairs share their columns of X
        q.i = r - q.j * rows;
    } else {
        const int cols = (m.rb + BOXES - 1) / BOXES;
        q.i = 0;
        for (;; ++q.i) {
            const int here = min(cols, (q.i + 1) * (4 / BOXES));
            if (r < here) break;
            r -= here;
        }
        q.j = r;
    }
    return q;
}

__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(op_smem(src)), "r"(bytes) : "memory");
}

// Two values as hi and lo words.
__device__ __forceinline__ void split_half2(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = pack2<__half>(x, y);
    const float2 f = unpack2<__half>(hi);
    lo = pack2<__half>(x - f.x, y - f.y);
}

// Eight values that a row's piece adds to.
__device__ __forceinline__ void add_piece(float* r, float f, const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int z = 0; z < 4; ++z) {
        const float2 h = unpack2<__half>(w[z]);
        r[2 * z] = fmaf(f, h.x, r[2 * z]);
        r[2 * z + 1] = fmaf(f, h.y, r[2 * z + 1]);
    }
}

// The same, each with a factor of its own: f + fd rests.
__device__ __forceinline__ void add_piece(float* r, float f, float fd, const float* rests, const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int z = 0; z < 4; ++z) {
        const float2 h = unpack2<__half>(w[z]);
        r[2 * z] = fmaf(fmaf(fd, rests[2 * z], f), h.x, r[2 * z]);
        r[2 * z + 1] = fmaf(fmaf(fd, rests[2 * z + 1], f), h.y, r[2 * z + 1]);
    }
}

// Byte of a lo part that no product reads: 8 columns of a row are a thread's 16 bytes, next to those of the rows above and below.
__device__ __forceinline__ int lane_place(int row, int col) { return (row >> 5) * 4096 + (col >> 3) * 512 + (row & 31) * 16 + (col & 7) * 2; }

// T: type of the caller's matrices (kLast).
template <typename T, int PARTS, int PASS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kOrthoThreads, 1) k_ortho(const __grid_constant__ OrthoArgs a, const OrthoPass pass) {
    using Shape = OrthoShape<PARTS>;
    constexpr int BN = Shape::kBN, S = Shape::kStages;
    constexpr bool SYMMETRIC = PASS < kApply;
    constexpr int TERMS = PASS == kGram || PASS == kSym0 ? 0 : PASS == kSym2 ? 2 : 1;      // that come in from memory
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* ring_b = smem + S * Shape::kA;
    unsigned char* epi = ring_b + S * Shape::kB;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Shape::kBars);   // [S] (even CTA's are used)
    uint64_t* empty = full + S;                                          // [S]
    uint64_t* acc_full = empty + S;                                      // [2]
    uint64_t* acc_empty = acc_full + 2;                                  // [2] (even CTA's are used)
    uint64_t* small_full = acc_empty + 2;                                // [2]: accumulators of the smaller products
    uint64_t* small_empty = small_full + 2;                              // [2] (even CTA's are used)
    uint64_t* epi_full = small_empty + 2;                                // [kOrthoEpiWarps]
    volatile int* s_abort = reinterpret_cast<volatile int*>(epi_full + kOrthoEpiWarps);
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(const_cast<int*>(s_abort) + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        *s_abort = 0;
        for (int s = 0; s < S; ++s) { op_mbar_init(&full[s], 1); op_mbar_init(&empty[s], 1); }
        for (int q = 0; q < 2; ++q) {
            op_mbar_init(&acc_full[q], 1); op_mbar_init(&acc_empty[q], 2 * kOrthoEpiWarps);
            op_mbar_init(&small_full[q], 1); op_mbar_init(&small_empty[q], 2 * kOrthoEpiWarps);
        }
        for (int q = 0; q < kOrthoEpiWarps; ++q) op_mbar_init(&epi_full[q], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3 && lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&a.map) : "memory");
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(op_smem(s_tmem)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = *s_tmem;
    // Set up, and the first tile looked up, while the kernel before this one finishes; whoever reads its results, or what others do with
    // them, waits for its end.
    auto wait_before = [] { asm volatile("griddepcontrol.wait;" ::: "memory"); };
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1, tiles = a.tiles[SYMMETRIC ? 0 : 1];
    const int from = pass.from;
    OrthoWalk walk;

    if (warp == 0 || warp == 3) {
        // warp 0 fetches the left operand (and announces a stage's bytes), warp 3 the right one
        if (elect_one()) {
            int s = 0, round = 0;
            OrthoPos upcoming = ortho_pos<PARTS, PASS>(a, walk, pair);
            wait_before();
            for (int t = pair; t < tiles; t += pairs) {
                const OrthoPos q = upcoming;                                  // (the one after it is looked up under the copies)
                const OrthoMat& g = a.mat[q.k];
                const bool left = warp == 0;
                const long long x = g.x[from] + q.p * g.x_rep, sym = g.s[left ? pass.l : pass.r] + q.p * g.s_rep;
                const int ksteps = PASS == kGram ? g.cb : g.rb;
                constexpr int RIGHT = BN / 128;                           // boxes of the right operand that a CTA fetches
                const int limit = left || SYMMETRIC ? g.rb : g.cb;
                // The two operands of a tile on the diagonal are the same rows of one matrix: fetched once, a box by either warp.
                const bool share = PARTS == 1 && SYMMETRIC && q.i == q.j;
                // Boxes of an operand that a CTA fetches: those that are there (what the other rows and columns of D become, nobody stores), but one at
                // least.  Every fetching thread has a part in every stage that way: one without could fall two rounds behind, take the phase of
                // `empty` for the one before, and wait for good.  (An arrival from each instead, across the pair: 4.9 -> 7.5 ms for the largest case.)
                auto boxes = [&](bool of_left, int r) {
                    const int wide = of_left ? 2 : RIGHT, first = of_left ? q.i * 4 + r * 2 : q.j * (2 * RIGHT) + r * RIGHT;
                    return share ? 1 : max(1, min(wide, (of_left || SYMMETRIC ? g.rb : g.cb) - first));
                };
                const int have = boxes(left, (int)rank);
                const int box0 = min(share ? q.i * 4 + (int)rank * 2 + (left ? 0 : 1) : left ? q.i * 4 + (int)rank * 2 : q.j * (2 * RIGHT) + (int)rank * RIGHT,
                                     limit - 1);
                const int block = left ? q.i : q.j * (2 * RIGHT) / 4;     // rows or columns of 256
                uint32_t bytes = 0;
                if (left && rank == 0) bytes = (uint32_t)(boxes(true, 0) + boxes(true, 1) + boxes(false, 0) + boxes(false, 1)) * kBoxBytes * PARTS;
                if (*s_abort) break;                                      // (after a time-out nobody starts anything more)
                for (int k = 0; k < ksteps; ++k) {
                    if (round > 0) mbar_wait(&empty[s], (round - 1) & 1, s_abort, a.err);
                    if (*s_abort) break;
                    unsigned char* to = left ? smem + s * Shape::kA : share ? smem + s * Shape::kA + kBoxBytes : ring_b + s * Shape::kB;
                    const uint32_t bar = map_to_rank(op_smem(&full[s]), 0);
                    if (left && rank == 0) op_mbar_expect(&full[s], bytes);
                    // (row, k) of a stored box; above the diagonal of a symmetric operand its mirror image; X by its columns
                    long long box, next, lo;
                    const bool is_x = PASS == kGram || (!SYMMETRIC && !left);
                    if (is_x) {
                        const bool by_column = !SYMMETRIC;
                        box = x + (by_column ? (long long)box0 * g.rb + k : (long long)k * g.rb + box0);
                        next = by_column ? g.rb : 1;
                        lo = g.lo[from] - g.x[from];
                    } else {
                        const bool mirror = k / 4 > block;
                        box = sym + (mirror ? (long long)box0 * g.rb + k : (long long)k * g.rb + box0);
                        next = mirror ? g.rb : 1;
                        lo = g.s_rep / 2;
                    }
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (h < have)
                                tma_load_pair(to + (part * (left ? 2 : RIGHT) + h) * kBoxBytes, &a.map, 0, (int)((box + h * next + part * lo) * kBox), 0, bar);
                        }
                    }
                    if (++s == S) { s = 0; ++round; }
                    if (k == 0 && t + pairs < tiles) upcoming = ortho_pos<PARTS, PASS>(a, walk, t + pairs);
                }
            }
            // the last arrivals on this CTA's barriers, which the even CTA's products send, come in before it ends
            for (int j = max(0, round * S + s - S); j < round * S + s; ++j) mbar_wait(&empty[j % S], (j / S) & 1, s_abort, a.err);
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            int s = 0, round = 0, count = 0, turn = 0;          // count: accumulators handed over; turn: tiles
            OrthoPos upcoming = ortho_pos<PARTS, PASS>(a, walk, pair);
            wait_before();                                      // (reads nothing of that kernel's, but the limits of its waits start here)
            for (int t = pair; t < tiles; t += pairs, ++turn) {
                const OrthoPos q = upcoming;                                  // (the one after it is looked up under the products)
                const OrthoMat& g = a.mat[q.k];
                const int ksteps = PASS == kGram ? g.cb : g.rb, right_block = q.j * (BN / kBox) / 4;
                const bool share = PARTS == 1 && SYMMETRIC && q.i == q.j;
                uint32_t add = 0, add_small = 0;
                const uint32_t small = tmem + (2 + (turn & 1)) * 128;
                if (PARTS == 2 && turn >= 2) mbar_wait(&small_empty[turn & 1], ((turn >> 1) - 1) & 1, s_abort, a.err);
                for (int k = 0; k < ksteps; ++k) {
                    const bool a_mn = PASS != kGram && k / 4 > q.i, b_mn = PASS >= kApply || (PASS != kGram && k / 4 > right_block);
                    const uint32_t idesc = (1u << 4) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(BN >> 3) << 17) |
                                           ((uint32_t)(kGemmM >> 4) << 24);
                    const uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
                    if (!add) {
                        if (count >= 2) mbar_wait(&acc_empty[count & 1], ((count >> 1) - 1) & 1, s_abort, a.err);
                        tc_fence_after();
                    }
                    const uint32_t d = tmem + (count & 1) * BN;
                    mbar_wait(&full[s], round & 1, s_abort, a.err);
                    if (*s_abort) break;
                    tc_fence_after();
                    auto product = [&](uint32_t to, int pa, int pb, uint32_t& add_to) {
                        unsigned char* l = smem + s * Shape::kA + pa * 2 * kBoxBytes;
                        const uint64_t da = smem_desc(op_smem(l), a_mn);
                        const uint64_t db = smem_desc(op_smem(share ? l : ring_b + s * Shape::kB + pb * (BN / 128) * kBoxBytes), b_mn);
#pragma unroll
                        for (int u = 0; u < kGemmK / 16; ++u) {
                            tc_mma_pair(to, da + u * a_step, db + u * b_step, idesc, add_to);
                            add_to = 1;
                        }
                    };
                    product(d, 0, 0, add);
                    if constexpr (PARTS == 2) {
                        product(small, 0, 1, add_small);
                        product(small, 1, 0, add_small);
                    }
                    tc_commit_pair(&empty[s]);
                    if (++s == S) { s = 0; ++round; }
                    if (k == 0 && t + pairs < tiles) upcoming = ortho_pos<PARTS, PASS>(a, walk, t + pairs);
                    if (PARTS == 2 && k + 1 < ksteps && (k + 1) % ortho_chunk<PASS>(ksteps) == 0) {
                        tc_commit_pair(&acc_full[count & 1]);
                        ++count;
                        add = 0;
                    }
                }
                if (*s_abort) break;
                tc_commit_pair(&acc_full[count & 1]);
                ++count;
                if (PARTS == 2) tc_commit_pair(&small_full[turn & 1]);
            }
        }
    } else if (warp >= 4) {
        // rows 32 * quad of the CTA's 128; PARTS == 1: the 64 columns of one box;  2: 32 columns, half of a box that two warps share
        const int w = warp - 4, quad = w & 3, group = w >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        int count = 0, turn = 0, uses = 0;
        OrthoPos q = ortho_pos<PARTS, PASS>(a, walk, pair);
        wait_before();
        for (int t = pair; t < tiles; t += pairs, ++turn) {
            // (after a time-out nobody starts anything more; warps that share a box leave together)
            if (PARTS == 1 ? (bool)__any_sync(0xffffffffu, *s_abort) : op_leave_together(1 + quad + 4 * (group >> 1), 64, s_abort)) break;
            if (t != pair) q = ortho_pos<PARTS, PASS>(a, walk, t);
            const OrthoMat& g = a.mat[q.k];
            const int ksteps = PASS == kGram ? g.cb : g.rb;
            const int rbox = q.i * 4 + (int)rank * 2 + (quad >> 1), cbox = q.j * (BN / kBox) + (PARTS == 1 ? group : group >> 1);
            const bool inside = rbox < g.rb && cbox < (SYMMETRIC ? g.rb : g.cb);
            const long long x = g.x[from] + q.p * g.x_rep, to = SYMMETRIC ? g.s[pass.to] + q.p * g.s_rep : g.x[from ^ 1] + q.p * g.x_rep;
            const float left_of = pass.first && (PASS == kGram || PASS >= kApply) ? a.turn[g.first + q.p] : 1.f;
            const float by = PASS == kGram ? left_of * left_of : left_of;
            // half a box, 32 rows: 4 KB in one piece
            auto place = [&](long long matrix) { return a.ws + (matrix + (long long)cbox * g.rb + rbox) * kBoxBytes + (quad & 1) * 4096; };
            const int row0 = rbox * kBox + (quad & 1) * 32;
            const float scale = a.out * g.scale;
            T* const out = PASS == kLast ? static_cast<T*>(g.out.p) + q.p * g.out.rep : nullptr;
            if constexpr (PARTS == 1) {
                unsigned char* box = epi + w * 4096;
                uint4 low[PASS >= kApply ? 8 : 1];
                unsigned char* const low_at = PASS >= kApply ? place(g.lo[0] + q.p * g.x_rep) + lane * 16 : nullptr;
                float* const rest_a = reinterpret_cast<float*>(a.ws + (g.rest + q.p * g.rest_rep) * kBoxBytes);
                float* const diagonal_b = rest_a + g.rb * kBox;
                const bool diagonal = SYMMETRIC && rbox == cbox;
                // of this thread's row: what is put back; its value on the diagonal, formed (symmetric) or read (applications, of B)
                float rest = 0.f, own = 0.f;
                auto rounded_by = [](float v) { return v - __half2float(__float2half_rn(v)); };
                if (inside && TERMS > 0) {                        // what the result is added to comes in under the products
                    store_wait_read<0>();
                    __syncwarp();
                    if (elect_one()) {
                        op_mbar_expect(&epi_full[w], 4096);
                        op_bulk_load(box, place(SYMMETRIC ? g.s[pass.e0] + q.p * g.s_rep : x), 4096, &epi_full[w]);
                    }
                    if constexpr (SYMMETRIC) {
                        rest = rest_a[row0 + lane];
                    } else {
                        own = diagonal_b[row0 + lane];
                        rest = rounded_by(own);
                    }
                    if constexpr (PASS == kSym1) {
                        if (lane < 2) asm volatile("prefetch.global.L1 [%0];" ::"l"(rest_a + cbox * kBox + lane * 32));
                    }
                    if constexpr (PASS >= kApply) {
#pragma unroll
                        for (int z = 0; z < 8; ++z) low[z] = pass.read_lower ? *reinterpret_cast<const uint4*>(low_at + z * 512) : make_uint4(0, 0, 0, 0);
                    }
                }
                mbar_wait(&acc_full[count & 1], (count >> 1) & 1, s_abort, a.err);
                tc_fence_after();
                const uint32_t acc = tmem + (count & 1) * BN + lanes + group * 64;
                const float f0 = fmaf(pass.fd, rest, pass.f0), f0_low = PASS >= kApply ? fmaf(pass.fd, own, pass.f0) : 0.f;
                if (inside) {
                    if (TERMS == 0) {
                        store_wait_read<0>();
                        __syncwarp();
                    } else {
                        mbar_wait(&epi_full[w], uses & 1, s_abort, a.err);
                        ++uses;
                    }
#pragma unroll
                    for (int x0 = 0; x0 < 64; x0 += 16) {
                        uint32_t d[16];
                        tc_load(d, acc + x0);
#pragma unroll
                        for (int e = 0; e < 16; e += 8) {
                            const int piece = (x0 + e) >> 3;
                            unsigned char* at = box + lane * 128 + ((piece ^ (lane & 7)) << 4);
                            float r[8];
#pragma unroll
                            for (int z = 0; z < 8; ++z) r[z] = pass.fd * __uint_as_float(d[e + z]);
                            if constexpr (PASS == kSym1) {
                                float rests[8];
                                *reinterpret_cast<float4*>(rests) = *reinterpret_cast<const float4*>(rest_a + cbox * kBox + x0 + e);
                                *reinterpret_cast<float4*>(rests + 4) = *reinterpret_cast<const float4*>(rest_a + cbox * kBox + x0 + e + 4);
                                add_piece(r, f0, pass.fd, rests, *reinterpret_cast<const uint4*>(at));
                            } else if constexpr (TERMS > 0) {
                                add_piece(r, f0, *reinterpret_cast<const uint4*>(at));
                            }
                            if constexpr (PASS >= kApply) add_piece(r, f0_low, low[piece]);
                            if constexpr (PASS == kGram || PASS >= kApply) {
#pragma unroll
                                for (int z = 0; z < 8; ++z) r[z] *= by;
                            }
                            if (diagonal) {
#pragma unroll
                                for (int z = 0; z < 8; ++z) {
                                    if (x0 + e + z != (quad & 1) * 32 + lane) continue;
                                    if constexpr (PASS == kSym1) r[z] = fmaf(fmaf(pass.fd, rest, pass.f0), rest, r[z]);
                                    own = r[z];
                                }
                            }
                            uint32_t hw[4], lw[4];
#pragma unroll
                            for (int z = 0; z < 4; ++z) {
                                if constexpr (PASS == kLast && sizeof(T) == 2) hw[z] = pack2<T>(r[2 * z] * scale, r[2 * z + 1] * scale);
                                else split_half2(r[2 * z], r[2 * z + 1], hw[z], lw[z]);
                            }
                            *reinterpret_cast<uint4*>(at) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
                            if constexpr (PASS == kApply) *reinterpret_cast<uint4*>(low_at + piece * 512) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_rank(op_smem(&acc_empty[count & 1]), 0));
                ++count;
                if (!inside) continue;
                if (diagonal) (PASS == kGram ? rest_a : diagonal_b)[row0 + lane] = PASS == kGram ? rounded_by(own) : own;
                if constexpr (PASS != kLast) {
                    fence_async_shared();
                    __syncwarp();
                    if (elect_one()) {
                        bulk_store(place(to), box, 4096);
                        store_commit();
                    }
                } else if constexpr (sizeof(T) == 2) {
                    const int col0 = cbox * kBox, rows = min(32, g.m - row0), n = min(64, g.n - col0);
                    if (g.flip) {                                 // a row of X is a column of the result
                        if (lane < rows) {
                            T* line = out + (long long)col0 * g.out.row + row0 + lane;
#pragma unroll 8
                            for (int e = 0; e < n; ++e)
                                line[e * g.out.row] = *reinterpret_cast<const T*>(box + lane * 128 + (((e >> 3) ^ (lane & 7)) << 4) + (e & 7) * 2);
                        }
                    } else {                                      // runs along the rows
                        T* line = out + (long long)row0 * g.out.row + col0;
                        const bool words = ((uintptr_t)line & 3) == 0 && (g.out.row & 1) == 0;
#pragma unroll 4
                        for (int r = 0; r < rows; ++r, line += g.out.row) {
                            const uint32_t v = *reinterpret_cast<const uint32_t*>(box + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4);
                            if (words && 2 * lane + 1 < n) {
                                *reinterpret_cast<uint32_t*>(line + 2 * lane) = v;
                            } else {
                                uint16_t* o = reinterpret_cast<uint16_t*>(line + 2 * lane);
                                if (2 * lane < n) o[0] = (uint16_t)v;
                                if (2 * lane + 1 < n) o[1] = (uint16_t)(v >> 16);
                            }
                        }
                    }
                    // the next box's copy comes by another way than these reads
                    fence_async_shared();
                    __syncwarp();
                }
            } else {
                const int sub = group & 1, pair_of = quad + 4 * (group >> 1);      // the two warps of a box
                unsigned char* box = epi + pair_of * kBoxBytes;
                auto together = [&] { op_named_barrier(1 + pair_of, 64); };
                const long long lo = SYMMETRIC ? g.s_rep / 2 : g.lo[from] - g.x[from], lo_to = SYMMETRIC ? g.s_rep / 2 : g.lo[from ^ 1] - g.x[from ^ 1];
                auto fetch = [&](int term) {                      // by the first of the two warps
                    if (sub == 0) {
                        store_wait_read<0>();
                        __syncwarp();
                        if (elect_one() && !*s_abort) {           // (a time-out in this tile: the barrier may still be armed)
                            const long long matrix = SYMMETRIC ? g.s[term ? pass.e1 : pass.e0] + q.p * g.s_rep : x;
                            op_mbar_expect(&epi_full[pair_of], 8192);
                            op_bulk_load(box, place(matrix), 4096, &epi_full[pair_of]);
                            op_bulk_load(box + 4096, place(matrix + lo), 4096, &epi_full[pair_of]);
                        }
                    }
                };
                auto piece_at = [&](int z) { return box + lane * 128 + (((sub * 4 + z) ^ (lane & 7)) << 4); };
                if (inside && TERMS > 0) fetch(0);
                float sum[32];                                    // this row's 32 columns: the terms, then the products' chunks
#pragma unroll
                for (int e = 0; e < 32; ++e) sum[e] = 0.f;
                if (inside) {
#pragma unroll 1
                    for (int term = 0; term < TERMS; ++term) {
                        if (term > 0) {
                            together();                           // both have read the first one
                            fetch(term);
                        }
                        mbar_wait(&epi_full[pair_of], uses & 1, s_abort, a.err);
                        ++uses;
                        const float f = term ? pass.f1 : pass.f0;
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            add_piece(sum + z * 8, f, *reinterpret_cast<const uint4*>(piece_at(z) + 4096));
                            add_piece(sum + z * 8, f, *reinterpret_cast<const uint4*>(piece_at(z)));
                        }
                    }
                }
                auto take = [&](uint32_t acc) {
                    tc_fence_after();
                    uint32_t v[32];
                    tc_load(v, acc + lanes + group * 32);
#pragma unroll
                    for (int z = 0; z < 32; ++z) sum[z] = fmaf(pass.fd, __uint_as_float(v[z]), sum[z]);
                    tc_fence_before();
                    __syncwarp();
                };
                const int chunk = ortho_chunk<PASS>(ksteps);
                for (int z = 0; z < (ksteps + chunk - 1) / chunk; ++z, ++count) {
                    mbar_wait(&acc_full[count & 1], (count >> 1) & 1, s_abort, a.err);
                    take(tmem + (count & 1) * BN);
                    if (lane == 0) mbar_arrive_cluster(map_to_rank(op_smem(&acc_empty[count & 1]), 0));
                }
                mbar_wait(&small_full[turn & 1], (turn >> 1) & 1, s_abort, a.err);
                take(tmem + (2 + (turn & 1)) * 128);
                if (lane == 0) mbar_arrive_cluster(map_to_rank(op_smem(&small_empty[turn & 1]), 0));
                if (!inside) continue;
                if constexpr (PASS == kGram || PASS >= kApply) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) sum[e] *= by;
                }
                if (TERMS == 0 || PASS == kLast) {                // the box is free: its store has been read; both have read what it held
                    if (sub == 0) store_wait_read<0>();
                    together();
                }
                if constexpr (PASS != kLast) {
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        uint32_t hw[4], lw[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y) split_half2(sum[z * 8 + 2 * y], sum[z * 8 + 2 * y + 1], hw[y], lw[y]);
                        *reinterpret_cast<uint4*>(piece_at(z)) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
                        *reinterpret_cast<uint4*>(piece_at(z) + 4096) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
                    }
                    fence_async_shared();
                    together();
                    if (sub == 0 && elect_one()) {
                        bulk_store(place(to), box, 4096);
                        bulk_store(place(to + lo_to), box + 4096, 4096);
                        store_commit();
                    }
                } else {
                    const int col0 = cbox * kBox + sub * 32, rows = min(32, g.m - row0), n = min(32, g.n - col0);
                    if (g.flip) {                                 // a row of X is a column of the result
                        if (lane < rows) {
                            T* line = out + (long long)col0 * g.out.row + row0 + lane;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (e < n) line[e * g.out.row] = from_f32<T>(sum[e] * scale);
                        }
                    } else {
                        // through this warp's half of the box, 32 rows of 32 values, to runs along the rows
                        unsigned char* mine = box + sub * 4096;
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            *reinterpret_cast<float4*>(mine + lane * 128 + (((e >> 2) ^ (lane & 7)) << 4)) =
                                make_float4(sum[e] * scale, sum[e + 1] * scale, sum[e + 2] * scale, sum[e + 3] * scale);
                        __syncwarp();
                        T* line = out + (long long)row0 * g.out.row + col0;
#pragma unroll 8
                        for (int r = 0; r < rows; ++r, line += g.out.row) {
                            const float f = *reinterpret_cast<const float*>(mine + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4);
                            if (lane < n) line[lane] = from_f32<T>(f);
                        }
                    }
                    // the next box's copy comes by another way than these accesses
                    fence_async_shared();
                    together();
                }
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
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

}  // namespace eg
