// The gated feed-forward block of every replica (eg_feed_forward) and its gradients: the plan of
// buffers and products, and the launches.  The products run in eg_gemm.cuh.
//
//   forward   1. [G | U] = x [Wg | Wu]^T with H = act(G) * U formed from the accumulators   (one launch)
//             2. y = H Wd^T
//   backward  3. dH = dy Wd with dU = dH * act(G), dG = dH * U act'(G) formed from the accumulators and the
//                saved factors (which the forward pass has in fp32: one rounding each, and no exponential here)
//             4. dx = dG Wg + dU Wu,  dWd = dy^T H,  dWg = dG^T x,  dWu = dU^T x           (one launch)
//
// Without `saved`, few tokens take two streams over the weights instead (eg_ffn_few.cuh).
#include <initializer_list>

#include "eg_ffn_few.cuh"
#include "eg_gemm.cuh"
#include "eg_tensor_map.cuh"

namespace eg {
namespace {

struct Mat {
    void* p;
    long long rep, row;
};

// ----------------------------------------------------------------------------------- tensor maps
// Rows on 16-byte boundaries, which the copies need.
bool in_place(const Mat& m, long long P, long long rows, size_t size) {
    return aligned16(m.p) && (rows <= 1 || m.row * (long long)size % 16 == 0) && (P <= 1 || m.rep * (long long)size % 16 == 0);
}

// [P][rows][cols] matrix in boxes of box_rows x box_cols.
bool encode(CUtensorMap* map, int dtype, const Mat& m, long long P, long long rows, long long cols, int box_cols, int box_rows) {
    EncodeFn fn = encoder();
    if (!fn) return false;
    const size_t size = dtype == EG_F32 ? 4 : 2;
    const long long pad = (cols * (long long)size + 15) / 16 * 16;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)P};
    const cuuint64_t row = rows > 1 ? (cuuint64_t)(m.row * (long long)size) : (cuuint64_t)pad;
    const cuuint64_t strides[2] = {row, P > 1 ? (cuuint64_t)(m.rep * (long long)size) : row * (cuuint64_t)rows};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
    const int bytes = box_cols * (int)size;
    return fn(map,
              dtype == EG_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                              : dtype == EG_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
              3, m.p, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
              bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ----------------------------------------------------------------------------------- copies
// Operands that the products cannot read in place: 16-bit rows of any stride and alignment go to rows on 16-byte
// boundaries, fp32 rows to their three bf16 parts (matrices `plane` elements apart).  One launch for all of a
// call; a warp takes 512 columns of one row in aligned pieces of 16 bytes, all its loads ahead of its stores, and shifts
// them into place.  Bound by memory: 6 x 3 matrices of 1905 x 5909 in bf16 take 166 us (4.9 TB/s).
constexpr int kCopyMax = 5, kCopyTurns = 2, kCopyCols = kCopyTurns * 256;
struct CopyArgs {
    struct { Mat src, dst; long long plane, rows, begin; int cols, chunks; } m[kCopyMax];   // begin: first unit of the matrix
    long long units;
    int count;
};

template <typename T> __global__ void __launch_bounds__(256) k_copy_in(const __grid_constant__ CopyArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int WORDS = 2 * (int)sizeof(T), V = 16 / (int)sizeof(T);    // 8 values in words; values of 16 bytes
    const int lane = threadIdx.x & 31;
    for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < a.units; u += (long long)gridDim.x * 8) {
        int k = 0;
        while (k + 1 < a.count && u >= a.m[k + 1].begin) ++k;
        const auto& m = a.m[k];
        const long long at = u - m.begin, line = at / m.chunks, i = line / m.rows, r = line % m.rows;
        const int c0 = (int)(at % m.chunks) * kCopyCols;
        const T* s = static_cast<const T*>(m.src.p) + i * m.src.rep + r * m.src.row + c0;
        uint16_t* d = static_cast<uint16_t*>(m.dst.p) + i * m.dst.rep + r * m.dst.row + c0;
        const int n = m.cols - c0;                          // columns of the row from here on
        const int shift = (int)((uintptr_t)s / sizeof(T)) & (V - 1);
        const uint4* from = reinterpret_cast<const uint4*>(s - shift);
        // lane's 8 values of turn q begin `shift` values into its 16-byte pieces; what lies behind comes from the next
        // lane, behind the last lane's from the next turn's first.  Pieces without a value of the row stay unread.
        uint32_t w[kCopyTurns][WORDS];
#pragma unroll
        for (int q = 0; q < kCopyTurns; ++q) {
#pragma unroll
            for (int z = 0; z < WORDS / 4; ++z) {
                const int piece = (q * 32 + lane) * (WORDS / 4) + z;
                const uint4 x = piece * V - shift < n ? from[piece] : make_uint4(0, 0, 0, 0);
                w[q][4 * z] = x.x; w[q][4 * z + 1] = x.y; w[q][4 * z + 2] = x.z; w[q][4 * z + 3] = x.w;
            }
        }
        uint4 tail = make_uint4(0, 0, 0, 0);
        if (lane == 0 && shift > 0 && kCopyCols - shift < n) tail = from[kCopyCols / V];
#pragma unroll
        for (int q = 0; q < kCopyTurns; ++q) {
            uint32_t x[WORDS + 4];
#pragma unroll
            for (int z = 0; z < WORDS; ++z) x[z] = w[q][z];
            if (shift > 0) {                                // the same for the whole warp
                const uint32_t next[4] = {tail.x, tail.y, tail.z, tail.w};
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const uint32_t first = q + 1 < kCopyTurns ? w[q + 1 < kCopyTurns ? q + 1 : q][z] : next[z];
                    x[WORDS + z] = __shfl_sync(0xffffffffu, lane == 0 ? first : w[q][z], (lane + 1) & 31);
                }
                const int words = shift * (int)sizeof(T) / 4;
                if (words & 2)
#pragma unroll
                    for (int z = 0; z < WORDS + 2; ++z) x[z] = x[z + 2];
                if (words & 1)
#pragma unroll
                    for (int z = 0; z < WORDS + 1; ++z) x[z] = x[z + 1];
                if (sizeof(T) == 2 && (shift & 1))
#pragma unroll
                    for (int z = 0; z < WORDS; ++z) x[z] = __funnelshift_r(x[z], x[z + 1], 16);
            }
            const int c = (q * 32 + lane) * 8;              // the pitch is a multiple of 64: what follows the last value is room
            if (c >= n) continue;
            if constexpr (sizeof(T) == 4) {
                uint32_t p[4][kParts];
#pragma unroll
                for (int z = 0; z < 4; ++z) split2(__uint_as_float(x[2 * z]), __uint_as_float(x[2 * z + 1]), p[z]);
#pragma unroll
                for (int z = 0; z < kParts; ++z)
                    *reinterpret_cast<uint4*>(d + z * m.plane + c) = make_uint4(p[0][z], p[1][z], p[2][z], p[3][z]);
            } else {
                *reinterpret_cast<uint4*>(d + c) = make_uint4(x[0], x[1], x[2], x[3]);
            }
        }
    }
}

// ----------------------------------------------------------------------------------- plan
struct Bump {
    char* base = nullptr;                         // nullptr: only the size is wanted
    long long at = 0;
    void* take(long long bytes) {
        void* p = base ? base + at : nullptr;
        at += (bytes + 255) / 256 * 256;
        return p;
    }
};

struct Operand {
    Mat src, use;                                 // as given; as the products read it (fp32: the first part)
    long long plane = 0;                          // elements from one part to the next
    long long rows = 0, cols = 0;
    bool copied = false;
};

struct Block {
    const eg_feed_forward_args* q;
    long long P, n, d, f, fp;
    int dtype, parts;
    size_t size;
    Operand x, wg, wu, wd, dy;
    Mat ma, mb;                                   // act(G), U act'(G): dU and dG are dH times these
    Operand h, dg, du;
    int few = 0;                                  // 1: k_few_mma, 2: k_few_dot; 0: tiles
};

Mat mat(const eg_matrix& m) { return Mat{m.data, (long long)m.replica_stride, (long long)m.row_stride}; }

long long pitch_of(long long cols) { return (cols + 63) / 64 * 64; }

void place(Operand* o, const eg_matrix& m, const Block& b, long long rows, long long cols, Bump* w) {
    o->src = o->use = mat(m);
    o->rows = rows;
    o->cols = cols;
    if (b.dtype != EG_F32 && in_place(o->src, b.P, rows, b.size)) return;
    o->copied = true;
    const long long pitch = pitch_of(cols);
    o->plane = b.P * rows * pitch;
    o->use = Mat{w->take(o->plane * 2 * b.parts), rows * pitch, pitch};
}

bool valid(const eg_feed_forward_args* q, bool backward) {
    if (!q) return false;
    if (q->dtype != EG_F32 && q->dtype != EG_BF16 && q->dtype != EG_F16) return false;
    if (q->activation != EG_ACT_SILU && q->activation != EG_ACT_GELU && q->activation != EG_ACT_RELU) return false;
    if (q->P < 1 || q->P > 65535 || q->rows < 0 || q->rows > (1ll << 30) || q->d_model < 1 || q->d_model > (1ll << 24) ||
        q->d_ff < 1 || q->d_ff > (1ll << 24))
        return false;
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    struct { const eg_matrix* m; bool needed, written; long long rows, cols; } all[] = {
        {&q->x, true, false, q->rows, q->d_model},         {&q->w_gate, true, false, q->d_ff, q->d_model},
        {&q->w_up, true, false, q->d_ff, q->d_model},      {&q->w_down, true, false, q->d_model, q->d_ff},
        {&q->y, !backward, !backward, q->rows, q->d_model}, {&q->dy, backward, false, q->rows, q->d_model},
        {&q->dx, false, backward, q->rows, q->d_model},    {&q->d_gate, false, backward, q->d_ff, q->d_model},
        {&q->d_up, false, backward, q->d_ff, q->d_model},  {&q->d_down, false, backward, q->d_model, q->d_ff}};
    for (const auto& e : all) {
        if (!e.m->data) {
            if (e.needed && e.rows > 0) return false;
            continue;
        }
        if ((uintptr_t)e.m->data % size || e.m->row_stride < 0 || e.m->replica_stride < 0) return false;
        // neither the rows of a matrix nor the replicas' matrices overlap: the replicas' lie one after the other, or take
        // turns row by row
        if (e.rows > 1 && (e.m->row_stride < e.cols || e.m->row_stride >= (1ll << 36))) return false;
        if (q->P > 1) {
            const long long rep = e.m->replica_stride, row = e.m->row_stride;
            const bool apart = rep >= (e.rows - 1) * row + e.cols, in_turn = rep >= e.cols && row >= (q->P - 1) * rep + e.cols;
            if (rep >= (1ll << 36) || !(apart || in_turn)) return false;
        }
    }
    return true;
}

// Layout of `saved`: act(G), U act'(G), each [P][rows][fp] of the type, then H (fp32: its three parts).
long long saved_bytes(const eg_feed_forward_args* q) {
    return q->P * q->rows * pitch_of(q->d_ff) * (q->dtype == EG_F32 ? 2 * 4 + 2 * kParts : 3 * 2);
}

// Which kernels a forward call without `saved` takes.  Measured with 4 replicas, us:
//   bf16 1024 x 2816   k_few_mma 15 for 1 token, 17 for 8, 22 for 16, 40 for 32; tiles 26 from 17 to 64
//   fp32 1024 x 2816   k_few_dot 31 for 1 token, 91 for 8;           tiles 159
//   bf16 1001 x 2817   k_few_dot 49 for 1 token, 47 for 2, 90 for 4;             tiles 55
// and, with the tokens in groups (fp32: 8, 16-bit: 2), the tiles' time behind the stroke:
//   fp32 2 x 1024 x 2816   16 tokens 62 / 105, 24 98 / 105, 32 129 / 106;    3 x 401 x 896   16 28 / 39, 24 36 / 39, 32 48 / 39
//   fp32 8 x 128 x 280     16 tokens 17 / 26, 64 23 / 26;                    bf16 8 x 129 x 280   4 8 / 14, 8 14 / 16, 12 19 / 15
//   bf16 3 x 401 x 896     4 tokens 14 / 16, 6 18 / 16;                      bf16 2 x 1001 x 2817   4 43 / 33
int few_kind(const eg_feed_forward_args* q) {
    if (q->saved || q->P > 65535) return 0;
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    const bool rows16 = in_place(mat(q->x), q->P, q->rows, size) && in_place(mat(q->w_gate), q->P, q->d_ff, size) &&
                        in_place(mat(q->w_up), q->P, q->d_ff, size) && in_place(mat(q->w_down), q->P, q->d_model, size) &&
                        q->d_model * size % 16 == 0 && q->d_ff * size % 16 == 0;
    if (q->dtype != EG_F32 && rows16 && q->rows <= kFewMmaTokens) return 1;
    // k_few_dot reads the weights once for every group of tokens, the tiles copy them once and have longer launches
    // (the limits are fits to the figures above, no sizes of the chip: what the further groups read again, fp32 from the third on,
    // 16-bit from the second, is 12.9 and 6.5 MB where k_few_dot is last ahead and 25.9 and 8.7 MB where it first is behind; fp32 at
    // 8 x 128 x 280 is ahead at 20.6 MB too.  Weights above 134 and 67 MB were not measured and go to the tiles)
    const bool f32 = q->dtype == EG_F32;
    const int64_t each = f32 ? kFewDotTokens32 : kFewDotTokens16, groups = (q->rows + each - 1) / each;
    const double bytes = 3.0 * q->P * q->d_model * q->d_ff * size;
    if (groups <= 1) return 2;
    return q->rows <= 64 && bytes <= (f32 ? 134e6 : 67e6) && bytes * (groups - (f32 ? 2 : 1)) <= (f32 ? 14e6 : 6.6e6) ? 2 : 0;
}

void plan(Block* b, const eg_feed_forward_args* q, bool backward, Bump* w) {
    b->q = q;
    b->P = q->P; b->n = q->rows; b->d = q->d_model; b->f = q->d_ff;
    b->fp = pitch_of(b->f);
    b->dtype = (int)q->dtype;
    b->size = q->dtype == EG_F32 ? 4 : 2;
    b->parts = q->dtype == EG_F32 ? kParts : 1;
    if (!backward && (b->few = few_kind(q)) != 0) {
        b->h.use = Mat{w->take(b->P * b->n * b->fp * (long long)b->size), b->n * b->fp, b->fp};
        return;
    }
    place(&b->x, q->x, *b, b->n, b->d, w);
    place(&b->wg, q->w_gate, *b, b->f, b->d, w);
    place(&b->wu, q->w_up, *b, b->f, b->d, w);
    place(&b->wd, q->w_down, *b, b->d, b->f, w);
    const long long plane = b->P * b->n * b->fp;
    char* s = static_cast<char*>(q->saved);
    b->ma = Mat{s, b->n * b->fp, b->fp};
    b->mb = Mat{s ? s + plane * b->size : nullptr, b->n * b->fp, b->fp};
    auto hidden = [&](Operand* o, void* p) {
        o->use = Mat{p, b->n * b->fp, b->fp};
        o->plane = plane;
        o->rows = b->n;
        o->cols = b->f;
    };
    hidden(&b->h, s ? s + 2 * plane * b->size : nullptr);
    if (backward) {
        place(&b->dy, q->dy, *b, b->n, b->d, w);
        hidden(&b->dg, w->take(plane * 2 * b->parts));
        hidden(&b->du, w->take(plane * 2 * b->parts));
    } else if (!s) {
        hidden(&b->h, w->take(plane * 2 * b->parts));
    }
}

cudaError_t copy_in(const Block& b, std::initializer_list<const Operand*> operands, cudaStream_t stream) {
    CopyArgs a;
    a.count = 0;
    a.units = 0;
    for (const Operand* o : operands) {
        if (!o->copied) continue;
        auto& m = a.m[a.count++];
        m.src = o->src; m.dst = o->use; m.plane = o->plane; m.rows = o->rows; m.cols = (int)o->cols;
        m.chunks = (m.cols + kCopyCols - 1) / kCopyCols;
        m.begin = a.units;
        a.units += b.P * o->rows * m.chunks;
    }
    if (a.units == 0) return cudaSuccess;
    const long long blocks = (a.units + 7) / 8, most = (long long)sm_count() * 8;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    return b.dtype == EG_F32 ? launch_after(k_copy_in<float>, dim3(grid), dim3(256), 0, stream, a)
                             : launch_after(k_copy_in<uint16_t>, dim3(grid), dim3(256), 0, stream, a);
}

// ----------------------------------------------------------------------------------- products
struct Builder {
    GemmArgs a;
    int maps = 0;
    bool ok = true;
    const Block& b;
    int BN;

    Builder(const Block& blk, int bn, unsigned int* err) : b(blk), BN(bn) {
        a.problems = a.tiles = 0;
        a.idesc = (1u << 4) | (b.dtype != EG_F16 ? (1u << 7) | (1u << 10) : 0u);
        a.err = err;
        a.act = (int)b.q->activation;
        a.map_a = a.map_b = a.map_h = a.map_dg = a.map_du = -1;
    }
    int map(const Mat& m, int dtype, long long rows, long long cols, int box_cols, int box_rows) {
        if (maps >= kGemmMaxMaps) { ok = false; return 0; }
        ok = ok && encode(&a.maps[maps], dtype, m, b.P, rows, cols, box_cols, box_rows);
        return maps++;
    }
    // a matrix of the block's type, or its parts one after the other (16-bit), in small boxes
    int boxes(const Mat& m, int box_cols) { return map(m, b.dtype, b.n, b.f, box_cols, 32); }
    int boxes(const Operand& o, int box_cols) {
        const int first = maps;
        for (int k = 0; k < b.parts; ++k) map(part(o, k), operand_type(), o.rows, o.cols, box_cols, 32);
        return first;
    }
    int operand_type() const { return b.dtype == EG_F32 ? EG_BF16 : b.dtype; }
    Mat part(const Operand& o, int k) const {
        Mat m = o.use;
        m.p = static_cast<uint16_t*>(m.p) + k * o.plane;
        return m;
    }
    // operand of A (128 rows a CTA) or B (BN / 2): stored [mn][k] or, transposed, [k][mn]; the first of its maps
    int operand(const Operand& o, bool mn, bool is_a) {
        const int first = maps;
        for (int k = 0; k < b.parts; ++k) {
            if (mn) map(part(o, k), operand_type(), o.rows, o.cols, 64, 64);
            else map(part(o, k), operand_type(), o.rows, o.cols, kGemmK, is_a ? a_box(o.rows) : BN / 2);
        }
        return first;
    }
    static int a_box(long long M) { return M < 128 ? (int)(M + 7) / 8 * 8 : 128; }
    GemmProblem* problem(long long M, long long N, bool a_mn, bool b_mn, bool pair) {
        GemmProblem* g = &a.p[a.problems++];
        const int cols = pair ? BN / 2 : BN;
        g->mt = (int)((M + kGemmM - 1) / kGemmM);
        g->nt = (int)((N + cols - 1) / cols);
        const long long tiles = b.P * g->mt * g->nt;
        if (tiles + a.tiles > 0x7fffffffll) ok = false;
        g->tiles = (int)tiles;
        a.tiles += g->tiles;
        g->nseg = 0;
        g->a_box = a_box(M);
        g->a_mn = a_mn; g->b_mn = b_mn; g->b_pair = pair;
        g->M = (int)M; g->N = (int)N;
        g->out = -1;
        return g;
    }
    // sum of A B^T over K of one or two pairs
    struct Pair { int ma, mb0, mb1; };
    void product(GemmProblem* g, std::initializer_list<Pair> pairs, long long K) {
        for (const Pair& p : pairs) {
            if (g->nseg >= kGemmMaxSegs) { ok = false; return; }
            g->seg[g->nseg++] = GemmSeg{p.ma, p.mb0, p.mb1, (int)((K + kGemmK - 1) / kGemmK)};
        }
    }
    void store_to(GemmProblem* g, const Mat& m, long long rows, long long cols) {
        const int columns = BN / 2 < 32 ? BN / 2 : 32;
        g->ptr = m.p; g->rep = m.rep; g->row = m.row;
        g->out = in_place(m, b.P, rows, b.size) ? map(m, b.dtype, rows, cols, columns, 32) : -1;
    }
};

template <typename T, int EPI, int BN, int G> cudaError_t launch_kernel(const GemmArgs& a, cudaStream_t stream) {
    constexpr int smem = GemmShape<T, EPI, BN>::kSmem;
    static std::atomic<bool> raised[64];
    const cudaError_t e = raise_smem(k_gemm<T, EPI, BN, G>, smem, raised);
    if (e != cudaSuccess) return e;
    const int pairs = sm_count() / 2;
    if (pairs < 1) return cudaErrorInvalidDevice;
    return launch_after(k_gemm<T, EPI, BN, G>, dim3(2 * (a.tiles < pairs ? a.tiles : pairs)), dim3(kGemmThreads), smem, stream, a);
}

template <typename T, int EPI, int BN> cudaError_t launch_shape(const GemmArgs& args, cudaStream_t stream) {
    using Shape = GemmShape<T, EPI, BN>;
    static_assert(Shape::kRing / 1024 * 1024 / (128 * kGemmK * 2 + Shape::kBBytes) >= 4, "stages");
    GemmArgs a = args;
    a.a_pitch = 0;
    for (int k = 0; k < a.problems; ++k) {
        const int rows = !a.p[k].a_mn ? a.p[k].a_box : a.p[k].M > 64 ? 128 : 64;
        if (a.a_pitch < rows * 128) a.a_pitch = rows * 128;
    }
    a.heavy = a.extra = 0;
    if (a.problems > 1 && a.tiles > sm_count() / 2) {      // (pairs: as launch_kernel counts them)
        // a tile's time in stages: its epilogue, which runs under the next tile's products, takes some 8 (plain stores 16)
        auto stages_of = [](const GemmProblem& g) {
            int n = 0;
            for (int e = 0; e < g.nseg; ++e) n += g.seg[e].ksteps * (sizeof(T) == 4 ? 6 : 1);
            const int epilogue = g.out >= 0 ? 8 : 16;
            return n > epilogue ? n : epilogue;
        };
        const int pairs = sm_count() / 2, first = stages_of(a.p[0]), other = stages_of(a.p[1]), r = a.p[0].tiles % pairs;
        if (other > 0 && first > other && r > 0) {
            a.heavy = a.p[0].tiles;
            const int fit = (a.tiles - a.heavy) / (pairs - r);
            a.extra = first / other < fit ? first / other : fit;
        }
    }
    const int stages = Shape::stages(a.a_pitch);
    // (fp32 hands its accumulator over every few stages and counts them one by one)
    if constexpr (sizeof(T) == 2 && EPI != kEpiDact) {
        if (stages >= 16) {
            a.stages = stages / 4;
            return launch_kernel<T, EPI, BN, 4>(a, stream);
        }
        if (stages >= 8) {
            a.stages = stages / 2;
            return launch_kernel<T, EPI, BN, 2>(a, stream);
        }
    }
    a.stages = stages;
    return launch_kernel<T, EPI, BN, 1>(a, stream);
}

template <typename T, int EPI> cudaError_t launch_gemm(Builder& w, cudaStream_t stream) {
    if (!w.ok) return cudaErrorInvalidValue;
    w.a.n_maps = w.maps;
    if (w.a.tiles == 0) return cudaSuccess;
    if constexpr (sizeof(T) == 2) {
        if (w.BN == 256) return launch_shape<T, EPI, 256>(w.a, stream);
    }
    if (w.BN == 128) return launch_shape<T, EPI, 128>(w.a, stream);
    if constexpr (EPI == kEpiStore || (EPI == kEpiGateUp && sizeof(T) == 2)) {
        if (w.BN == 64) return launch_shape<T, EPI, 64>(w.a, stream);
    }
    if constexpr (EPI == kEpiStore) {
        if (w.BN == 32) return launch_shape<T, EPI, 32>(w.a, stream);
    }
    return cudaErrorInvalidValue;
}

// Tile width of a launch: the one whose last pair of multiprocessors should be done first.  A stage of 64 of K
// takes 2 cycles a column of the tile on the tensor cores, but no less than 300 for its copies and barriers (fp32: six
// products of three stages);
// filling and draining a tile's pipeline costs about 2500 and its epilogue 8 a column.  `cols`: columns of the
// result for a tile of 256.
int tile_width(const Block& b, long long M, long long N, long long K, int cols, int least) {
    const long long mt = (M + kGemmM - 1) / kGemmM, ksteps = (K + kGemmK - 1) / kGemmK;
    const long long pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
    int best = 0;
    long long best_time = 0;
    for (int bn = b.dtype == EG_F32 ? 128 : 256; bn >= least; bn /= 2) {       // fp32: a tile's sums in registers, 64 a thread
        const long long c = (long long)cols * bn / 256, tiles = b.P * mt * ((N + c - 1) / c), waves = (tiles + pairs - 1) / pairs;
        const int step = b.dtype == EG_F32 ? (12 * bn > 900 ? 12 * bn : 900) : 2 * bn > 300 ? 2 * bn : 300;
        const long long time = waves * (ksteps * step + 8 * bn) + 2500;
        if (!best || time < best_time) {
            best = bn;
            best_time = time;
        }
    }
    return best;
}

// Tile width of the gradients' launch: 128 where the pairs of multiprocessors would wait for a few long tiles.  Measured
// in bf16, us of a training step with 256 and 128: 300 tokens, 1024 x 4096 84 and 66; 49, 2512 x 8064 148 and 140; 3 x
// 4485, 88 x 200 64 and 57; 2 x 428, 1408 x 4800, which the rule leaves at 256, 140 and 156.
int gradient_width(const Block& b) {
    if (b.dtype == EG_F32) return 128;
    const long long pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
    long long best = 0;
    int width = 256;
    for (int bn = 256; bn >= 128; bn /= 2) {
        auto tiles = [&](long long M, long long N) { return b.P * ((M + kGemmM - 1) / kGemmM) * ((N + bn - 1) / bn); };
        const long long step = bn == 256 ? 512 : 400, epilogue = 16 * bn;      // cycles; narrow tiles copy more for each product
        const long long long_tile = b.q->dx.data ? 2 * ((b.f + kGemmK - 1) / kGemmK) * step : 0;
        const long long n = (b.n + kGemmK - 1) / kGemmK * step, tile = n > epilogue ? n : epilogue;
        const long long others = (b.q->d_down.data ? tiles(b.d, b.f) : 0) + ((b.q->d_gate.data ? 1 : 0) + (b.q->d_up.data ? 1 : 0)) * tiles(b.f, b.d);
        const long long all = (tiles(b.n, b.d) * long_tile + others * tile) / pairs;
        const long long longest = long_tile > tile ? long_tile : tile, time = all > longest ? all : longest;
        if (bn == 256 || time * 10 < best * 9) {
            best = time;
            width = bn;
        }
    }
    return width;
}

template <typename T> cudaError_t few_tokens(const Block& b, cudaStream_t stream) {
    const eg_feed_forward_args* q = b.q;
    FewArgs up{q->w_gate.data, q->w_up.data, q->w_gate.replica_stride, q->w_gate.row_stride, q->w_up.replica_stride,
               q->w_up.row_stride, q->x.data, q->x.replica_stride, q->x.row_stride, b.h.use.p, b.h.use.rep, b.h.use.row,
               (int)b.P, (int)b.n, (int)b.f, (int)b.d, (int)q->activation, 1};
    FewArgs down{q->w_down.data, nullptr, q->w_down.replica_stride, q->w_down.row_stride, 0, 0, b.h.use.p, b.h.use.rep,
                 b.h.use.row, q->y.data, q->y.replica_stride, q->y.row_stride, (int)b.P, (int)b.n, (int)b.d, (int)b.f, (int)q->activation, 1};
    cudaError_t e;
    if constexpr (sizeof(T) == 2) {
        if (b.few == 1) {
            e = launch_few_mma<T, true>(up, stream);
            return e != cudaSuccess ? e : launch_few_mma<T, false>(down, stream);
        }
    }
    const bool v = sizeof(T) == 4 && in_place(mat(q->x), b.P, b.n, 4) && in_place(mat(q->w_gate), b.P, b.f, 4) &&
                   in_place(mat(q->w_up), b.P, b.f, 4) && in_place(mat(q->w_down), b.P, b.d, 4) && b.d % 4 == 0 && b.f % 4 == 0;
    if constexpr (sizeof(T) == 4) {
        if (v) {
            e = launch_few_dot<T, 4, true>(up, (int)b.P, stream);
            return e != cudaSuccess ? e : launch_few_dot<T, 4, false>(down, (int)b.P, stream);
        }
    }
    e = launch_few_dot<T, 1, true>(up, (int)b.P, stream);
    return e != cudaSuccess ? e : launch_few_dot<T, 1, false>(down, (int)b.P, stream);
}

template <typename T> cudaError_t forward(const Block& b, unsigned int* err, cudaStream_t stream) {
    if (b.few) return few_tokens<T>(b, stream);
    cudaError_t e;
    if ((e = copy_in(b, {&b.x, &b.wg, &b.wu, &b.wd}, stream)) != cudaSuccess) return e;
    {
        Builder w(b, tile_width(b, b.n, b.f, b.d, 128, b.dtype == EG_F32 ? 128 : 64), err);
        GemmProblem* g = w.problem(b.n, b.f, false, false, true);
        const int mx = w.operand(b.x, false, true), mg = w.operand(b.wg, false, false), mu = w.operand(b.wu, false, false);
        w.product(g, {{mx, mg, mu}}, b.d);
        const int box = w.BN / 4 < 32 ? w.BN / 4 : 32;
        w.a.map_h = w.boxes(b.h, box);
        if (b.q->saved) {
            w.a.map_a = w.boxes(b.ma, box);
            w.a.map_b = w.boxes(b.mb, box);
        }
        if ((e = launch_gemm<T, kEpiGateUp>(w, stream)) != cudaSuccess) return e;
    }
    Builder w(b, tile_width(b, b.n, b.d, b.f, 256, 32), err);
    GemmProblem* g = w.problem(b.n, b.d, false, false, false);
    const int mb = w.operand(b.wd, false, false);
    w.product(g, {{w.operand(b.h, false, true), mb, mb}}, b.f);
    w.store_to(g, mat(b.q->y), b.n, b.d);
    return launch_gemm<T, kEpiStore>(w, stream);
}

template <typename T> cudaError_t backward(const Block& b, unsigned int* err, cudaStream_t stream) {
    cudaError_t e;
    const eg_feed_forward_args* q = b.q;
    if ((e = copy_in(b, {&b.x, &b.wg, &b.wu, &b.wd, &b.dy}, stream)) != cudaSuccess) return e;
    {
        Builder w(b, tile_width(b, b.n, b.f, b.d, 256, 128), err);
        GemmProblem* g = w.problem(b.n, b.f, false, true, false);
        const int mb = w.operand(b.wd, true, false);
        w.product(g, {{w.operand(b.dy, false, true), mb, mb}}, b.d);
        w.a.map_a = w.boxes(b.ma, 32);
        w.a.map_b = w.boxes(b.mb, 32);
        w.a.map_dg = w.boxes(b.dg, 32);
        w.a.map_du = w.boxes(b.du, 32);
        if ((e = launch_gemm<T, kEpiDact>(w, stream)) != cudaSuccess) return e;
    }
    Builder w(b, gradient_width(b), err);
    if (q->dx.data) {
        GemmProblem* g = w.problem(b.n, b.d, false, true, false);
        const int mg = w.operand(b.wg, true, false), mu = w.operand(b.wu, true, false);
        const int ag = w.operand(b.dg, false, true), au = w.operand(b.du, false, true);
        w.product(g, {{ag, mg, mg}, {au, mu, mu}}, b.f);
        w.store_to(g, mat(q->dx), b.n, b.d);
    }
    struct { const eg_matrix* out; const Operand *a, *bm; long long M, N; } grads[] = {
        {&q->d_down, &b.dy, &b.h, b.d, b.f}, {&q->d_gate, &b.dg, &b.x, b.f, b.d}, {&q->d_up, &b.du, &b.x, b.f, b.d}};
    for (const auto& t : grads) {
        if (!t.out->data) continue;
        GemmProblem* g = w.problem(t.M, t.N, true, true, false);
        const int mb = w.operand(*t.bm, true, false);
        w.product(g, {{w.operand(*t.a, true, true), mb, mb}}, b.n);
        w.store_to(g, mat(*t.out), t.M, t.N);
    }
    return launch_gemm<T, kEpiStore>(w, stream);
}

cudaError_t zero(const eg_matrix& m, long long P, long long rows, long long cols, size_t size, cudaStream_t stream) {
    for (long long i = 0; m.data && i < P; ++i) {
        const cudaError_t e = cudaMemset2DAsync(static_cast<char*>(m.data) + i * m.replica_stride * (long long)size,
                                                (rows > 1 ? m.row_stride : cols) * size, 0, cols * size, rows, stream);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// A wait on a barrier that nobody arrives on, with a limit of `cycles`.
__global__ void k_selftest_operator_wait(int which, long long cycles, unsigned int* err) {
    __shared__ __align__(8) uint64_t s_bar;
    __shared__ volatile int s_abort;
    if (threadIdx.x == 0) {
        s_abort = 0;
        op_mbar_init(&s_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (which == 0) (void)op_mbar_wait(&s_bar, 0, &s_abort, err, cycles);
    else if (which == 1) (void)op_mbar_wait_cluster(&s_bar, 0, &s_abort, err, cycles);
    else mbar_wait(&s_bar, 0, &s_abort, err, cycles);
}

}  // namespace
}  // namespace eg

using namespace eg;

extern "C" {

int64_t eg_feed_forward_saved_bytes(const eg_feed_forward_args* q) {
    if (!q || q->P < 1 || q->rows < 0 || q->d_ff < 1) return 0;
    return saved_bytes(q);
}

int64_t eg_feed_forward_workspace(const eg_feed_forward_args* q, int backward) {
    if (!valid(q, backward != 0)) return 0;
    Bump w;
    Block b;
    plan(&b, q, backward != 0, &w);
    return w.at;
}

eg_status eg_feed_forward(const eg_feed_forward_args* q, void* workspace, int64_t workspace_bytes, void* stream_v) {
    if (!valid(q, false)) return EG_ERR_INVALID;
    if (q->rows == 0) return EG_OK;
    if (q->saved && (!aligned16(q->saved) || q->saved_bytes < saved_bytes(q))) return EG_ERR_INVALID;
    Bump w;
    w.base = static_cast<char*>(workspace);
    Block b;
    plan(&b, q, false, &w);
    if (w.at > workspace_bytes || (w.at && (!workspace || !aligned16(workspace)))) return EG_ERR_INVALID;
    unsigned int* err = operator_error_word();
    if (!err) return EG_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    const cudaError_t e = q->dtype == EG_F32    ? forward<float>(b, err, stream)
                          : q->dtype == EG_BF16 ? forward<__nv_bfloat16>(b, err, stream)
                                                : forward<__half>(b, err, stream);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

eg_status eg_feed_forward_backward(const eg_feed_forward_args* q, void* workspace, int64_t workspace_bytes, void* stream_v) {
    if (!valid(q, true)) return EG_ERR_INVALID;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (q->rows == 0) {
        const size_t size = q->dtype == EG_F32 ? 4 : 2;
        const bool ok = zero(q->d_gate, q->P, q->d_ff, q->d_model, size, stream) == cudaSuccess &&
                        zero(q->d_up, q->P, q->d_ff, q->d_model, size, stream) == cudaSuccess &&
                        zero(q->d_down, q->P, q->d_model, q->d_ff, size, stream) == cudaSuccess;
        return ok ? EG_OK : EG_ERR_CUDA;
    }
    if (!q->saved || !aligned16(q->saved) || q->saved_bytes < saved_bytes(q)) return EG_ERR_INVALID;
    Bump w;
    w.base = static_cast<char*>(workspace);
    Block b;
    plan(&b, q, true, &w);
    if (w.at > workspace_bytes || (w.at && (!workspace || !aligned16(workspace)))) return EG_ERR_INVALID;
    unsigned int* err = operator_error_word();
    if (!err) return EG_ERR_CUDA;
    const cudaError_t e = q->dtype == EG_F32    ? backward<float>(b, err, stream)
                          : q->dtype == EG_BF16 ? backward<__nv_bfloat16>(b, err, stream)
                                                : backward<__half>(b, err, stream);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

eg_status eg_selftest_operator_wait(int which, void* stream_v) {
    if (which < 0 || which > 2) return EG_ERR_INVALID;
    unsigned int* err = operator_error_word();
    if (!err) return EG_ERR_CUDA;
    k_selftest_operator_wait<<<1, 64, 0, static_cast<cudaStream_t>(stream_v)>>>(which, 2000000ll /* about a millisecond */, err);
    return cudaGetLastError() == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

}  // extern "C"
