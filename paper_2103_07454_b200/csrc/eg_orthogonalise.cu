// Orthogonal updates (eg_orthogonalise): every matrix of every replica as its momentum's nearest orthogonal matrix, roughly.
//
//   v' = momentum * v + g,   u = v' or g + momentum * v'        (without a velocity u = g)
//   X = u / |u|,  transposed where it has more rows than columns (m x n, m <= n)
//   steps times   X <- a X + (b A + c A^2) X,   A = X X^T       (an odd polynomial of X's singular values, which pulls them to 1)
//   out = scale * X
//
// Launches: k_ortho_norm (velocity, sums of squares), k_ortho_in (X in the workspace's boxes), then the products (eg_orthogonal_gemm.cuh), each over all
// matrices of all replicas: a network's small matrices fill the machine together.
//
// Only a power of two of 1 / |u| goes into X at first, so that gradients of 16 bits enter the products without a rounding; the rest,
// between 1 and 2, is multiplied onto the first step's results in 32 bits.
#include <math.h>

#include "eg_orthogonal_gemm.cuh"
#include "eg_tensor_map.cuh"

namespace eg {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxItems = 128;                    // of an instance
constexpr long long kGroupBytes = 1ll << 30;      // workspace of one group of matrices that share their launches (one matrix may need more)

// Four neighbouring values of a row, as they lie in memory.
template <typename T> struct Quad {
    static constexpr int kWords = sizeof(T) == 4 ? 4 : 2;
    uint32_t w[kWords];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int q = 0; q < kWords; ++q) w[q] = 0;
    }
    // n of them are there; vec: on a boundary of four
    __device__ __forceinline__ void load(const T* p, int n, bool vec) {
        if (vec && n >= 4) {
            if constexpr (sizeof(T) == 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(p);
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            } else {
                const uint2 v = *reinterpret_cast<const uint2*>(p);
                w[0] = v.x; w[1] = v.y;
            }
            return;
        }
        clear();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e >= n) continue;
            if constexpr (sizeof(T) == 4) w[e] = *reinterpret_cast<const uint32_t*>(p + e);
            else w[e / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + e) << (16 * (e & 1));
        }
    }
    __device__ __forceinline__ void values(float (&v)[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) {
                v[e] = __uint_as_float(w[e]);
            } else {
                const float2 f = unpack2<T>(w[e / 2]);
                v[e] = e & 1 ? f.y : f.x;
            }
        }
    }
};

// Whether the rows of the gradient and the velocities begin on boundaries of four values.
__device__ __forceinline__ bool quads(const OrthoMat& m, size_t size) {
    auto fits = [](const Strided& s, size_t bytes) {
        return !s.p || (((uintptr_t)s.p | (uintptr_t)(s.rep * (long long)bytes) | (uintptr_t)(s.row * (long long)bytes)) & (4 * bytes - 1)) == 0;
    };
    return fits(m.grad, size) && fits(m.velocity, 4) && fits(m.velocity_out, 4);
}

// Walks over the boxes of an item, those of the gradient's rows of boxes one after another; a thread holds four quads of a box: rows
// 16 z + first, columns 4 * quad.  FORM: with the velocity before, otherwise with the one after the update.
// VEL: some matrices of the launch have a velocity.  Without, a thread's registers hold more boxes on their way: of 138 M 16-bit
// values the norm took 135 us with one box (16 KB a multiprocessor) ahead, 77 with four, the boxes 234 and 168.
template <typename T, bool FORM, bool VEL> struct Boxes {
    static constexpr int kSlots = VEL ? 2 : sizeof(T) == 2 ? 5 : 3;
    const OrthoArgs& a;
    const OrthoMat& m;
    int p, b, quad, first, rows, cols, wide, box0, box1;
    bool vec, need_g;
    Strided v;
    Quad<T> g[kSlots][4];
    Quad<float> w[VEL ? kSlots : 1][4];

    __device__ __forceinline__ Boxes(const OrthoArgs& args, int k, int item)
        : a(args), m(args.mat[k]), p((item - m.begin) / m.items), b(item - m.begin - p * m.items), quad(threadIdx.x & 15), first(threadIdx.x >> 4) {
        rows = m.flip ? m.n : m.m;
        cols = m.flip ? m.m : m.n;
        wide = m.flip ? m.rb : m.cb;
        const long long boxes = (long long)m.rb * m.cb;
        box0 = (int)(boxes * b / m.items);
        box1 = (int)(boxes * (b + 1) / m.items);
        vec = quads(m, sizeof(T));
        v = FORM ? m.velocity : m.velocity_out;
        need_g = !VEL || FORM || !v.p || a.nesterov;
    }
    __device__ __forceinline__ void fetch(int box, int slot) {
        const int grow = box / wide, c = (box - grow * wide) * kBox + quad * 4, n = cols - c;
        const long long r = grow * kBox + first;
        const T* from = static_cast<const T*>(m.grad.p) + p * m.grad.rep + r * m.grad.row + c;
        const float* speed = static_cast<const float*>(v.p) + p * v.rep + r * v.row + c;
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            const int have = r + z * 16 < rows ? n : 0;
            if (need_g) g[slot][z].load(from + z * 16 * m.grad.row, have, vec);
            if constexpr (VEL) {
                if (v.p) w[slot][z].load(speed + z * 16 * v.row, have, vec);
            }
        }
    }
    // work(box, slot) for each, with the next ones on their way
    __device__ __forceinline__ void start() {
#pragma unroll
        for (int q = 0; q < kSlots - 1; ++q)
            if (box0 + q < box1) fetch(box0 + q, q);
    }
    template <typename F> __device__ __forceinline__ void walk(F work) {
        for (int box = box0; box < box1; box += kSlots) {
#pragma unroll
            for (int q = 0; q < kSlots; ++q) {
                if (box + q >= box1) break;
                if (box + q + kSlots - 1 < box1) fetch(box + q + kSlots - 1, (q + kSlots - 1) % kSlots);
                work(box + q, q);
            }
        }
    }
    // u, four quads of it; FORM: stores the velocity.
    __device__ __forceinline__ void update(int box, int slot, float (&u)[4][4]) {
        const int grow = box / wide, c = (box - grow * wide) * kBox + quad * 4, n = cols - c;
        const long long r = grow * kBox + first;
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            if (need_g) g[slot][z].values(u[z]);
            if (!VEL || !v.p) continue;
            float s[4];
            w[VEL ? slot : 0][z].values(s);
            if (FORM) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = fmaf(a.momentum, s[e], u[z][e]);
                if (r + z * 16 < rows) {
                    float* to = static_cast<float*>(m.velocity_out.p) + p * m.velocity_out.rep + (r + z * 16) * m.velocity_out.row + c;
                    if (vec && n >= 4) {
                        store_vec<float, 4>(to, s);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < n) to[e] = s[e];
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) u[z][e] = a.nesterov ? fmaf(a.momentum, s[e], u[z][e]) : s[e];
        }
    }
};

__device__ __forceinline__ int matrix_of(const OrthoArgs& a, int item) {
    int k = 0;
    while (k + 1 < a.count && item >= a.mat[k + 1].begin) ++k;
    return k;
}

// The two kernels before the products read the same values; both are bound by memory, the next boxes on their way while one is worked on
// (4 x 2048 x 5504 three times, bf16 with a velocity: 235 and 272 us, 5.7 and 5.0 TB/s).
// Tried: both phases in one launch, the second a few hundred items behind the first so that it reads from the L2: 549 us against 502 for 8 x
// 2048 x 5504 with a velocity (an instance's 68 MB and what passes by do not stay there).
template <typename T, bool VEL> __global__ void __launch_bounds__(kThreads, 2) k_ortho_norm(const __grid_constant__ OrthoArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ double s_sum[kThreads / 32];
    Boxes<T, true, VEL> x(a, matrix_of(a, blockIdx.x), blockIdx.x);
    double sum = 0.0;
    x.start();
    x.walk([&](int box, int slot) {
        float u[4][4];
        x.update(box, slot, u);
#pragma unroll
        for (int z = 0; z < 4; ++z)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fma((double)u[z][e], (double)u[z][e], sum);
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) sum += s_sum[w];
        a.partial[(long long)(x.m.first + x.p) * kMaxItems + x.b] = sum;
    }
}

template <typename T, bool VEL> __global__ void __launch_bounds__(kThreads, 2) k_ortho_in(const __grid_constant__ OrthoArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ double s_sum[kThreads / 32];
    __shared__ float s_box[kBox][kBox + 1];
    Boxes<T, false, VEL> x(a, matrix_of(a, blockIdx.x), blockIdx.x);
    const OrthoMat& m = x.m;
    const int instance = m.first + x.p;
    x.start();
    static_assert(kMaxItems <= kThreads, "one partial sum a thread");
    double s = (int)threadIdx.x < m.items ? a.partial[(long long)instance * kMaxItems + threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = s;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) total += s_sum[w];
    const double norm = sqrt(total);
    int ex = 0;
    double fraction = 0.0;
    const bool finite = norm <= 1.7e308;                  // (false for NaN too)
    if (finite) fraction = frexp(norm, &ex);              // norm = fraction * 2^ex, 1/2 <= fraction < 1
    // sx / 2^ex as two factors, since it may pass the range of 32 bits
    const float by0 = (float)ldexp(1.0, -ex / 2), by1 = (float)ldexp((double)a.sx, -ex + ex / 2);
    if (x.b == 0 && threadIdx.x == 0)
        a.turn[instance] = !finite ? __int_as_float(0x7fffffff) : fraction > 0.0 ? (float)(1.0 / fraction) : 0.f;
    x.walk([&](int box, int slot) {
        float u[4][4];
        x.update(box, slot, u);
#pragma unroll
        for (int z = 0; z < 4; ++z)
#pragma unroll
            for (int e = 0; e < 4; ++e) u[z][e] = u[z][e] * by0 * by1;
        int rbox = box / x.wide, cbox = box - rbox * x.wide;
        if (m.flip) {
            const int r = rbox;
            rbox = cbox;
            cbox = r;
            __syncthreads();
#pragma unroll
            for (int z = 0; z < 4; ++z)
#pragma unroll
                for (int e = 0; e < 4; ++e) s_box[x.quad * 4 + e][z * 16 + x.first] = u[z][e];
            __syncthreads();
#pragma unroll
            for (int z = 0; z < 4; ++z)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[z][e] = s_box[z * 16 + x.first][x.quad * 4 + e];
        }
        unsigned char* hi = a.ws + (m.x[0] + x.p * m.x_rep + (long long)cbox * m.rb + rbox) * kBoxBytes;
        unsigned char* lo = a.ws + (m.lo[0] + x.p * m.x_rep + (long long)cbox * m.rb + rbox) * kBoxBytes;
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            uint32_t h0, h1, l0, l1;
            split_half2(u[z][0], u[z][1], h0, l0);
            split_half2(u[z][2], u[z][3], h1, l1);
            const uint32_t off = swz128((z * 16 + x.first) * 128 + x.quad * 8);
            *reinterpret_cast<uint2*>(hi + off) = make_uint2(h0, h1);
            // (a gradient of 8 bits has no lower part)
            if (VEL || sizeof(T) == 4 || a.parts == 2) *reinterpret_cast<uint2*>(lo + (a.parts == 1 ? lane_place(z * 16 + x.first, x.quad * 4) : off)) = make_uint2(l0, l1);
        }
    });
}

// ----------------------------------------------------------------------------------- host
constexpr int kMaxSteps = 64;
const double kDefault[3] = {3.4445, -4.7750, 2.0315};

struct Scales {
    float sx[kMaxSteps + 1];                              // powers of two before X: of every step, and of the result
    float sa[kMaxSteps], sb[kMaxSteps], sc[kMaxSteps];    // before A, B, C = A B
    double c[kMaxSteps][3], most[kMaxSteps];              // coefficients; bound of |B|
};

// The largest power of two with most * it <= 60000, but no more than takes `most` to 2^14 .. 2^15, nor than 2^114: values that a
// polynomial makes small keep their bits, down to a bound of 2^-100.
float power_below(double most) {
    most = fmax(most, 0x1p-100);
    int high = 0, low = 0;
    frexp(60000.0 / most, &high);
    frexp(most, &low);                                    // 2^(low - 1) <= most
    const int cap = low > 1 ? 14 : 15 - low;
    return (float)ldexp(1.0, high - 1 < cap ? high - 1 : cap);
}

// Bounds of the singular values, step by step, and the powers of two that they allow; false where the polynomials let them grow
// beyond 64.
bool scales(const eg_orthogonalise_args* q, Scales* s) {
    double bound = 1.0;
    for (int k = 0; k < q->steps; ++k) {
        for (int z = 0; z < 3; ++z) {
            s->c[k][z] = q->coefficients ? q->coefficients[3 * k + z] : kDefault[z];
            if (!(fabs(s->c[k][z]) <= 1e4)) return false;
        }
        const double a = s->c[k][0], b = s->c[k][1], c = s->c[k][2], top = bound * bound;
        // |B| in the spectral norm: b x + c x^2 on 0 .. bound^2
        double highest = fabs(b * top + c * top * top);
        if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < top) highest = fmax(highest, fabs(b * b / (4 * c)));
        s->most[k] = highest;
        s->sx[k] = power_below(bound * 1.02);
        s->sa[k] = power_below(top * 1.02);
        s->sb[k] = power_below(highest * 1.02);
        s->sc[k] = power_below(highest * top * 1.02);
        auto value = [&](double x) { return fabs(sqrt(x) * (a + x * (b + c * x))); };   // x: a square
        double next = value(top);
        // roots of a + 3 b x + 5 c x^2, each without a difference of like values (c may be next to nothing beside b)
        const double disc = 9 * b * b - 20 * a * c;
        if (disc >= 0.0) {
            const double far = -(3 * b + copysign(sqrt(disc), b)) / 2;
            for (double x : {c != 0.0 ? far / (5 * c) : -1.0, far != 0.0 ? a / far : -1.0})
                if (x > 0.0 && x < top) next = fmax(next, value(x));
        }
        bound = next * 1.01;
        if (bound > 64.0) return false;
    }
    s->sx[q->steps] = power_below(bound * 1.02);
    return true;
}

bool usable(const eg_matrix& m, int64_t P, int64_t rows, int64_t cols, size_t size, bool written) {
    if (!m.data || (uintptr_t)m.data % size || m.row_stride < 0 || m.replica_stride < 0 || m.row_stride >= (1ll << 36) ||
        m.replica_stride >= (1ll << 42))
        return false;
    if (!written) return true;
    if (rows > 1 && m.row_stride < cols) return false;
    if (P > 1) {
        const int64_t rep = m.replica_stride, row = rows > 1 ? m.row_stride : 0;
        if (!(rep >= (rows - 1) * row + cols || (rep >= cols && row >= (P - 1) * rep + cols))) return false;
    }
    return true;
}

size_t size_of(int64_t dtype) { return dtype == EG_F32 ? 4 : 2; }
bool known(int64_t dtype) { return dtype == EG_F32 || dtype == EG_BF16 || dtype == EG_F16; }

bool valid(const eg_orthogonalise_args* q, Scales* s) {
    if (!q || !known(q->dtype) || !known(q->out_dtype) || (q->out_dtype != q->dtype && q->out_dtype != EG_F32)) return false;
    if (q->P < 1 || q->P > 4096 || q->count < 0 || q->count > 65536 || (q->count > 0 && !q->matrices)) return false;
    if (q->steps < 1 || q->steps > kMaxSteps || !(fabs(q->momentum) <= 1e4) || !scales(q, s)) return false;
    for (int64_t i = 0; i < q->count; ++i) {
        const eg_orthogonal_matrix& m = q->matrices[i];
        if (m.rows < 1 || m.columns < 1 || m.rows > (1 << 20) || m.columns > (1 << 20) || !(fabs(m.scale) <= 3e38)) return false;
        const int64_t boxes = (m.rows + 63) / 64 * ((m.columns + 63) / 64);
        const int64_t side = ((m.rows < m.columns ? m.rows : m.columns) + 63) / 64;
        if (q->P * (4 * boxes + 6 * side * side) > (1ll << 24)) return false;              // 128 GB of workspace
        if (!usable(m.grad, q->P, m.rows, m.columns, size_of(q->dtype), false)) return false;
        if (!usable(m.out, q->P, m.rows, m.columns, size_of(q->out_dtype), true)) return false;
        if (m.velocity.data && !usable(m.velocity, q->P, m.rows, m.columns, 4, !m.velocity_out.data)) return false;
        if (m.velocity_out.data && (!m.velocity.data || !usable(m.velocity_out, q->P, m.rows, m.columns, 4, true))) return false;
    }
    return true;
}

// Parts of an operand.  Results of 8 bits take two where a matrix is longer than 2^18: with one, a product's sum stays in the accumulator, which
// truncates (64 x 2^18: error 2.1e-3 with one; 64 x 2^20: 5.7e-3, 1.7e-3 with two; 24 and 26 ms).
int parts_of(const eg_orthogonalise_args* q) {
    if (q->out_dtype != EG_BF16) return 2;
    for (int64_t i = 0; i < q->count; ++i)
        if (q->matrices[i].rows > (1 << 18) || q->matrices[i].columns > (1 << 18)) return 2;
    return 1;
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
struct Sides {
    int64_t rb, cb, boxes;                                // boxes: of one replica
};
Sides sides(int parts, const eg_orthogonal_matrix& m) {
    const int64_t r = m.rows <= m.columns ? m.rows : m.columns, c = m.rows <= m.columns ? m.columns : m.rows;
    Sides s{up(r, kBox) / kBox, up(c, kBox) / kBox, 0};
    s.boxes = parts == 2 ? 4 * s.rb * s.cb + 6 * s.rb * s.rb : 3 * s.rb * s.cb + 2 * s.rb * s.rb + (s.rb + 15) / 16;
    return s;
}
// Matrices [first, *end) share their launches.  Returns their boxes.
int64_t group(const eg_orthogonalise_args* q, int parts, int64_t first, int64_t* end) {
    int64_t boxes = 0, i = first;
    for (; i < q->count && i - first < kOrthoMats; ++i) {
        const int64_t more = q->P * sides(parts, q->matrices[i]).boxes;
        if (i > first && (boxes + more) * kBoxBytes > kGroupBytes) break;
        boxes += more;
    }
    *end = i;
    return boxes;
}
// Behind a group's boxes: partial sums, what is left of 1 / |u|.
struct Tail {
    int64_t partial, turn, bytes;
};
Tail tail(const eg_orthogonalise_args* q) {
    const int64_t instances = q->P * (q->count < kOrthoMats ? q->count : kOrthoMats);
    Tail t;
    t.partial = 0;
    t.turn = up(instances * kMaxItems * 8, 256);
    t.bytes = t.turn + up(instances * 4, 256);
    return t;
}
int64_t workspace_of(const eg_orthogonalise_args* q) {
    const int parts = parts_of(q);
    int64_t most = 0, end = 0;
    for (int64_t i = 0; i < q->count; i = end) {
        const int64_t boxes = group(q, parts, i, &end);
        most = boxes > most ? boxes : most;
    }
    return most * kBoxBytes + tail(q).bytes;
}

Strided strided(const eg_matrix& m) { return Strided{m.data, (long long)m.replica_stride, (long long)m.row_stride}; }

bool fill(OrthoArgs* a, const eg_orthogonalise_args* q, int parts, int64_t first, int64_t end, unsigned char* ws, int64_t boxes) {
    const Tail z = tail(q);
    unsigned char* behind = ws + boxes * kBoxBytes;
    a->ws = ws;
    a->partial = reinterpret_cast<double*>(behind + z.partial);
    a->turn = reinterpret_cast<float*>(behind + z.turn);
    a->P = (int)q->P;
    a->parts = parts;
    a->count = (int)(end - first);
    a->momentum = (float)q->momentum;
    a->nesterov = q->nesterov != 0;
    // longest products first: pairs of CTAs take the tiles in turn
    int64_t order[kOrthoMats];
    for (int64_t i = first; i < end; ++i) {
        int64_t j = i - first;
        auto longer = [&](int64_t x, int64_t y) {
            const Sides s = sides(parts, q->matrices[x]), t = sides(parts, q->matrices[y]);
            return s.cb != t.cb ? s.cb > t.cb : s.rb > t.rb;
        };
        for (; j > 0 && longer(i, order[j - 1]); --j) order[j] = order[j - 1];
        order[j] = i;
    }
    int64_t at = 0, begin = 0, tiles[2] = {0, 0};
    for (int i = 0; i < a->count; ++i) {
        const eg_orthogonal_matrix& s = q->matrices[order[i]];
        OrthoMat* m = &a->mat[i];
        const Sides z = sides(parts, s);
        m->flip = s.rows > s.columns;
        m->m = (int)(m->flip ? s.columns : s.rows);
        m->n = (int)(m->flip ? s.rows : s.columns);
        m->rb = (int)z.rb; m->cb = (int)z.cb;
        m->first = (int)(i * q->P);
        m->scale = (float)s.scale;
        const int64_t plane = z.rb * z.cb, square = z.rb * z.rb;
        // hi and lo of X twice and of three symmetric matrices; or hi of X twice, lo of X, hi of two and their diagonals (rounding, values)
        m->x_rep = parts * plane; m->s_rep = parts * square;
        m->x[0] = at;
        m->x[1] = at + q->P * parts * plane;
        m->lo[0] = parts == 2 ? m->x[0] + plane : at + q->P * 2 * plane;
        m->lo[1] = parts == 2 ? m->x[1] + plane : m->lo[0];
        for (int k = 0; k < 3; ++k) m->s[k] = at + q->P * (parts == 2 ? 4 * plane + 2 * square * k : 3 * plane + square * (k & 1));
        m->rest = at + q->P * (3 * plane + 2 * square);
        m->rest_rep = (z.rb + 15) / 16;
        at += q->P * z.boxes;
        m->grad = strided(s.grad); m->out = strided(s.out); m->velocity = strided(s.velocity);
        m->velocity_out = s.velocity_out.data ? strided(s.velocity_out) : m->velocity;
        const int wide = parts == 2 ? 2 : 4;              // boxes of a tile's columns
        const int64_t rt = (z.rb + 3) / 4, ct = (z.rb + wide - 1) / wide;
        int64_t low = 0;
        for (int64_t r = 0; r < rt; ++r) low += ct < (r + 1) * (4 / wide) ? ct : (r + 1) * (4 / wide);
        m->tiles[0] = (int)low;
        m->tiles[1] = (int)(rt * ((z.cb + wide - 1) / wide));
        tiles[0] += q->P * low;
        tiles[1] += q->P * (int64_t)m->tiles[1];
        const int64_t items = (plane + 3) / 4;            // four boxes or more each
        m->items = (int)(items < kMaxItems ? items : kMaxItems);
        m->begin = (int)begin;
        begin += q->P * m->items;
    }
    if (tiles[0] > 0x3fffffff || tiles[1] > 0x3fffffff || begin > 0x3fffffff) return false;
    a->tiles[0] = (int)tiles[0];
    a->tiles[1] = (int)tiles[1];
    a->items = (int)begin;
    EncodeFn fn = encoder();
    if (!fn) return false;
    const cuuint64_t dims[3] = {64, (cuuint64_t)(boxes * kBox), 1}, strides[2] = {128, (cuuint64_t)(boxes * kBoxBytes)};
    const cuuint32_t box[3] = {64, 64, 1}, one[3] = {1, 1, 1};
    return fn(&a->map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, ws, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int PARTS, int PASS> cudaError_t product(const OrthoArgs& a, const OrthoPass& pass, cudaStream_t stream) {
    constexpr int smem = OrthoShape<PARTS>::kSmem;
    static std::atomic<bool> raised[64];
    const cudaError_t e = raise_smem(k_ortho<T, PARTS, PASS>, smem, raised);
    if (e != cudaSuccess) return e;
    const int pairs = sm_count() / 2, tiles = a.tiles[PASS >= kApply ? 1 : 0];
    if (pairs < 1) return cudaErrorInvalidDevice;
    return launch_after(k_ortho<T, PARTS, PASS>, dim3(2 * (tiles < pairs ? tiles : pairs)), dim3(kOrthoThreads), smem, stream, a, pass);
}

template <typename T, int PARTS> cudaError_t run(OrthoArgs& a, const Scales& s, const eg_orthogonalise_args* q, cudaStream_t stream) {
    a.sx = s.sx[0];
    a.out = 1.f / s.sx[q->steps];
    bool any_velocity = false;
    double saved = 0;
    for (int i = 0; i < a.count; ++i) {
        any_velocity = any_velocity || a.mat[i].velocity.p;
        saved += (double)q->P * a.mat[i].m * a.mat[i].m * (a.mat[i].n - 2.0 * a.mat[i].m);
    }
    [[maybe_unused]] const bool pairs = saved >= 0x1p31;
    auto given = [&](auto value, auto vel) {
        using G = decltype(value);
        constexpr bool VEL = decltype(vel)::value;
        const cudaError_t e = launch_after(k_ortho_norm<G, VEL>, dim3(a.items), dim3(kThreads), 0, stream, a);
        return e != cudaSuccess ? e : launch_after(k_ortho_in<G, VEL>, dim3(a.items), dim3(kThreads), 0, stream, a);
    };
    auto of_type = [&](auto vel) { return q->dtype == EG_F32 ? given(0.f, vel) : q->dtype == EG_BF16 ? given(__nv_bfloat16{}, vel) : given(__half{}, vel); };
    cudaError_t e = any_velocity ? of_type(std::true_type{}) : of_type(std::false_type{});
    int from = 0;
    for (int k = 0; k < q->steps && e == cudaSuccess; from ^= 1) {
        const double *c0 = s.c[k], sx = s.sx[k], sa = s.sa[k], sb0 = s.sb[k];
        OrthoPass p{};
        p.from = from;
        p.first = k == 0;
        p.to = 0;
        p.fd = (float)(sa / (sx * sx));
        // (what only the last launch depends on is the caller's type: the others are shared)
        e = product<float, PARTS, kGram>(a, p, stream);
        auto sym = [&](int l, int r, int e0, int e1, int to, double f0, double f1, double fd) {
            p.l = l; p.r = r; p.e0 = e0; p.e1 = e1; p.to = to;
            p.f0 = (float)f0; p.f1 = (float)f1; p.fd = (float)fd;
        };
        // B0 = b A + c A^2
        sym(0, 0, 0, 0, 1, c0[1] * sb0 / sa, 0, c0[2] * sb0 / (sa * sa));
        if (e == cudaSuccess) e = product<float, PARTS, kSym1>(a, p, stream);
        double outer = c0[0], scale = sb0;
        p.l = 1;
        ++k;
        if constexpr (PARTS == 2) {
            // Two steps in one take m^2 (n - 2 m) fewer multiplications at about 6e13 a second (a square matrix would take 20 % longer), and double the
            // error. From 2^31 on, 35 us, the time counts: below, launches do (8 x 512 x 4608 638 -> 504 us, error 2.4e-6 -> 2.8e-6;
            // 8 x 128 x 1152 163 -> 166 us, 1.9e-6 -> 2.3e-6).
            // (polynomials that make small values smaller: their products of two steps would sink below the boxes' last bit, 2^-39)
            if (pairs && k < q->steps && fabs(c0[0]) >= 1.0 && fabs(s.c[k][0]) >= 1.0) {
                const double *c1 = s.c[k], sa1 = s.sa[k], sb1 = s.sb[k], sc = s.sc[k - 1];
                const double bound = fabs(c1[0]) * s.most[k - 1] + fabs(c0[0]) * s.most[k] + s.most[k - 1] * s.most[k], sr = power_below(bound * 1.02);
                // C = A B0
                sym(0, 1, 0, 0, 2, 0, 0, sc / (sa * sb0));
                if (e == cudaSuccess) e = product<float, PARTS, kSym0>(a, p, stream);
                // A1 = a0^2 A + 2 a0 C + C B0, in A's place
                sym(2, 1, 0, 2, 0, c0[0] * c0[0] * sa1 / sa, 2 * c0[0] * sa1 / sc, sa1 / (sc * sb0));
                if (e == cudaSuccess) e = product<float, PARTS, kSym2>(a, p, stream);
                // B1 = b A1 + c A1^2, in C's place
                sym(0, 0, 0, 0, 2, c1[1] * sb1 / sa1, 0, c1[2] * sb1 / (sa1 * sa1));
                if (e == cudaSuccess) e = product<float, PARTS, kSym1>(a, p, stream);
                // a1 B0 + a0 B1 + B1 B0, in A1's place
                sym(2, 1, 1, 2, 0, c1[0] * sr / sb0, c0[0] * sr / sb1, sr / (sb1 * sb0));
                if (e == cudaSuccess) e = product<float, PARTS, kSym2>(a, p, stream);
                outer = c0[0] * c1[0];
                scale = sr;
                p.l = 0;
                ++k;
            }
        }
        p.f0 = (float)(outer * s.sx[k] / sx);
        p.fd = (float)(s.sx[k] / (sx * scale));
        // The lower parts of X: there are none at first where u is the gradient of 8 bits.  Afterwards X, which the steps carry on, keeps them to
        // the end (without them in the last step two blocks of 1024 x 2816 on 8 replicas took 3.04 ms instead of 3.09, 2048 x 5504 on 4 replicas 5.05
        // instead of 5.10).
        p.read_lower = k > 1 || any_velocity;
        if (e != cudaSuccess) break;
        e = k < q->steps ? product<float, PARTS, kApply>(a, p, stream) : product<T, PARTS, kLast>(a, p, stream);
    }
    return e;
}

}  // namespace
}  // namespace eg

using namespace eg;

extern "C" {

int64_t eg_orthogonalise_workspace(const eg_orthogonalise_args* q) {
    Scales s;
    if (!valid(q, &s)) return 0;
    return workspace_of(q);
}

eg_status eg_orthogonalise(const eg_orthogonalise_args* q, void* workspace, int64_t workspace_bytes, void* stream_v) {
    Scales s;
    if (!valid(q, &s)) return EG_ERR_INVALID;
    if (q->count == 0) return EG_OK;
    if (!workspace || (uintptr_t)workspace % 128 || workspace_bytes < workspace_of(q)) return EG_ERR_INVALID;
    unsigned int* err = operator_error_word();
    if (!err) return EG_ERR_CUDA;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    const int parts = parts_of(q);
    int64_t end = 0;
    for (int64_t i = 0; i < q->count; i = end) {
        const int64_t boxes = group(q, parts, i, &end);
        OrthoArgs a;
        a.err = err;
        if (!fill(&a, q, parts, i, end, static_cast<unsigned char*>(workspace), boxes)) return EG_ERR_CUDA;
        const cudaError_t e = q->out_dtype == EG_F32   ? run<float, 2>(a, s, q, stream)
                              : q->out_dtype == EG_F16 ? run<__half, 2>(a, s, q, stream)
                              : parts == 2             ? run<__nv_bfloat16, 2>(a, s, q, stream)
                                                       : run<__nv_bfloat16, 1>(a, s, q, stream);
        if (e != cudaSuccess) return EG_ERR_CUDA;
    }
    return EG_OK;
}

}  // extern "C"
