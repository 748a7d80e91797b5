// Embedding of tokens (eg_embedding) and its gradient (eg_embedding_backward).
//
//   forward   y[t] = scale * W[token t]                      (a token outside of the table: zeros)
//   backward  dW[v] = scale * sum of dy over the places t of token v   (+ what dW holds, where it is to be added to)
//
// Bound by memory: the forward call moves a row in and a row out for every place; the gradient reads every row of dy
// once and writes the whole table, most of whose rows are zero (32000 rows and 1024 places on each of 8 replicas: 525 of
// 542 MB).
//
// The gradient sorts the places by token, so that every row of dW is one run of places, summed in the order of the places:
// no atomics on values, the same bits every time.
//   1. k_embed_sort: one CTA per range of the table's rows reads all tokens of its replica twice.  It counts the tokens
//      below its range (which is where its part of the sorted list begins) and each of its own, then puts the places into
//      the list.  The tokens come out of the L2 and nobody waits for another CTA; a sort in several passes would launch five kernels.
//      The reads are n V / 256 tokens: right for tables of some 10^4 rows; above 2 * 10^5 rows with 10^5 places they pass what is read of dy.
//      It notes which rows have a place.
//   2. k_embed_sum: a warp adds up one chunk of the list over some columns.  Chunks have equal length, however often a token
//      comes; a run that crosses chunks leaves a partial sum in each.
// The table's zeros are written by further blocks of these launches, the same number of rows each: beside the sort, for all rows, where
// there are fewer places than rows (the sort, 10 to 30 us of latencies, is then for nothing), beside the sums, for the rows
// without a place, where there are more.
//   3. k_embed_join: adds the partial sums of such runs, in order.
// Measured, bf16: 8 x 1024 places of 32000 x 1024: forward 11 us (launch and latency), sort and zeros 75 us (524 MB, 7 TB/s), sums 17, joins 7;
// 4 x 16384 places of 32000 x 2048: forward 63 us, sort and zeros 101, sums 91, joins 23.
#include "eg_ops.cuh"

namespace eg {
namespace {

constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kRangeMax = 512;             // rows of the table that a sorting CTA owns, at most
constexpr int kMaxVectors = 4;             // 16-byte vectors of a row that a warp's lane holds (forward)

struct Rows {
    void* p;
    long long rep, row;                    // strides in elements
};

struct EmbedArgs {
    int P;
    long long n, V;
    int d;
    float scale;
    const void* tokens;
    long long token_rep, token_step;
    int wide;                              // tokens of 64 bits
    Rows weight, out;                      // forward: table and y; backward: dy and the table's gradient
    int accumulate;
    // backward
    int range;                             // rows of the table per sorting CTA
    int chunk, chunks;                     // places of a chunk; chunks of a replica
    int pitch;                             // columns of a partial sum, up to whole vectors
    int sum_blocks;                        // of k_embed_sum, per replica; the rest write zeros
    int sort_blocks;                       // of k_embed_sort
    int *order, *key, *count;              // [P][n] places and tokens of the sorted list, [P] its length
    unsigned int* named;                   // [P][words] one bit for every row of the table that has a place
    int words;
    float* partial;                        // [P][chunks][2][pitch]: of a run from the chunk before, of one into the next
};

// The token at place t of replica i, -1 where it is none of the table's.
struct Tokens {
    const char* p;
    long long step;                        // bytes
    int wide;
    unsigned V;
    __device__ __forceinline__ Tokens(const EmbedArgs& a, int i)
        : p(static_cast<const char*>(a.tokens) + i * a.token_rep * (a.wide ? 8 : 4)), step(a.token_step * (a.wide ? 8 : 4)), wide(a.wide), V((unsigned)a.V) {}
    __device__ __forceinline__ int at(long long t) const {
        if (wide) {
            const unsigned long long v = __ldg(reinterpret_cast<const unsigned long long*>(p + t * step));
            return v < V ? (int)v : -1;
        }
        const unsigned v = __ldg(reinterpret_cast<const unsigned*>(p + t * step));
        return v < V ? (int)v : -1;
    }
};
template <typename T> __device__ __forceinline__ T* row_of(const Rows& m, int i, long long t) {
    return static_cast<T*>(m.p) + (long long)i * m.rep + t * m.row;
}

// ----------------------------------------------------------------------------------- forward
// A warp takes 32 * U vectors of one row, all its loads ahead of its stores.
template <typename T, int VEC, int U>
__global__ void __launch_bounds__(256) k_embed(const __grid_constant__ EmbedArgs a, int slices) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), rows = a.P * a.n;
    if (unit >= rows * slices) return;
    const long long line = unit / slices;
    const int i = (int)(line / a.n);
    const long long t = line - i * a.n;
    const int c0 = (int)(unit - line * slices) * 32 * U * VEC, token = Tokens(a, i).at(t);
    float v[U][VEC];
    const T* from = row_of<T>(a.weight, i, token < 0 ? 0 : token);
    T* to = row_of<T>(a.out, i, t);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + (u * 32 + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[u][e] = 0.f;
        if (c < a.d && token >= 0) load_vec<T, VEC>(from + c, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + (u * 32 + lane) * VEC;
        if (c >= a.d) continue;
        if (token >= 0) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[u][e] *= a.scale;
        }
        store_vec<T, VEC>(to + c, v[u]);
    }
}

// ----------------------------------------------------------------------------------- backward
// Zeros for block b's share of a replica's rows; `some`: only for rows without a place.
template <typename T, int VEC> __device__ __forceinline__ void write_zeros(const EmbedArgs& a, int i, int b, int blocks, bool some) {
    const float zero[VEC] = {};
    const long long v0 = a.V * b / blocks, v1 = a.V * (b + 1) / blocks;
    for (long long v = v0 + (threadIdx.x >> 5); v < v1; v += blockDim.x >> 5) {
        if (some && (a.named[(long long)i * a.words + v / 32] >> (v & 31) & 1)) continue;
        T* to = row_of<T>(a.out, i, v);
        for (int c = (int)(threadIdx.x & 31) * VEC; c < a.d; c += 32 * VEC) store_vec<T, VEC>(to + c, zero);
    }
}

// Sum over the CTA, valid in all threads; `red` holds kSortWarps values.
__device__ __forceinline__ int block_total(int v, int* red) {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    int s = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) s += red[w];
    return s;
}

template <typename T, int VEC> __global__ void __launch_bounds__(kSortThreads) k_embed_sort(const __grid_constant__ EmbedArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ int s_at[kSortWarps][kRangeMax];          // first how often, then where to
    __shared__ int s_red[kSortWarps];
    const int i = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x >= a.sort_blocks) {
        write_zeros<T, VEC>(a, i, blockIdx.x - a.sort_blocks, gridDim.x - a.sort_blocks, false);
        return;
    }
    const long long first = (long long)blockIdx.x * a.range;
    const int mine = (int)(a.V - first < a.range ? a.V - first : a.range);
    for (int q = threadIdx.x; q < kSortWarps * kRangeMax; q += kSortThreads) (&s_at[0][0])[q] = 0;
    __syncthreads();
    // every warp takes its own stretch of the places, 32 at a time, SCAN of them on their way at once
    constexpr int SCAN = 8;
    const long long each = ((a.n + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
    const long long t0 = warp * each, t1 = t0 + each < a.n ? t0 + each : a.n;
    const Tokens tokens(a, i);
    const int first_row = (int)first;
    int below = 0;
    for (long long t = t0; t < t1; t += 32 * SCAN) {
        int v[SCAN];
#pragma unroll
        for (int u = 0; u < SCAN; ++u) v[u] = t + u * 32 + lane < t1 ? tokens.at(t + u * 32 + lane) : -1;
#pragma unroll
        for (int u = 0; u < SCAN; ++u) {
            const unsigned at = (unsigned)(v[u] - first_row);
            below += v[u] >= 0 && v[u] < first_row;
            if (v[u] >= 0 && at < (unsigned)mine) atomicAdd(&s_at[warp][at], 1);
        }
    }
    const int base = block_total(below, s_red);          // (its barriers also end the counting)
    // where the places of row r go that warp w finds: behind those of the rows before and of the warps before
    const int r = threadIdx.x;
    int total = 0;
    if (r < mine) {
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) total += s_at[w][r];
    }
    int upto = total;                                    // sum over the rows up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    __syncthreads();
    if (lane == 31) s_red[warp] = upto;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
        before += w < warp ? s_red[w] : 0;
        all += s_red[w];
    }
    const unsigned some = __ballot_sync(0xffffffffu, total > 0);
    if (lane == 0 && r < mine) a.named[(long long)i * a.words + (first + r) / 32] = some;     // (ranges are whole words)
    if (r < mine) {
        int at = base + before + upto - total;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            const int x = s_at[w][r];
            s_at[w][r] = at;
            at += x;
        }
    }
    if (threadIdx.x == 0 && first + mine == a.V) a.count[i] = base + all;
    __syncthreads();
    if (all > 0) {
        int *order = a.order + i * a.n, *key = a.key + i * a.n;
        for (long long t = t0; t < t1; t += 32 * SCAN) {
            int v[SCAN];
#pragma unroll
            for (int u = 0; u < SCAN; ++u) v[u] = t + u * 32 + lane < t1 ? tokens.at(t + u * 32 + lane) : -1;
#pragma unroll
            for (int u = 0; u < SCAN; ++u) {
                const unsigned rel = (unsigned)(v[u] - first_row);
                const bool in = v[u] >= 0 && rel < (unsigned)mine;
                if (!__any_sync(0xffffffffu, in)) continue;
                const unsigned same = __match_any_sync(0xffffffffu, in ? v[u] : -1);
                const int rank = __popc(same & ((1u << lane) - 1));
                int at = 0;
                if (in) at = s_at[warp][rel];
                __syncwarp();
                if (in) {
                    order[at + rank] = (int)(t + u * 32 + lane);
                    key[at + rank] = v[u];
                    if (rank == 0) s_at[warp][rel] = at + __popc(same);
                }
                __syncwarp();
            }
        }
    }
}

// Adds to or writes a row's columns.
template <typename T, int VEC> __device__ __forceinline__ void finish(const EmbedArgs& a, int i, int token, int c, const float* sum) {
    T* to = row_of<T>(a.out, i, token) + c;
    float v[VEC];
    if (a.accumulate) load_vec<T, VEC>(to, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = a.accumulate ? fmaf(a.scale, sum[e], v[e]) : a.scale * sum[e];
    store_vec<T, VEC>(to, v);
}

// Values as they lie in memory.
template <typename T, int VEC> struct Raw {
    uint4 v;
    __device__ __forceinline__ void load(const T* p) { v = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void add_to(float* sum) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (sizeof(T) == 4) {
                sum[q] += __uint_as_float(w[q]);
            } else {
                const float2 f = unpack2<T>(w[q]);
                sum[2 * q] += f.x;
                sum[2 * q + 1] += f.y;
            }
        }
    }
};
template <typename T> struct Raw<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = *p; }
    __device__ __forceinline__ void add_to(float* sum) const { sum[0] += to_f32(v); }
};

// A warp: one chunk of the sorted list, 32 * U vectors of columns; or zeros for rows without a place.
template <typename T, int VEC, int U> __global__ void __launch_bounds__(256, 4) k_embed_sum(const __grid_constant__ EmbedArgs a, int slices) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int AHEAD = 4;                             // rows on their way at once
    const int lane = threadIdx.x & 31, i = blockIdx.y;
    if ((int)blockIdx.x >= a.sum_blocks) {
        write_zeros<T, VEC>(a, i, blockIdx.x - a.sum_blocks, gridDim.x - a.sum_blocks, true);
        return;
    }
    const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const long long chunk = unit / slices;
    if (chunk >= a.chunks) return;
    const int c0 = (int)(unit - chunk * slices) * 32 * U * VEC + lane * VEC, count = a.count[i];
    const long long first = chunk * a.chunk;
    if (first >= count) return;
    const int n = count - first < a.chunk ? (int)(count - first) : a.chunk;
    const int *order = a.order + i * a.n + first, *key = a.key + i * a.n + first;
    const bool from_before = first > 0 && key[-1] == key[0], into_next = first + n < count && key[n] == key[n - 1];
    float* partial = a.partial + ((long long)i * a.chunks + chunk) * 2 * a.pitch;
    float sum[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[u][e] = 0.f;
    bool at_first = true;                                // in the chunk's first run
    for (int j0 = 0; j0 < n; j0 += 32) {
        const int m = n - j0 < 32 ? n - j0 : 32;
        const int place = lane < m ? order[j0 + lane] : 0, token = lane < m ? key[j0 + lane] : -1;
        const int after = j0 + lane + 1 < n && lane < m ? key[j0 + lane + 1] : -1;
        for (int j = 0; j < m; j += AHEAD) {
            Raw<T, VEC> v[AHEAD][U];
#pragma unroll
            for (int h = 0; h < AHEAD; ++h) {
                const T* from = row_of<T>(a.weight, i, __shfl_sync(0xffffffffu, place, (j + h) & 31)) + c0;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (j + h < m && c0 + u * 32 * VEC < a.d) v[h][u].load(from + u * 32 * VEC);
            }
#pragma unroll
            for (int h = 0; h < AHEAD; ++h) {
                if (j + h >= m) break;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c0 + u * 32 * VEC < a.d) v[h][u].add_to(sum[u]);
                const int here = __shfl_sync(0xffffffffu, token, j + h), next = __shfl_sync(0xffffffffu, after, j + h);
                if (here == next) continue;
                // the end of a run, or of the chunk
                const bool last = j0 + j + h + 1 == n;
                const int slot = at_first && from_before ? 0 : last && into_next ? 1 : -1;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int c = c0 + u * 32 * VEC;
                    if (c < a.d) {
                        if (slot < 0) {
                            finish<T, VEC>(a, i, here, c, sum[u]);
                        } else {
#pragma unroll
                            for (int e = 0; e < VEC; ++e) partial[slot * a.pitch + c + e] = sum[u][e];
                        }
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[u][e] = 0.f;
                }
                at_first = false;
            }
        }
    }
}

// A block: the run that begins in one chunk and goes on into the next, 1024 columns.
template <typename T> __global__ void __launch_bounds__(256) k_embed_join(const __grid_constant__ EmbedArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int AHEAD = 16;
    const int lane = threadIdx.x & 31, i = blockIdx.y;
    const long long chunk = blockIdx.x, first = chunk * a.chunk, end = first + a.chunk;
    const int* key = a.key + i * a.n;
    const int count = a.count[i];
    if (end >= count) return;
    const int token = key[end - 1], next = key[end], before = first > 0 ? key[first - 1] : -1;
    if (next != token || before == token) return;
    // chunks that the run goes on through: those that begin with its token
    long long more = 1;
    for (long long q = chunk + 1;; q += 32) {
        const long long begin = (q + lane) * a.chunk;
        const unsigned on = __ballot_sync(0xffffffffu, begin < count && key[begin < count ? begin : 0] == token);
        if (on != 0xffffffffu) {
            more = q - chunk - 1 + __popc(on);           // (sorted: the ones with the token come first)
            break;
        }
    }
    const int c = ((int)blockIdx.z * 256 + (int)threadIdx.x) * 4;
    if (c < a.d) {
        const float* partial = a.partial + ((long long)i * a.chunks + chunk) * 2 * a.pitch + c;
        float sum[4];
        load_vec<float, 4>(partial + a.pitch, sum);
        for (long long q = 1; q <= more; q += AHEAD) {
            float v[AHEAD][4];
#pragma unroll
            for (int h = 0; h < AHEAD; ++h) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[h][e] = 0.f;
                if (q + h <= more) load_vec<float, 4>(partial + (q + h) * 2 * a.pitch, v[h]);
            }
#pragma unroll
            for (int h = 0; h < AHEAD; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += v[h][e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.d) finish<T, 1>(a, i, token, c + e, sum + e);
    }
}

// Few places: one launch.  A block owns some rows of the table and 32 * U vectors of their columns, sorts the places of its rows in
// shared memory (warps one after another, so that the order is that of the places), and then a warp adds up and writes one row after
// another.  Rows with many places are added up by all warps.  For how many places and how large a table, us, against the three launches:
// 16 places of 1 x 500 x 64 in bf16 3.1 / 8.7; 122 of 2 x 1443 x 752 8.3 / 11.0; 209 of 6 x 224 x 48 7.3 / 11.3; 777 of 3 x 1009 x 509 in fp32 23 / 17;
// 1024 of 16 x 300 x 512 in bf16 30 / 21; 1 of 4 x 32000 x 64 (16 MB) 31 / 12.
constexpr int kFewPlaces = 256, kFewRange = 256, kFewMany = 16;
constexpr double kFewBytes = 8e6;
template <typename T, int VEC, int U> __global__ void __launch_bounds__(256, 4) k_embed_few(const __grid_constant__ EmbedArgs a) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int AHEAD = 8, EACH = kFewPlaces / 8;
    __shared__ int s_at[8][kFewRange], s_from[kFewRange + 1], s_red[8];
    __shared__ unsigned short s_place[kFewPlaces];
    __shared__ float s_sum[8][32 * U * VEC];
    const int i = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int first = (int)blockIdx.x * a.range, mine = (int)(a.V - first < a.range ? a.V - first : a.range);
    const int c0 = (int)blockIdx.z * 32 * U * VEC + lane * VEC;
    for (int q = threadIdx.x; q < 8 * kFewRange; q += 256) (&s_at[0][0])[q] = 0;
    const Tokens tokens(a, i);
    unsigned rel[EACH / 32];                             // rows of this lane's places, of the block's; beyond `mine`: none
#pragma unroll
    for (int u = 0; u < EACH / 32; ++u) {
        const int t = warp * EACH + u * 32 + lane, v = t < a.n ? tokens.at(t) : -1;
        rel[u] = v >= first ? (unsigned)(v - first) : 0xffffffffu;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < EACH / 32; ++u)
        if (rel[u] < (unsigned)mine) atomicAdd(&s_at[warp][rel[u]], 1);
    __syncthreads();
    // where the places of row r go that warp w finds: behind those of the rows before and of the warps before
    const int r = threadIdx.x;
    int total = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) total += s_at[w][r];
    int upto = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) s_red[warp] = upto;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) before += w < warp ? s_red[w] : 0;
    int at = before + upto - total;
    s_from[r] = at;
    if (r == kFewRange - 1) s_from[kFewRange] = at + total;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const int x = s_at[w][r];
        s_at[w][r] = at;
        at += x;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < EACH / 32; ++u) {
        const bool in = rel[u] < (unsigned)mine;
        const unsigned same = __match_any_sync(0xffffffffu, in ? rel[u] : 0xffffffffu);
        const int rank = __popc(same & ((1u << lane) - 1));
        int to = 0;
        if (in) to = s_at[warp][rel[u]];
        __syncwarp();
        if (in) {
            s_place[to + rank] = (unsigned short)(warp * EACH + u * 32 + lane);
            if (rank == 0) s_at[warp][rel[u]] = to + __popc(same);
        }
        __syncwarp();
    }
    __syncthreads();
    // sum over the places q0, q0 + step, ... below q1
    auto add_up = [&](int q0, int q1, int step, float (&sum)[U][VEC]) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[u][e] = 0.f;
        for (int q = q0; q < q1; q += AHEAD * step) {
            Raw<T, VEC> v[AHEAD][U];
#pragma unroll
            for (int h = 0; h < AHEAD; ++h) {
                if (q + h * step >= q1) continue;
                const T* from = row_of<T>(a.weight, i, s_place[q + h * step]) + c0;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c0 + u * 32 * VEC < a.d) v[h][u].load(from + u * 32 * VEC);
            }
#pragma unroll
            for (int h = 0; h < AHEAD; ++h) {
                if (q + h * step >= q1) continue;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c0 + u * 32 * VEC < a.d) v[h][u].add_to(sum[u]);
            }
        }
    };
    for (int q = warp; q < mine; q += 8) {
        const int q0 = s_from[q], q1 = s_from[q + 1];
        if (q1 - q0 > kFewMany || (q1 == q0 && a.accumulate)) continue;
        float sum[U][VEC];
        add_up(q0, q1, 1, sum);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * 32 * VEC;
            if (c >= a.d) continue;
            if (q1 > q0) finish<T, VEC>(a, i, first + q, c, sum[u]);
            else store_vec<T, VEC>(row_of<T>(a.out, i, first + q) + c, sum[u]);
        }
    }
    for (int q = 0; q < mine; ++q) {
        const int q0 = s_from[q], q1 = s_from[q + 1];
        if (q1 - q0 <= kFewMany) continue;
        float sum[U][VEC];
        add_up(q0 + warp, q1, 8, sum);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s_sum[warp][(u * 32 + lane) * VEC + e] = sum[u][e];
        __syncthreads();
        for (int x = threadIdx.x; x < 32 * U * VEC; x += 256) {
            const int c = (int)blockIdx.z * 32 * U * VEC + x;
            if (c >= a.d) continue;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) v += s_sum[w][x];
            finish<T, 1>(a, i, first + q, c, &v);
        }
        __syncthreads();
    }
}

// ----------------------------------------------------------------------------------- host
Rows rows(const eg_matrix& m) { return Rows{m.data, (long long)m.replica_stride, (long long)m.row_stride}; }

bool whole_vectors(const eg_matrix& m, int64_t P, int64_t rows, size_t size) {
    return aligned16(m.data) && (P <= 1 || m.replica_stride * (int64_t)size % 16 == 0) && (rows <= 1 || m.row_stride * (int64_t)size % 16 == 0);
}

// written: neither the rows of a replica nor the replicas fall on one another; the replicas lie one after the other, or take
// turns row by row.
bool usable(const eg_matrix& m, int64_t P, int64_t rows, int64_t cols, size_t size, bool written) {
    if (!m.data || (uintptr_t)m.data % size || m.row_stride < 0 || m.replica_stride < 0 || m.row_stride >= (1ll << 36) ||
        m.replica_stride >= (1ll << 42))
        return false;
    if (!written) return true;
    if (rows > 1 && m.row_stride < cols) return false;
    if (P > 1) {
        const __int128 rep = m.replica_stride, row = rows > 1 ? m.row_stride : 0;       // (2^30 rows 2^36 apart)
        if (!(rep >= (rows - 1) * row + cols || (rep >= cols && row >= (P - 1) * rep + cols))) return false;
    }
    return true;
}

bool valid(const eg_embedding_args* q, bool backward) {
    if (!q) return false;
    if (q->dtype != EG_F32 && q->dtype != EG_BF16 && q->dtype != EG_F16) return false;
    if (q->P < 1 || q->P > 65535 || q->rows < 0 || q->rows > (1ll << 30) || q->vocabulary < 1 || q->vocabulary > (1ll << 30) ||
        q->width < 1 || q->width > (1ll << 24))
        return false;
    if (!(q->scale >= -3e38 && q->scale <= 3e38)) return false;
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    if (q->rows > 0) {
        if (q->token_bytes != 4 && q->token_bytes != 8) return false;
        if (!q->tokens || (uintptr_t)q->tokens % (size_t)q->token_bytes || q->token_replica_stride < 0 || q->token_stride < 0 ||
            q->token_replica_stride >= (1ll << 42) || q->token_stride >= (1ll << 36))
            return false;
        if (!usable(backward ? q->dy : q->out, q->P, q->rows, q->width, size, !backward)) return false;
    }
    if (!usable(backward ? q->d_weight : q->weight, q->P, q->vocabulary, q->width, size, backward)) return false;
    return true;
}

// Chunks of 8 to 32 places, so that there are some eight warps for every multiprocessor (3 x 777 rows of 509 in fp32: chunks of 32 took 42 us);
// of more where a run over all places would have more than 1024 partial sums to join: a bound of what one block adds up, not a measured one.
int chunk_of(const eg_embedding_args* q) {
    const int64_t n = q->rows, columns = q->dtype == EG_F32 ? 128 : 256;
    const double all = (double)q->P * (double)n * (double)((q->width + columns - 1) / columns);
    int c = 32;
    while (c > 8 && all / c < 8.0 * 148) c /= 2;
    while (c * 1024ll < n) c *= 2;
    return c;
}
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

struct Layout {
    int64_t order, key, count, named, partial, bytes;
    int chunk, chunks, pitch, words;
};
Layout layout(const eg_embedding_args* q) {
    Layout l;
    const int64_t n = q->rows > 0 ? q->rows : 1;
    l.chunk = chunk_of(q);
    l.chunks = (int)((n + l.chunk - 1) / l.chunk);
    l.pitch = (int)((q->width + 7) / 8 * 8);
    l.order = 0;
    l.key = up16(4 * q->P * n);
    l.count = l.key + up16(4 * q->P * n);
    l.named = l.count + up16(4 * q->P);
    l.words = (int)((q->vocabulary + 31) / 32);
    l.partial = l.named + up16(4 * q->P * (int64_t)l.words);
    l.bytes = l.partial + q->P * (int64_t)l.chunks * 2 * l.pitch * 4;
    return l;
}

void fill(EmbedArgs* a, const eg_embedding_args* q, bool backward) {
    *a = EmbedArgs{};
    a->P = (int)q->P; a->n = q->rows; a->V = q->vocabulary; a->d = (int)q->width;
    a->scale = (float)q->scale;
    a->tokens = q->tokens; a->token_rep = q->token_replica_stride; a->token_step = q->token_stride;
    a->wide = q->token_bytes == 8;
    a->weight = rows(backward ? q->dy : q->weight);
    a->out = rows(backward ? q->d_weight : q->out);
    a->accumulate = q->accumulate != 0;
}

template <typename T, int VEC> cudaError_t forward(const EmbedArgs& a, cudaStream_t stream) {
    auto launch = [&](auto kernel, int U) {
        const int per = 32 * U * VEC, slices = (a.d + per - 1) / per;
        const long long blocks = (a.P * a.n * slices + 7) / 8;
        if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
        return launch_after(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a, slices);
    };
    if (a.d <= 32 * VEC) return launch(k_embed<T, VEC, 1>, 1);
    if (a.d <= 64 * VEC) return launch(k_embed<T, VEC, 2>, 2);
    return launch(k_embed<T, VEC, kMaxVectors>, kMaxVectors);
}

template <typename T, int VEC> cudaError_t backward(EmbedArgs a, cudaStream_t stream) {
    // zeros: 64 KB or so a block, at least a few blocks for every multiprocessor
    long long zeros = 0;
    if (!a.accumulate) {
        zeros = (long long)((double)a.V * a.d * sizeof(T) / 65536.0) + 1;
        const long long least = (4ll * sm_count() + a.P - 1) / a.P, most = (a.V + 7) / 8;
        if (zeros < least) zeros = least;
        if (zeros > most) zeros = most;
    }
    cudaError_t e;
    constexpr int U = VEC > 1 ? 1 : 4;
    const int slices = (a.d + 32 * U * VEC - 1) / (32 * U * VEC);
    if (a.n > 0 && a.n <= kFewPlaces && (double)a.P * a.V * a.d * sizeof(T) <= kFewBytes) {
        // rows of a block: as many as still leave four blocks for every multiprocessor
        a.range = kFewRange;
        while (a.range > 4 && (double)a.P * slices * ((a.V + a.range - 1) / a.range) < 4.0 * sm_count()) a.range /= 2;
        return launch_after(k_embed_few<T, VEC, U>, dim3((unsigned)((a.V + a.range - 1) / a.range), a.P, slices), dim3(256), 0, stream, a);
    }
    // Zeros beside the sort, for all rows, or beside the sums, for those without a place.  Measured, us, early / late, tokens as often as words
    // and (uniform): 4 replicas of 32000 x 1024 in bf16 with 960 places 55 / 60 (55 / 58), 4000 78 / 80 (76 / 78), 16000 135 / 137 (132 / 127), 32000
    // 219 / 217 (213 / 192), 64000 355 / 348 (347 / 311), 128000 631 / 608 (594 / 542); 4 x 1009 x 512 in fp32 with 504 21 / 18, 4036 40 / 37.
    const bool early = a.n <= a.V;
    a.sort_blocks = a.n > 0 ? (int)((a.V + a.range - 1) / a.range) : 0;
    e = launch_after(k_embed_sort<T, VEC>, dim3((unsigned)(a.sort_blocks + (early ? zeros : 0)), a.P), dim3(kSortThreads), 0, stream, a);
    if (e != cudaSuccess || a.n == 0) return e;
    a.sum_blocks = (int)(((long long)a.chunks * slices + 7) / 8);
    e = launch_after(k_embed_sum<T, VEC, U>, dim3((unsigned)(a.sum_blocks + (early ? 0 : zeros)), a.P), dim3(256), 0, stream, a, slices);
    if (e != cudaSuccess || a.chunks == 1) return e;
    return launch_after(k_embed_join<T>, dim3((unsigned)a.chunks, a.P, (a.d + 1023) / 1024), dim3(256), 0, stream, a);
}

}  // namespace
}  // namespace eg

using namespace eg;

extern "C" {

eg_status eg_embedding(const eg_embedding_args* q, void* stream_v) {
    if (!valid(q, false)) return EG_ERR_INVALID;
    if (q->rows == 0) return EG_OK;
    EmbedArgs a;
    fill(&a, q, false);
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    const bool vec = q->width * size % 16 == 0 && whole_vectors(q->weight, q->P, q->vocabulary, size) && whole_vectors(q->out, q->P, q->rows, size);
    cudaStream_t s = static_cast<cudaStream_t>(stream_v);
    cudaError_t e;
    if (q->dtype == EG_F32) e = vec ? forward<float, 4>(a, s) : forward<float, 1>(a, s);
    else if (q->dtype == EG_BF16) e = vec ? forward<__nv_bfloat16, 8>(a, s) : forward<__nv_bfloat16, 1>(a, s);
    else e = vec ? forward<__half, 8>(a, s) : forward<__half, 1>(a, s);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

int64_t eg_embedding_workspace(const eg_embedding_args* q) {
    if (!valid(q, true)) return 0;
    return layout(q).bytes;
}

eg_status eg_embedding_backward(const eg_embedding_args* q, void* workspace, int64_t workspace_bytes, void* stream_v) {
    if (!valid(q, true)) return EG_ERR_INVALID;
    if (q->rows == 0 && q->accumulate) return EG_OK;
    const Layout l = layout(q);
    if (!workspace || !aligned16(workspace) || workspace_bytes < l.bytes) return EG_ERR_INVALID;
    const int sms = sm_count();
    if (sms < 1) return EG_ERR_CUDA;
    EmbedArgs a;
    fill(&a, q, true);
    char* w = static_cast<char*>(workspace);
    a.order = reinterpret_cast<int*>(w + l.order);
    a.key = reinterpret_cast<int*>(w + l.key);
    a.count = reinterpret_cast<int*>(w + l.count);
    a.named = reinterpret_cast<unsigned int*>(w + l.named);
    a.words = l.words;
    a.partial = reinterpret_cast<float*>(w + l.partial);
    a.chunk = l.chunk; a.chunks = l.chunks; a.pitch = l.pitch;
    // ranges long enough that the tokens are not read more often than needed, short enough that every multiprocessor has some (us with ranges
    // of 512 and of 64: 4 replicas of 32000 x 1024 in bf16 with 960 places 55 and 70, 32000 217 and 371; 4 x 8000 x 1024 with 1000 31 and 35; 1 x 32000
    // x 2048 with 64000 240 and 275, with the 128 that the rule takes 234; 4 x 1009 x 512 in fp32 with 4036 39 and 37, the rule's)
    a.range = kRangeMax;
    while (a.range > 64 && a.P * ((a.V + a.range - 1) / a.range) < sms) a.range /= 2;
    const size_t size = q->dtype == EG_F32 ? 4 : 2;
    const bool vec = q->width * size % 16 == 0 && (q->rows == 0 || whole_vectors(q->dy, q->P, q->rows, size)) &&
                     whole_vectors(q->d_weight, q->P, q->vocabulary, size);
    cudaStream_t s = static_cast<cudaStream_t>(stream_v);
    cudaError_t e;
    if (q->dtype == EG_F32) e = vec ? backward<float, 4>(a, s) : backward<float, 1>(a, s);
    else if (q->dtype == EG_BF16) e = vec ? backward<__nv_bfloat16, 8>(a, s) : backward<__nv_bfloat16, 1>(a, s);
    else e = vec ? backward<__half, 8>(a, s) : backward<__half, 1>(a, s);
    return e == cudaSuccess ? EG_OK : EG_ERR_CUDA;
}

}  // extern "C"
