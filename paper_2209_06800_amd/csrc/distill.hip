// The loss of a student against a teacher's top logits, and its gradient.
//
// With q = softmax(z / T) over a row of logits and p = softmax(t / T) over its teacher entries, the loss needs the row's maximum m
// and s = sum exp((z - m) / T): sum p (log p - log q) = sum p (log p - (z - m) / T) + log s; the gradient is w T (q - p).
// Bound by HBM: the logits read once, the gradient written once.  What a row costs besides is kept small in three ways, by the
// length of a row and their number (launch_distill):
//   - short rows: a few lanes each, in registers, several rows per wavefront;
//   - rows that the registers of a workgroup hold: one workgroup each, one reading;
//   - few rows, or longer ones: pieces of rows; each piece's maximum and sum first, then the gradient from a second reading
//     (out of the caches where it is for few rows).
// 4096 rows of 128 k bf16 with gradient: 0.47 ms, 1.99 GB at 4.2 TB/s, the row in the registers of 1024 threads (a block per row that
// reads it three times: 1.84 ms); 306 k rows of 47 fp32: loss alone 27 us, 2.7 TB/s, with gradient 49 us, 2.8 TB/s; 37 rows of 50 k with gradient:
// 17 us, two launches; 2000 rows with gradient in pieces, read twice: 151,936 bf16 345 us, 262,144 bf16 577, 128,000 fp32 549 (1.16, 1.99 and 1.95 GB
// at 3.4 - 3.5 TB/s, once counted); 4096 rows of 128 k bf16, loss alone: 174 us, 5.4 TB/s.
#include <cmath>

#include "train_common.h"

namespace mgg {

namespace {

using namespace train;

constexpr int kMaxTop = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct DistillArgs {
    const void *logits, *top_ids, *top_logits;
    const float *row_weight;
    float *loss;
    void *grad;
    float *stats;           // pieces: [rows x (2 pieces + 3)]: what piece 0 knows, then a maximum and a sum each
    int64_t n_rows, ld_logits, ld_ids, ld_top, ld_grad;
    int32_t n_classes, k;
    float temperature, inv_t;
    int32_t ids64, top_bf16;
    int32_t lanes_log2;     // short rows: lanes of a row
    int32_t piece, pieces;  // classes of a piece, a multiple of 8; pieces of a row
};

__device__ __forceinline__ int32_t entry_id(const DistillArgs &p, int64_t row, int j)       // -1: not there
{
    const int64_t id = p.ids64 ? static_cast<const int64_t *>(p.top_ids)[row * p.ld_ids + j] : static_cast<const int32_t *>(p.top_ids)[row * p.ld_ids + j];
    return id >= 0 && id < p.n_classes ? static_cast<int32_t>(id) : -1;
}
__device__ __forceinline__ float entry_logit(const DistillArgs &p, int64_t row, int j)
{
    return p.top_bf16 ? to_f32(static_cast<const Bf16 *>(p.top_logits)[row * p.ld_top + j]) : static_cast<const float *>(p.top_logits)[row * p.ld_top + j];
}

// exp((x - m) / T) with c = log2(e) / T.  The difference comes first: with masks of the type's lowest value the product alone would not
// cancel.
__device__ __forceinline__ float soft(float x, float m, float c) { return __builtin_amdgcn_exp2f((x - m) * c); }
__device__ __forceinline__ float log_of(float x) { return __builtin_amdgcn_logf(x) * kLn2; }

// 16 bytes of a row at column c, as they lie; -infinity in the places of columns that are not this vector's: those behind the
// row's end, and, in the last vector, which is moved back to end with the row, those of the vector before
template <typename T> struct Vec { static constexpr int N = 16 / sizeof(T); uint32_t u[4]; };

__device__ __forceinline__ float element(const Vec<float> &v, int e) { return __uint_as_float(v.u[e]); }
__device__ __forceinline__ float element(const Vec<Bf16> &v, int e) { return __uint_as_float(e & 1 ? v.u[e >> 1] & 0xffff0000u : v.u[e >> 1] << 16); }

template <typename T>
__device__ __forceinline__ Vec<T> load_own(const T *row, int64_t c, int64_t n)
{
    constexpr int N = Vec<T>::N;
    Vec<T> v;
    if (c + N <= n) {
        __builtin_memcpy(v.u, __builtin_assume_aligned(row + c, sizeof(T)), 16);
        return v;
    }
    T e[N];
    if (n >= N && c < n) {
        __builtin_memcpy(e, __builtin_assume_aligned(row + n - N, sizeof(T)), 16);
    } else if (c < n) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) e[i] = row[i];
    }
    const int64_t col = n >= N ? n - N : 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (col + i < c || col + i >= n) {
            if constexpr (sizeof(T) == 2) e[i].bits = 0xff80u;
            else e[i] = -INFINITY;
        }
    __builtin_memcpy(v.u, e, 16);
    return v;
}

// the same of a row of N elements at least, without a branch before the load (a vector behind the row loads its last one)
template <typename T>
__device__ __forceinline__ Vec<T> load_own_long(const T *row, int c, int n)
{
    constexpr int N = Vec<T>::N;
    const int col = c + N <= n ? c : n - N;
    Vec<T> v;
    __builtin_memcpy(v.u, __builtin_assume_aligned(row + col, sizeof(T)), 16);
    if (c + N > n) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (col + i < c) {
                if constexpr (sizeof(T) == 2) v.u[i >> 1] = i & 1 ? (v.u[i >> 1] & 0xffffu) | 0xff800000u : (v.u[i >> 1] & 0xffff0000u) | 0xff80u;
                else v.u[i] = 0xff800000u;
            }
    }
    return v;
}

// the values of such a vector to the same columns of another row
template <typename T, int N>
__device__ __forceinline__ void store_own(T *row, int64_t c, int64_t n, const float (&v)[N])
{
    if (c + N <= n) {
        store_n<N>(row + c, v);
    } else if (c < n) {
        const int64_t col = n >= N ? n - N : 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (col + i >= c && col + i < n) from_f32(v[i], row[col + i]);
    }
}

// The row stays in registers as it lies: without this the compiler keeps what a pass has unpacked, twice the registers, for the next.
template <typename T, int NV>
__device__ __forceinline__ void pin(Vec<T> (&x)[NV])
{
#pragma unroll
    for (int v = 0; v < NV; ++v) asm volatile("" : "+v"(x[v].u[0]), "+v"(x[v].u[1]), "+v"(x[v].u[2]), "+v"(x[v].u[3]));
}

// maximum m (NaN aside) and s = sum of soft(x, m) of what has been seen
struct Running {
    float m, s;
    __device__ __forceinline__ void join(float om, float os, float c)
    {
        const float high = fmaxf(m, om), at = high == -INFINITY ? 0.f : high;
        s = s * soft(m, at, c) + os * soft(om, at, c);
        m = high;
    }
};

// over a workgroup: the wavefronts' values meet in LDS, and every wavefront joins them for itself
template <int THREADS>
__device__ __forceinline__ Running block_join(Running r, float c, float (&part)[2][THREADS / kWave])
{
    constexpr int W = THREADS / kWave;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) r.join(__shfl_xor(r.m, off), __shfl_xor(r.s, off), c);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { part[0][threadIdx.x >> 6] = r.m; part[1][threadIdx.x >> 6] = r.s; }
    __syncthreads();
    r = Running{part[0][threadIdx.x % W], part[1][threadIdx.x % W]};
#pragma unroll
    for (int off = W / 2; off >= 1; off >>= 1) r.join(__shfl_xor(r.m, off), __shfl_xor(r.s, off), c);
    return r;
}
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float (&part)[2][THREADS / kWave])
{
    constexpr int W = THREADS / kWave;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[0][threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0][threadIdx.x % W];
#pragma unroll
    for (int off = W / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// ---- short rows ----------------------------------------------------------------------------------------------
// 2^lanes_log2 lanes hold a row, NV vectors each; a class's teacher mass is taken off as its entries go round the lanes
constexpr int kShortThreads = 256, kShortMax = 4;

template <typename In, typename Out, int NV>
__global__ __launch_bounds__(kShortThreads) void distill_short_kernel(const DistillArgs p)
{
    constexpr int N = Vec<In>::N;
    const int lanes = 1 << p.lanes_log2, lane = threadIdx.x & (lanes - 1), base = threadIdx.x & 63 & ~(lanes - 1);
    const int64_t row = ((static_cast<int64_t>(blockIdx.x) * kShortThreads) + threadIdx.x) >> p.lanes_log2;
    if (row >= p.n_rows) return;            // (whole groups of lanes)
    const In *z = static_cast<const In *>(p.logits) + row * p.ld_logits;
    const float weight = p.row_weight ? p.row_weight[row] : 1.f, c2 = p.inv_t * kLog2e;
    Vec<In> x[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) x[v] = load_own(z, static_cast<int64_t>(v * lanes + lane) * N, p.n_classes);
    Running t{-INFINITY, 0.f};
    for (int j = lane; j < p.k; j += lanes)
        if (entry_id(p, row, j) >= 0) t.join(entry_logit(p, row, j), 1.f, c2);
    Running r{-INFINITY, 0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < N; ++e) r.m = fmaxf(r.m, element(x[v], e));
    const float at = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < N; ++e) r.s += soft(element(x[v], e), at, c2);
    for (int off = lanes >> 1; off >= 1; off >>= 1) {
        t.join(__shfl_xor(t.m, off), __shfl_xor(t.s, off), c2);
        r.join(__shfl_xor(r.m, off), __shfl_xor(r.s, off), c2);
    }
    const bool empty = weight == 0.f || (t.m == -INFINITY && t.s == 0.f) || (r.m == -INFINITY && r.s == 0.f);
    const float log_s = log_of(r.s), log_t = log_of(t.s), inv_s = 1.f / r.s, inv_ts = 1.f / t.s;
    float loss = 0.f;
    for (int j = lane; j < p.k; j += lanes) {
        const int32_t id = entry_id(p, row, j);
        if (id < 0 || empty) continue;
        const float v = entry_logit(p, row, j), prob = soft(v, t.m, c2) * inv_ts;
        if (prob != 0.f) loss += prob * (((v - t.m) * p.inv_t - log_t) - ((to_f32(z[id]) - r.m) * p.inv_t - log_s));
    }
    for (int off = lanes >> 1; off >= 1; off >>= 1) loss += __shfl_xor(loss, off);
    if (lane == 0) p.loss[row] = empty ? 0.f : weight * p.temperature * p.temperature * loss;
    if (!p.grad) return;
    float g[NV][N];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < N; ++e) g[v][e] = empty ? 0.f : soft(element(x[v], e), r.m, c2) * inv_s;
    // in place of the logits: every lane of the row has read what it needs of them (a wavefront's accesses are in order)
    const int first_own = p.n_classes >= N ? p.n_classes - N : 0;       // column of the moved-back vector
    for (int j0 = 0; j0 < p.k; j0 += lanes) {
        int32_t id = -1;
        float prob = 0.f;
        if (j0 + lane < p.k && !empty) {
            id = entry_id(p, row, j0 + lane);
            if (id >= 0) prob = soft(entry_logit(p, row, j0 + lane), t.m, c2) * inv_ts;
        }
        const int count = p.k - j0 < lanes ? p.k - j0 : lanes;
        for (int j = 0; j < count; ++j) {
            const int32_t other = __shfl(id, base + j);
            const float mass = __shfl(prob, base + j);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * lanes + lane) * N, col = c + N <= p.n_classes ? c : first_own;
#pragma unroll
                for (int e = 0; e < N; ++e) g[v][e] -= other == col + e ? mass : 0.f;
            }
        }
    }
    Out *dz = static_cast<Out *>(p.grad) + row * p.ld_grad;
    const float factor = weight * p.temperature;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int e = 0; e < N; ++e) g[v][e] = empty ? 0.f : factor * g[v][e];
        store_own(dz, static_cast<int64_t>(v * lanes + lane) * N, p.n_classes, g[v]);
    }
}

// ---- the teacher's side of a row, by a workgroup ---------------------------------------------------------------
struct Teacher {
    int32_t id[kMaxTop];
    float p[kMaxTop];       // logit, then probability
    float z[kMaxTop];       // the student's logit of the class
};

// ids and logits to LDS; the student's logits of their classes behind them
template <typename In, int THREADS>
__device__ __forceinline__ Running teacher_load(const DistillArgs &p, int64_t row, const In *z, Teacher &t, float c2)
{
    Running r{-INFINITY, 0.f};
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        const int32_t id = entry_id(p, row, j);
        const float v = entry_logit(p, row, j);
        t.id[j] = id;
        t.p[j] = v;
        if (id >= 0) r.join(v, 1.f, c2);
        t.z[j] = id >= 0 ? to_f32(z[id]) : 0.f;
    }
    return r;
}

// logits to probabilities; returns this thread's part of sum p (log p - (z - ref) / T), ref being any number near the z
template <int THREADS>
__device__ __forceinline__ float teacher_loss(const DistillArgs &p, Teacher &t, const Running &top, float ref, float c2)
{
    const float log_t = log_of(top.s), inv_ts = 1.f / top.s;
    float loss = 0.f;
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        const float v = t.p[j], prob = t.id[j] >= 0 ? soft(v, top.m, c2) * inv_ts : 0.f;
        if (prob != 0.f) loss += prob * (((v - top.m) * p.inv_t - log_t) - (t.z[j] - ref) * p.inv_t);
        t.p[j] = prob;
    }
    return loss;
}

// the gradient at the teacher's classes in [lo, hi), each by its first entry, over what was written there without them
template <typename Out, int THREADS>
__device__ __forceinline__ void teacher_grad(const DistillArgs &p, const Teacher &t, Out *dz, int64_t lo, int64_t hi, float m, float inv_s, float factor, float c2)
{
    for (int j = threadIdx.x; j < p.k; j += THREADS) {
        const int32_t id = t.id[j];
        if (id < lo || id >= hi) continue;
        float prob = 0.f;
        bool first = true;
        for (int i = 0; i < p.k; ++i)
            if (t.id[i] == id) {
                first = first && i >= j;
                prob += t.p[i];
            }
        if (first) from_f32(factor * (soft(t.z[j], m, c2) * inv_s - prob), dz[id]);
    }
}

// ---- a workgroup per row, the row in its registers -------------------------------------------------------------
template <typename In, typename Out, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void distill_row_kernel(const DistillArgs p)
{
    constexpr int N = Vec<In>::N;
    __shared__ Teacher t;
    __shared__ float part[2][THREADS / kWave];
    const int64_t row = blockIdx.x;
    const In *z = static_cast<const In *>(p.logits) + row * p.ld_logits;
    Out *dz = static_cast<Out *>(p.grad) + row * p.ld_grad;
    const float weight = p.row_weight ? p.row_weight[row] : 1.f, c2 = p.inv_t * kLog2e;
    const float zero[N] = {};
    if (weight == 0.f) {
        if (threadIdx.x == 0) p.loss[row] = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) store_own(dz, static_cast<int64_t>(v * THREADS + threadIdx.x) * N, p.n_classes, zero);
        return;
    }
    Vec<In> x[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) x[v] = load_own_long(z, static_cast<int>(v * THREADS + threadIdx.x) * N, p.n_classes);
    Running top = teacher_load<In, THREADS>(p, row, z, t, c2);
    Running r{-INFINITY, 0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < N; ++e) r.m = fmaxf(r.m, element(x[v], e));
    pin(x);
    const float at = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < N; ++e) r.s += soft(element(x[v], e), at, c2);
    pin(x);
    r = block_join<THREADS>(r, c2, part);
    top = block_join<THREADS>(top, c2, part);
    const bool empty = (top.m == -INFINITY && top.s == 0.f) || (r.m == -INFINITY && r.s == 0.f);
    if (empty) {
        if (threadIdx.x == 0) p.loss[row] = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) store_own(dz, static_cast<int64_t>(v * THREADS + threadIdx.x) * N, p.n_classes, zero);
        return;
    }
    const float log_s = log_of(r.s), inv_s = 1.f / r.s, factor = weight * p.temperature, scale = factor * inv_s;
    const float loss = block_sum<THREADS>(teacher_loss<THREADS>(p, t, top, r.m, c2), part);
    if (threadIdx.x == 0) p.loss[row] = weight * p.temperature * p.temperature * (loss + log_s);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float g[N];
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = scale * soft(element(x[v], e), r.m, c2);
        store_own(dz, static_cast<int64_t>(v * THREADS + threadIdx.x) * N, p.n_classes, g);
    }
    __syncthreads();
    teacher_grad<Out, THREADS>(p, t, dz, 0, p.n_classes, r.m, inv_s, factor, c2);
}

// ---- pieces of rows ------------------------------------------------------------------------------------------
constexpr int kPieceThreads = 256;

// maximum and sum of a piece; with piece 0 the teacher's side: sum p (log p - (z - ref) / T), ref, and whether there is a teacher.
// ONE: a row is one piece, and this is the loss.
template <typename In, bool ONE>
__global__ __launch_bounds__(kPieceThreads) void distill_stats_kernel(const DistillArgs p)
{
    constexpr int N = Vec<In>::N, U = 4;
    __shared__ Teacher t;
    __shared__ float part[2][kPieceThreads / kWave];
    const int64_t row = blockIdx.x / p.pieces, index = blockIdx.x % p.pieces;
    const In *z = static_cast<const In *>(p.logits) + row * p.ld_logits;
    const float weight = p.row_weight ? p.row_weight[row] : 1.f, c2 = p.inv_t * kLog2e;
    if (weight == 0.f) {                     // (nothing of it is read later)
        if (ONE && threadIdx.x == 0) p.loss[row] = 0.f;
        return;
    }
    float *stats = p.stats + row * (2 * static_cast<int64_t>(p.pieces) + 3);
    const int64_t lo = index * p.piece, hi = lo + p.piece < p.n_classes ? lo + p.piece : p.n_classes;
    Running top{-INFINITY, 0.f};
    if (index == 0) top = teacher_load<In, kPieceThreads>(p, row, z, t, c2);
    Running r{-INFINITY, 0.f};
    for (int64_t c = lo + threadIdx.x * N; c < hi; c += U * kPieceThreads * N) {
        Vec<In> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load_own(z, c + u * kPieceThreads * N, hi);
        float high = r.m;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) high = fmaxf(high, element(x[u], e));
        const float at = high == -INFINITY ? 0.f : high;
        float s = r.s * soft(r.m, at, c2);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) s += soft(element(x[u], e), at, c2);
        r.m = high;
        r.s = s;
    }
    r = block_join<kPieceThreads>(r, c2, part);
    if (!ONE && threadIdx.x == 0) { stats[3 + 2 * index] = r.m; stats[4 + 2 * index] = r.s; }
    if (index != 0) return;
    top = block_join<kPieceThreads>(top, c2, part);
    const bool none = top.m == -INFINITY && top.s == 0.f;
    if constexpr (ONE) {
        const bool empty = none || (r.m == -INFINITY && r.s == 0.f);
        const float loss = empty ? 0.f : block_sum<kPieceThreads>(teacher_loss<kPieceThreads>(p, t, top, r.m, c2), part);
        if (threadIdx.x == 0) p.loss[row] = empty ? 0.f : weight * p.temperature * p.temperature * (loss + log_of(r.s));
    } else {
        // the classes' logits relative to their largest, which the row's maximum replaces when it is known
        Running ref{-INFINITY, 0.f};
        for (int j = threadIdx.x; j < p.k; j += kPieceThreads)
            if (t.id[j] >= 0) ref.m = fmaxf(ref.m, t.z[j]);
        ref = block_join<kPieceThreads>(ref, c2, part);
        const float at = ref.m == -INFINITY ? 0.f : ref.m;
        const float loss = none ? 0.f : block_sum<kPieceThreads>(teacher_loss<kPieceThreads>(p, t, top, at, c2), part);
        if (threadIdx.x == 0) { stats[0] = loss; stats[1] = at; stats[2] = none ? 1.f : 0.f; }
    }
}

// the row's maximum and sum from its pieces', the loss (piece 0), and the piece's gradient
template <typename In, typename Out>
__global__ __launch_bounds__(kPieceThreads) void distill_pieces_kernel(const DistillArgs p, int blocks_per_row)
{
    constexpr int N = Vec<In>::N, U = 4;
    __shared__ Teacher t;
    __shared__ float part[2][kPieceThreads / kWave];
    const int64_t row = blockIdx.x / blocks_per_row, index = blockIdx.x % blocks_per_row;
    const In *z = static_cast<const In *>(p.logits) + row * p.ld_logits;
    Out *dz = static_cast<Out *>(p.grad) + row * p.ld_grad;
    const float weight = p.row_weight ? p.row_weight[row] : 1.f, c2 = p.inv_t * kLog2e;
    const float *stats = p.stats + row * (2 * static_cast<int64_t>(p.pieces) + 3);
    Running r{-INFINITY, 0.f};
    bool empty = weight == 0.f;
    if (!empty) {
        for (int i = threadIdx.x; i < p.pieces; i += kPieceThreads) r.join(stats[3 + 2 * i], stats[4 + 2 * i], c2);
        r = block_join<kPieceThreads>(r, c2, part);
        empty = stats[2] != 0.f || (r.m == -INFINITY && r.s == 0.f);
    }
    if (index == 0 && threadIdx.x == 0)
        p.loss[row] = empty ? 0.f : weight * p.temperature * p.temperature * (stats[0] + (r.m - stats[1]) * p.inv_t + log_of(r.s));
    if (!p.grad) return;
    const int64_t lo = index * p.piece, hi = lo + p.piece < p.n_classes ? lo + p.piece : p.n_classes;
    const float inv_s = 1.f / r.s, factor = weight * p.temperature, scale = factor * inv_s;
    if (!empty) {
        // the teacher's entries of this piece, their logits of the student before anything is written in their place
        Running top{-INFINITY, 0.f};
        for (int j = threadIdx.x; j < p.k; j += kPieceThreads) {
            const int32_t id = entry_id(p, row, j);
            t.id[j] = id;
            t.p[j] = entry_logit(p, row, j);
            if (id >= 0) top.join(t.p[j], 1.f, c2);
            t.z[j] = id >= lo && id < hi ? to_f32(z[id]) : 0.f;
        }
        top = block_join<kPieceThreads>(top, c2, part);
        (void)teacher_loss<kPieceThreads>(p, t, top, 0.f, c2);
        __syncthreads();
    }
    for (int64_t c = lo + threadIdx.x * N; c < hi; c += U * kPieceThreads * N) {
        Vec<In> x[U];
        if (!empty) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = load_own(z, c + u * kPieceThreads * N, hi);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float g[N];
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = empty ? 0.f : scale * soft(element(x[u], e), r.m, c2);
            store_own(dz, c + u * kPieceThreads * N, hi, g);
        }
    }
    if (empty) return;
    __syncthreads();
    teacher_grad<Out, kPieceThreads>(p, t, dz, lo, hi, r.m, inv_s, factor, c2);
}

// Pieces of a row where it is taken in pieces: workgroups enough for the chip, but not more pieces than there are 4096 classes, begun
// ones counted (4097 classes are two pieces of some 2 k).
int pieces_of(int64_t n_rows, int32_t n_classes)
{
    const int64_t wanted = n_rows < 2048 ? ceil_div(2048, n_rows > 0 ? n_rows : 1) : 1, most = ceil_div(n_classes, 4096);
    return static_cast<int>(wanted < most ? wanted : most);
}

// The longest rows, in vectors, that the registers of a workgroup hold, and those that are short.
constexpr int kShortVecs = kWave * kShortMax, kRow256Vecs = 256 * 8, kRow1024Vecs = 1024 * 16;

// rows of more than kShortVecs vectors, with a gradient, by 256 or 1024 threads
template <typename In, typename Out, int THREADS>
void launch_rows(const DistillArgs &p, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(p.n_rows)), block(THREADS);
    const int64_t per = ceil_div(ceil_div(p.n_classes, Vec<In>::N), THREADS);
#define MGG_ROWS(NV) hipLaunchKernelGGL((distill_row_kernel<In, Out, THREADS, NV>), grid, block, 0, stream, p)
    if constexpr (THREADS == 256) {
        static_assert(kShortVecs >= 256 && kRow256Vecs == 256 * 8, "two to eight vectors of a thread");
        if (per <= 2) MGG_ROWS(2);
        else if (per <= 4) MGG_ROWS(4);
        else MGG_ROWS(8);
    } else {
        static_assert(THREADS == 1024 && kRow1024Vecs == 1024 * 16, "up to sixteen");
        if (per <= 4) MGG_ROWS(4);
        else if (per <= 8) MGG_ROWS(8);
        else MGG_ROWS(16);
    }
#undef MGG_ROWS
}

template <typename In, typename Out>
mgg_status_t launch_typed(DistillArgs p, hipStream_t stream)
{
    constexpr int N = Vec<In>::N;
    const char *const refused = "too many rows for one launch";
    const int64_t vecs = ceil_div(p.n_classes, N);
    if (vecs <= kShortVecs) {
        // four lanes at least, which share the teacher's entries; four vectors at most per lane
        p.lanes_log2 = ceil_log2(ceil_div(vecs, kShortMax));
        if (p.lanes_log2 < 2) p.lanes_log2 = 2;
        const int64_t blocks = ceil_div(p.n_rows << p.lanes_log2, kShortThreads), per = ceil_div(vecs, static_cast<int64_t>(1) << p.lanes_log2);
        if (!launchable(blocks, kShortThreads)) return fail(MGG_ERR_UNSUPPORTED, "%s", refused);
        const dim3 grid(static_cast<unsigned>(blocks));
        if (per <= 1) hipLaunchKernelGGL((distill_short_kernel<In, Out, 1>), grid, dim3(kShortThreads), 0, stream, p);
        else if (per <= 2) hipLaunchKernelGGL((distill_short_kernel<In, Out, 2>), grid, dim3(kShortThreads), 0, stream, p);
        else if (per <= 3) hipLaunchKernelGGL((distill_short_kernel<In, Out, 3>), grid, dim3(kShortThreads), 0, stream, p);
        else hipLaunchKernelGGL((distill_short_kernel<In, Out, 4>), grid, dim3(kShortThreads), 0, stream, p);
    } else if (p.grad && vecs <= kRow256Vecs) {
        if (!launchable(p.n_rows, 256)) return fail(MGG_ERR_UNSUPPORTED, "%s", refused);
        launch_rows<In, Out, 256>(p, stream);
    } else if (p.grad && vecs <= kRow1024Vecs && (p.n_rows >= 64 || vecs <= 4 * 1024)) {
        // (100 rows of 128 k bf16: 31 us, in pieces 35; 16 rows: 28 and 21; 4 rows of 30 k: 13 and 17)
        if (!launchable(p.n_rows, 1024)) return fail(MGG_ERR_UNSUPPORTED, "%s", refused);
        launch_rows<In, Out, 1024>(p, stream);
    } else {
        p.pieces = pieces_of(p.n_rows, p.n_classes);
        p.piece = static_cast<int32_t>(ceil_div(ceil_div(p.n_classes, p.pieces), 8) * 8);
        const int64_t blocks = p.n_rows * p.pieces;
        if (!launchable(blocks, kPieceThreads)) return fail(MGG_ERR_UNSUPPORTED, "%s", refused);
        const dim3 grid(static_cast<unsigned>(blocks)), block(kPieceThreads);
        if (p.pieces == 1 && !p.grad) {
            hipLaunchKernelGGL((distill_stats_kernel<In, true>), grid, block, 0, stream, p);
        } else {
            hipLaunchKernelGGL((distill_stats_kernel<In, false>), grid, block, 0, stream, p);
            const int per_row = p.grad ? p.pieces : 1;
            hipLaunchKernelGGL((distill_pieces_kernel<In, Out>), dim3(static_cast<unsigned>(p.n_rows * per_row)), block, 0, stream, p, per_row);
        }
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, "distillation kernel launch");
}

}  // namespace

size_t distill_workspace(int64_t n_rows, int32_t n_classes)
{
    return static_cast<size_t>(n_rows) * (2 * static_cast<size_t>(pieces_of(n_rows, n_classes)) + 3) * 4 + 256;
}

mgg_status_t launch_distill(const Distill &q, void *workspace, hipStream_t stream)
{
    DistillArgs p{};
    p.logits = q.logits; p.top_ids = q.top_ids; p.top_logits = q.top_logits; p.row_weight = q.row_weight; p.loss = q.loss; p.grad = q.grad;
    p.stats = static_cast<float *>(workspace);
    p.n_rows = q.n_rows; p.ld_logits = q.ld_logits; p.ld_ids = q.ld_ids; p.ld_top = q.ld_top; p.ld_grad = q.ld_grad;
    p.n_classes = q.n_classes; p.k = q.k; p.temperature = q.temperature; p.inv_t = 1.f / q.temperature;
    p.ids64 = q.id_type == MGG_I64; p.top_bf16 = q.top_dtype == MGG_BF16;
    const bool in16 = q.logits_dtype == MGG_BF16, out16 = q.grad ? q.grad_dtype == MGG_BF16 : in16;
    if (in16) return out16 ? launch_typed<Bf16, Bf16>(p, stream) : launch_typed<Bf16, float>(p, stream);
    return out16 ? launch_typed<float, Bf16>(p, stream) : launch_typed<float, float>(p, stream);
}

}  // namespace mgg
