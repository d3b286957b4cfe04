// Lookup of scaled table rows by ids on the device, and the gradient of the table by sorted ids.
#include "train_common.h"

namespace mgg {

namespace {

using namespace train;

constexpr int kThreads = 256;

// ---- out[i] = scale * table[ids[i]] --------------------------------------------------------------------------
// A copy of rows: bound by HBM (the distinct rows read, all rows written).
template <typename In, typename Out, typename Id>
struct EmbedArgs {
    const Id *ids;
    const In *table;
    Out *out;
    int64_t n, ld_table, ld_out;
    int64_t table_rows;
    int32_t dim, lanes_log2;
    float scale;
};

// 2^lanes_log2 threads of a block take a row, VEC elements each; the last vector of a row is moved back to end with it
// (what it shares with its neighbour is written twice, with the same bits)
template <typename In, typename Out, typename Id, int VEC, int U>
__global__ __launch_bounds__(kThreads) void embed_kernel(const EmbedArgs<In, Out, Id> p)
{
    const int lanes = 1 << p.lanes_log2, rows_per_block = kThreads >> p.lanes_log2;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * rows_per_block * U + (threadIdx.x >> p.lanes_log2);
    const In *src[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t row = row0 + static_cast<int64_t>(u) * rows_per_block;
        const int64_t id = row < p.n ? static_cast<int64_t>(p.ids[row]) : -1;
        src[u] = id >= 0 && id < p.table_rows ? p.table + id * p.ld_table : nullptr;
    }
    for (int64_t c = (static_cast<int64_t>(blockIdx.y) << p.lanes_log2) + (threadIdx.x & (lanes - 1)); c * VEC < p.dim; c += static_cast<int64_t>(gridDim.y) << p.lanes_log2) {
        const int64_t col = c * VEC + VEC <= p.dim ? c * VEC : p.dim - VEC;
        float v[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (src[u]) {
                load_n<VEC>(src[u] + col, v[u]);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[u][e] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row0 + static_cast<int64_t>(u) * rows_per_block;
            if (row >= p.n) continue;
            if (src[u]) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[u][e] *= p.scale;
            }
            store_n<VEC>(p.out + row * p.ld_out + col, v[u]);
        }
    }
}

template <typename In, typename Out, typename Id>
hipError_t embed_typed(int64_t n, const void *ids, int64_t table_rows, const void *table, int32_t dim, int64_t ld_table, float scale, void *out, int64_t ld_out,
                       hipStream_t stream)
{
    constexpr int VEC = sizeof(In) == 4 && sizeof(Out) == 4 ? 4 : 8;
    const int64_t vecs = dim < VEC ? dim : ceil_div(dim, VEC);
    int lanes_log2 = ceil_log2(vecs);
    if (lanes_log2 > 8) lanes_log2 = 8;
    const EmbedArgs<In, Out, Id> p{static_cast<const Id *>(ids), static_cast<const In *>(table), static_cast<Out *>(out), n, ld_table, ld_out, table_rows, dim,
                                   lanes_log2, scale};
    const int64_t slabs = ceil_div(vecs, static_cast<int64_t>(1) << lanes_log2);
    const int64_t rows_per_block = kThreads >> lanes_log2;
    const bool four = n / rows_per_block >= 4096;           // blocks enough for the chip at four rows per thread
    const dim3 grid(static_cast<unsigned>(ceil_div(n, rows_per_block * (four ? 4 : 1))), static_cast<unsigned>(slabs < 1024 ? slabs : 1024));
    if (dim < VEC) {
        hipLaunchKernelGGL((embed_kernel<In, Out, Id, 1, 1>), dim3(static_cast<unsigned>(ceil_div(n, rows_per_block)), grid.y), dim3(kThreads), 0, stream, p);
    } else if (four) {
        hipLaunchKernelGGL((embed_kernel<In, Out, Id, VEC, 4>), grid, dim3(kThreads), 0, stream, p);
    } else {
        hipLaunchKernelGGL((embed_kernel<In, Out, Id, VEC, 1>), grid, dim3(kThreads), 0, stream, p);
    }
    return hipGetLastError();
}

// ---- the ids in order ----------------------------------------------------------------------------------------
// A stable radix sort of (id, position), least significant digit first; an id outside the table has the key table_rows,
// behind all others.  Per digit: counts per block, their prefix sums over the blocks, and the scatter.
constexpr int kDigitBits = 8, kBins = 1 << kDigitBits;
constexpr int kPerThread = 16, kTile = kThreads * kPerThread;

struct SortArgs {
    const void *ids;                    // of the first pass
    const uint32_t *key_in, *pos_in;    // of the others
    uint32_t *key_out, *pos_out;
    uint32_t *count;                    // [kBins x tiles]: per digit and block, then its exclusive prefix over the blocks
    uint32_t *total;                    // [kBins]
    int64_t n, table_rows;
    int32_t tiles, shift, bits;
};

template <typename Id, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortArgs &p, int64_t i)
{
    if constexpr (FIRST) {
        const int64_t id = static_cast<const Id *>(p.ids)[i];
        return id >= 0 && id < p.table_rows ? static_cast<uint32_t>(id) : static_cast<uint32_t>(p.table_rows);
    } else {
        return p.key_in[i];
    }
}

template <typename Id, bool FIRST>
__global__ __launch_bounds__(kThreads) void sort_count_kernel(const SortArgs p)
{
    __shared__ uint32_t bins[kBins];
    bins[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kTile;
#pragma unroll 4
    for (int r = 0; r < kPerThread; ++r) {
        const int64_t i = first + r * kThreads + threadIdx.x;
        if (i < p.n) atomicAdd(&bins[(sort_key<Id, FIRST>(p, i) >> p.shift) & ((1u << p.bits) - 1)], 1u);
    }
    __syncthreads();
    p.count[static_cast<int64_t>(threadIdx.x) * p.tiles + blockIdx.x] = bins[threadIdx.x];
}

// a block per digit: counts of the blocks -> exclusive prefix sums
__global__ __launch_bounds__(kThreads) void sort_scan_kernel(const SortArgs p)
{
    __shared__ uint32_t part[kThreads / kWave];
    uint32_t *row = p.count + static_cast<int64_t>(blockIdx.x) * p.tiles;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t before = 0;
    for (int base = 0; base < p.tiles; base += kThreads) {
        const int t = base + threadIdx.x;
        const uint32_t c = t < p.tiles ? row[t] : 0u;
        uint32_t incl = c;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const uint32_t o = __shfl_up(incl, off);
            if (lane >= off) incl += o;
        }
        if (lane == 63) part[wave] = incl;
        __syncthreads();
        uint32_t prev = before, all = 0;
#pragma unroll
        for (int w = 0; w < kThreads / kWave; ++w) {
            if (w < wave) prev += part[w];
            all += part[w];
        }
        if (t < p.tiles) row[t] = prev + incl - c;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) p.total[blockIdx.x] = before;
}

// Wave w of a block takes a quarter of its keys in order, 64 at a time; the place of a key is the digit's start + the keys of
// the digit in earlier blocks + in earlier waves + in earlier steps of the wave + in earlier lanes of the step.
template <typename Id, bool FIRST>
__global__ __launch_bounds__(kThreads) void sort_scatter_kernel(const SortArgs p)
{
    constexpr int kWaves = kThreads / kWave;
    __shared__ uint32_t seen[kWaves][kBins];
    __shared__ uint32_t part[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) seen[w][threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kTile + wave * (kTile / kWaves) + lane;
    uint32_t key[kPerThread], rank[kPerThread];
#pragma unroll
    for (int r = 0; r < kPerThread; ++r) {
        const int64_t i = first + r * kWave;
        key[r] = i < p.n ? sort_key<Id, FIRST>(p, i) : 0u;
    }
#pragma unroll
    for (int r = 0; r < kPerThread; ++r) {
        const bool there = first + r * kWave < p.n;
        const uint32_t digit = (key[r] >> p.shift) & ((1u << p.bits) - 1);
        uint64_t peers = __ballot(there);
        for (int b = 0; b < p.bits; ++b) {
            const bool set = (digit >> b) & 1u;
            const uint64_t with = __ballot(set);
            peers &= set ? with : ~with;
        }
        const int leader = there ? __ffsll(static_cast<unsigned long long>(peers)) - 1 : lane;
        uint32_t old = 0;
        if (there && lane == leader) old = atomicAdd(&seen[wave][digit], static_cast<uint32_t>(__popcll(peers)));
        old = __shfl(old, leader);
        rank[r] = old + static_cast<uint32_t>(__popcll(peers & ((1ull << lane) - 1)));
    }
    __syncthreads();
    // thread t holds digit t: where its keys of each wave begin
    {
        const uint32_t mine = p.total[threadIdx.x];
        uint32_t incl = mine;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const uint32_t o = __shfl_up(incl, off);
            if (lane >= off) incl += o;
        }
        if (lane == 63) part[wave] = incl;
        __syncthreads();
        uint32_t start = incl - mine + p.count[static_cast<int64_t>(threadIdx.x) * p.tiles + blockIdx.x];
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            if (w < wave) start += part[w];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = seen[w][threadIdx.x];
            seen[w][threadIdx.x] = start;
            start += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kPerThread; ++r) {
        const int64_t i = first + r * kWave;
        if (i >= p.n) continue;
        const uint32_t to = seen[wave][(key[r] >> p.shift) & ((1u << p.bits) - 1)] + rank[r];
        p.key_out[to] = key[r];
        p.pos_out[to] = FIRST ? static_cast<uint32_t>(i) : p.pos_in[i];
    }
}

struct SortPlan {
    int passes, bits;
    int64_t tiles;
    size_t key0, pos0, key1, pos1, count, total, bytes;     // offsets in the workspace
};

SortPlan plan_sort(int64_t n, int64_t table_rows)
{
    SortPlan s;
    const int bits = ceil_log2(table_rows + 1) < 1 ? 1 : ceil_log2(table_rows + 1);
    s.passes = static_cast<int>(ceil_div(bits, kDigitBits));
    s.bits = static_cast<int>(ceil_div(bits, s.passes));
    s.tiles = ceil_div(n, kTile);
    const size_t list = round_up(static_cast<size_t>(n) * 4, 256);
    s.key0 = 0; s.pos0 = list; s.key1 = 2 * list; s.pos1 = 3 * list; s.count = 4 * list;
    s.total = s.count + round_up(static_cast<size_t>(s.tiles) * kBins * 4, 256);
    s.bytes = s.total + kBins * 4;
    return s;
}

template <typename Id>
hipError_t sort_ids(const SortPlan &s, int64_t n, const void *ids, int64_t table_rows, char *ws, const uint32_t **keys, const uint32_t **pos, hipStream_t stream)
{
    uint32_t *key[2] = {reinterpret_cast<uint32_t *>(ws + s.key0), reinterpret_cast<uint32_t *>(ws + s.key1)};
    uint32_t *at[2] = {reinterpret_cast<uint32_t *>(ws + s.pos0), reinterpret_cast<uint32_t *>(ws + s.pos1)};
    SortArgs p{};
    p.ids = ids; p.n = n; p.table_rows = table_rows; p.tiles = static_cast<int32_t>(s.tiles); p.bits = s.bits;
    p.count = reinterpret_cast<uint32_t *>(ws + s.count);
    p.total = reinterpret_cast<uint32_t *>(ws + s.total);
    const dim3 grid(static_cast<unsigned>(s.tiles)), block(kThreads);
    for (int pass = 0; pass < s.passes; ++pass) {
        p.shift = pass * s.bits;
        p.key_in = key[(pass + 1) & 1]; p.pos_in = at[(pass + 1) & 1];
        p.key_out = key[pass & 1]; p.pos_out = at[pass & 1];
        if (pass == 0) hipLaunchKernelGGL((sort_count_kernel<Id, true>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((sort_count_kernel<Id, false>), grid, block, 0, stream, p);
        hipLaunchKernelGGL(sort_scan_kernel, dim3(kBins), block, 0, stream, p);
        if (pass == 0) hipLaunchKernelGGL((sort_scatter_kernel<Id, true>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((sort_scatter_kernel<Id, false>), grid, block, 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    *keys = key[(s.passes - 1) & 1];
    *pos = at[(s.passes - 1) & 1];
    return hipSuccess;
}

// ---- grad_table[v] = scale * the sum of the rows of id v -----------------------------------------------------
template <typename In, typename Out>
struct SumArgs {
    const uint32_t *keys, *pos;
    const In *grad;
    Out *out;
    int64_t n, table_rows, ld_grad, ld_out;
    int32_t dim;
    float scale;
    int32_t accumulate;
};

__device__ __forceinline__ int64_t lower_bound(const uint32_t *a, int64_t n, uint32_t v)
{
    int64_t lo = 0;
    while (n > 0) {
        const int64_t half = n >> 1;
        if (a[lo + half] < v) { lo += half + 1; n -= half + 1; }
        else n = half;
    }
    return lo;
}

// a wavefront per table row and slab of 64 * VEC columns
template <typename In, typename Out, int VEC>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(const SumArgs<In, Out> p)
{
    const int lane = threadIdx.x & 63;
    const int64_t v = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + (threadIdx.x >> 6);
    if (v >= p.table_rows) return;
    const int64_t beg = lower_bound(p.keys, p.n, static_cast<uint32_t>(v)), end = beg + lower_bound(p.keys + beg, p.n - beg, static_cast<uint32_t>(v + 1));
    if (beg == end && p.accumulate) return;
    for (int64_t c = (static_cast<int64_t>(blockIdx.y) * kWave + lane) * VEC; c < p.dim; c += static_cast<int64_t>(gridDim.y) * kWave * VEC) {
        float sum[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
        const bool whole = c + VEC <= p.dim;
        for (int64_t i = beg; i < end; ++i) {
            const In *g = p.grad + static_cast<int64_t>(p.pos[i]) * p.ld_grad + c;
            if (whole) {
                float x[VEC];
                load_n<VEC>(g, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += x[e];
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e < p.dim) sum[e] += to_f32(g[e]);
            }
        }
        Out *o = p.out + v * p.ld_out + c;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (c + e < p.dim) from_f32((p.accumulate ? to_f32(o[e]) : 0.f) + p.scale * sum[e], o[e]);
    }
}

template <typename In, typename Out>
hipError_t embed_sum(const uint32_t *keys, const uint32_t *pos, int64_t n, int64_t table_rows, const void *grad, int32_t dim, int64_t ld_grad, float scale,
                     bool accumulate, void *out, int64_t ld_out, hipStream_t stream)
{
    constexpr int VEC = 4;
    const SumArgs<In, Out> p{keys, pos, static_cast<const In *>(grad), static_cast<Out *>(out), n, table_rows, ld_grad, ld_out, dim, scale, accumulate};
    const int64_t slabs = ceil_div(dim, kWave * VEC);
    hipLaunchKernelGGL((embed_sum_kernel<In, Out, VEC>), dim3(static_cast<unsigned>(ceil_div(table_rows, kThreads / kWave)), static_cast<unsigned>(slabs < 1024 ? slabs : 1024)),
                       dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

mgg_status_t launch_embed(int64_t n, mgg_index_t id_type, const void *ids, int64_t table_rows, mgg_dtype_t table_dtype, const void *table, int32_t dim,
                          int64_t ld_table, float scale, mgg_dtype_t out_dtype, void *out, int64_t ld_out, hipStream_t stream)
{
    if (n > static_cast<int64_t>(INT32_MAX)) return fail(MGG_ERR_UNSUPPORTED, "%lld ids", (long long)n);
    hipError_t e;
#define MGG_EMBED(IN, OUT)                                                                                                              \
    e = id_type == MGG_I64 ? embed_typed<IN, OUT, int64_t>(n, ids, table_rows, table, dim, ld_table, scale, out, ld_out, stream)         \
                           : embed_typed<IN, OUT, int32_t>(n, ids, table_rows, table, dim, ld_table, scale, out, ld_out, stream)
    if (table_dtype == MGG_BF16) { if (out_dtype == MGG_BF16) MGG_EMBED(Bf16, Bf16); else MGG_EMBED(Bf16, float); }
    else { if (out_dtype == MGG_BF16) MGG_EMBED(float, Bf16); else MGG_EMBED(float, float); }
#undef MGG_EMBED
    return e == hipSuccess ? MGG_OK : hip_fail(e, "lookup kernel launch");
}

size_t embed_grad_workspace(int64_t n, int64_t table_rows, int32_t dim) { return round_up(plan_sort(n, table_rows).bytes, 256); }

mgg_status_t launch_embed_grad(int64_t n, mgg_index_t id_type, const void *ids, int64_t table_rows, mgg_dtype_t grad_dtype, const void *grad, int32_t dim,
                               int64_t ld_grad, float scale, bool accumulate, mgg_dtype_t out_dtype, void *out, int64_t ld_out, void *workspace,
                               hipStream_t stream)
{
    const SortPlan s = plan_sort(n, table_rows);
    const uint32_t *keys = nullptr, *pos = nullptr;
    hipError_t e = hipSuccess;
    if (n > 0) {
        e = id_type == MGG_I64 ? sort_ids<int64_t>(s, n, ids, table_rows, static_cast<char *>(workspace), &keys, &pos, stream)
                               : sort_ids<int32_t>(s, n, ids, table_rows, static_cast<char *>(workspace), &keys, &pos, stream);
        if (e != hipSuccess) return hip_fail(e, "sort kernel launch");
    }
#define MGG_SUM(IN, OUT) e = embed_sum<IN, OUT>(keys, pos, n, table_rows, grad, dim, ld_grad, scale, accumulate, out, ld_out, stream)
    if (grad_dtype == MGG_BF16) { if (out_dtype == MGG_BF16) MGG_SUM(Bf16, Bf16); else MGG_SUM(Bf16, float); }
    else { if (out_dtype == MGG_BF16) MGG_SUM(float, Bf16); else MGG_SUM(float, float); }
#undef MGG_SUM
    return e == hipSuccess ? MGG_OK : hip_fail(e, "table gradient kernel launch");
}

}  // namespace mgg
