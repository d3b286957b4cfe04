// Lookup of scaled table rows by ids on the device, and the gradient of the table by sorted ids.
#include "train_common.h"

namespace mgg {

namespace {

using namespace train;

constexpr int kThreads = 256;

// ---- out[i] = scale * table[ids[i]] --------------------------------------------------------------------------
// A copy of rows: bound by HBM (the distinct rows read, all rows written).  64 k rows of 4 KB: 77 - 79 us, 347 MB at 4.4 - 4.5 TB/s; a large
// copy reaches 5.1.
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
mgg_status_t embed_typed(int64_t n, const void *ids, int64_t table_rows, const void *table, int32_t dim, int64_t ld_table, float scale, void *out, int64_t ld_out,
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
    const bool four = dim >= VEC && n / rows_per_block >= 4096;         // blocks enough for the chip at four rows per thread
    const int64_t blocks = ceil_div(n, rows_per_block * (four ? 4 : 1));
    if (!launchable(blocks, kThreads)) return fail(MGG_ERR_UNSUPPORTED, "%lld ids of %d columns need too many threads for one launch", (long long)n, dim);
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(slabs < 1024 ? slabs : 1024));
    if (dim < VEC) {
        hipLaunchKernelGGL((embed_kernel<In, Out, Id, 1, 1>), grid, dim3(kThreads), 0, stream, p);
    } else if (four) {
        hipLaunchKernelGGL((embed_kernel<In, Out, Id, VEC, 4>), grid, dim3(kThreads), 0, stream, p);
    } else {
        hipLaunchKernelGGL((embed_kernel<In, Out, Id, VEC, 1>), grid, dim3(kThreads), 0, stream, p);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, "lookup kernel launch");
}

// ---- the ids in order ----------------------------------------------------------------------------------------
// A stable radix sort of (id, position), least significant digit first; an id outside the table has the key table_rows,
// behind all others.  The work is small beside the sums (8 bytes an id), so what counts is the number of launches: up to
// kSmall ids one block sorts them in LDS (2 k ids of 13 bits: 10 us); beyond, a digit takes two launches (counts per block; the scatter, whose blocks add up
// the counts of the blocks before them), three where there are more blocks than that pays for.
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kPerThread = 8, kTile = kThreads * kPerThread;
constexpr int kScanTiles = 256;                     // up to so many blocks the scatter adds up their counts itself
constexpr int kSmallThreads = 1024, kSmallBits = 8, kSmall = kSmallThreads * 8;

struct SortArgs {
    const void *ids;                    // of the first pass
    const uint32_t *key_in, *pos_in;    // of the others
    uint32_t *key_out, *pos_out;
    uint32_t *count;                    // [tiles x kBins]: per block and digit, then, after the scan, those of the blocks before
    uint32_t *total;                    // [kBins], written by the scan
    int64_t n, table_rows;
    int32_t tiles, shift, bits, passes;
};

template <typename Id>
__device__ __forceinline__ uint32_t id_key(const SortArgs &p, int64_t i)
{
    const int64_t id = static_cast<const Id *>(p.ids)[i];
    return id >= 0 && id < p.table_rows ? static_cast<uint32_t>(id) : static_cast<uint32_t>(p.table_rows);
}
template <typename Id, bool FIRST>
__device__ __forceinline__ uint32_t sort_key(const SortArgs &p, int64_t i)
{
    if constexpr (FIRST) return id_key<Id>(p, i);
    else return p.key_in[i];
}

// The rank of this lane's key among those of its wavefront with the same digit: those of earlier steps, counted in
// `seen`, and of earlier lanes.
__device__ __forceinline__ uint32_t wave_rank(uint32_t *seen, uint32_t digit, int bits, bool there, int lane)
{
    uint64_t peers = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const bool set = (digit >> b) & 1u;
        const uint64_t with = __ballot(set);
        peers &= set ? with : ~with;
    }
    const int leader = there ? __ffsll(static_cast<unsigned long long>(peers)) - 1 : lane;
    uint32_t old = 0;
    if (there && lane == leader) old = atomicAdd(&seen[digit], static_cast<uint32_t>(__popcll(peers)));
    old = __shfl(old, leader);
    return old + static_cast<uint32_t>(__popcll(peers & ((1ull << lane) - 1)));
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t v, int lane)
{
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const uint32_t o = __shfl_up(v, off);
        if (lane >= off) v += o;
    }
    return v;
}

// exclusive prefix sums of one value per thread; part: a word per wavefront
template <int THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t incl = wave_scan(v, lane);
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    uint32_t before = incl - v;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w)
        if (w < wave) before += part[w];
    return before;
}

template <typename Id>
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(const SortArgs p)
{
    constexpr int kWaves = kSmallThreads / kWave, kB = 1 << kSmallBits;
    __shared__ uint32_t key_at[kSmall], pos_at[kSmall];
    __shared__ uint32_t seen[kWaves][kB];
    __shared__ uint32_t part[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = static_cast<int>(p.n);
    const int steps = (n + kSmallThreads - 1) / kSmallThreads;          // of a wavefront: it takes steps * 64 keys in a row
    const int first = wave * steps * kWave + lane;
    uint32_t key[8], pos[8], rank[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int i = first + r * kWave;
        if (r < steps && i < n) { key[r] = id_key<Id>(p, i); pos[r] = static_cast<uint32_t>(i); }
    }
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * p.bits;
        const uint32_t mask = (1u << p.bits) - 1;
        for (int b = threadIdx.x; b < kWaves * kB; b += kSmallThreads) seen[b / kB][b % kB] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < steps) rank[r] = wave_rank(seen[wave], (key[r] >> shift) & mask, p.bits, first + r * kWave < n, lane);
        __syncthreads();
        uint32_t sum = 0;
        if (threadIdx.x < kB) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum += seen[w][threadIdx.x];
        }
        uint32_t start = block_scan<kSmallThreads>(sum, part);
        if (threadIdx.x < kB) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t c = seen[w][threadIdx.x];
                seen[w][threadIdx.x] = start;
                start += c;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < steps && first + r * kWave < n) {
                const uint32_t to = seen[wave][(key[r] >> shift) & mask] + rank[r];
                key_at[to] = key[r];
                pos_at[to] = pos[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const int i = first + r * kWave;
            if (r < steps && i < n) { key[r] = key_at[i]; pos[r] = pos_at[i]; }
        }
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int i = first + r * kWave;
        if (r < steps && i < n) { p.key_out[i] = key[r]; p.pos_out[i] = pos[r]; }
    }
}

template <typename Id, bool FIRST>
__global__ __launch_bounds__(kThreads) void sort_count_kernel(const SortArgs p)
{
    __shared__ uint32_t bins[kBins];
    for (int b = threadIdx.x; b < kBins; b += kThreads) bins[b] = 0;
    __syncthreads();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kTile;
#pragma unroll
    for (int r = 0; r < kPerThread; ++r) {
        const int64_t i = first + r * kThreads + threadIdx.x;
        if (i < p.n) atomicAdd(&bins[(sort_key<Id, FIRST>(p, i) >> p.shift) & ((1u << p.bits) - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads) p.count[static_cast<int64_t>(blockIdx.x) * kBins + b] = bins[b];
}

// counts of the blocks -> those of the blocks before: a thread per digit, wavefront w taking a quarter of the blocks
__global__ __launch_bounds__(kThreads) void sort_scan_kernel(const SortArgs p)
{
    constexpr int kWaves = kThreads / kWave;
    __shared__ uint32_t part[kWaves][kWave];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.x * kWave + lane;
    const int share = (p.tiles + kWaves - 1) / kWaves, from = wave * share, to = from + share < p.tiles ? from + share : p.tiles;
    uint32_t sum = 0;
#pragma unroll 8
    for (int t = from; t < to; ++t) sum += p.count[static_cast<int64_t>(t) * kBins + b];
    part[wave][lane] = sum;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (w < wave) before += part[w][lane];
    for (int t = from; t < to; ++t) {
        uint32_t *c = p.count + static_cast<int64_t>(t) * kBins + b;
        const uint32_t mine = *c;
        *c = before;
        before += mine;
    }
    if (wave == kWaves - 1) p.total[b] = before;
}

// Wave w of a block takes a quarter of its keys in order, 64 at a time; the place of a key is the digit's start + the keys of
// the digit in earlier blocks + in earlier waves + in earlier steps of the wave + in earlier lanes of the step.
template <typename Id, bool FIRST, bool SCANNED>
__global__ __launch_bounds__(kThreads) void sort_scatter_kernel(const SortArgs p)
{
    constexpr int kWaves = kThreads / kWave, kPer = kBins / kThreads;
    __shared__ uint32_t seen[kWaves][kBins];
    __shared__ uint32_t part[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t mask = (1u << p.bits) - 1;
    for (int b = threadIdx.x; b < kWaves * kBins; b += kThreads) seen[b / kBins][b % kBins] = 0;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kTile + wave * (kTile / kWaves) + lane;
    uint32_t key[kPerThread], rank[kPerThread];
#pragma unroll
    for (int r = 0; r < kPerThread; ++r) {
        const int64_t i = first + r * kWave;
        key[r] = i < p.n ? sort_key<Id, FIRST>(p, i) : 0u;
    }
    // thread t holds digits kPer t .. kPer t + kPer - 1: all their keys, and those of the blocks before
    uint32_t before[kPer], total[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const int b = threadIdx.x * kPer + e;
        if constexpr (SCANNED) {
            before[e] = p.count[static_cast<int64_t>(blockIdx.x) * kBins + b];
            total[e] = p.total[b];
        } else {
            before[e] = total[e] = 0;
        }
    }
    if constexpr (!SCANNED) {
#pragma unroll 8
        for (int t = 0; t < p.tiles; ++t) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const uint32_t c = p.count[static_cast<int64_t>(t) * kBins + threadIdx.x * kPer + e];
                total[e] += c;
                before[e] += t < static_cast<int>(blockIdx.x) ? c : 0u;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kPerThread; ++r) rank[r] = wave_rank(seen[wave], (key[r] >> p.shift) & mask, p.bits, first + r * kWave < p.n, lane);
    __syncthreads();
    uint32_t mine = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) mine += total[e];
    uint32_t at = block_scan<kThreads>(mine, part);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        uint32_t start = at + before[e];
        at += total[e];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = seen[w][threadIdx.x * kPer + e];
            seen[w][threadIdx.x * kPer + e] = start;
            start += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kPerThread; ++r) {
        const int64_t i = first + r * kWave;
        if (i >= p.n) continue;
        const uint32_t to = seen[wave][(key[r] >> p.shift) & mask] + rank[r];
        p.key_out[to] = key[r];
        p.pos_out[to] = FIRST ? static_cast<uint32_t>(i) : p.pos_in[i];
    }
}

// ---- grad_table[v] = scale * the sum of the rows of id v -----------------------------------------------------
// The sorted positions are cut into chunks of equal length, whatever the ids, so that a token that makes up a tenth of the batch
// costs no more than others.  A chunk's rows are added up id by id; a sum that began and ended inside the chunk is a
// finished row, one that reaches over its border goes to the workspace (slot 0 of the chunk: it began before; slot 1: it goes on), and
// embed_join_kernel adds those up chunk by chunk.  Bound by HBM: the rows of grad_out read once, grad_table written once.  32 k ids over
// 128 k rows of 2048, bf16 to fp32: the sums and zeros 185 - 220 us (1.17 GB at 5.3 - 6.3 TB/s), the sort 30, the join 12.  1 M ids over
// 100 k rows of 64 fp32: 65, the sort 87 (40 of them its two scans), the join 20, where bytes allow 53 in all.  Stores that pass the caches by took
// 14 % longer in all (277 to 317 us, before the zeros went in larger shares).
constexpr int chunk_of(int64_t n) { return n <= 4096 ? 8 : (n <= 16384 ? 16 : (n <= 262144 ? 32 : 64)); }     // enough chunks for the chip, few partial sums

struct EmbedGradPlan {
    bool small;
    int passes, bits;
    int64_t tiles, chunks;
    int chunk;
    int64_t ld_part;
    size_t key0, pos0, key1, pos1, count, total, part, bytes;     // offsets in the workspace
};

EmbedGradPlan plan_embed_grad(int64_t n, int64_t table_rows, int32_t dim)
{
    EmbedGradPlan s;
    const int bits = ceil_log2(table_rows + 1) < 1 ? 1 : ceil_log2(table_rows + 1);
    s.small = n <= kSmall;
    s.passes = static_cast<int>(ceil_div(bits, s.small ? kSmallBits : kDigitBits));
    s.bits = static_cast<int>(ceil_div(bits, s.passes));
    s.tiles = ceil_div(n, kTile);
    s.chunk = chunk_of(n);
    s.chunks = ceil_div(n, s.chunk);
    s.ld_part = static_cast<int64_t>(round_up(static_cast<size_t>(dim), 8));
    const size_t list = round_up(static_cast<size_t>(n) * 4, 256);
    s.key0 = 0; s.pos0 = list; s.key1 = 2 * list; s.pos1 = 3 * list;
    s.count = s.small ? 2 * list : 4 * list;
    s.total = s.count + (s.small ? 0 : static_cast<size_t>(s.tiles) * kBins * 4);
    s.part = s.total + (s.small ? 0 : kBins * 4);
    s.bytes = s.part + static_cast<size_t>(s.chunks) * 2 * s.ld_part * 4 + 256;
    return s;
}

template <typename Id>
hipError_t sort_ids(const EmbedGradPlan &s, int64_t n, const void *ids, int64_t table_rows, char *ws, const uint32_t **keys, const uint32_t **pos, hipStream_t stream)
{
    uint32_t *key[2] = {reinterpret_cast<uint32_t *>(ws + s.key0), reinterpret_cast<uint32_t *>(ws + s.key1)};
    uint32_t *at[2] = {reinterpret_cast<uint32_t *>(ws + s.pos0), reinterpret_cast<uint32_t *>(ws + s.pos1)};
    SortArgs p{};
    p.ids = ids; p.n = n; p.table_rows = table_rows; p.tiles = static_cast<int32_t>(s.tiles); p.bits = s.bits; p.passes = s.passes;
    if (s.small) {
        p.key_out = key[0]; p.pos_out = at[0];
        *keys = key[0]; *pos = at[0];
        hipLaunchKernelGGL((sort_small_kernel<Id>), dim3(1), dim3(kSmallThreads), 0, stream, p);
        return hipGetLastError();
    }
    p.count = reinterpret_cast<uint32_t *>(ws + s.count);
    p.total = reinterpret_cast<uint32_t *>(ws + s.total);
    const dim3 grid(static_cast<unsigned>(s.tiles)), block(kThreads);
    for (int pass = 0; pass < s.passes; ++pass) {
        p.shift = pass * s.bits;
        p.key_in = key[(pass + 1) & 1]; p.pos_in = at[(pass + 1) & 1];
        p.key_out = key[pass & 1]; p.pos_out = at[pass & 1];
        if (pass == 0) hipLaunchKernelGGL((sort_count_kernel<Id, true>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((sort_count_kernel<Id, false>), grid, block, 0, stream, p);
        if (s.tiles > kScanTiles) {
            hipLaunchKernelGGL(sort_scan_kernel, dim3(kBins / kWave), block, 0, stream, p);
            if (pass == 0) hipLaunchKernelGGL((sort_scatter_kernel<Id, true, true>), grid, block, 0, stream, p);
            else hipLaunchKernelGGL((sort_scatter_kernel<Id, false, true>), grid, block, 0, stream, p);
        } else {
            if (pass == 0) hipLaunchKernelGGL((sort_scatter_kernel<Id, true, false>), grid, block, 0, stream, p);
            else hipLaunchKernelGGL((sort_scatter_kernel<Id, false, false>), grid, block, 0, stream, p);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    *keys = key[(s.passes - 1) & 1];
    *pos = at[(s.passes - 1) & 1];
    return hipSuccess;
}

template <typename In, typename Out>
struct SumArgs {
    const uint32_t *keys, *pos;
    const In *grad;
    Out *out;
    float *part;
    int64_t n, table_rows, ld_grad, ld_out, ld_part, sum_blocks;
    int32_t dim, chunk, chunks, lanes_log2, slabs, fill_rows;
    float scale;
    int32_t accumulate;
};

// the first place in sorted a[lo, hi) whose key is not below v, by a wavefront: 64 places at a time, so that a list of 2^18 takes three loads one after the other
__device__ __forceinline__ int64_t wave_lower_bound(const uint32_t *a, int64_t lo, int64_t hi, uint32_t v, int lane)
{
    while (hi - lo > kWave) {
        const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
        const int below = __popcll(__ballot(at < hi && a[at] < v));
        if (below == 0) return lo;
        hi = lo + below * step < hi ? lo + below * step : hi;
        lo += (below - 1) * step + 1;
    }
    return lo + __popcll(__ballot(lo + lane < hi && a[lo + lane] < v));
}

// which of the `count` (up to 64) ids from `first` on the sorted list has: a bit each.  A step passes 64 keys, or all of the last one's kind.
__device__ __forceinline__ uint64_t ids_present(const uint32_t *keys, int64_t n, uint32_t first, uint32_t count, int lane)
{
    uint64_t present = 0;
    int64_t at = wave_lower_bound(keys, 0, n, first, lane);
    while (at < n) {
        const uint32_t key = at + lane < n ? keys[at + lane] : 0xffffffffu;
        const bool mine = key - first < count;
        uint64_t bit = mine ? 1ull << (key - first) : 0ull;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) bit |= __shfl_xor(bit, off);
        present |= bit;
        const uint32_t last = __builtin_amdgcn_readlane(key, 63);
        if (last - first >= count) break;
        at = wave_lower_bound(keys, at + kWave, n, last + 1, lane);
    }
    return present;
}

// columns [c, c + VEC) of a finished row; with the last vector moved back to `col` the columns before c are the neighbour's
template <typename In, typename Out, int VEC>
__device__ __forceinline__ void put_row(const SumArgs<In, Out> &p, uint32_t row, int64_t c, int64_t col, const float (&sum)[VEC])
{
    Out *o = p.out + static_cast<int64_t>(row) * p.ld_out;
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = p.scale * sum[e];
    if (c == col) {
        if (p.accumulate) {
            float old[VEC];
            load_n<VEC>(o + c, old);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] += old[e];
        }
        store_n<VEC>(o + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (col + e >= c) from_f32(v[e] + (p.accumulate ? to_f32(o[col + e]) : 0.f), o[col + e]);
    }
}

// Blocks up to sum_blocks: 2^lanes_log2 lanes per chunk (and slab of columns).  The others write zeros to the rows that no id names.
template <typename In, typename Out, int VEC>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(const SumArgs<In, Out> p)
{
    const int lanes = 1 << p.lanes_log2;
    if (static_cast<int64_t>(blockIdx.x) >= p.sum_blocks) {
        const int lane = threadIdx.x & 63;
        const int64_t row0 = ((static_cast<int64_t>(blockIdx.x) - p.sum_blocks) * (kThreads / kWave) + (threadIdx.x >> 6)) * p.fill_rows;
        if (row0 >= p.table_rows) return;
        const int count = static_cast<int>(min(p.table_rows - row0, static_cast<int64_t>(p.fill_rows)));
        const uint64_t rows = ~ids_present(p.keys, p.n, static_cast<uint32_t>(row0), count, lane);
        constexpr int VO = VEC == 1 ? 1 : 16 / static_cast<int>(sizeof(Out));
        const float zero[VO] = {};
        for (int r = lane >> p.lanes_log2; r < count; r += kWave >> p.lanes_log2)
            if ((rows >> r) & 1)
                for (int64_t c = (lane & (lanes - 1)) * VO; c < p.dim; c += lanes * VO)
                    store_n<VO>(p.out + (row0 + r) * p.ld_out + (c + VO <= p.dim ? c : p.dim - VO), zero);
        return;
    }
    constexpr int U = 8;
    const int64_t group = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> p.lanes_log2;
    const int64_t chunk = group / p.slabs;
    const int64_t c = (((group % p.slabs) << p.lanes_log2) + (threadIdx.x & (lanes - 1))) * VEC;
    if (chunk >= p.chunks || c >= p.dim) return;
    const int64_t col = c + VEC <= p.dim ? c : p.dim - VEC;
    const int64_t beg = chunk * p.chunk, end = beg + p.chunk < p.n ? beg + p.chunk : p.n;
    const uint32_t none = static_cast<uint32_t>(p.table_rows);
    uint32_t cur = p.keys[beg];
    bool head = beg > 0 && p.keys[beg - 1] == cur;
    float sum[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
    auto finish = [&](bool tail) {
        if (cur != none) {
            if (head || tail) store_n<VEC>(p.part + (2 * chunk + (head ? 0 : 1)) * p.ld_part + c, sum);
            else put_row<In, Out, VEC>(p, cur, c, col, sum);
        }
        head = false;
    };
    for (int64_t i = beg; i < end; i += U) {
        uint32_t key[U], pos[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            key[u] = i + u < end ? p.keys[i + u] : none;
            pos[u] = i + u < end ? p.pos[i + u] : 0u;
        }
        float x[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (key[u] != none) {
                load_n<VEC>(p.grad + static_cast<int64_t>(pos[u]) * p.ld_grad + col, x[u]);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[u][e] = 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u < end && key[u] != cur) {
                finish(false);
                cur = key[u];
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += x[u][e];
        }
    }
    finish(end < p.n && p.keys[end] == cur);
}

// The sums that reach over a chunk's end: a block per chunk and slab in which one begins.  Its groups of lanes add up equal shares of
// the partial sums, which then meet in LDS, in order.
template <typename In, typename Out, int VEC>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(const SumArgs<In, Out> p)
{
    __shared__ float joined[kThreads * VEC];
    const int64_t chunk = blockIdx.x / p.slabs, beg = chunk * p.chunk, end = beg + p.chunk;
    if (end >= p.n) return;
    const uint32_t id = p.keys[end - 1];
    if (id != p.keys[end] || id == static_cast<uint32_t>(p.table_rows)) return;
    if (p.keys[beg] == id && beg > 0 && p.keys[beg - 1] == id) return;              // it began in an earlier one
    const int64_t last = (wave_lower_bound(p.keys, end, p.n, id + 1, threadIdx.x & 63) - 1) / p.chunk;
    const int lanes = 1 << p.lanes_log2, groups = kThreads >> p.lanes_log2, group = threadIdx.x >> p.lanes_log2;
    const int64_t c = (static_cast<int64_t>((blockIdx.x % p.slabs) << p.lanes_log2) + (threadIdx.x & (lanes - 1))) * VEC;
    const int64_t count = last - chunk + 1, share = (count + groups - 1) / groups, from = group * share, to = from + share < count ? from + share : count;
    float sum[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
    if (c < p.dim) {
#pragma unroll 8
        for (int64_t i = from; i < to; ++i) {
            float x[VEC];
            load_n<VEC>(p.part + (2 * (chunk + i) + (i == 0 ? 1 : 0)) * p.ld_part + c, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += x[e];
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) joined[e * kThreads + threadIdx.x] = sum[e];
    __syncthreads();
    if (group != 0 || c >= p.dim) return;
    for (int g = 1; g < groups && g * share < count; ++g) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += joined[e * kThreads + (g << p.lanes_log2) + threadIdx.x];
    }
    put_row<In, Out, VEC>(p, id, c, c + VEC <= p.dim ? c : p.dim - VEC, sum);
}

// the sort and the sums; what does not fit a launch is refused before either
template <typename In, typename Out, int VEC>
mgg_status_t embed_sum(const EmbedGradPlan &s, SumArgs<In, Out> p, mgg_index_t id_type, const void *ids, char *ws, hipStream_t stream)
{
    const int64_t vecs = ceil_div(p.dim, VEC);
    p.lanes_log2 = ceil_log2(vecs) < 6 ? ceil_log2(vecs) : 6;
    p.slabs = static_cast<int32_t>(ceil_div(vecs, static_cast<int64_t>(1) << p.lanes_log2));
    p.sum_blocks = ceil_div((s.chunks * p.slabs) << p.lanes_log2, kThreads);
    // some 32 KB of zeros to a wavefront, up to 64 rows (2 k ids in 5 k rows of 2.4 KB: 64 rows 16 us, 8 rows 8)
    const int64_t fill = 32768 / (static_cast<int64_t>(p.dim) * static_cast<int64_t>(sizeof(Out)));
    p.fill_rows = static_cast<int32_t>(fill < 1 ? 1 : (fill < kWave ? fill : kWave));
    const int64_t fill_blocks = p.accumulate ? 0 : ceil_div(p.table_rows, static_cast<int64_t>(p.fill_rows) * (kThreads / kWave));
    if (!launchable(p.sum_blocks + fill_blocks, kThreads) || !launchable(s.chunks * p.slabs, kThreads))
        return fail(MGG_ERR_UNSUPPORTED, "%lld ids of %d columns need too many threads for one launch", (long long)p.n, p.dim);
    if (p.sum_blocks + fill_blocks == 0) return MGG_OK;
    if (p.n > 0) {
        const hipError_t e = id_type == MGG_I64 ? sort_ids<int64_t>(s, p.n, ids, p.table_rows, ws, &p.keys, &p.pos, stream)
                                                : sort_ids<int32_t>(s, p.n, ids, p.table_rows, ws, &p.keys, &p.pos, stream);
        if (e != hipSuccess) return hip_fail(e, "sort kernel launch");
    }
    hipLaunchKernelGGL((embed_sum_kernel<In, Out, VEC>), dim3(static_cast<unsigned>(p.sum_blocks + fill_blocks)), dim3(kThreads), 0, stream, p);
    if (s.chunks > 1) hipLaunchKernelGGL((embed_join_kernel<In, Out, VEC>), dim3(static_cast<unsigned>(s.chunks * p.slabs)), dim3(kThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, "table gradient kernel launch");
}

}  // namespace

mgg_status_t launch_embed(int64_t n, mgg_index_t id_type, const void *ids, int64_t table_rows, mgg_dtype_t table_dtype, const void *table, int32_t dim,
                          int64_t ld_table, float scale, mgg_dtype_t out_dtype, void *out, int64_t ld_out, hipStream_t stream)
{
    if (n > static_cast<int64_t>(INT32_MAX)) return fail(MGG_ERR_UNSUPPORTED, "%lld ids", (long long)n);
#define MGG_EMBED(IN, OUT)                                                                                                              \
    return id_type == MGG_I64 ? embed_typed<IN, OUT, int64_t>(n, ids, table_rows, table, dim, ld_table, scale, out, ld_out, stream)         \
                                : embed_typed<IN, OUT, int32_t>(n, ids, table_rows, table, dim, ld_table, scale, out, ld_out, stream)
    if (table_dtype == MGG_BF16) { if (out_dtype == MGG_BF16) MGG_EMBED(Bf16, Bf16); else MGG_EMBED(Bf16, float); }
    else { if (out_dtype == MGG_BF16) MGG_EMBED(float, Bf16); else MGG_EMBED(float, float); }
#undef MGG_EMBED
}

size_t embed_grad_workspace(int64_t n, int64_t table_rows, int32_t dim) { return plan_embed_grad(n, table_rows, dim).bytes; }

mgg_status_t launch_embed_grad(int64_t n, mgg_index_t id_type, const void *ids, int64_t table_rows, mgg_dtype_t grad_dtype, const void *grad, int32_t dim,
                               int64_t ld_grad, float scale, bool accumulate, mgg_dtype_t out_dtype, void *out, int64_t ld_out, void *workspace,
                               hipStream_t stream)
{
    const EmbedGradPlan s = plan_embed_grad(n, table_rows, dim);
    char *ws = static_cast<char *>(workspace);
#define MGG_SUM(IN, OUT)                                                                                                                                      \
    do {                                                                                                                                                      \
        const SumArgs<IN, OUT> p{nullptr, nullptr, static_cast<const IN *>(grad), static_cast<OUT *>(out), reinterpret_cast<float *>(ws + s.part), n, table_rows,       \
                                 ld_grad, ld_out, s.ld_part, 0, dim, s.chunk, static_cast<int32_t>(s.chunks), 0, 0, 0, scale, accumulate};                         \
        constexpr int VEC = 16 / sizeof(IN);                                                                                                                  \
        return dim < 8 ? embed_sum<IN, OUT, 1>(s, p, id_type, ids, ws, stream) : embed_sum<IN, OUT, VEC>(s, p, id_type, ids, ws, stream);                      \
    } while (0)
    if (grad_dtype == MGG_BF16) { if (out_dtype == MGG_BF16) MGG_SUM(Bf16, Bf16); else MGG_SUM(Bf16, float); }
    else { if (out_dtype == MGG_BF16) MGG_SUM(float, Bf16); else MGG_SUM(float, float); }
#undef MGG_SUM
}

}  // namespace mgg
