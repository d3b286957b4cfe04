// The Update by groups of rows and its gradients: products of ragged row blocks with a matrix per group, on the matrix cores.
//
// One tile kernel serves the three products; they differ in which index of an operand is contiguous in memory:
//   forward   out[r][n]  = sum_k a[r][k]  w[k][n]      a along the sum, w across it
//   rows'     da[r][k]   = sum_n dz[r][n] w[k][n]      both along the sum
//   weights'  dw[k][n]   = sum_r a[r][k]  dz[r][n]     both across it
// An operand along the sum is kept in LDS by rows of 128 bytes and read 16 bytes a lane; one across it is kept by rows of the
// tile's width, and bf16 is turned on the way out of LDS (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 elements, a lane gets
// the four elements of a column).
#include "train_common.h"

namespace mgg {

namespace {

using namespace train;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct Vec16 { uint32_t u[4]; };

// ---- which rows a block has ----------------------------------------------------------------------------------
struct Span { int32_t group, row, end, index, total; };     // rows [row, end) of the group: piece `index` of `total` in all

// The groups cut every `step` rows: piece number `index`, found by every wavefront for itself (64 groups at a time, a group per
// lane).  With xcds > 1 `index` counts through pieces dealt in contiguous runs to the XCDs (block b runs on XCD b mod 8).
__device__ __forceinline__ void group_range(const int64_t *ptr, int g, int n_groups, int64_t n_rows, int32_t *lo, int32_t *hi)
{
    *lo = *hi = 0;
    if (g >= n_groups) return;
    const int64_t a = ptr[g], b = ptr[g + 1];
    *lo = static_cast<int32_t>(a < 0 ? 0 : (a > n_rows ? n_rows : a));
    *hi = static_cast<int32_t>(b < *lo ? *lo : (b > n_rows ? n_rows : b));
}

__device__ __forceinline__ int wave_scan(int v, int lane)
{
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const int o = __shfl_up(v, off);
        if (lane >= off) v += o;
    }
    return v;
}


__device__ __forceinline__ bool find_piece(const int64_t *ptr, int n_groups, int64_t n_rows, int step, int index, Span *s)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int g0 = 0; g0 < n_groups; g0 += kWave) {
        int32_t lo, hi;
        group_range(ptr, g0 + lane, n_groups, n_rows, &lo, &hi);
        const int count = (hi - lo) / step + ((hi - lo) % step != 0);
        const int incl = wave_scan(count, lane);
        const uint64_t past = __ballot(before + incl > index);
        if (past) {
            const int at = __ffsll(static_cast<unsigned long long>(past)) - 1;
            s->group = g0 + at;
            const int first = __shfl(lo, at) + (index - before - __shfl(incl - count, at)) * step, last = __shfl(hi, at);
            s->row = __builtin_amdgcn_readfirstlane(first);
            s->end = __builtin_amdgcn_readfirstlane(last - first < step ? last : first + step);
            s->group = __builtin_amdgcn_readfirstlane(s->group);
            return true;
        }
        before += __shfl(incl, 63);
    }
    return false;
}

// ---- an operand's tile on its way from memory to the matrix cores ----------------------------------------------
template <typename T> struct Elem;
template <> struct Elem<Bf16> { static constexpr int N = 8, BK = 64; };      // elements of 16 bytes; depth of a tile: 128 bytes
template <> struct Elem<float> { static constexpr int N = 4, BK = 32; };

template <typename T>
__device__ __forceinline__ Vec16 load16(const T *p)
{
    Vec16 v;
    __builtin_memcpy(&v, __builtin_assume_aligned(p, sizeof(T)), 16);
    return v;
}

// the first `have` elements at p, zeros behind them; reads nothing outside a row of `len` elements that begins at `row`
template <typename T>
__device__ __forceinline__ Vec16 load16_edge(const T *row, int64_t at, int have, int64_t len)
{
    constexpr int N = Elem<T>::N;
    Vec16 v{{0u, 0u, 0u, 0u}};
    if (have >= N) return load16(row + at);
    if (have <= 0) return v;
    if (len >= N) {
        // ends with the row: what lies before `at` is shifted out
        const Vec16 w = load16(row + at + have - N);
        const int bits = (N - have) * static_cast<int>(sizeof(T)) * 8, dwords = bits >> 5, rest = bits & 31;
        uint32_t u[5] = {w.u[0], w.u[1], w.u[2], w.u[3], 0u};
        if (dwords & 1) { u[0] = u[1]; u[1] = u[2]; u[2] = u[3]; u[3] = 0u; }
        if (dwords & 2) { u[0] = u[2]; u[1] = u[3]; u[2] = 0u; u[3] = 0u; }
#pragma unroll
        for (int i = 0; i < 4; ++i) v.u[i] = __builtin_amdgcn_alignbit(i < 3 ? u[i + 1] : 0u, u[i], rest);
        return v;
    }
    T e[N];
    __builtin_memset(e, 0, sizeof e);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < have) e[i] = row[at + i];
    __builtin_memcpy(&v, e, 16);
    return v;
}

// ALONG: rows of the tile are rows of the matrix, the sum runs along them.  Else the sum runs over the matrix's rows and the tile's
// R rows are R of its columns.
template <typename T, int R, bool ALONG, int THREADS>
struct Operand {
    static constexpr int N = Elem<T>::N, BK = Elem<T>::BK;
    static constexpr int kBytes = R * 128;
    static constexpr int kPer = kBytes / 16 / THREADS;
    static constexpr int kRowChunks = ALONG ? 8 : R / N;        // 16-byte chunks per row in LDS
    static_assert(kPer * THREADS * 16 == kBytes, "a tile is whole chunks of every thread");

    const T *base;      // ALONG: first row of the tile; else first row of the sum
    int64_t ld;
    int32_t rows;       // ALONG: rows of the tile that exist; else columns of the matrix from the tile's first on
    int32_t col0;       // else: the tile's first column
    int32_t depth;      // length of the sum
    Vec16 v[kPer];

    // chunk c of row r lies where neighbouring rows' chunks of one column meet different banks
    static __device__ __forceinline__ int place(int r, int c)
    {
        if constexpr (ALONG) return r * 128 + ((c ^ (r & 7)) << 4);
        else {
            constexpr int G = sizeof(T) == 2 ? 4 : 8;            // chunks of 32 columns
            constexpr int M = R / 32 < 4 ? R / 32 - 1 : 3;
            const int key = (sizeof(T) == 2 ? r : r >> 2) & M;
            return r * R * static_cast<int>(sizeof(T)) + ((((c / G) ^ key) * G + c % G) << 4);
        }
    }
    __device__ __forceinline__ void load(int k0)
    {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = threadIdx.x + i * THREADS, r = id / kRowChunks, c = id % kRowChunks;
            if constexpr (ALONG) {
                const T *row = base + static_cast<int64_t>(r < rows ? r : rows - 1) * ld;
                v[i] = load16_edge(row, k0 + c * N, depth - k0 - c * N, depth);
            } else {
                const bool there = k0 + r < depth;
                const T *row = base + static_cast<int64_t>(there ? k0 + r : 0) * ld;
                v[i] = load16_edge(row, col0 + c * N, there ? rows - c * N : 0, static_cast<int64_t>(col0) + rows);
            }
        }
    }
    __device__ __forceinline__ void store(char *lds) const
    {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = threadIdx.x + i * THREADS;
            __builtin_memcpy(__builtin_assume_aligned(lds + place(id / kRowChunks, id % kRowChunks), 16), &v[i], 16);
        }
    }
    // step s of the tile's depth (32 bytes of it) for the 32 rows from r0 on: lane (i, h) gets row r0 + i and, bf16, elements
    // 16 s + 8 h .. + 7, fp32, elements 8 s + 4 h .. + 3
    static __device__ __forceinline__ Vec16 frag(const char *lds, int r0, int s, int lane)
    {
        const int i = lane & 31, h = lane >> 5;
        Vec16 f;
        if constexpr (ALONG) {
            __builtin_memcpy(&f, __builtin_assume_aligned(lds + place(r0 + i, 2 * s + h), 16), 16);
        } else if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int q = lane & 15, col = r0 + (lane & 16) + (q & 3) * 4;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int k = 16 * s + 8 * h + 4 * j + (q >> 2);
                const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + place(k, col / 8) + (col & 7) * 2));
                __builtin_memcpy(&f.u[2 * j], &t, 8);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = 8 * s + 4 * h + j, col = r0 + i;
                __builtin_memcpy(&f.u[j], __builtin_assume_aligned(lds + place(k, col / 4) + (col & 3) * 4, 4), 4);
            }
        }
        return f;
    }
};

template <typename T>
__device__ __forceinline__ f32x16 multiply(const Vec16 &cols, const Vec16 &rows, f32x16 acc)
{
    if constexpr (sizeof(T) == 2) {
        union { Vec16 v; bf16x8 b; } x{cols}, y{rows};
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b, y.b, acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(cols.u[j]), __uint_as_float(rows.u[j]), acc, 0, 0, 0);
        return acc;
    }
}

// The columns' fragment goes in first, so that the accumulator holds the tile turned: register r of lane (m, h) is row m, column
// 8 (r / 4) + 4 h + r % 4, and a lane owns four neighbouring columns.
struct Sink {
    void *out;
    int64_t ld;
    const float *bias;
    int32_t n_cols;         // columns of the matrix
    int32_t bf16, relu, add;
};

template <typename Out>
__device__ __forceinline__ void put4(Out *o, float (&v)[4], int cols, bool add)
{
    if (cols >= 4) {
        if (add) {
            float old[4];
            load_n<4>(o, old);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += old[e];
        }
        store_n<4>(o, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < cols) from_f32(v[e] + (add ? to_f32(o[e]) : 0.f), o[e]);
    }
}

__device__ __forceinline__ void put_tile(const Sink &p, const f32x16 &acc, int64_t row, int64_t end, int col0, int lane)
{
    const int64_t r = row + (lane & 31);
    if (r >= end) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int col = col0 + 8 * q + 4 * (lane >> 5);
        if (col >= p.n_cols) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = acc[4 * q + e] + (p.bias && col + e < p.n_cols ? p.bias[col + e] : 0.f);
            if (p.relu) v[e] = v[e] > 0.f || v[e] != v[e] ? v[e] : 0.f;
        }
        if (p.bf16) put4(static_cast<Bf16 *>(p.out) + r * p.ld + col, v, p.n_cols - col, p.add);
        else put4(static_cast<float *>(p.out) + r * p.ld + col, v, p.n_cols - col, p.add);
    }
}

template <typename T, int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG>
struct Tile {
    static constexpr int THREADS = 64 * WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    using A = Operand<T, BM, A_ALONG, THREADS>;
    using B = Operand<T, BN, B_ALONG, THREADS>;
    static constexpr int kLds = A::kBytes + B::kBytes;

    // acc = the product of the two operands' tiles over their whole depth
    static __device__ __forceinline__ void run(A &a, B &b, char *lds, f32x16 (&acc)[TM][TN])
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        constexpr int BK = Elem<T>::BK;
        const int steps = (a.depth + BK - 1) / BK;
        for (int t = 0; t < steps; ++t) {
            a.load(t * BK);
            b.load(t * BK);
            __syncthreads();
            a.store(lds);
            b.store(lds + A::kBytes);
            __syncthreads();
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                Vec16 fa[TM], fb[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[i] = A::frag(lds, (wm * TM + i) * 32, s, lane);
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[j] = B::frag(lds + A::kBytes, (wn * TN + j) * 32, s, lane);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
            }
        }
    }
    static __device__ __forceinline__ void put(const Sink &p, const f32x16 (&acc)[TM][TN], int64_t row0, int64_t end, int col0)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) put_tile(p, acc[i][j], row0 + (wm * TM + i) * 32, end, col0 + (wn * TN + j) * 32, lane);
    }
};

struct RowsArgs {
    const void *a, *w;
    const int64_t *ptr;
    int64_t n_rows, ld_a;
    int64_t w_group;        // elements of a group's matrix
    int32_t ld_w;
    int32_t n_groups, depth, col_tiles;
    Sink sink;              // bias: of group 0
};

// forward and rows' gradient: pieces of BM rows of the groups x column tiles
template <typename T, int BM, int BN, int WM, int WN, bool B_ALONG>
__global__ __launch_bounds__(64 * WM * WN) void grouped_rows_kernel(const RowsArgs p)
{
    using K = Tile<T, BM, BN, WM, WN, true, B_ALONG>;
    __shared__ __attribute__((aligned(16))) char lds[K::kLds];
    Span s;
    if (!find_piece(p.ptr, p.n_groups, p.n_rows, BM, static_cast<int>(blockIdx.x) / p.col_tiles, &s)) return;
    const int col0 = static_cast<int>(blockIdx.x) % p.col_tiles * BN;
    typename K::A a;
    typename K::B b;
    a.base = static_cast<const T *>(p.a) + s.row * p.ld_a;
    a.ld = p.ld_a; a.rows = s.end - s.row; a.col0 = 0; a.depth = p.depth;
    const T *w = static_cast<const T *>(p.w) + s.group * p.w_group;
    b.ld = p.ld_w; b.depth = p.depth; b.col0 = col0; b.rows = p.sink.n_cols - col0;
    b.base = B_ALONG ? w + static_cast<int64_t>(col0) * p.ld_w : w;
    f32x16 acc[K::TM][K::TN];
    K::run(a, b, lds, acc);
    Sink sink = p.sink;
    if (sink.bias) sink.bias += static_cast<int64_t>(s.group) * sink.n_cols;
    K::put(sink, acc, s.row, s.end, col0);
}

struct WeightArgs {
    const void *a, *dz;
    const int64_t *ptr;
    int64_t n_rows, ld_a, ld_dz;
    int32_t n_groups, d_in, d_out, row_tiles, col_tiles;
    int32_t step;           // rows of a piece; 0: a group is one
    Sink sink;              // of group or piece 0
};

// weights' gradient: tiles of [d_in x d_out] per group, or per piece of `step` rows (partial sums, joined by sum_pieces_kernel)
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void grouped_weight_kernel(const WeightArgs p)
{
    using K = Tile<T, BM, BN, WM, WN, false, false>;
    __shared__ __attribute__((aligned(16))) char lds[K::kLds];
    const int64_t tiles = static_cast<int64_t>(p.row_tiles) * p.col_tiles;
    const int64_t index = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    Span s;
    if (p.step) {
        if (!find_piece(p.ptr, p.n_groups, p.n_rows, p.step, static_cast<int>(index), &s)) return;
    } else {
        s.group = static_cast<int>(index);
        group_range(p.ptr, s.group, p.n_groups, p.n_rows, &s.row, &s.end);
    }
    const int row0 = static_cast<int>(tile / p.col_tiles) * BM, col0 = static_cast<int>(tile % p.col_tiles) * BN;
    typename K::A a;
    typename K::B b;
    a.base = static_cast<const T *>(p.a) + s.row * p.ld_a;
    a.ld = p.ld_a; a.rows = p.d_in - row0; a.col0 = row0; a.depth = s.end - s.row;
    b.base = static_cast<const T *>(p.dz) + s.row * p.ld_dz;
    b.ld = p.ld_dz; b.rows = p.d_out - col0; b.col0 = col0; b.depth = a.depth;
    f32x16 acc[K::TM][K::TN];
    K::run(a, b, lds, acc);
    Sink sink = p.sink;
    const int64_t first = index * p.d_in;
    sink.out = static_cast<char *>(sink.out) + first * p.d_out * (sink.bf16 ? 2 : 4);
    K::put(sink, acc, row0, p.d_in, col0);
}

// out[g] (+)= the sum of the partial sums of the group's pieces, front to back; `width` values each
struct JoinArgs {
    const float *part;
    const int64_t *ptr;
    void *out;
    int64_t n_rows, width;
    int32_t n_groups, step, bf16, add;
};
__global__ __launch_bounds__(256) void sum_pieces_kernel(const JoinArgs p)
{
    const int g = blockIdx.y;
    const int lane = threadIdx.x & 63;
    int first = 0;
    for (int g0 = 0; g0 < g; g0 += kWave) {
        int32_t lo, hi;
        group_range(p.ptr, g0 + lane, g0 + lane < g ? p.n_groups : 0, p.n_rows, &lo, &hi);
        first += (hi - lo) / p.step + ((hi - lo) % p.step != 0);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) first += __shfl_xor(first, off);
    int32_t lo, hi;
    group_range(p.ptr, g, p.n_groups, p.n_rows, &lo, &hi);
    const int count = (hi - lo) / p.step + ((hi - lo) % p.step != 0);
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= p.width) return;
    float sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < count; ++i) sum += p.part[(first + i) * p.width + c];
    const int64_t at = static_cast<int64_t>(g) * p.width + c;
    if (p.bf16) { Bf16 *o = static_cast<Bf16 *>(p.out) + at; from_f32(sum + (p.add ? to_f32(*o) : 0.f), *o); }
    else { float *o = static_cast<float *>(p.out) + at; *o = sum + (p.add ? *o : 0.f); }
}

// dz = grad_out where out > 0 (RELU; written for the two products), and its column sums over pieces of rows
struct MaskArgs {
    const void *grad, *out;
    void *dz;               // NULL: grad is dz already
    float *part;            // NULL: no column sums
    const int64_t *ptr;
    int64_t n_rows, ld_grad, ld_out, ld_dz;
    int32_t n_groups, d_out, step, out_bf16;
};
template <typename T>
__global__ __launch_bounds__(256) void mask_rows_kernel(const MaskArgs p)
{
    __shared__ float joined[4][64];
    Span s;
    if (!find_piece(p.ptr, p.n_groups, p.n_rows, p.step, static_cast<int>(blockIdx.x), &s)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t c0 = static_cast<int64_t>(blockIdx.y) * 64; c0 < p.d_out; c0 += static_cast<int64_t>(gridDim.y) * 64) {
        const int64_t c = c0 + lane;
        float sum = 0.f;
        if (c < p.d_out)
            for (int64_t r = s.row + wave; r < s.end; r += 4) {
                T g = static_cast<const T *>(p.grad)[r * p.ld_grad + c];
                if (p.out) {
                    const float o = p.out_bf16 ? to_f32(static_cast<const Bf16 *>(p.out)[r * p.ld_out + c]) : static_cast<const float *>(p.out)[r * p.ld_out + c];
                    if (!(o > 0.f)) from_f32(0.f, g);
                }
                if (p.dz) static_cast<T *>(p.dz)[r * p.ld_dz + c] = g;
                sum += to_f32(g);
            }
        if (p.part) {
            joined[wave][lane] = sum;
            __syncthreads();
            if (wave == 0 && c < p.d_out) p.part[static_cast<int64_t>(blockIdx.x) * p.d_out + c] = joined[0][lane] + joined[1][lane] + joined[2][lane] + joined[3][lane];
            __syncthreads();
        }
    }
}

constexpr int kMaskRows = 256;

struct GradPlan {
    int32_t step;                   // rows of a piece of the weights' gradient, 0: groups whole
    int64_t pieces, mask_pieces;    // at most
    int64_t ld_dz;
    size_t dz, part, bias_part, bytes;
};

GradPlan plan_grad(int64_t n_rows, int32_t n_groups, int32_t d_in, int32_t d_out, mgg_dtype_t dtype, bool relu)
{
    GradPlan g;
    const int64_t tiles = ceil_div(d_in, 128) * ceil_div(d_out, 128);
    g.step = 0;
    g.pieces = n_groups;
    if (tiles < 256 && n_rows > 0) {
        const int64_t wanted = ceil_div(512, tiles);
        int64_t step = ceil_div(ceil_div(n_rows, wanted), 64) * 64;
        if (step < 256) step = 256;
        g.step = static_cast<int32_t>(step < (1 << 30) ? step : 1 << 30);
        g.pieces = n_rows / g.step + (n_groups < n_rows ? n_groups : n_rows);
    }
    g.mask_pieces = n_rows / kMaskRows + (n_groups < n_rows ? n_groups : n_rows);
    g.ld_dz = static_cast<int64_t>(round_up(static_cast<size_t>(d_out), 8));
    size_t at = 0;
    g.dz = at; at += relu ? round_up(static_cast<size_t>(n_rows) * g.ld_dz * (dtype == MGG_BF16 ? 2 : 4), 256) : 0;
    g.part = at; at += g.step ? round_up(static_cast<size_t>(g.pieces) * d_in * d_out * 4, 256) : 0;
    g.bias_part = at; at += round_up(static_cast<size_t>(g.mask_pieces) * d_out * 4, 256);
    g.bytes = at + 256;
    return g;
}

template <typename T>
mgg_status_t rows_product(RowsArgs p, bool b_along, hipStream_t stream)
{
    constexpr int BM = 128, BN = 128;
    p.col_tiles = static_cast<int32_t>(ceil_div(p.sink.n_cols, BN));
    const int64_t blocks = (p.n_rows / BM + (p.n_groups < p.n_rows ? p.n_groups : p.n_rows)) * p.col_tiles;
    if (blocks > INT32_MAX) return fail(MGG_ERR_UNSUPPORTED, "too many tiles for one launch");
    const dim3 grid(static_cast<unsigned>(blocks));
    if (b_along) hipLaunchKernelGGL((grouped_rows_kernel<T, BM, BN, 2, 2, true>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((grouped_rows_kernel<T, BM, BN, 2, 2, false>), grid, dim3(256), 0, stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, "grouped product launch");
}

template <typename T>
mgg_status_t weight_product(WeightArgs p, int64_t pieces, hipStream_t stream)
{
    constexpr int BM = 128, BN = 128;
    p.row_tiles = static_cast<int32_t>(ceil_div(p.d_in, BM));
    p.col_tiles = static_cast<int32_t>(ceil_div(p.d_out, BN));
    const int64_t blocks = pieces * p.row_tiles * p.col_tiles;
    if (blocks > INT32_MAX) return fail(MGG_ERR_UNSUPPORTED, "too many tiles for one launch");
    hipLaunchKernelGGL((grouped_weight_kernel<T, BM, BN, 2, 2>), dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, "grouped weight gradient launch");
}

mgg_status_t join_pieces(const JoinArgs &p, hipStream_t stream)
{
    const int64_t blocks = ceil_div(p.width, 256);
    if (blocks > INT32_MAX) return fail(MGG_ERR_UNSUPPORTED, "too many columns for one launch");
    hipLaunchKernelGGL(sum_pieces_kernel, dim3(static_cast<unsigned>(blocks), p.n_groups), dim3(256), 0, stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, "partial sum launch");
}

}  // namespace

mgg_status_t launch_update_grouped(int64_t n_rows, int32_t n_groups, const int64_t *group_ptr, mgg_dtype_t dtype, const void *a, int64_t ld_a, int32_t d_in,
                                   const void *w, const float *bias, int32_t d_out, bool relu, mgg_dtype_t out_dtype, void *out, int64_t ld_out,
                                   hipStream_t stream)
{
    RowsArgs p{};
    p.a = a; p.w = w; p.ptr = group_ptr; p.n_rows = n_rows; p.ld_a = ld_a; p.n_groups = n_groups;
    p.w_group = static_cast<int64_t>(d_in) * d_out; p.ld_w = d_out; p.depth = d_in;
    p.sink = Sink{out, ld_out, bias, d_out, out_dtype == MGG_BF16, relu, 0};
    return dtype == MGG_BF16 ? rows_product<Bf16>(p, false, stream) : rows_product<float>(p, false, stream);
}

size_t grouped_grad_workspace(int64_t n_rows, int32_t n_groups, int32_t d_in, int32_t d_out, mgg_dtype_t dtype, bool relu)
{
    return plan_grad(n_rows, n_groups, d_in, d_out, dtype, relu).bytes;
}

mgg_status_t launch_update_grouped_grad(const GroupedGrad &q, void *workspace, hipStream_t stream)
{
    const GradPlan g = plan_grad(q.n_rows, q.n_groups, q.d_in, q.d_out, q.dtype, q.relu);
    char *ws = static_cast<char *>(workspace);
    const bool bf16 = q.dtype == MGG_BF16;
    const void *dz = q.grad_out;
    int64_t ld_dz = q.ld_grad;
    mgg_status_t s = MGG_OK;
    if (q.n_rows > 0 && (q.relu || q.grad_bias) && (q.grad_a || q.grad_w || q.grad_bias)) {
        MaskArgs m{};
        m.grad = q.grad_out; m.ptr = q.group_ptr; m.n_rows = q.n_rows; m.ld_grad = q.ld_grad; m.n_groups = q.n_groups; m.d_out = q.d_out; m.step = kMaskRows;
        if (q.relu) {
            m.out = q.out; m.ld_out = q.ld_out; m.out_bf16 = q.out_dtype == MGG_BF16;
            if (q.grad_a || q.grad_w) { m.dz = ws + g.dz; m.ld_dz = g.ld_dz; dz = m.dz; ld_dz = m.ld_dz; }
        }
        if (q.grad_bias) m.part = reinterpret_cast<float *>(ws + g.bias_part);
        const int64_t slabs = ceil_div(q.d_out, 64);
        const dim3 grid(static_cast<unsigned>(g.mask_pieces), static_cast<unsigned>(slabs < 1024 ? slabs : 1024));
        if (bf16) hipLaunchKernelGGL(mask_rows_kernel<Bf16>, grid, dim3(256), 0, stream, m);
        else hipLaunchKernelGGL(mask_rows_kernel<float>, grid, dim3(256), 0, stream, m);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "mask launch");
    }
    if (q.grad_bias) {
        s = join_pieces(JoinArgs{reinterpret_cast<float *>(ws + g.bias_part), q.group_ptr, q.grad_bias, q.n_rows, q.d_out, q.n_groups, kMaskRows, 0, q.add_bias}, stream);
        if (s != MGG_OK) return s;
    }
    if (q.grad_a) {
        RowsArgs p{};
        p.a = dz; p.w = q.w; p.ptr = q.group_ptr; p.n_rows = q.n_rows; p.ld_a = ld_dz; p.n_groups = q.n_groups;
        p.w_group = static_cast<int64_t>(q.d_in) * q.d_out; p.ld_w = q.d_out; p.depth = q.d_out;
        p.sink = Sink{q.grad_a, q.ld_grad_a, nullptr, q.d_in, q.grad_a_dtype == MGG_BF16, 0, 0};
        s = bf16 ? rows_product<Bf16>(p, true, stream) : rows_product<float>(p, true, stream);
        if (s != MGG_OK) return s;
    }
    if (q.grad_w) {
        WeightArgs p{};
        p.a = q.a; p.dz = dz; p.ptr = q.group_ptr; p.n_rows = q.n_rows; p.ld_a = q.ld_a; p.ld_dz = ld_dz;
        p.n_groups = q.n_groups; p.d_in = q.d_in; p.d_out = q.d_out; p.step = g.step;
        if (g.step) p.sink = Sink{ws + g.part, q.d_out, nullptr, q.d_out, 0, 0, 0};
        else p.sink = Sink{q.grad_w, q.d_out, nullptr, q.d_out, q.grad_w_dtype == MGG_BF16, 0, q.add_w};
        s = bf16 ? weight_product<Bf16>(p, g.pieces, stream) : weight_product<float>(p, g.pieces, stream);
        if (s != MGG_OK || !g.step) return s;
        s = join_pieces(JoinArgs{reinterpret_cast<float *>(ws + g.part), q.group_ptr, q.grad_w, q.n_rows, static_cast<int64_t>(q.d_in) * q.d_out, q.n_groups, g.step,
                                 q.grad_w_dtype == MGG_BF16, q.add_w}, stream);
    }
    return s;
}

}  // namespace mgg
