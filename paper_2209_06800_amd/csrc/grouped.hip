// The Update by groups of rows and its gradients: products of ragged row blocks with a matrix per group, on the matrix cores.
//
// One tile kernel serves the three products; they differ in which index of an operand is contiguous in memory:
//   forward   out[r][n]  = sum_k a[r][k]  w[k][n]      a along the sum, w across it
//   rows'     da[r][k]   = sum_n dz[r][n] w[k][n]      both along the sum
//   weights'  dw[k][n]   = sum_r a[r][k]  dz[r][n]     both across it
// An operand along the sum is kept in LDS by rows of 128 bytes and read 16 bytes a lane; one across it is kept by rows of the
// tile's width, and bf16 is turned on the way out of LDS (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 elements, a lane gets
// the four elements of a column).
//
// What bounds it and what it reaches (one MI355X; a large library product runs at 1285 TFLOP/s bf16 and 154 fp32, a copy at 5.1 TB/s):
//   - many rows, bf16: the matrix cores, as far as the clock holds (by the cycle counter 2.0 GHz in launches of 0.3 ms, 1.5 in a run of the one below).  32 k rows over
//     8 groups 4096 -> 4096: 1.03 - 1.17 ms by the clock, 940 - 1070 TFLOP/s; rows' gradient of 16 k rows 2048 <- 4096:
//     0.30 ms, weights': 0.28.
//   - many rows, fp32: the fp32 matrix instruction.  8 k rows 2048 -> 2048 over 4 groups: 0.62 - 0.64 ms, 107 - 111 TFLOP/s.
//   - few rows to a group: reading the weights.  64 rows over 64 groups 1024 -> 2048 bf16, 41 of them with rows: 38 us, 172 MB at 4.6 TB/s
//     (30 where the Infinity Cache still holds a part).
//   - short sums (widths up to some hundred): the chain of a block from its group's offsets over its operands to its stores, a few
//     microseconds for each of the rounds that fill the chip.  233 k rows 100 -> 256 fp32: 181 - 192 us, where bytes and instructions allow 77;
//     60 k rows 300 -> 200 bf16 over 7 groups: 36 us, bytes allow 12.
//   - widths below 16 bytes: plain sums, one result per thread, bound by the latency of loads a row apart (tiny_rows_kernel).
#include "train_common.h"

namespace mgg {

namespace {

using namespace train;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct Vec16 { uint32_t u[4]; };

constexpr int kBandRows = 1024;     // rows of a band of tiles

// ---- which rows a block has ----------------------------------------------------------------------------------
struct Span { int32_t group, row, end; };       // rows [row, end) of the group

__device__ __forceinline__ void group_range(const int64_t *ptr, int g, int n_groups, int64_t n_rows, int32_t *lo, int32_t *hi)
{
    *lo = *hi = 0;
    if (g >= n_groups) return;
    const int64_t a = ptr[g], b = ptr[g + 1];
    *lo = static_cast<int32_t>(a < 0 ? 0 : (a > n_rows ? n_rows : a));
    *hi = static_cast<int32_t>(b < *lo ? *lo : (b > n_rows ? n_rows : b));
}

// inclusive prefix sums over a wavefront, by DPP: within rows of 16 lanes, then the rows' last ones to the rows behind
__device__ __forceinline__ int wave_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);      // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // row_bcast:15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);     // row_bcast:31 to rows 2 and 3
    return v;
}

__device__ __forceinline__ int pieces_in(int32_t rows, int step) { return rows / step + (rows % step != 0); }

// pieces of `step` rows in the first n_groups groups, those of groups of fewer than `least` left out, by a wavefront, a group per lane;
// `most` where overlapping groups would give more
__device__ __forceinline__ int count_pieces(const int64_t *ptr, int n_groups, int64_t n_rows, int step, int most, int least = 1)
{
    int total = 0;
    for (int g0 = 0; g0 < n_groups; g0 += kWave) {
        int32_t lo, hi;
        group_range(ptr, g0 + (threadIdx.x & 63), n_groups, n_rows, &lo, &hi);
        const int pieces = pieces_in(hi - lo, step);
        total = min(total + min(__builtin_amdgcn_readlane(wave_scan(pieces < least ? 0 : pieces), 63), most), most);
    }
    return total;
}

// piece number `index`, found by every wavefront for itself, 64 groups at a time; SLOT: also its number among the pieces of groups of
// several
template <bool SLOT = false>
__device__ __forceinline__ bool find_piece(const int64_t *ptr, int n_groups, int64_t n_rows, int step, int index, Span *s, int *slot = nullptr)
{
    int before = 0, slots = 0;
    for (int g0 = 0; g0 < n_groups; g0 += kWave) {
        int32_t lo, hi;
        group_range(ptr, g0 + (threadIdx.x & 63), n_groups, n_rows, &lo, &hi);
        const int count = pieces_in(hi - lo, step), incl = wave_scan(count);
        const int several = count < 2 ? 0 : count, several_incl = SLOT ? wave_scan(several) : 0;
        const uint64_t past = __ballot(before + incl > index);
        if (past) {
            const int at = __builtin_amdgcn_readfirstlane(__ffsll(static_cast<unsigned long long>(past)) - 1);
            const int in = index - before - __builtin_amdgcn_readlane(incl - count, at), first = __builtin_amdgcn_readlane(lo, at) + in * step;
            const int last = __builtin_amdgcn_readlane(hi, at);
            if (first < __builtin_amdgcn_readlane(lo, at) || first >= last) return false;       // (sums of overlapping groups can overflow)
            s->group = g0 + at;
            s->row = first;
            s->end = last - first < step ? last : first + step;
            if constexpr (SLOT) *slot = slots + __builtin_amdgcn_readlane(several_incl - several, at) + in;
            return true;
        }
        before += __builtin_amdgcn_readlane(incl, 63);
        if constexpr (SLOT) slots += __builtin_amdgcn_readlane(several_incl, 63);
    }
    return false;
}

// tile number `index` of rows x cols, in bands of `band` rows, each walked column by column
__device__ __forceinline__ void band_order(int index, int rows, int cols, int band, int *row, int *col)
{
    const int b = index / (band * cols), in = index % (band * cols), high = rows - b * band < band ? rows - b * band : band;
    *col = in / high;
    *row = b * band + in % high;
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

// the elements of v from number `skip` (0 .. N) on, zeros behind them
template <typename T>
__device__ __forceinline__ Vec16 drop(const Vec16 &v, int skip)
{
    const int bits = skip * static_cast<int>(sizeof(T)) * 8;
    const bool one = bits & 32, two = bits & 64, all = bits & 128;
    const uint32_t a0 = one ? v.u[1] : v.u[0], a1 = one ? v.u[2] : v.u[1], a2 = one ? v.u[3] : v.u[2], a3 = one ? 0u : v.u[3];
    const uint32_t b0 = two ? a2 : a0, b1 = two ? a3 : a1, b2 = two ? 0u : a2, b3 = two ? 0u : a3;
    const uint32_t rest = bits & 31;
    Vec16 r;
    r.u[0] = all ? 0u : __builtin_amdgcn_alignbit(b1, b0, rest);
    r.u[1] = all ? 0u : __builtin_amdgcn_alignbit(b2, b1, rest);
    r.u[2] = all ? 0u : __builtin_amdgcn_alignbit(b3, b2, rest);
    r.u[3] = all ? 0u : b3 >> rest;
    return r;
}

// ALONG: rows of the tile are rows of the matrix, the sum runs along them.  Else the sum runs over the matrix's rows and the tile's
// R rows are R of its columns.  ODD: rows need not be whole chunks of 16 bytes (they have one at least).
// Nothing outside the matrix is read: rows and columns that are not there are read from the nearest ones that are, 16 bytes that would
// reach over a row's end from so far before it that they end with the row, and shifted.  What that leaves in places of the sum that do not exist
// is zeroed, what it leaves in rows or columns of the result that do not exist is never written.
template <typename T, int R, bool ALONG, int THREADS, bool ODD>
struct Operand {
    static constexpr int N = Elem<T>::N, BK = Elem<T>::BK;
    static constexpr int kBytes = R * 128;
    static constexpr int kPer = kBytes / 16 / THREADS;
    static constexpr int kRowChunks = ALONG ? 8 : R / N;        // 16-byte chunks per row in LDS
    static_assert(kPer * THREADS * 16 == kBytes, "a tile is whole chunks of every thread");

    const T *base;      // ALONG: first row of the tile; else first row of the sum (column 0 of the matrix)
    int64_t ld;
    int32_t rows;       // ALONG: rows of the tile that exist; else columns of the matrix from the tile's first on
    int32_t col0;       // else: the tile's first column
    int32_t depth;      // length of the sum
    uint32_t off[kPer]; // bytes from `base`
    Vec16 v[kPer];      // a step on its way

    // Chunk c of row r lies where what is read at once meets different banks: along, 16 lanes read a chunk of 16 rows (256 bytes, all
    // banks); across, 32 lanes read 64 bytes of 4 rows (bf16) or 64 lanes 128 bytes of 2 rows, 4 apart (fp32).
    static __device__ __forceinline__ int place(int r, int c)
    {
        if constexpr (ALONG) return r * 128 + ((c ^ ((r >> 1) & 7)) << 4);
        else {
            constexpr int G = sizeof(T) == 2 ? 4 : 8;            // chunks of 32 columns
            const int key = sizeof(T) == 4 ? (r >> 2) & 1 : (R >= 128 ? r & 3 : (r >> 1) & 1);
            return r * R * static_cast<int>(sizeof(T)) + ((((c / G) ^ key) * G + c % G) << 4);
        }
    }
    static __device__ __forceinline__ int chunk_row(int i) { return (threadIdx.x % THREADS + i * THREADS) / kRowChunks; }
    static __device__ __forceinline__ int chunk_col(int i) { return (threadIdx.x % THREADS + i * THREADS) % kRowChunks; }
    // place of this thread's chunk i: where all of them have the same key, one address and constants
    static __device__ __forceinline__ int chunk_place(int i)
    {
        constexpr int kStep = THREADS / kRowChunks;
        if constexpr (kStep % (ALONG ? 16 : 8) == 0) return place(chunk_row(0), chunk_col(0)) + i * kStep * (ALONG ? 128 : R * static_cast<int>(sizeof(T)));
        else return place(chunk_row(i), chunk_col(i));
    }
    // (32 bits hold an offset: at most 256 rows of 2^22 elements of 4 bytes)
    __device__ __forceinline__ void init()
    {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = ALONG ? min(chunk_row(i), rows - 1) : chunk_row(i), c = ALONG ? chunk_col(i) * N : min(col0 + chunk_col(i) * N, col0 + rows - N);
            off[i] = (static_cast<uint32_t>(r) * static_cast<uint32_t>(ld) + static_cast<uint32_t>(c)) * static_cast<uint32_t>(sizeof(T));
        }
    }
    __device__ __forceinline__ const char *step_base(int k0) const
    {
        return reinterpret_cast<const char *>(base) + (ALONG ? static_cast<int64_t>(k0) : static_cast<int64_t>(k0) * ld) * static_cast<int64_t>(sizeof(T));
    }
    // a step whose BK places of the sum all exist
    __device__ __forceinline__ void load_chunk(const char *at, int i) { v[i] = load16(reinterpret_cast<const T *>(at + off[i])); }
    // the last one, where they do not
    __device__ __forceinline__ void load_last(int k0)
    {
        const char *at = step_base(k0);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int over = ALONG ? max(k0 + chunk_col(i) * N + N - depth, 0) : max(k0 + chunk_row(i) - (depth - 1), 0);
            const Vec16 x = load16(reinterpret_cast<const T *>(at + off[i]) - (ALONG ? over : over * ld));
            if (ALONG && ODD) {
                v[i] = drop<T>(x, min(over, N));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i].u[e] = over ? 0u : x.u[e];
            }
        }
    }
    __device__ __forceinline__ void load(int t)
    {
        const int k0 = t * BK;
        if (k0 + BK <= depth) {
            const char *at = step_base(k0);
#pragma unroll
            for (int i = 0; i < kPer; ++i) load_chunk(at, i);
        } else if (k0 < depth) {
            load_last(k0);
        }
    }
    __device__ __forceinline__ void store_chunk(char *lds, int i) const
    {
        Vec16 x = v[i];
        if (ODD && !ALONG && rows < R) x = drop<T>(x, min(max(chunk_col(i) * N + N - rows, 0), N));
        __builtin_memcpy(__builtin_assume_aligned(lds + chunk_place(i), 16), &x, 16);
    }
    __device__ __forceinline__ void store(char *lds) const
    {
#pragma unroll
        for (int i = 0; i < kPer; ++i) store_chunk(lds, i);
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

// the first `cols` of N values to o, on top of what is there where `add` says so
template <int N, typename Out>
__device__ __forceinline__ void put_cols(Out *o, float (&v)[N], int cols, bool add)
{
    if (cols >= N) {
        if (add) {
            float old[N];
            load_n<N>(o, old);
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] += old[e];
        }
        store_n<N>(o, v);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < cols) from_f32(v[e] + (add ? to_f32(o[e]) : 0.f), o[e]);
    }
}

// The two halves of a wavefront change registers, so that a lane has eight neighbouring columns: 16 (q + h), q = 0, 1, of row m.
__device__ __forceinline__ void put_tile(const Sink &p, const f32x16 &acc, int64_t row, int64_t end, int col0, int lane)
{
    const int64_t r = row + (lane & 31);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * q + e]), __float_as_uint(acc[8 * q + 4 + e]), false, false);
            v[e] = __uint_as_float(both[0]);
            v[4 + e] = __uint_as_float(both[1]);
        }
        const int col = col0 + 16 * q + 8 * (lane >> 5);
        if (r >= end || col >= p.n_cols) continue;
        if (p.bias) {
            float b[8];
            if (col + 8 <= p.n_cols) {
                load_n<8>(p.bias + col, b);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) b[e] = p.bias[min(col + e, p.n_cols - 1)];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += b[e];
        }
        if (p.relu) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];
        }
        if (p.bf16) put_cols<8>(static_cast<Bf16 *>(p.out) + r * p.ld + col, v, p.n_cols - col, p.add);
        else put_cols<8>(static_cast<float *>(p.out) + r * p.ld + col, v, p.n_cols - col, p.add);
    }
}

// A tile of BM x BN of the result by THREADS threads: WM x WN wavefronts, TM x TN pieces of 32 x 32 each
template <typename T, int BM, int BN, int WM, int WN, bool A_ALONG, bool B_ALONG, bool ODD>
struct Tile {
    static constexpr int THREADS = 64 * WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, BK = Elem<T>::BK;
    using A = Operand<T, BM, A_ALONG, THREADS, ODD>;
    using B = Operand<T, BN, B_ALONG, THREADS, ODD>;
    static constexpr int kStage = A::kBytes + B::kBytes;
    typedef f32x16 Acc[TM][TN];

    static __device__ __forceinline__ int wave_row() { return threadIdx.x % THREADS / 64 / WN * TM * 32; }
    static __device__ __forceinline__ int wave_col() { return threadIdx.x % THREADS / 64 % WN * TN * 32; }
    static __device__ __forceinline__ void clear(Acc &acc)
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }
    // quarter s of a step out of LDS
    static __device__ __forceinline__ void read(const char *lds, int s, Vec16 (&fa)[TM], Vec16 (&fb)[TN])
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[j] = B::frag(lds + A::kBytes, wave_col() + j * 32, s, lane);
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[i] = A::frag(lds, wave_row() + i * 32, s, lane);
    }
    static __device__ __forceinline__ void multiply_quarter(const Vec16 (&fa)[TM], const Vec16 (&fb)[TN], Acc &acc)
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = multiply<T>(fb[j], fa[i], acc[i][j]);
    }
    static __device__ __forceinline__ void multiply_step(const char *lds, Acc &acc, int quarters = 4)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s >= quarters) break;
            Vec16 fa[TM], fb[TN];
            read(lds, s, fa, fb);
            multiply_quarter(fa, fb, acc);
        }
    }
    // quarters of the last step that hold anything
    static __device__ __forceinline__ int last_quarters(int depth) { return ((depth - 1) % BK * 4 + BK) / BK; }
    static __device__ __forceinline__ void load(A &a, B &b, int t)
    {
        a.load(t);
        b.load(t);
    }
    static __device__ __forceinline__ void load_plain(A &a, B &b, int t)
    {
        const char *at_a = a.step_base(t * BK), *at_b = b.step_base(t * BK);
#pragma unroll
        for (int i = 0; i < A::kPer; ++i) a.load_chunk(at_a, i);
#pragma unroll
        for (int i = 0; i < B::kPer; ++i) b.load_chunk(at_b, i);
    }
    static __device__ __forceinline__ void store(const A &a, const B &b, char *lds)
    {
        a.store(lds);
        b.store(lds + A::kBytes);
    }

    // acc = the product of the two operands' tiles over their whole depth, by all threads of the block; lds: two stages.  While a
    // step is multiplied out of one, the next one goes from registers to the other and the one after it is on its way from memory.
    static __device__ __forceinline__ void run(A &a, B &b, char *lds, Acc &acc)
    {
        clear(acc);
        const int steps = (a.depth + BK - 1) / BK;
        if (steps == 0) return;
        a.init();
        b.init();
        load(a, b, 0);
        store(a, b, lds);
        load(a, b, 1);
        __syncthreads();
        int t = 0;
        for (; t + 2 < a.depth / BK; ++t) {
            store(a, b, lds + ((t + 1) & 1) * kStage);
            load_plain(a, b, t + 2);
            multiply_step(lds + (t & 1) * kStage, acc);
            __syncthreads();
        }
        for (; t + 1 < steps; ++t) {
            store(a, b, lds + ((t + 1) & 1) * kStage);
            load(a, b, t + 2);
            multiply_step(lds + (t & 1) * kStage, acc);
            __syncthreads();
        }
        multiply_step(lds + (t & 1) * kStage, acc, last_quarters(a.depth));
    }

    // The same for large tiles with two wavefronts on a SIMD, in turns: in every quarter step one of them fetches (its fragments out of LDS,
    // a part of the next step into it) while the other multiplies, and they change places at a barrier; the second half of the block
    // is one turn late throughout.  All that a quarter multiplies is in registers when its turn begins, so the matrix cores
    // of a SIMD wait for LDS only where the other wavefront's fetching takes longer than the multiplying.
    template <bool NEXT, bool PLAIN>
    static __device__ __forceinline__ void turns_step(A &a, B &b, char *lds, int t, Acc &acc)
    {
        const char *from = lds + (t & 1) * kStage;
        char *to = lds + ((t + 1) & 1) * kStage;
        constexpr int P = (A::kPer + B::kPer) / 4;          // chunks of a quarter
        static_assert(P * 4 == A::kPer + B::kPer, "quarters alike");
        const char *at_a = a.step_base((t + 2) * BK), *at_b = b.step_base((t + 2) * BK);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            Vec16 fa[TM], fb[TN];
            read(from, s, fa, fb);
            if (NEXT) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = s * P; i < (s + 1) * P; ++i) {
                    if (i < A::kPer) a.store_chunk(to, i);
                    else b.store_chunk(to + A::kBytes, i - A::kPer);
                }
                if (!PLAIN && s == 3) load(a, b, t + 2);
            }
            // the fragments are here (LDS answers in order; what is written has to be there at the step's end only)
            if (NEXT && PLAIN && s < 3) asm volatile("s_waitcnt lgkmcnt(%0)" :: "i"(P) : "memory");
            else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            if (NEXT && PLAIN) {
#pragma unroll
                for (int i = s * P; i < (s + 1) * P; ++i) {
                    if (i < A::kPer) a.load_chunk(at_a, i);
                    else b.load_chunk(at_b, i - A::kPer);
                }
            }
            multiply_quarter(fa, fb, acc);
            if (NEXT && PLAIN) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);      // two matrix instructions,
                    __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);      // a load
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    static __device__ __forceinline__ void run_in_turns(A &a, B &b, char *lds, Acc &acc)
    {
        static_assert(THREADS == 512, "wavefronts w and w + 4 share a SIMD");
        clear(acc);
        const int steps = (a.depth + BK - 1) / BK;
        if (steps == 0) return;
        a.init();
        b.init();
        load(a, b, 0);
        store(a, b, lds);
        load(a, b, 1);
        __syncthreads();
        const bool late = __builtin_amdgcn_readfirstlane(threadIdx.x) >= THREADS / 2;      // (a scalar: a barrier takes no notice of masked lanes)
        if (late) __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        int t = 0;
        for (; t + 2 < a.depth / BK; ++t) turns_step<true, true>(a, b, lds, t, acc);
        for (; t + 1 < steps; ++t) turns_step<true, false>(a, b, lds, t, acc);
        turns_step<false, false>(a, b, lds, t, acc);
        if (!late) __builtin_amdgcn_s_barrier();
    }

    // Steps [t, end) by one wavefront for itself; lds: one stage of its own.  (A wavefront's LDS accesses are in order.)
    static __device__ __forceinline__ void run_alone(A &a, B &b, char *lds, int t, int end, Acc &acc)
    {
        static_assert(THREADS == 64, "one wavefront");
        clear(acc);
        if (t >= end) return;
        a.init();
        b.init();
        load(a, b, t);
        const int plain = min(end, a.depth / BK);
        for (; t + 1 < plain; ++t) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            store(a, b, lds);
            load_plain(a, b, t + 1);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            multiply_step(lds, acc);
        }
        for (; t < end; ++t) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            store(a, b, lds);
            if (t + 1 < end) load(a, b, t + 1);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            multiply_step(lds, acc);
        }
    }

    static __device__ __forceinline__ void put(const Sink &p, const Acc &acc, int64_t row0, int64_t end, int col0)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) put_tile(p, acc[i][j], row0 + wave_row() + i * 32, end, col0 + wave_col() + j * 32, lane);
    }
};

// The kinds of tiles.  LARGE: 256 x 256 in turns, bf16 and whole chunks only (its registers are full).  MEDIUM: 128 x 128, two blocks to a CU.
// NARROW: 128 x 64, SMALL: 64 x 64, for results of few columns; SMALL for all of fp32, too, whose products take so long that what counts is how
// evenly the chip is filled (20 k rows 512 -> 512 over 10 groups: 106 us against 132 with MEDIUM).
enum Kind { LARGE, MEDIUM, NARROW, SMALL };
constexpr int kind_rows(Kind k) { return k == LARGE ? 256 : (k == SMALL ? 64 : 128); }
constexpr int kind_cols(Kind k) { return k == LARGE ? 256 : (k == MEDIUM ? 128 : 64); }
constexpr int kind_threads(Kind k) { return k == LARGE ? 512 : 256; }
template <typename T, Kind KIND, bool A_ALONG, bool B_ALONG, bool ODD>
using KindTile = Tile<T, kind_rows(KIND), kind_cols(KIND), 2, KIND == LARGE ? 4 : 2, A_ALONG, B_ALONG, ODD>;

template <typename K, Kind KIND>
__device__ __forceinline__ void run_kind(typename K::A &a, typename K::B &b, char *lds, typename K::Acc &acc)
{
    if constexpr (KIND == LARGE) K::run_in_turns(a, b, lds, acc);
    else K::run(a, b, lds, acc);
}

struct RowsArgs {
    const void *a, *w;
    const int64_t *ptr;
    int64_t n_rows, ld_a;
    int64_t w_group;        // elements of a group's matrix
    int32_t ld_w;
    int32_t n_groups, depth, col_tiles;
    int32_t most;           // pieces there can be
    Sink sink;              // bias: of group 0
};

template <typename K, typename T, bool B_ALONG>
__device__ __forceinline__ void rows_operands(const RowsArgs &p, const Span &s, int col0, typename K::A &a, typename K::B &b, Sink &sink)
{
    a.base = static_cast<const T *>(p.a) + s.row * p.ld_a;
    a.ld = p.ld_a; a.rows = s.end - s.row; a.col0 = 0; a.depth = p.depth;
    const T *w = static_cast<const T *>(p.w) + s.group * p.w_group;
    b.base = B_ALONG ? w + static_cast<int64_t>(col0) * p.ld_w : w;
    b.ld = p.ld_w; b.rows = p.sink.n_cols - col0; b.col0 = B_ALONG ? 0 : col0; b.depth = p.depth;
    sink = p.sink;
    if (sink.bias) sink.bias += static_cast<int64_t>(s.group) * sink.n_cols;
}

// forward and rows' gradient: pieces of the groups' rows x column tiles
template <typename T, Kind KIND, bool B_ALONG, bool ODD>
__global__ __launch_bounds__(kind_threads(KIND)) __attribute__((amdgpu_waves_per_eu(2))) void grouped_rows_kernel(const RowsArgs p)
{
    using K = KindTile<T, KIND, true, B_ALONG, ODD>;
    constexpr int BM = kind_rows(KIND), BN = kind_cols(KIND);
    __shared__ __attribute__((aligned(16))) char lds[2 * K::kStage];
    const int pieces = count_pieces(p.ptr, p.n_groups, p.n_rows, BM, p.most);
    if (static_cast<int>(blockIdx.x) >= pieces * p.col_tiles) return;
    int piece, col;
    band_order(blockIdx.x, pieces, p.col_tiles, kBandRows / BM, &piece, &col);
    Span s;
    if (!find_piece(p.ptr, p.n_groups, p.n_rows, BM, piece, &s)) return;
    typename K::A a;
    typename K::B b;
    Sink sink;
    rows_operands<K, T, B_ALONG>(p, s, col * BN, a, b, sink);
    typename K::Acc acc;
    run_kind<K, KIND>(a, b, lds, acc);
    K::put(sink, acc, s.row, s.end, col * BN);
}

// The same where a group has few rows, and what takes the time is reading its weights: tiles of 32 x BN by WAVES wavefronts, which share
// the depth, each for itself and without a barrier until their sums meet in LDS, in order.
template <typename T, int BN, int WAVES, bool B_ALONG, bool ODD>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2))) void grouped_few_rows_kernel(const RowsArgs p)
{
    using K = Tile<T, 32, BN, 1, 1, true, B_ALONG, ODD>;
    constexpr int J = BN / 32, kSums = J * 16 * 64 * 4;
    static_assert(WAVES >= J, "a wavefront per 32 columns at the end");
    static_assert(K::kStage >= kSums, "a wavefront's sums fit where its tiles were");
    __shared__ __attribute__((aligned(16))) char lds[WAVES * K::kStage];
    Span s;
    if (!find_piece(p.ptr, p.n_groups, p.n_rows, 32, static_cast<int>(blockIdx.x) / p.col_tiles, &s)) return;
    const int col0 = static_cast<int>(blockIdx.x) % p.col_tiles * BN, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    typename K::A a;
    typename K::B b;
    Sink sink;
    rows_operands<K, T, B_ALONG>(p, s, col0, a, b, sink);
    typename K::Acc acc;
    const int steps = (p.depth + K::BK - 1) / K::BK;
    K::run_alone(a, b, lds + wave * K::kStage, wave * steps / WAVES, (wave + 1) * steps / WAVES, acc);
    __syncthreads();
    float *sums = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[((wave * J + j) * 16 + r) * 64 + lane] = acc[0][j][r];
    __syncthreads();
    if (wave >= J) return;
    // wavefront j takes the sums of 32 columns
    f32x16 all;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        all[r] = sums[(wave * 16 + r) * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) all[r] += sums[((w * J + wave) * 16 + r) * 64 + lane];
    }
    put_tile(sink, all, s.row, s.end, col0 + wave * 32, lane);
}

struct WeightArgs {
    const void *a, *dz;
    const int64_t *ptr;
    int64_t n_rows, ld_a, ld_dz;
    int32_t n_groups, d_in, d_out, row_tiles, col_tiles;
    int32_t step;           // rows of a piece; 0: a group is one
    int32_t slots;          // partial sums there is room for: one for each piece of the groups of several
    Sink sink;              // of group 0
    float *part;            // the first partial sums
};

// The rows of group or piece number `index`, and where its product goes: to the result where it is all of a group, else to the partial sums
template <bool PIECES>
__device__ __forceinline__ bool weight_span(const WeightArgs &p, int index, Span *s, Sink *sink)
{
    int64_t at;
    *sink = p.sink;
    if (PIECES && p.step) {
        int slot;
        if (!find_piece<true>(p.ptr, p.n_groups, p.n_rows, p.step, index, s, &slot)) return false;
        int32_t lo, hi;
        group_range(p.ptr, s->group, p.n_groups, p.n_rows, &lo, &hi);
        at = s->group;
        if (hi - lo > p.step) {
            if (slot >= p.slots) return false;      // (overlapping groups)
            *sink = Sink{p.part, p.sink.ld, nullptr, p.sink.n_cols, 0, 0, 0};
            at = slot;
        }
    } else {
        s->group = index;
        group_range(p.ptr, index, p.n_groups, p.n_rows, &s->row, &s->end);
        at = index;
    }
    sink->out = static_cast<char *>(sink->out) + at * p.d_in * p.d_out * (sink->bf16 ? 2 : 4);
    return true;
}

// weights' gradient: tiles of [d_in x d_out] per group, or, but for LARGE, per piece of `step` rows (joined by sum_pieces_kernel)
template <typename T, Kind KIND, bool ODD>
__global__ __launch_bounds__(kind_threads(KIND)) __attribute__((amdgpu_waves_per_eu(2))) void grouped_weight_kernel(const WeightArgs p)
{
    using K = KindTile<T, KIND, false, false, ODD>;
    constexpr int BM = kind_rows(KIND), BN = kind_cols(KIND);
    __shared__ __attribute__((aligned(16))) char lds[2 * K::kStage];
    const int tiles = p.row_tiles * p.col_tiles, index = static_cast<int>(blockIdx.x) / tiles;
    Span s;
    Sink sink;
    if (!weight_span<KIND != LARGE>(p, index, &s, &sink)) return;
    int row, col;
    band_order(static_cast<int>(blockIdx.x) % tiles, p.row_tiles, p.col_tiles, kBandRows / BM, &row, &col);
    const int row0 = row * BM, col0 = col * BN;
    typename K::A a;
    typename K::B b;
    a.base = static_cast<const T *>(p.a) + s.row * p.ld_a;
    a.ld = p.ld_a; a.rows = p.d_in - row0; a.col0 = row0; a.depth = s.end - s.row;
    b.base = static_cast<const T *>(p.dz) + s.row * p.ld_dz;
    b.ld = p.ld_dz; b.rows = p.d_out - col0; b.col0 = col0; b.depth = a.depth;
    typename K::Acc acc;
    run_kind<K, KIND>(a, b, lds, acc);
    K::put(sink, acc, row0, p.d_in, col0);
}

// ---- widths of less than 16 bytes: plain sums ------------------------------------------------------------------
// 100 k rows over 5 groups: 500 -> 3 fp32 368 us forward (201 MB, which HBM allows in 39), 120 and 451 for the gradients of rows and weights;
// 64 -> 7 bf16 85, 39 and 183.
__device__ __forceinline__ void put1(const Sink &p, float v, int64_t row, int col)
{
    if (p.bias) v += p.bias[col];
    if (p.relu && v < 0.f) v = 0.f;
    if (p.bf16) {
        Bf16 *o = static_cast<Bf16 *>(p.out) + row * p.ld + col;
        from_f32(v + (p.add ? to_f32(*o) : 0.f), *o);
    } else {
        float *o = static_cast<float *>(p.out) + row * p.ld + col;
        *o = v + (p.add ? *o : 0.f);
    }
}

// blocks of 64 rows of a group; a thread per element
template <typename T, bool B_ALONG>
__global__ __launch_bounds__(256) void tiny_rows_kernel(const RowsArgs p)
{
    Span s;
    if (!find_piece(p.ptr, p.n_groups, p.n_rows, 64, static_cast<int>(blockIdx.x) / p.col_tiles, &s)) return;
    const T *w = static_cast<const T *>(p.w) + s.group * p.w_group;
    Sink sink = p.sink;
    if (sink.bias) sink.bias += static_cast<int64_t>(s.group) * sink.n_cols;
    const int col0 = static_cast<int>(blockIdx.x) % p.col_tiles * 64, cols = min(64, sink.n_cols - col0);
    for (int e = threadIdx.x; e < (s.end - s.row) * cols; e += 256) {
        const int64_t row = s.row + e / cols;
        const int col = col0 + e % cols;
        const T *a = static_cast<const T *>(p.a) + row * p.ld_a;
        float sum = 0.f;
        for (int k = 0; k < p.depth; ++k) sum += to_f32(a[k]) * to_f32(B_ALONG ? w[static_cast<int64_t>(col) * p.ld_w + k] : w[static_cast<int64_t>(k) * p.ld_w + col]);
        put1(sink, sum, row, col);
    }
}

// a block per group or piece and 256 elements of the result
template <typename T>
__global__ __launch_bounds__(256) void tiny_weight_kernel(const WeightArgs p)
{
    const int tiles = p.row_tiles * p.col_tiles, index = static_cast<int>(blockIdx.x) / tiles;
    Span s;
    Sink sink;
    if (!weight_span<true>(p, index, &s, &sink)) return;
    const int64_t e = static_cast<int64_t>(blockIdx.x % tiles) * 256 + threadIdx.x;
    if (e >= static_cast<int64_t>(p.d_in) * p.d_out) return;
    const int k = static_cast<int>(e / p.d_out), n = static_cast<int>(e % p.d_out);
    float sum = 0.f;
    for (int64_t r = s.row; r < s.end; ++r) sum += to_f32(static_cast<const T *>(p.a)[r * p.ld_a + k]) * to_f32(static_cast<const T *>(p.dz)[r * p.ld_dz + n]);
    put1(sink, sum, k, n);
}

// out[g] (+)= the sum of the partial sums of the group's pieces, `width` values each: the wavefronts of a block share them,
// each front to back.  `whole`: what a group of one piece has is in `out` already, and there are no partial sums of it.
constexpr int kJoinWaves = 16, kJoinCols = 4;
struct JoinArgs {
    const float *part;
    const int64_t *ptr;
    void *out;
    int64_t n_rows, width;
    int32_t n_groups, step, most, bf16, add, whole;
};
// the values of columns [col, col + kJoinCols), those from c on
template <typename Out>
__device__ __forceinline__ void put_own(Out *row, float (&v)[kJoinCols], int64_t c, int64_t col, int64_t width, bool add)
{
    if (c == col && c + kJoinCols <= width) {
        put_cols<kJoinCols>(row + c, v, kJoinCols, add);
    } else {
#pragma unroll
        for (int e = 0; e < kJoinCols; ++e)
            if (col + e >= c && col + e < width) from_f32(v[e] + (add ? to_f32(row[col + e]) : 0.f), row[col + e]);
    }
}
__global__ __launch_bounds__(64 * kJoinWaves) void sum_pieces_kernel(const JoinArgs p)
{
    __shared__ float joined[kJoinCols][kJoinWaves][64];
    const int g = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t lo, hi;
    group_range(p.ptr, g, p.n_groups, p.n_rows, &lo, &hi);
    const int64_t base = static_cast<int64_t>(g) * p.width;
    if (lo == hi) {
        if (p.add) return;
        for (int64_t c = static_cast<int64_t>(blockIdx.x) * 64 * kJoinWaves + threadIdx.x; c < p.width; c += static_cast<int64_t>(gridDim.x) * 64 * kJoinWaves) {
            if (p.bf16) static_cast<Bf16 *>(p.out)[base + c].bits = 0;
            else static_cast<float *>(p.out)[base + c] = 0.f;
        }
        return;
    }
    if (p.whole && hi - lo <= p.step) return;
    // (overlapping groups could have more pieces than there is room for)
    const int first = count_pieces(p.ptr, g, p.n_rows, p.step, p.most, p.whole ? 2 : 1), count = min(pieces_in(hi - lo, p.step), p.most - first);
    // four pieces at least to a wavefront; the wavefronts that are left take other columns
    int split = 1;
    while (split < kJoinWaves && count >= 8 * split) split *= 2;
    const int share = wave % split, from = share * count / split, to = (share + 1) * count / split;
    const int64_t block_cols = kJoinWaves / split * 64 * kJoinCols;
    for (int64_t c0 = static_cast<int64_t>(blockIdx.x) * block_cols; c0 < p.width; c0 += static_cast<int64_t>(gridDim.x) * block_cols) {
        // (the last columns' vector is moved back to end with the row; what it has of its neighbour's is not written)
        const int64_t c = c0 + (wave / split * 64 + lane) * kJoinCols, col = max(min(c, p.width - kJoinCols), static_cast<int64_t>(0));
        float sum[kJoinCols] = {};
        if (p.width >= kJoinCols) {
#pragma unroll 4
            for (int i = from; i < to; ++i) {
                float x[kJoinCols];
                load_n<kJoinCols>(p.part + (first + i) * p.width + col, x);
#pragma unroll
                for (int e = 0; e < kJoinCols; ++e) sum[e] += x[e];
            }
        } else {
#pragma unroll 4
            for (int i = from; i < to; ++i)
#pragma unroll
                for (int e = 0; e < kJoinCols; ++e) sum[e] += p.part[(first + i) * p.width + min(static_cast<int64_t>(e), p.width - 1)];
        }
        if (split > 1) {
#pragma unroll
            for (int e = 0; e < kJoinCols; ++e) joined[e][wave][lane] = sum[e];
            __syncthreads();
            if (share == 0) {
                for (int w = 1; w < split; ++w)
#pragma unroll
                    for (int e = 0; e < kJoinCols; ++e) sum[e] += joined[e][wave + w][lane];
            }
        }
        if (share == 0 && c < p.width) {
            if (p.bf16) put_own(static_cast<Bf16 *>(p.out) + base, sum, c, col, p.width, p.add);
            else put_own(static_cast<float *>(p.out) + base, sum, c, col, p.width, p.add);
        }
        if (split > 1) __syncthreads();
    }
}

// dz = grad_out where out > 0 (RELU; written for the two products), and its column sums over pieces of rows.  Bound by HBM.
struct MaskArgs {
    const void *grad, *out;
    void *dz;               // NULL: grad is dz already
    float *part;            // NULL: no column sums
    const int64_t *ptr;
    int64_t n_rows, ld_grad, ld_out, ld_dz;
    int32_t n_groups, d_out, out_bf16, lanes_log2, step;
};
// 2^lanes_log2 lanes take a row, V columns each; a wavefront 64 / 2^lanes_log2 rows at a time
template <typename T, int V>
__global__ __launch_bounds__(256) void mask_rows_kernel(const MaskArgs p)
{
    __shared__ float joined[256 * V];
    Span s;
    if (!find_piece(p.ptr, p.n_groups, p.n_rows, p.step, static_cast<int>(blockIdx.x), &s)) return;
    const int lanes = 1 << p.lanes_log2, groups = 256 >> p.lanes_log2, group = threadIdx.x >> p.lanes_log2;
    const int64_t c = ((static_cast<int64_t>(blockIdx.y) << p.lanes_log2) + (threadIdx.x & (lanes - 1))) * V;
    const int64_t col = c + V <= p.d_out ? c : p.d_out - V;         // the last vector ends with the row; the columns before c are its neighbour's
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    if (c < p.d_out) {
        constexpr int U = 4;
        for (int64_t r0 = s.row + group; r0 < s.end; r0 += U * groups) {
            float g[U][V], o[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t r = min(r0 + u * groups, static_cast<int64_t>(s.end) - 1);
                load_n<V>(static_cast<const T *>(p.grad) + r * p.ld_grad + col, g[u]);
                if (p.out) {
                    if (p.out_bf16) load_n<V>(static_cast<const Bf16 *>(p.out) + r * p.ld_out + col, o[u]);
                    else load_n<V>(static_cast<const float *>(p.out) + r * p.ld_out + col, o[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r0 + u * groups >= s.end) break;
                if (p.out) {
#pragma unroll
                    for (int e = 0; e < V; ++e) g[u][e] = o[u][e] > 0.f ? g[u][e] : 0.f;
                }
                if (p.dz) store_n<V>(static_cast<T *>(p.dz) + (r0 + u * groups) * p.ld_dz + col, g[u]);
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += g[u][e];
            }
        }
    }
    if (!p.part) return;
#pragma unroll
    for (int e = 0; e < V; ++e) joined[e * 256 + threadIdx.x] = sum[e];
    __syncthreads();
    if (group != 0 || c >= p.d_out) return;
    for (int i = 1; i < groups; ++i) {
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += joined[e * 256 + (i << p.lanes_log2) + threadIdx.x];
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (col + e >= c) p.part[static_cast<int64_t>(blockIdx.x) * p.d_out + col + e] = sum[e];
}

// ---- which tiles ---------------------------------------------------------------------------------------------
constexpr int kCus = 256;

// LARGE or MEDIUM, by how often the chip is filled: a CU takes one large tile at a time or two medium ones, and a large one (four
// times the work) takes some 2.9 times as long as a medium one beside another
bool large_pays(int64_t large_tiles, int64_t medium_tiles) { return ceil_div(large_tiles, kCus) * 29 <= ceil_div(medium_tiles, 2 * kCus) * 20; }

struct GradPlan {
    bool tiny;
    Kind kind;
    int32_t step;                   // rows of a piece of the weights' gradient, 0: groups whole
    int64_t row_tiles, col_tiles;
    int64_t pieces, mask_pieces;    // at most
    int64_t slots;                  // partial sums: pieces of groups longer than one piece, at most
    int32_t mask_step;
    int64_t ld_dz;
    size_t dz, part, bias_part, bytes;
};

GradPlan plan_grad(int64_t n_rows, int32_t n_groups, int32_t d_in, int32_t d_out, mgg_dtype_t dtype, bool relu)
{
    GradPlan g{};
    const int32_t chunk = dtype == MGG_BF16 ? 8 : 4;
    const int64_t present = n_groups < n_rows ? n_groups : n_rows;      // groups that can have rows
    g.tiny = d_in < chunk || d_out < chunk;
    g.kind = dtype == MGG_F32 || (d_in <= 64 && d_out <= 64) ? SMALL : (d_out > 64 ? MEDIUM : NARROW);
    if (dtype == MGG_BF16 && g.kind == MEDIUM && d_in % chunk == 0 && d_out % chunk == 0 &&
        large_pays(n_groups * ceil_div(d_in, 256) * ceil_div(d_out, 256), n_groups * ceil_div(d_in, 128) * ceil_div(d_out, 128)))
        g.kind = LARGE;
    g.row_tiles = g.tiny ? ceil_div(static_cast<int64_t>(d_in) * d_out, 256) : ceil_div(d_in, kind_rows(g.kind));
    g.col_tiles = g.tiny ? 1 : ceil_div(d_out, kind_cols(g.kind));
    // pieces of rows where the tiles of the groups do not fill the chip (counted as if one group had all rows)
    const int64_t tiles = g.row_tiles * g.col_tiles;
    g.pieces = n_groups;
    if (g.kind != LARGE && tiles < kCus && n_rows > 0) {
        const int64_t step = ceil_div(ceil_div(n_rows, ceil_div(2 * kCus, tiles)), 64) * 64;
        g.step = static_cast<int32_t>(step < 256 ? 256 : (step < (1 << 30) ? step : 1 << 30));
        g.pieces = n_rows / g.step + present;
        // (ceil(c / step) is at most 2 floor(c / step) where c > step)
        const int64_t full = n_rows / g.step;
        g.slots = n_rows <= g.step ? 0 : (full < present ? 2 * full : full + present);
    }
    // some 2048 blocks of the mask, 64 rows and 64 x 16 bytes at least
    g.mask_step = static_cast<int32_t>(ceil_div(ceil_div(n_rows * ceil_div(d_out, 64 * chunk), 2048), 64) * 64);
    if (g.mask_step < 64) g.mask_step = 64;
    g.mask_pieces = n_rows / g.mask_step + present;
    g.ld_dz = static_cast<int64_t>(round_up(static_cast<size_t>(d_out), 8));
    size_t at = 0;
    g.dz = at; at += relu ? round_up(static_cast<size_t>(n_rows) * g.ld_dz * (dtype == MGG_BF16 ? 2 : 4), 256) : 0;
    g.part = at; at += round_up(static_cast<size_t>(g.slots) * d_in * d_out * 4, 256);
    g.bias_part = at; at += round_up(static_cast<size_t>(g.mask_pieces) * d_out * 4, 256);
    g.bytes = at + 256;
    return g;
}

mgg_status_t launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, what);
}

// dry: nothing is launched, the answer is whether it could be
template <typename T, bool B_ALONG, bool ODD>
mgg_status_t rows_product(RowsArgs p, bool dry, hipStream_t stream)
{
    constexpr int N = Elem<T>::N;
    const int32_t cols = p.sink.n_cols;
    const int64_t present = p.n_groups < p.n_rows ? p.n_groups : p.n_rows;
    auto grid = [&](int rows, int tile_cols) {
        p.col_tiles = static_cast<int32_t>(ceil_div(cols, tile_cols));
        const int64_t most = p.n_rows / rows + present;
        p.most = static_cast<int32_t>(most < INT32_MAX ? most : INT32_MAX);
        return most * p.col_tiles;
    };
    const char *const refused = "too many tiles for one launch";
#define MGG_GRID(ROWS, COLS, THREADS)                                                      \
    const int64_t blocks = grid(ROWS, COLS);                                               \
    if (!launchable(blocks, THREADS)) return fail(MGG_ERR_UNSUPPORTED, "%s", refused);      \
    if (dry) return MGG_OK;                                                                \
    const dim3 blocks_dim(static_cast<unsigned>(blocks))
    if (cols < N || p.depth < N) {
        MGG_GRID(64, 64, 256);
        hipLaunchKernelGGL((tiny_rows_kernel<T, B_ALONG>), blocks_dim, dim3(256), 0, stream, p);
        return launched("grouped product launch");
    }
    // few rows to a group, where reading the weights is what takes the time, or tiles too few to fill the chip, where the depth is
    // (1500 rows over 2 groups 2048 -> 1024, 104 tiles of 128 x 128: 26 us, with those 41; 2500 rows: 36 and 42; 3000 rows 512 -> 1024, 192
    // tiles: 19 and 18; fp32 512 rows 2048 -> 1024: 33 and 72)
    const int64_t tiles = (p.n_rows / 128 + present / 2 + 1) * ceil_div(cols, 128);
    if (p.n_rows <= 24 * static_cast<int64_t>(p.n_groups) || tiles <= kCus / 2) {
        // (8 wavefronts where blocks are few; 64 rows over 64 groups 1024 -> 2048 with 4: 40 us, with 8: 50; one row 4096 -> 4096 with
        // 8: 23 us, with 4: 27, as its 64 blocks fill a quarter of the chip)
        MGG_GRID(32, 64, blocks < 2 * kCus ? 512 : 256);
        if (blocks < 2 * kCus) hipLaunchKernelGGL((grouped_few_rows_kernel<T, 64, 8, B_ALONG, ODD>), blocks_dim, dim3(512), 0, stream, p);
        else hipLaunchKernelGGL((grouped_few_rows_kernel<T, 64, 4, B_ALONG, ODD>), blocks_dim, dim3(256), 0, stream, p);
        return launched("grouped product launch");
    }
    if constexpr (!ODD && sizeof(T) == 2) {
        // (a group's last piece is half full on average; one group's pieces are known.  One group 4096 -> 32000, microseconds with large and
        // medium tiles: 25 rows 93 and 73, 128 rows 93 and 74, 256 rows 99 and 102, 300 rows 113 and 156; 2048 -> 128000, 200 rows: 133
        // and 199)
        auto pieces = [&](int rows) {
            const int64_t some = p.n_rows / rows + present / 2, least = ceil_div(p.n_rows, rows);
            return some > least ? some : least;
        };
        if (large_pays(pieces(256) * ceil_div(cols, 256), pieces(128) * ceil_div(cols, 128))) {
            MGG_GRID(256, 256, 512);
            hipLaunchKernelGGL((grouped_rows_kernel<T, LARGE, B_ALONG, ODD>), blocks_dim, dim3(512), 0, stream, p);
            return launched("grouped product launch");
        }
    }
    if constexpr (sizeof(T) == 4) {
        MGG_GRID(64, 64, 256);
        hipLaunchKernelGGL((grouped_rows_kernel<T, SMALL, B_ALONG, ODD>), blocks_dim, dim3(256), 0, stream, p);
        return launched("grouped product launch");
    } else if (cols <= 64) {
        MGG_GRID(128, 64, 256);
        hipLaunchKernelGGL((grouped_rows_kernel<T, NARROW, B_ALONG, ODD>), blocks_dim, dim3(256), 0, stream, p);
    } else {
        MGG_GRID(128, 128, 256);
        hipLaunchKernelGGL((grouped_rows_kernel<T, MEDIUM, B_ALONG, ODD>), blocks_dim, dim3(256), 0, stream, p);
    }
#undef MGG_GRID
    return launched("grouped product launch");
}

template <typename T>
mgg_status_t rows_product_of(const RowsArgs &p, bool b_along, bool dry, hipStream_t stream)
{
    const bool odd = p.depth % Elem<T>::N != 0 || p.sink.n_cols % Elem<T>::N != 0;
    if (b_along) return odd ? rows_product<T, true, true>(p, dry, stream) : rows_product<T, true, false>(p, dry, stream);
    return odd ? rows_product<T, false, true>(p, dry, stream) : rows_product<T, false, false>(p, dry, stream);
}

template <typename T, bool ODD>
mgg_status_t weight_product(WeightArgs p, const GradPlan &g, bool dry, hipStream_t stream)
{
    p.row_tiles = static_cast<int32_t>(g.row_tiles);
    p.col_tiles = static_cast<int32_t>(g.col_tiles);
    const int threads = !g.tiny && g.kind == LARGE ? 512 : 256;
    if (g.row_tiles > INT32_MAX || g.pieces * g.row_tiles > INT32_MAX / g.col_tiles || !launchable(g.pieces * g.row_tiles * g.col_tiles, threads))
        return fail(MGG_ERR_UNSUPPORTED, "too many tiles for one launch");
    if (dry) return MGG_OK;
    const dim3 grid(static_cast<unsigned>(g.pieces * g.row_tiles * g.col_tiles));
    if (g.tiny) hipLaunchKernelGGL((tiny_weight_kernel<T>), grid, dim3(256), 0, stream, p);
    else if (g.kind == SMALL) hipLaunchKernelGGL((grouped_weight_kernel<T, SMALL, ODD>), grid, dim3(256), 0, stream, p);
    else if constexpr (sizeof(T) == 2) {
        if (g.kind == MEDIUM) hipLaunchKernelGGL((grouped_weight_kernel<T, MEDIUM, ODD>), grid, dim3(256), 0, stream, p);
        else if (g.kind == NARROW) hipLaunchKernelGGL((grouped_weight_kernel<T, NARROW, ODD>), grid, dim3(256), 0, stream, p);
        else if constexpr (!ODD) hipLaunchKernelGGL((grouped_weight_kernel<T, LARGE, ODD>), grid, dim3(512), 0, stream, p);
    }
    return launched("grouped weight gradient launch");
}

template <typename T>
mgg_status_t weight_product_of(const WeightArgs &p, const GradPlan &g, bool dry, hipStream_t stream)
{
    return p.d_in % Elem<T>::N != 0 || p.d_out % Elem<T>::N != 0 ? weight_product<T, true>(p, g, dry, stream) : weight_product<T, false>(p, g, dry, stream);
}

mgg_status_t join_pieces(const JoinArgs &p, hipStream_t stream)
{
    const int64_t columns = ceil_div(p.width, 64 * kJoinCols), some = 1024 / p.n_groups + 1;
    hipLaunchKernelGGL(sum_pieces_kernel, dim3(static_cast<unsigned>(columns < some ? columns : some), p.n_groups), dim3(64 * kJoinWaves), 0, stream, p);
    return launched("partial sum launch");
}

template <typename T>
mgg_status_t mask_rows(MaskArgs m, int64_t pieces, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T);
    const int64_t vecs = m.d_out < V ? m.d_out : ceil_div(m.d_out, V);
    m.lanes_log2 = ceil_log2(vecs) < 6 ? ceil_log2(vecs) : 6;
    const dim3 grid(static_cast<unsigned>(pieces), static_cast<unsigned>(ceil_div(vecs, static_cast<int64_t>(1) << m.lanes_log2)));
    if (m.d_out < V) hipLaunchKernelGGL((mask_rows_kernel<T, 1>), grid, dim3(256), 0, stream, m);
    else hipLaunchKernelGGL((mask_rows_kernel<T, V>), grid, dim3(256), 0, stream, m);
    return launched("mask launch");
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
    return dtype == MGG_BF16 ? rows_product_of<Bf16>(p, false, false, stream) : rows_product_of<float>(p, false, false, stream);
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
    auto rows = [&](bool dry) {
        RowsArgs p{};
        p.a = dz; p.w = q.w; p.ptr = q.group_ptr; p.n_rows = q.n_rows; p.ld_a = ld_dz; p.n_groups = q.n_groups;
        p.w_group = static_cast<int64_t>(q.d_in) * q.d_out; p.ld_w = q.d_out; p.depth = q.d_out;
        p.sink = Sink{q.grad_a, q.ld_grad_a, nullptr, q.d_in, q.grad_a_dtype == MGG_BF16, 0, 0};
        return bf16 ? rows_product_of<Bf16>(p, true, dry, stream) : rows_product_of<float>(p, true, dry, stream);
    };
    auto weights = [&](bool dry) {
        WeightArgs p{};
        p.a = q.a; p.dz = dz; p.ptr = q.group_ptr; p.n_rows = q.n_rows; p.ld_a = q.ld_a; p.ld_dz = ld_dz;
        p.n_groups = q.n_groups; p.d_in = q.d_in; p.d_out = q.d_out; p.step = g.step; p.slots = static_cast<int32_t>(g.slots);
        p.sink = Sink{q.grad_w, q.d_out, nullptr, q.d_out, q.grad_w_dtype == MGG_BF16, 0, q.add_w};
        p.part = reinterpret_cast<float *>(ws + g.part);
        return bf16 ? weight_product_of<Bf16>(p, g, dry, stream) : weight_product_of<float>(p, g, dry, stream);
    };
    // what does not fit a launch is refused before anything is written
    if (q.grad_a && (s = rows(true)) != MGG_OK) return s;
    if (q.grad_w && (s = weights(true)) != MGG_OK) return s;
    if (q.n_rows > 0 && (q.grad_bias || (q.relu && (q.grad_a || q.grad_w)))) {
        MaskArgs m{};
        m.grad = q.grad_out; m.ptr = q.group_ptr; m.n_rows = q.n_rows; m.ld_grad = q.ld_grad; m.n_groups = q.n_groups; m.d_out = q.d_out; m.step = g.mask_step;
        if (q.relu) {
            m.out = q.out; m.ld_out = q.ld_out; m.out_bf16 = q.out_dtype == MGG_BF16;
            if (q.grad_a || q.grad_w) { m.dz = ws + g.dz; m.ld_dz = g.ld_dz; dz = m.dz; ld_dz = m.ld_dz; }
        }
        if (q.grad_bias) m.part = reinterpret_cast<float *>(ws + g.bias_part);
        s = bf16 ? mask_rows<Bf16>(m, g.mask_pieces, stream) : mask_rows<float>(m, g.mask_pieces, stream);
        if (s != MGG_OK) return s;
    }
    if (q.grad_bias) {
        s = join_pieces(JoinArgs{reinterpret_cast<float *>(ws + g.bias_part), q.group_ptr, q.grad_bias, q.n_rows, q.d_out, q.n_groups, g.mask_step,
                                 static_cast<int32_t>(g.mask_pieces), 0, q.add_bias, 0}, stream);
        if (s != MGG_OK) return s;
    }
    if (q.grad_a) {
        s = rows(false);
        if (s != MGG_OK) return s;
    }
    if (q.grad_w) {
        s = weights(false);
        if (s != MGG_OK || !g.step) return s;
        s = join_pieces(JoinArgs{reinterpret_cast<float *>(ws + g.part), q.group_ptr, q.grad_w, q.n_rows, static_cast<int64_t>(q.d_in) * q.d_out, q.n_groups, g.step,
                                 static_cast<int32_t>(g.slots), q.grad_w_dtype == MGG_BF16, q.add_w, 1}, stream);
    }
    return s;
}

}  // namespace mgg
