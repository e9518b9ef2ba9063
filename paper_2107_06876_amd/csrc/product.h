// Matrix products of the embedding operators on the bf16 matrix instruction: the sum over k of A[m][k] B[n][k],
// both operands in memory as planes of bf16, with an epilogue that reads the accumulators in registers.
//
// bf16 inputs are one plane.  A float x is three: x1 = bf16(x), x2 = bf16(x - x1), x3 = bf16(x - x1 - x2); what is left
// is below 2^-26 |x|.  Of the nine products of planes the six with x_i y_j, i + j <= 4, are added (the others are below
// 2^-25 of the product), the small ones first.  Six bf16 products cost less than one on the fp32 matrix instruction,
// whose rate is 1/16.  Two planes of the second operand alone (two products) serve where a rounding of it to one would
// show in the result.
//
// An operand is stored either with k contiguous (`rows`: A[m][k] at m * ld + k) or with its own index contiguous
// (`columns`: A[k][m] at k * ld + m).  Tiles of 32 or 64 values of k go from memory straight into LDS (16 bytes a lane; what is
// outside the operand is read as zero by the buffer's bounds), two tiles of LDS in turn, so that the next tile is on its
// way while the matrix instructions work on this one.  The 16-byte pieces of a tile are permuted so that neither the
// 128-bit reads of `rows` tiles nor the transposing 64-bit reads of `columns` tiles meet in a bank.
//
// The accumulators' row index (four consecutive values in a lane) is m: outputs are stored with m contiguous.
//
// Bound by the matrix instruction while k is long: 8192^3 in bf16 1.25 PFLOP/s (the library's product there 1.14), in three
// planes 233 TFLOP/s of float products (library 154).  With short k the epilogue counts, which nothing overlaps (a
// workgroup of the largest shape fills a compute unit): bf16, 16384 rows, 4096 -> 1024 values 1.3 PFLOP/s, 1024 -> 4096
// 0.95, k = 300 0.72.  A resident workgroup that loads its next tile during the epilogue was 1 to 3 % faster and spilled; not kept.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lcn {

// ---- launches of many workgroups --------------------------------------------
// A dimension of a grid has fewer than 2^32 threads; what is beyond is cut off without an error.  More workgroups than GRID_ROW
// are laid out in rows of so many, which are numbered through (the last row may be longer than what is left).
constexpr long long GRID_ROW = 1 << 22;
inline dim3 grid_of(long long groups)
{
    return groups <= GRID_ROW ? dim3((unsigned)groups) : dim3((unsigned)GRID_ROW, (unsigned)((groups + GRID_ROW - 1) / GRID_ROW));
}
__device__ __forceinline__ unsigned group_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct Operand {
    const void *p;     // first plane, 16-byte aligned
    long long plane;   // bytes from one plane to the next
    long long ld;      // elements from a row (`rows`) or a k (`columns`) to the next, a multiple of 8
};

struct ProductArgs {
    Operand a, b;
    int m, n, k;         // k is padded by zeros up to a multiple of 8 in `rows` operands
    int planes;          // 1; 2: two of the second operand; 3: three of both
    int splits;          // workgroups that share a tile's k
    int tiles_m, tiles_n;   // their product is below 2^31 (sizes_fit)
    int n_first, n_last;   // the columns of a launch
};

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Permutation of the 16-byte pieces of a tile of BK values of k: of row r (`rows`), of value k (`columns`, W indices wide).  A 128-bit
// read is served for lanes 0 .. 3, 12 .. 15 and 20 .. 27 of a half at a time, then for its others: with BK = 32 and (r >> 2) & 3
// every read met another in its bank, as counted (two planes, 128 x 128 tiles, 4 products of 1024^3: 49 us, with this 45).
template <int BK>
__device__ __forceinline__ int rows_swizzle(int r) { return BK == 64 ? (r >> 1) & 7 : (r >> 3 & 1) * 3; }
template <int W>
__device__ __forceinline__ int columns_swizzle(int k)
{
    if (W % 128 == 0) return ((k & 3) | ((k >> 1) & 4)) << 1;
    if (W % 64) return (k >> 3 & 1) << 1;
    return (((k >> 1) & 1) | ((k >> 2) & 2)) << 1;
}

// Whether an epilogue takes the rows of the first operand in pairs: the matrix has 2 m rows, row i and row m + i belong together, and
// of every 32 rows of a tile 16 are rows i .. i + 15 and 16 are rows m + i .. m + i + 15, so that a lane gets both.
template <class Epi>
constexpr bool paired_rows = false;

// One operand's part of the tiles of a workgroup: W indices from i0, BK values of k at a time, into LDS.
template <int W, int BK, bool COLUMNS, int THREADS, bool PAIRED = false>
struct TileLoader {
    static constexpr int PIECES = W * BK / 8, LOADS = (PIECES + THREADS - 1) / THREADS;   // 16 bytes each
    static_assert(PIECES % 64 == 0, "whole wavefronts of pieces");
    static constexpr int ROW = COLUMNS ? W / 8 : BK / 8;   // pieces of a row of the tile
    // From one of a thread's pieces to the next: so many rows, the same place in them where that is a whole number that
    // the permutation does not see.
    static constexpr bool EVEN = THREADS % ROW == 0 && THREADS / ROW % 16 == 0;
    static constexpr int KEPT = EVEN ? 1 : LOADS;
    static_assert(!PAIRED || (!COLUMNS && (LOADS == 1 || THREADS / ROW % 32 == 0)), "a wavefront's loads are all of one half");
    const char *first;        // the workgroup's first index, k = 0, first plane
    long long k_bytes;        // from one tile's k to the next
    unsigned row_bytes, tail; // from a row to the next; bytes of the last row that are read
    int rows;                 // `rows`: rows there are
    unsigned off[KEPT];
    int need[KEPT];           // `rows`: values of k the piece needs to be left

    __device__ __forceinline__ void init(const Operand &o, long long i0, int count, int wave, int lane)
    {
        const int left = count - (int)i0;
        row_bytes = (unsigned)(o.ld * 2);
        first = (const char *)o.p + (COLUMNS ? i0 : i0 * o.ld) * 2;
        if (PAIRED && (wave * (64 / ROW) >> 4) & 1) first += count * o.ld * 2;
        k_bytes = COLUMNS ? (long long)BK * o.ld * 2 : BK * 2;
        rows = left < W / (PAIRED ? 2 : 1) ? left : W / (PAIRED ? 2 : 1);
        tail = (unsigned)(((left + 7) & ~7) * 2);
#pragma unroll
        for (int u = 0; u < KEPT; ++u) {
            const int c = (u * (THREADS / 64) + wave) * 64 + lane, row = c / ROW;
            const int piece = (c % ROW) ^ (COLUMNS ? columns_swizzle<W>(row) : rows_swizzle<BK>(row));
            off[u] = (unsigned)(PAIRED ? (row >> 5) * 16 + (row & 15) : row) * row_bytes + (unsigned)piece * 16;
            need[u] = piece * 8;
            if (COLUMNS && piece * 8 >= left) off[u] = 0x80000000u;   // outside, also with rows added
        }
    }
    // tile number `step` of the plane that lies `plane` bytes behind the first; k: all values of k
    __device__ __forceinline__ void load(long long plane, int step, int k, char *lds, int wave) const
    {
        const int left = k - step * BK;
        const char *base = first + plane + step * k_bytes;
        const int r = COLUMNS ? (left < BK ? left : BK) : rows;
        const unsigned end = COLUMNS ? tail : (unsigned)(((left + 7) & ~7) * 2);
        __amdgpu_buffer_rsrc_t res =
            __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (unsigned)(r - 1) * row_bytes + end, 0x00020000);
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            if (PIECES % THREADS && (u * (THREADS / 64) + wave) * 64 >= PIECES) break;
            unsigned o = off[EVEN ? 0 : u];
            if (!COLUMNS) o = need[EVEN ? 0 : u] < left ? o : 0x80000000u;
            if (EVEN) o += u * (THREADS / ROW) / (PAIRED ? 2 : 1) * row_bytes;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (lds_void *)(lds + (u * (THREADS / 64) + wave) * 1024), 16, (int)o,
                                                     0, 0, 0);
        }
    }
};

// The matrix instruction's operand for indices i .. i + 15 (i a multiple of 16) and the 32 values of k from 32 kk: lane l
// has index i + l % 16 and k = 32 kk + 8 (l / 16) + 0 .. 7.  `at` is the lane's place for i = 0 and kk = 0.
template <int W, int BK, bool COLUMNS>
__device__ __forceinline__ int fragment_place(int lane)
{
    if constexpr (!COLUMNS) {
        return (lane & 15) * (BK * 2) + (((lane >> 4) ^ rows_swizzle<BK>(lane & 15)) << 4);
    } else {
        // a group of 16 lanes reads 4 values of k x 16 indices, each lane 4 indices of one k, and gets 4 values of
        // k of one index; the second read is 4 values of k further
        const int k = (lane >> 4) * 8 + ((lane & 15) >> 2);
        return k * (W * 2) + ((((lane & 3) >> 1) ^ columns_swizzle<W>(k)) << 4) + (lane & 1) * 8;
    }
}
template <int W, int BK, bool COLUMNS>
__device__ __forceinline__ bf16x8 load_fragment(const char *lds, int at, int i, int kk)
{
    if constexpr (!COLUMNS) {
        return *(const bf16x8 *)(lds + (at ^ (kk * 64)) + i * (BK * 2));
    } else {
        union {
            s16x4 h[2];
            bf16x8 v;
        } f;
        static_assert(W == 32 || W % 64 == 0, "a row of the tile is whole units of 128 bytes, or half a one");
        constexpr int LOW = W % 128 == 0 ? 255 : W % 64 == 0 ? 127 : 63;   // what the permutation moves within
        const char *q = lds + (at ^ (i * 2 & LOW)) + (i * 2 & ~LOW) + kk * 32 * (W * 2);
        f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)q);
        f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(q + 4 * (W * 2)));
        return f.v;
    }
}

__device__ __forceinline__ f32x4 mfma_bf16(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The tile that a workgroup works on.  Workgroups are dealt to the eight dies in turn: a die gets a run of
// consecutive tiles, and tiles follow each other in strips of four along n, so that the tiles in flight on a die share
// their operands in its cache.
__device__ __forceinline__ void tile_of(const ProductArgs &p, int id, int &tm, int &tn)
{
    const int total = p.tiles_m * p.tiles_n;
    const int base = total / 8, more = total % 8, die = id % 8, nth = id / 8;
    const int t = die * base + (die < more ? die : more) + nth;
    const int strip = t / (4 * p.tiles_m), in = t % (4 * p.tiles_m);
    const int wide = p.tiles_n - strip * 4 < 4 ? p.tiles_n - strip * 4 : 4;
    tm = in / wide;
    tn = strip * 4 + in % wide;
}

// Row by row through LDS: a wavefront's accumulators of 16 columns n (v[i]: rows 16 i + 4 (lane / 16) + 0 .. 3 of column
// lane % 16) come back as pieces of eight consecutive m, neighbours in neighbouring lanes, so that memory is read and written
// in whole lines.  ahead(r, c) is called for every piece before (loads that its store will need), then
// store(r, c, values, what ahead returned), r: column 0 .. 15, c: first m.  `region`: RowRegion<TM>::BYTES of the
// wavefront's own.
template <int TM>
struct RowRegion {
    static constexpr int PITCH = TM * 16 + 4, BYTES = 16 * PITCH * 4;   // 16 rows of a 128-bit write meet in no bank
};
struct Nothing {};
template <int TM, class Ahead, class Store>
__device__ __forceinline__ void by_rows(char *region, const f32x4 (&v)[TM], int lane, Ahead ahead, Store store)
{
    constexpr int PITCH = RowRegion<TM>::PITCH, ROW = 2 * TM, PIECES = 16 * ROW, S = (PIECES + 63) / 64;
    float *f = (float *)region;
    decltype(ahead(0, 0)) early[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int q = s * 64 + lane;
        if (PIECES % 64 == 0 || q < PIECES) early[s] = ahead(q / ROW, q % ROW * 8);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) *(f32x4 *)(f + (lane & 15) * PITCH + i * 16 + 4 * (lane >> 4)) = v[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // LDS serves a wavefront in order
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1   // a loop: unrolled, epilogues with an activation no longer fit beside unrolled accumulators
    for (int q = lane; q < PIECES; q += 64) {
        f32x4 w[2];
        w[0] = *(const f32x4 *)(f + q / ROW * PITCH + q % ROW * 8);
        w[1] = *(const f32x4 *)(f + q / ROW * PITCH + q % ROW * 8 + 4);
        store(q / ROW, q % ROW * 8, w, early[0]);
#pragma unroll
        for (int s = 0; s + 1 < S; ++s) early[s] = early[s + 1];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// WM x WN wavefronts of 64, each BM/WM x BN/WN of the tile; NP: 3 planes of both operands at a time, or 1.  Epi: struct with Args and
// run<TM, TN, WM, WN>(args, product args, acc, m0, n0, split, lds, tile) for the wavefront's accumulators.
template <int BM, int BN, int BK, int WM, int WN, int NP, bool ACOL, bool BCOL, class Epi>
__global__ __launch_bounds__(WM *WN * 64, 2) void product_kernel(ProductArgs p, typename Epi::Args e)
{
    constexpr int THREADS = WM * WN * 64, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int ABYTES = BM * BK * 2, BBYTES = BN * BK * 2;
    constexpr int ROWS = WM * WN * RowRegion<TM>::BYTES, TILE = NP * (ABYTES + BBYTES);
    __shared__ __align__(1024) char lds0[TILE > ROWS ? TILE : ROWS];
    __shared__ __align__(1024) char lds1[TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned id = blockIdx.z * gridDim.x + blockIdx.x;   // y: splits
    if (id >= (unsigned)(p.tiles_m * p.tiles_n)) return;
    int tm, tn;
    tile_of(p, (int)id, tm, tn);
    constexpr int PAIR = paired_rows<Epi> ? 2 : 1;   // rows of the tile that make an index m
    const long long m0 = (long long)tm * (BM / PAIR), n0 = p.n_first + (long long)tn * BN;
    const int wm = (wave % WM) * (BM / WM), wn = (wave / WM) * (BN / WN);

    const int at_a = fragment_place<BM, BK, ACOL>(lane), at_b = fragment_place<BN, BK, BCOL>(lane);
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int ksteps = (p.k + BK - 1) / BK, pairs = NP == 3 ? 1 : p.planes;
    const int all = ksteps * pairs, per = (all + p.splits - 1) / p.splits;
    const int first = (int)blockIdx.y * per, last = first + per < all ? first + per : all;

    TileLoader<BM, BK, ACOL, THREADS, paired_rows<Epi>> load_a;
    TileLoader<BN, BK, BCOL, THREADS> load_b;
    load_a.init(p.a, m0, p.m, wave, lane);
    load_b.init(p.b, n0, p.n, wave, lane);
    int pair = first / ksteps, step = first - pair * ksteps;   // of the next fetch
    auto fetch = [&](char *lds) {
        if constexpr (NP == 3) {
#pragma unroll
            for (int u = 0; u < 3; ++u) {
                load_a.load(u * p.a.plane, step, p.k, lds + u * ABYTES, wave);
                load_b.load(u * p.b.plane, step, p.k, lds + 3 * ABYTES + u * BBYTES, wave);
            }
            ++step;
        } else {   // two planes of B: the second one first
            load_a.load(0, step, p.k, lds, wave);
            load_b.load(pairs == 2 ? (1 - pair) * p.b.plane : 0, step, p.k, lds + ABYTES, wave);
            if (++step == ksteps) {
                step = 0;
                ++pair;
            }
        }
    };
    auto work = [&](const char *lds) {
        // places are formed anew for every tile: kept in registers they would not fit beside the accumulators
        int pa = at_a, pb = at_b;
        asm volatile("" : "+v"(pa), "+v"(pb));
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
            if constexpr (NP == 3) {
                bf16x8 b[3][TN];
#pragma unroll
                for (int u = 0; u < 3; ++u)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        b[u][j] = load_fragment<BN, BK, BCOL>(lds + 3 * ABYTES + u * BBYTES, pb, wn + j * 16, kk);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    bf16x8 a[3];
#pragma unroll
                    for (int u = 0; u < 3; ++u) a[u] = load_fragment<BM, BK, ACOL>(lds + u * ABYTES, pa, wm + i * 16, kk);
                    // the five small products are added up by themselves, so that the sum is rounded twice in a step
                    f32x4 t[TN];
#pragma unroll
                    for (int j = 0; j < TN; ++j) t[j] = mfma_bf16(a[2], b[0][j], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int j = 0; j < TN; ++j) t[j] = mfma_bf16(a[1], b[1][j], t[j]);
#pragma unroll
                    for (int j = 0; j < TN; ++j) t[j] = mfma_bf16(a[0], b[2][j], t[j]);
#pragma unroll
                    for (int j = 0; j < TN; ++j) t[j] = mfma_bf16(a[1], b[0][j], t[j]);
#pragma unroll
                    for (int j = 0; j < TN; ++j) t[j] = mfma_bf16(a[0], b[1][j], t[j]);
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma_bf16(a[0], b[0][j], acc[i][j]) + t[j];
                }
            } else {
                bf16x8 a[TM], b[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) a[i] = load_fragment<BM, BK, ACOL>(lds, pa, wm + i * 16, kk);
#pragma unroll
                for (int j = 0; j < TN; ++j) b[j] = load_fragment<BN, BK, BCOL>(lds + ABYTES, pb, wn + j * 16, kk);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma_bf16(a[i], b[j], acc[i][j]);
            }
        }
    };
    auto arrived = [&]() {   // this wavefront's loads are in LDS, and so are all others'
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
        __syncthreads();
    };
    if (first < last) {
        fetch(lds0);
        int t = first;
        for (; t + 2 <= last; t += 2) {
            arrived();
            fetch(lds1);
            work(lds0);
            arrived();
            if (t + 2 < last) fetch(lds0);
            work(lds1);
        }
        if (t < last) {
            arrived();
            work(lds0);
        }
    }
    __syncthreads();
    Epi::template run<TM, TN, WM, WN>(e, p, acc, m0 + wm / PAIR, n0 + wn, (int)blockIdx.y, lds0, tm, tn);
}

template <int BM, int BN, int BK, int WM, int WN, int NP, bool ACOL, bool BCOL, class Epi>
hipError_t launch_product(ProductArgs p, const typename Epi::Args &e, hipStream_t s)
{
    constexpr int M = BM / (paired_rows<Epi> ? 2 : 1);
    p.tiles_m = (p.m + M - 1) / M;
    p.tiles_n = (p.n_last - p.n_first + BN - 1) / BN;
    const dim3 tiles = grid_of((long long)p.tiles_m * p.tiles_n);
    hipLaunchKernelGGL((product_kernel<BM, BN, BK, WM, WN, NP, ACOL, BCOL, Epi>), dim3(tiles.x, p.splits, tiles.y), dim3(WM * WN * 64),
                       0, s, p, e);
    return hipGetLastError();
}

}  // namespace lcn
