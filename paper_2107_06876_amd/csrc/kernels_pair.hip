// Products of matrices in planes of fp16 (orthogonal.h), on the tiles, loads and fragments of product.h.
//
// 256 x 256 tiles, two buffers of LDS: large products, 1.2 PFLOP/s of fp16 (4 of 8192 x 1024 x 1024, two planes: 170 us).
// 128 x 128 tiles, two buffers, two workgroups to a compute unit: products of some hundred tiles (4 symmetric ones of 1024^3: 33 us,
// of which the rate above would be 13: 144 tiles do not fill 256 compute units, and one wave after another reads LDS and multiplies;
// four buffers, fragments ahead in registers and other orders of k were no faster, 64 x 64 tiles 34 to 38).
// 64 x 64 tiles, 64 values of k at a time in four buffers: products of few tiles, where what counts is the way from memory
// (1024^3: 13 us; as 128 x 128 25, with 32 values of k at a time 17).
// 32 x 32 tiles, the same: of even fewer, where what counts is what a workgroup has to bring (300^3: 4.9 us, as 64 x 64 7.0, with 128
// values of k at a time 4.8; 896^3, symmetric: 11, as 64 x 64 10).
#include "orthogonal.h"

namespace lcn {

// The tile of a workgroup: matrices follow each other, workgroups are dealt to the eight dies in turn (tile_of); of a symmetric
// result tiles with tm <= tn.
template <bool SYMMETRIC>
__device__ __forceinline__ bool pair_tile(const PairArgs &p, int &number, int &batch, int &tm, int &tn)
{
    const unsigned id = blockIdx.z * gridDim.x + blockIdx.x;   // y: splits
    const int tiles = SYMMETRIC ? p.tiles_n * (p.tiles_n + 1) / 2 : p.tiles_m * p.tiles_n;
    const int total = tiles * p.batches;
    if (id >= (unsigned)total) return false;
    const int base = total / 8, more = total % 8, die = (int)(id % 8), nth = (int)(id / 8);
    number = die * base + (die < more ? die : more) + nth;
    batch = number / tiles;
    const int in = number - batch * tiles;
    if constexpr (SYMMETRIC) {
        tn = (int)((__builtin_sqrtf(8.f * (float)in + 1.f) - 1.f) * 0.5f);
        while (tn * (tn + 1) / 2 > in) --tn;
        while ((tn + 1) * (tn + 2) / 2 <= in) ++tn;
        tm = in - tn * (tn + 1) / 2;
    } else {
        const int strip = in / (4 * p.tiles_m), inside = in % (4 * p.tiles_m);
        const int wide = p.tiles_n - strip * 4 < 4 ? p.tiles_n - strip * 4 : 4;
        tm = inside / wide;
        tn = strip * 4 + inside % wide;
    }
    return true;
}

template <int N>
struct Count {
    static constexpr int value = N;
};

template <bool SYM>   // false: of few tiles all are computed, which costs no time and saves writing twice
struct GramEpilogue {
    typedef GramArgs Args;
    static constexpr bool SYMMETRIC = SYM, ROWS = false;   // ROWS: goes through LDS row by row
    // What the result needs of `gram`, requested before the product where there is room for it
    template <int TM, int TN>
    struct Early {
        static constexpr bool HERE = TM * TN <= 4;
        f16x4 hi[HERE ? TM : 1][HERE ? TN : 1], lo[HERE ? TM : 1][HERE ? TN : 1];
    };
    template <int TM, int TN>
    static __device__ void early(const Args &e, const PairArgs &p, Early<TM, TN> &g, int m0, int n0, int batch)
    {
        const int lane = threadIdx.x & 63, ld = (int)e.out.ld;
        if constexpr (Early<TM, TN>::HERE)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int n = n0 + j * 16 + (lane & 15), m = m0 + i * 16 + 4 * (lane >> 4);
                    const bool in = e.gram.p && n < p.n && m < ld;
                    const long long at = batch * e.batch + (long long)n * ld + m;
                    g.hi[i][j] = in ? *(const f16x4 *)(e.gram.p + at) : f16x4{};
                    g.lo[i][j] = in ? *(const f16x4 *)(e.gram.p + e.gram.plane + at) : f16x4{};
                }
    }
    template <int TM, int TN>
    static __device__ void run(const Args &e, const PairArgs &p, f32x4 (&acc)[TM][TN], const Early<TM, TN> &g, int m0, int n0, int batch,
                               bool mirror, char *)
    {
        const int lane = threadIdx.x & 63;
        const float r = e.ratio ? e.ratio[batch] : 1.f, factor = e.ratio ? e.factor * r * r : e.factor;
        f16 *hi = e.out.p + batch * e.batch, *lo = hi + e.out.plane;
        const f16 *gram = e.gram.p ? e.gram.p + batch * e.batch : nullptr;
        const int ld = (int)e.out.ld;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int n = n0 + j * 16 + (lane & 15);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int m = m0 + i * 16 + 4 * (lane >> 4);
                if (m >= ld) continue;
                const long long at = (long long)n * ld + m;
                f32x4 v = acc[i][j] * factor;
                if (gram && n < p.n) {
                    f16x4 a, b;
                    if constexpr (Early<TM, TN>::HERE) {
                        a = g.hi[i][j];
                        b = g.lo[i][j];
                    } else {
                        a = *(const f16x4 *)(gram + at);
                        b = *(const f16x4 *)(gram + e.gram.plane + at);
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        v[u] += e.linear * ((float)a[u] + (float)b[u]);
                        if (m + u == n) v[u] += e.constant;
                    }
                }
                f16x4 x, y;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    x[u] = (f16)v[u];
                    y[u] = (f16)(v[u] - (float)x[u]);
                }
                if (n < p.n) {
                    *(f16x4 *)(hi + at) = x;
                    *(f16x4 *)(lo + at) = y;
                }
                if (SYM && mirror && n < ld) {   // also zeros behind the rows' ends
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (m + u < p.m) {
                            hi[(long long)(m + u) * ld + n] = x[u];
                            lo[(long long)(m + u) * ld + n] = y[u];
                        }
                }
            }
        }
    }
};

struct ApplyEpilogue {
    typedef ApplyArgs Args;
    static constexpr bool SYMMETRIC = false, ROWS = true;
    template <int TM, int TN>
    struct Early {};
    template <int TM, int TN>
    static __device__ void early(const Args &, const PairArgs &, Early<TM, TN> &, int, int, int) {}
    template <int TM, int TN>
    static __device__ void run(const Args &e, const PairArgs &p, f32x4 (&acc)[TM][TN], const Early<TM, TN> &, int m0, int n0, int batch, bool, char *region)
    {
        const int lane = threadIdx.x & 63;
        const float factor = e.ratio ? e.factor * e.ratio[batch] : e.factor;
        const Planes out{e.out.p + batch * e.batch, e.out.plane, e.out.ld};
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) col[i] = acc[i][j] * factor;
            by_rows<TM>(
                region, col, lane, [](int, int) { return Nothing{}; },
                [&](int r, int c, f32x4 (&v)[2], Nothing) {
                    const int n = n0 + j * 16 + r, m = m0 + c;
                    if (n < p.n && m < p.m) store_planes(out, n * out.ld + m, v);   // zeros behind the row's end
                });
        }
    }
};

template <class T>
struct LastEpilogue {
    typedef LastArgs Args;
    static constexpr bool SYMMETRIC = false, ROWS = true;
    template <int TM, int TN>
    struct Early {};
    template <int TM, int TN>
    static __device__ void early(const Args &, const PairArgs &, Early<TM, TN> &, int, int, int) {}
    template <int TM, int TN>
    static __device__ void run(const Args &e, const PairArgs &p, f32x4 (&acc)[TM][TN], const Early<TM, TN> &, int m0, int n0, int batch, bool, char *region)
    {
        const int lane = threadIdx.x & 63;
        const float factor = e.ratio ? e.factor * e.ratio[batch] : e.factor;
        T *out = (T *)e.out + batch * e.batch;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) col[i] = acc[i][j] * factor;
            by_rows<TM>(
                region, col, lane, [](int, int) { return Nothing{}; },
                [&](int r, int c, f32x4 (&v)[2], Nothing) {
                    const int n = n0 + j * 16 + r, m = m0 + c;
                    if (n < p.n && m < p.m) store_eight(out + n * e.ld + m, v, p.m - m);
                });
        }
    }
};

// PA, PB: planes of the operands; LOW: the small products have accumulators of their own; STAGES: tiles of LDS in turn
template <int BM, int BN, int BK, int WM, int WN, int STAGES, bool ACOL, bool BCOL, int PA, int PB, bool LOW, class Epi>
__global__ __launch_bounds__(WM *WN * 64, WM *WN == 4 ? 1 : BM == 128 ? 4 : 2) void pair_kernel(PairArgs p, typename Epi::Args e)
{
    constexpr int THREADS = WM * WN * 64, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int ABYTES = BM * BK * 2, BBYTES = BN * BK * 2, STAGE = PA * ABYTES + PB * BBYTES;
    constexpr int ROWS = Epi::ROWS ? WM * WN * RowRegion<TM>::BYTES : 0;
    typedef TileLoader<BM, BK, ACOL, THREADS> LoadA;
    typedef TileLoader<BN, BK, BCOL, THREADS> LoadB;
    static_assert(LoadA::PIECES % THREADS == 0 && LoadB::PIECES % THREADS == 0, "a wavefront's loads of a tile are counted");
    constexpr int LOADS = PA * LoadA::LOADS + PB * LoadB::LOADS;   // of a wavefront, for a tile
    __shared__ __align__(1024) char lds0[STAGE > ROWS ? STAGE : ROWS];
    __shared__ __align__(1024) char lds1[STAGE];
    __shared__ __align__(1024) char lds2[STAGES > 2 ? STAGE : 16];
    __shared__ __align__(1024) char lds3[STAGES > 3 ? STAGE : 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int number, batch, tm, tn;
    if (!pair_tile<Epi::SYMMETRIC>(p, number, batch, tm, tn)) return;
    const int m0 = tm * BM, n0 = tn * BN, wm = (wave % WM) * (BM / WM), wn = (wave / WM) * (BN / WN);
    const int at_a = fragment_place<BM, BK, ACOL>(lane), at_b = fragment_place<BN, BK, BCOL>(lane);
    f32x4 acc[TM][TN], low[LOW ? TM : 1][LOW ? TN : 1];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (LOW) low[i][j] = acc[i][j];
        }
    const int all = (p.k + BK - 1) / BK, per = (all + p.splits - 1) / p.splits;
    const int first = (int)blockIdx.y * per, last = first + per < all ? first + per : all;
    Operand a = p.a, b = p.b;
    a.p = (const char *)a.p + batch * p.a_batch;
    b.p = (const char *)b.p + batch * p.b_batch;
    typename Epi::template Early<TM, TN> wanted{};
    if (!Epi::SYMMETRIC || p.splits == 1) Epi::template early<TM, TN>(e, p, wanted, m0 + wm, n0 + wn, batch);
    LoadA load_a;
    LoadB load_b;
    load_a.init(a, m0, p.m, wave, lane);
    load_b.init(b, n0, p.n, wave, lane);
    auto fetch = [&](int step, char *lds) {
#pragma unroll
        for (int u = 0; u < PA; ++u) load_a.load(u * a.plane, step, p.k, lds + u * ABYTES, wave);
#pragma unroll
        for (int u = 0; u < PB; ++u) load_b.load(u * b.plane, step, p.k, lds + PA * ABYTES + u * BBYTES, wave);
    };
    auto work = [&](const char *lds) {
        // places are formed anew for every tile: kept in registers they would not fit beside the accumulators
        int pa = at_a, pb = at_b;
        asm volatile("" : "+v"(pa), "+v"(pb));
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
            bf16x8 fb[PB][TN];
#pragma unroll
            for (int u = 0; u < PB; ++u)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    fb[u][j] = load_fragment<BN, BK, BCOL>(lds + PA * ABYTES + u * BBYTES, pb, wn + j * 16, kk);
            auto read = [&](int i, bf16x8(&fa)[PA]) {
#pragma unroll
                for (int u = 0; u < PA; ++u) fa[u] = load_fragment<BM, BK, ACOL>(lds + u * ABYTES, pa, wm + i * 16, kk);
            };
            auto multiply = [&](int i, const bf16x8(&fa)[PA]) {
                f32x4(&small)[TN] = *(LOW ? (f32x4(*)[TN])&low[LOW ? i : 0] : &acc[i]);
                if constexpr (PA == 2)
#pragma unroll
                    for (int j = 0; j < TN; ++j) small[j] = mfma_f16(fa[1], fb[0][j], small[j]);
                if constexpr (PB == 2)
#pragma unroll
                    for (int j = 0; j < TN; ++j) small[j] = mfma_f16(fa[0], fb[1][j], small[j]);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = mfma_f16(fa[0], fb[0][j], acc[i][j]);
            };
            if constexpr (TM <= 4) {   // room for all: one way to LDS instead of TM
                bf16x8 fa[TM][PA];
#pragma unroll
                for (int i = 0; i < TM; ++i) read(i, fa[i]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < TM; ++i) multiply(i, fa[i]);
            } else {
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    bf16x8 fa[PA];
                    read(i, fa);
                    multiply(i, fa);
                }
            }
        }
    };
    // A tile is in LDS, of every wavefront, and every wavefront has read the tile before: those of `more` later tiles may be under
    // way.  Loads end in the order of their issue, as the counter is defined (the compiler's own waits rest on it), also those that are
    // out of range as a whole: they go the same way and bring zeros.
    auto arrived = [&](auto more) {
        constexpr int MORE = decltype(more)::value * LOADS;
        static_assert(MORE < 64, "the counter");
        __builtin_amdgcn_s_waitcnt((MORE & 15) | (MORE >> 4) << 14 | 0x0f70);
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    static_assert(STAGES == 2 || STAGES == 4, "buffers of the turns below");
    if (first < last) {
        fetch(first, lds0);
        if (STAGES > 2) {
            if (first + 1 < last) fetch(first + 1, lds1);
            if (first + 2 < last) fetch(first + 2, lds2);
        }
        int t = first;
        // tile t, in `now`; `then`: the buffer of the tile before
        auto turn = [&](const char *now, char *then) {
            arrived(Count<STAGES - 2>());
            fetch(t + STAGES - 1, then);
            work(now);
            ++t;
        };
        auto last_turn = [&](const char *now, char *then) {
            if (t >= last) return;
            if (t + STAGES - 2 < last)
                arrived(Count<STAGES - 2>());
            else
                arrived(Count<0>());
            if (t + STAGES - 1 < last) fetch(t + STAGES - 1, then);
            work(now);
            ++t;
        };
        // a loop without a branch inside: the compiler's own waits then count as these do
        while (t + 2 * STAGES - 2 < last) {
            turn(lds0, STAGES == 2 ? lds1 : lds3);
            turn(lds1, lds0);
            if constexpr (STAGES > 2) {
                turn(lds2, lds1);
                turn(lds3, lds2);
            }
        }
        while (t < last) {
            last_turn(lds0, STAGES == 2 ? lds1 : lds3);
            last_turn(lds1, lds0);
            if constexpr (STAGES > 2) {
                last_turn(lds2, lds1);
                last_turn(lds3, lds2);
            }
        }
    }
    if (LOW)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] += low[LOW ? i : 0][LOW ? j : 0];
    if (Epi::SYMMETRIC && p.splits > 1) {
        const long long tiles = (long long)p.tiles_n * (p.tiles_n + 1) / 2 * p.batches;
        f32x4 *to = (f32x4 *)(p.part + (blockIdx.y * tiles + number) * (BM * BN));
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) to[(i * TN + j) * THREADS + tid] = acc[i][j];
        return;
    }
    __syncthreads();
    Epi::template run<TM, TN>(e, p, acc, wanted, m0 + wm, n0 + wn, batch, tm != tn, lds0 + (Epi::ROWS ? wave * RowRegion<TM>::BYTES : 0));
}

// adds up the partial sums of a symmetric product, tile by tile in the order that pair_kernel left them
template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64, 2) void pair_join_kernel(PairArgs p, GramArgs e)
{
    constexpr int THREADS = WM * WN * 64, TM = BM / WM / 16, TN = BN / WN / 16;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int number, batch, tm, tn;
    if (!pair_tile<true>(p, number, batch, tm, tn)) return;
    const long long tiles = (long long)p.tiles_n * (p.tiles_n + 1) / 2 * p.batches;
    const int j = (int)blockIdx.y;   // 16 of a wavefront's columns n
    f32x4 acc[TM][1];
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[i][0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
    for (int s = 0; s < p.splits; ++s) {
        const f32x4 *from = (const f32x4 *)(p.part + (s * tiles + number) * (BM * BN));
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][0] += from[(i * TN + j) * THREADS + tid];
    }
    const int m0 = tm * BM + (wave % WM) * (BM / WM), n0 = tn * BN + (wave / WM) * (BN / WN) + j * 16;
    typedef GramEpilogue<true> Epi;
    Epi::Early<TM, 1> wanted{};
    Epi::early<TM, 1>(e, p, wanted, m0, n0, batch);
    Epi::run<TM, 1>(e, p, acc, wanted, m0, n0, batch, tm != tn, nullptr);
}

// ---- host ---------------------------------------------------------------------

// The tile and split with the least estimated time: a round of workgroups costs its steps of 32 values of k, as measured with two
// planes of both operands, and about 4 us of start, first loads and epilogue; a split its sums' way through memory and a launch.
// The largest tile has no room for sums of a float's precision.
PairPlan plan_pair(long long m, long long n, long long k, long long batches, bool symmetric, bool bf16)
{
    static const int resident[PAIR_SHAPES] = {1, 2, 1, 2};
    static const double alone_us[PAIR_SHAPES] = {2.4, 0.85, 0.32, 0.2}, full_us[PAIR_SHAPES] = {2.6, 1.35, 0.37, 0.25};
    PairPlan best{PAIR_64, 1};
    double least = 1e300;
    for (int t = bf16 ? 0 : 1; t < PAIR_SHAPES; ++t) {
        const int w = pair_tile_of(t);
        const long long tm = (m + w - 1) / w, tn = (n + w - 1) / w;
        const long long count = (symmetric ? tn * (tn + 1) / 2 : tm * tn) * batches, steps = (k + 31) / 32;
        for (int splits = 1; splits <= 16; ++splits) {
            if (splits > 1 && (!symmetric || steps / splits < 8)) break;
            const long long groups = count * splits, room = 256LL * resident[t], each = (steps + splits - 1) / splits;
            const long long rounds = groups / room, rest = groups % room;
            double us = (double)rounds * (full_us[t] * (double)each + 4.0);
            if (rest) us += (rest <= 256 ? alone_us[t] : full_us[t]) * (double)each + 4.0;
            if (splits > 1) us += 5.0 + (double)groups * w * w * 8e-6 / 4.0;
            if (us < least) {
                least = us;
                best = PairPlan{t, splits};
            }
        }
    }
    return best;
}

template <int BM, int BK, int WM, int WN, int STAGES, bool ACOL, bool BCOL, int PA, int PB, bool LOW, class Epi>
static hipError_t launch_pair(const PairPlan &plan, PairArgs p, const typename Epi::Args &e, hipStream_t s)
{
    p.splits = plan.splits;
    p.tiles_m = (p.m + BM - 1) / BM;
    p.tiles_n = (p.n + BM - 1) / BM;
    const long long tiles = (Epi::SYMMETRIC ? (long long)p.tiles_n * (p.tiles_n + 1) / 2 : (long long)p.tiles_m * p.tiles_n) * p.batches;
    if (tiles >= 1LL << 31) return hipErrorInvalidValue;
    const dim3 grid = grid_of(tiles);
    hipLaunchKernelGGL((pair_kernel<BM, BM, BK, WM, WN, STAGES, ACOL, BCOL, PA, PB, LOW, Epi>), dim3(grid.x, p.splits, grid.y),
                       dim3(WM * WN * 64), 0, s, p, e);
    const hipError_t st = hipGetLastError();
    if constexpr (Epi::SYMMETRIC)
        if (st == hipSuccess && p.splits > 1) {
            hipLaunchKernelGGL((pair_join_kernel<BM, BM, WM, WN>), dim3(grid.x, BM / WN / 16, grid.y), dim3(WM * WN * 64), 0, s, p, e);
            return hipGetLastError();
        }
    return st;
}

template <bool ACOL, bool BCOL, int PA, int PB, bool LOW, class Epi>
static hipError_t launch_tile(const PairPlan &plan, const PairArgs &p, const typename Epi::Args &e, hipStream_t s)
{
    if constexpr (!LOW)
        if (plan.shape == PAIR_256) return launch_pair<256, 32, 2, 4, 2, ACOL, BCOL, PA, PB, LOW, Epi>(plan, p, e, s);
    return plan.shape == PAIR_128  ? launch_pair<128, 32, 2, 4, 2, ACOL, BCOL, PA, PB, LOW, Epi>(plan, p, e, s)
           : plan.shape == PAIR_64 ? launch_pair<64, 64, 2, 2, 4, ACOL, BCOL, PA, PB, LOW, Epi>(plan, p, e, s)
                                   : launch_pair<32, 64, 2, 2, 4, ACOL, BCOL, PA, PB, LOW, Epi>(plan, p, e, s);
}
template <bool ACOL, bool BCOL, int PA, int PB, bool LOW>
static hipError_t launch_symmetric(const PairPlan &plan, const PairArgs &p, const GramArgs &e, hipStream_t s)
{
    const long long w = pair_tile_of(plan.shape), t = (p.n + w - 1) / w;
    if (plan.shape >= PAIR_64 && plan.splits == 1 && t * t * p.batches <= 256)
        return plan.shape == PAIR_64 ? launch_pair<64, 64, 2, 2, 4, ACOL, BCOL, PA, PB, LOW, GramEpilogue<false>>(plan, p, e, s)
                                     : launch_pair<32, 64, 2, 2, 4, ACOL, BCOL, PA, PB, LOW, GramEpilogue<false>>(plan, p, e, s);
    return launch_tile<ACOL, BCOL, PA, PB, LOW, GramEpilogue<true>>(plan, p, e, s);
}

hipError_t launch_gram(const PairPlan &plan, const PairArgs &p, const GramArgs &e, bool wide, int planes, hipStream_t s)
{
    if (wide)
        return planes == PAIR_ONE   ? launch_symmetric<false, false, 1, 1, false>(plan, p, e, s)
               : planes == PAIR_TWO ? launch_symmetric<false, false, 2, 2, false>(plan, p, e, s)
                                    : launch_symmetric<false, false, 2, 2, true>(plan, p, e, s);
    return planes == PAIR_ONE   ? launch_symmetric<true, true, 1, 1, false>(plan, p, e, s)
           : planes == PAIR_TWO ? launch_symmetric<true, true, 2, 2, false>(plan, p, e, s)
                                : launch_symmetric<true, true, 2, 2, true>(plan, p, e, s);
}

template <bool ACOL, bool BCOL, int PA, int PB, class Epi>
static hipError_t launch_bf16(const PairPlan &plan, const PairArgs &p, const typename Epi::Args &e, bool one, hipStream_t s)
{
    return one ? launch_tile<ACOL, BCOL, PA, PB, false, Epi>(plan, p, e, s) : launch_tile<ACOL, BCOL, 2, 2, false, Epi>(plan, p, e, s);
}
hipError_t launch_apply(const PairPlan &plan, const PairArgs &p, const ApplyArgs &e, bool wide, int planes, hipStream_t s)
{
    if (planes == PAIR_FLOAT)
        return wide ? launch_tile<true, false, 2, 2, true, ApplyEpilogue>(plan, p, e, s)
                    : launch_tile<false, false, 2, 2, true, ApplyEpilogue>(plan, p, e, s);
    return wide ? launch_bf16<true, false, 1, 2, ApplyEpilogue>(plan, p, e, planes == PAIR_ONE, s)
                : launch_bf16<false, false, 2, 1, ApplyEpilogue>(plan, p, e, planes == PAIR_ONE, s);
}
hipError_t launch_apply_last(const PairPlan &plan, const PairArgs &p, const LastArgs &e, bool wide, int planes, hipStream_t s)
{
    if (planes == PAIR_FLOAT)
        return wide ? launch_tile<true, false, 2, 2, true, LastEpilogue<float>>(plan, p, e, s)
                    : launch_tile<false, false, 2, 2, true, LastEpilogue<float>>(plan, p, e, s);
    return wide ? launch_bf16<true, false, 1, 2, LastEpilogue<__bf16>>(plan, p, e, planes == PAIR_ONE, s)
                : launch_bf16<false, false, 2, 1, LastEpilogue<__bf16>>(plan, p, e, planes == PAIR_ONE, s);
}

}  // namespace lcn
