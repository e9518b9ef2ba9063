// Shared by the operators that produce and train the points: activations, planes of bf16, host-side choices.
#pragma once

#include "lcn_internal.h"
#include "product.h"

namespace lcn {

// what the host takes for granted about sizes: offsets within a tile stay below 2^31 bytes
constexpr int32_t MAX_WIDTH = 1 << 20;
constexpr int64_t MAX_ROWS = (int64_t)1 << 30;
// a product's tiles are numbered in 31 bits: 64 x 64 of them at least in a result of up to 2^42 values
constexpr int64_t MAX_AREA = (int64_t)1 << 42;
inline bool sizes_fit(int64_t a, int64_t b) { return a * b <= MAX_AREA; }

template <class T>
struct Four;   // four consecutive values, one load or store
template <>
struct Four<float> {
    typedef f32x4 type;
};
template <>
struct Four<__bf16> {
    typedef bf16x4 type;
};

// Four consecutive values from `p` (only the first `left` exist) and back, in one piece wherever p lies: rows of odd widths are then
// nearly as fast as others (planes, epilogues and slopes of 4000 rows, 1001 -> 2003 bf16: 72 -> 44 us and 130 -> 108).
template <class T>
__device__ __forceinline__ f32x4 load_four(const T *p, int left)
{
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if (left >= 4) {
        typedef typename Four<T>::type any __attribute__((aligned(sizeof(T))));
        const typename Four<T>::type v = *(const any *)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) r[e] = (float)p[e];
    }
    return r;
}
template <class T>
__device__ __forceinline__ void store_four(T *p, f32x4 v, int left)
{
    if (left >= 4) {
        typedef typename Four<T>::type any __attribute__((aligned(sizeof(T))));
        typename Four<T>::type o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (T)v[e];
        *(any *)p = o;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (T)v[e];
    }
}

// The same for eight values in two halves.
template <class T>
__device__ __forceinline__ void load_eight(const T *p, int left, f32x4 (&r)[2])
{
    if constexpr (sizeof(T) == 2) {
        if (left >= 8) {
            typedef bf16x8 any __attribute__((aligned(2)));
            const bf16x8 v = *(const any *)p;
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e >> 2][e & 3] = (float)v[e];
            return;
        }
    }
    r[0] = load_four(p, left);
    r[1] = load_four(p + 4, left - 4);
}
// The same as they are in memory.
template <class T>
struct Eight {
    T v[8];
};
template <class T>
__device__ __forceinline__ Eight<T> read_eight(const T *p, int left)
{
    Eight<T> r;
    if (left >= 8) {
        typedef T piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            const piece q = ((const piece *)p)[h];
#pragma unroll
            for (int e = 0; e < 16 / (int)sizeof(T); ++e) r.v[h * (16 / (int)sizeof(T)) + e] = q[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = e < left ? p[e] : (T)0.f;
    }
    return r;
}
template <class T>
__device__ __forceinline__ void store_eight(T *p, const f32x4 (&v)[2], int left)
{
    if constexpr (sizeof(T) == 2) {
        if (left >= 8) {
            typedef bf16x8 any __attribute__((aligned(2)));
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (T)v[e >> 2][e & 3];
            *(any *)p = o;
            return;
        }
    }
    store_four(p, v[0], left);
    store_four(p + 4, v[1], left - 4);
}
// Whether rows of `width` values at p are whole aligned 16-byte pieces (of four floats, eight bf16).
template <class T>
inline bool whole_rows(const void *p, long long width)
{
    return ((uintptr_t)p & 15) == 0 && width % (16 / (int)sizeof(T)) == 0;
}

// x as the sum of three bf16 (to 2^-26).  A value beyond the largest bf16 is cut, not rounded to infinity; what
// is not finite stands in the first plane alone.
__device__ __forceinline__ void split_planes(float x, __bf16 &a, __bf16 &b, __bf16 &c)
{
    a = (__bf16)x;
    const float whole = __builtin_fabsf(x);
    if (__builtin_isinf((float)a) && whole < __builtin_huge_valf())
        a = __builtin_bit_cast(__bf16, (unsigned short)(__builtin_bit_cast(unsigned, x) >> 16));
    float r = x - (float)a;
    if (!(whole < __builtin_huge_valf())) r = 0.f;
    b = (__bf16)r;
    c = (__bf16)(r - (float)b);
}

// 2^x by the instruction alone: results below the smallest normal float are zero
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == LCN_ACT_TANH) return tanhf(z);
    if constexpr (ACT == LCN_ACT_RELU) return z > 0.f ? z : z == z ? 0.f : z;
    if constexpr (ACT == LCN_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    if constexpr (ACT == LCN_ACT_SILU) return z / (1.f + expf(-z));
    return z;
}
template <int ACT>
__device__ __forceinline__ float activate_slope(float z)
{
    if constexpr (ACT == LCN_ACT_TANH) {
        const float t = tanhf(z);
        return 1.f - t * t;
    }
    if constexpr (ACT == LCN_ACT_RELU) return z > 0.f ? 1.f : z == z ? 0.f : z;
    if constexpr (ACT == LCN_ACT_GELU)
        return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    if constexpr (ACT == LCN_ACT_SILU) {
        const float f = 1.f / (1.f + expf(-z));
        return f * (1.f + z * (1.f - f));
    }
    return 1.f;
}

// up to so many rows a layer takes dot products of its own (few_rows_dot) instead of the matrix instruction
constexpr int FEW_ROWS = 8;

template <int ACT>
struct Activation {
    static constexpr int value = ACT;
};
// calls f with the activation as a type
template <class F>
hipError_t by_activation(int act, F f)
{
    switch (act) {
    case LCN_ACT_TANH: return f(Activation<LCN_ACT_TANH>());
    case LCN_ACT_RELU: return f(Activation<LCN_ACT_RELU>());
    case LCN_ACT_GELU: return f(Activation<LCN_ACT_GELU>());
    case LCN_ACT_SILU: return f(Activation<LCN_ACT_SILU>());
    default: return f(Activation<LCN_ACT_NONE>());
    }
}

// ---- planes (kernels_planes.hip) --------------------------------------------
inline __host__ __device__ long long padded(long long d) { return (d + 7) & ~7LL; }
inline int planes_of(int32_t dtype) { return dtype == LCN_F32 ? 3 : 1; }
// bytes of an operand of rows x d in planes
inline size_t planes_bytes(long long rows, long long d, int planes)
{
    return ((size_t)rows * (size_t)padded(d) * 2 * planes + 255) & ~(size_t)255;
}
// Planes of the gradients dz and G on the way into their products.  One rounding of them to bf16 is as large as that of
// the result; where few rows are added it can be larger than it in some of the result, so up to FEW_GRADIENT_ROWS rows
// they have a second plane (the products are then bound by the other operand's bytes).
constexpr int64_t FEW_GRADIENT_ROWS = 512;
inline int gradient_planes(int64_t rows, int32_t dtype) { return dtype == LCN_F32 ? 3 : rows <= FEW_GRADIENT_ROWS ? 2 : 1; }
// Whether a bf16 matrix can be an operand as it lies: rows of whole 16-byte pieces, aligned.
inline bool in_place(const void *p, long long d, int32_t dtype)
{
    return dtype == LCN_BF16 && d % 8 == 0 && ((uintptr_t)p & 15) == 0;
}
// Matrices to lay out in planes, all by one launch: rows x d into planes at dst, rows padded with zeros to a multiple of 8;
// rows whose `target` is negative become zero (target: nullable).
struct PlaneJobs {
    enum { MOST = 3 };
    struct Job {
        const void *src;
        void *dst;
        const int64_t *target;
        long long rows;
        int d, dp;
        unsigned end;   // workgroups of this job and those before
    } job[MOST];
    int count = 0;
};
// The operand of a matrix: as it lies where that can be, else its planes at `space`, which become one of the jobs.
Operand add_operand(PlaneJobs &jobs, const void *p, long long rows, int d, int32_t dtype, void *space);
// The same, always in planes, with the rows whose target is negative zero.
Operand add_masked(PlaneJobs &jobs, const void *p, long long rows, int d, int32_t dtype, const int64_t *target, void *space);
hipError_t launch_planes(const PlaneJobs &jobs, int32_t dtype, hipStream_t s);
// planes that a kernel has written to dst
inline Operand plane_operand(const void *dst, long long rows, long long d) { return Operand{dst, rows * padded(d) * 2, padded(d)}; }

// out[n][m] (dtype, m dense, width m) = scale * the sum of `splits` partial products (float, [split][n][ldp])
hipError_t launch_add_partials(const float *part, int splits, long long n, int m, long long ldp, float scale, int32_t dtype,
                               void *out, hipStream_t s);

// ---- host-side choice of a product's tile and split --------------------------
struct ProductPlan {
    int tile;      // index of the tile shape, see launch_planned
    int splits;
    bool tail;     // columns behind the last whole tile: by small tiles, in a launch of their own
    double us;     // estimated
};
// workgroups of a tile shape that are on the chip at a time; the estimated time of a launch without partial sums' way
long long product_room(int tile, int planes);
double product_us(int tile, long long m, long long columns, long long k, int planes, int splits);
ProductPlan plan_product(long long m, long long n, long long k, int planes, bool may_split, bool may_tail, bool may_320 = true);

// A float product's partial sums: [split][n][ldp]; `add` adds to what is there.
struct PartialEpilogue {
    struct Args {
        float *part;
        long long ldp, stride;   // elements from a row, from a split to the next; ldp is a multiple of 8
        int add;
    };
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0,
                               int split, char *lds, int, int)
    {
        const int lane = threadIdx.x & 63;
        char *region = lds + (threadIdx.x >> 6) * RowRegion<TM>::BYTES;
        float *first = e.part + split * e.stride + m0;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) col[i] = acc[i][j];
            by_rows<TM>(
                region, col, lane,
                [&](int r, int c) {
                    const long long n = n0 + j * 16 + r;
                    return e.add && n < p.n && m0 + c < p.m ? read_eight(first + n * e.ldp + c, 8) : Eight<float>{};
                },
                [&](int r, int c, f32x4 (&v)[2], const Eight<float> &o) {
                    const long long n = n0 + j * 16 + r;
                    if (n >= p.n || m0 + c >= p.m) return;
#pragma unroll
                    for (int u = 0; u < 8; ++u) v[u >> 2][u & 3] += o.v[u];
                    store_eight(first + n * e.ldp + c, v, 8);
                });
        }
    }
};

// scale * the product, rounded to T, at out[n][m]
template <class T>
struct ScaledEpilogue {
    struct Args {
        T *out;
        long long ld;
        float scale;
    };
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0, int,
                               char *lds, int, int)
    {
        const int lane = threadIdx.x & 63;
        char *region = lds + (threadIdx.x >> 6) * RowRegion<TM>::BYTES;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) col[i] = acc[i][j] * e.scale;
            by_rows<TM>(
                region, col, lane, [](int, int) { return Nothing{}; },
                [&](int r, int c, f32x4 (&v)[2], Nothing) {
                    const long long n = n0 + j * 16 + r, m = m0 + c;
                    if (n < p.n && m < p.m) store_eight(e.out + n * e.ld + m, v, (int)(p.m - m));
                });
        }
    }
};

// Tile shapes: index -> BM x BN.  256 x 256 has the best rate; the smaller ones fill the chip where the result is
// small, the 320 wide one keeps a row of up to 320 values in one tile.  With three planes a tile has 32 values of k and
// all planes of both operands in LDS, so the large ones are half as wide in n.
enum { TILE_256 = 0, TILE_128 = 1, TILE_64 = 2, TILE_320 = 3, TILE_COUNT = 4 };
inline int tile_m(int tile) { return tile == TILE_256 ? 256 : tile == TILE_128 ? 128 : tile == TILE_64 ? 64 : 320; }
inline int tile_n(int tile, int planes)
{
    if (planes == 3) return tile == TILE_256 || tile == TILE_128 ? 128 : 64;
    return tile == TILE_256 ? 256 : tile == TILE_64 ? 64 : 128;
}
template <int NP, bool ACOL, bool BCOL, class Epi>
hipError_t launch_tiles(int tile, const ProductArgs &p, const typename Epi::Args &e, hipStream_t s)
{
    if constexpr (NP == 3) {
        switch (tile) {
        case TILE_256: return launch_product<256, 128, 32, 4, 2, 3, ACOL, BCOL, Epi>(p, e, s);
        case TILE_320:   // 80 rows of a wavefront are no whole pairs
            if constexpr (paired_rows<Epi>) return hipErrorInvalidValue;
            else return launch_product<320, 64, 32, 4, 2, 3, ACOL, BCOL, Epi>(p, e, s);
        case TILE_128: return launch_product<128, 128, 32, 2, 2, 3, ACOL, BCOL, Epi>(p, e, s);
        default: return launch_product<64, 64, 32, 2, 2, 3, ACOL, BCOL, Epi>(p, e, s);
        }
    } else {
        switch (tile) {
        case TILE_256: return launch_product<256, 256, 64, 2, 4, 1, ACOL, BCOL, Epi>(p, e, s);
        case TILE_320:
            if constexpr (paired_rows<Epi>) return hipErrorInvalidValue;
            else return launch_product<320, 128, 64, 4, 2, 1, ACOL, BCOL, Epi>(p, e, s);
        case TILE_128: return launch_product<128, 128, 64, 2, 2, 1, ACOL, BCOL, Epi>(p, e, s);
        default: return launch_product<64, 64, 64, 2, 2, 1, ACOL, BCOL, Epi>(p, e, s);
        }
    }
}
template <int NP, bool ACOL, bool BCOL, class Epi>
hipError_t launch_planned(const ProductPlan &plan, ProductArgs p, const typename Epi::Args &e, hipStream_t s)
{
    const int whole = p.n - p.n % tile_n(plan.tile, NP);
    p.splits = plan.splits;
    p.n_first = 0;
    p.n_last = plan.tail && whole ? whole : p.n;
    const hipError_t st = launch_tiles<NP, ACOL, BCOL, Epi>(plan.tile, p, e, s);
    if (st != hipSuccess || p.n_last == p.n) return st;
    p.n_first = whole;
    p.n_last = p.n;
    return launch_tiles<NP, ACOL, BCOL, Epi>(TILE_64, p, e, s);
}

// out[n][m] = scale * product, in one launch or as partial sums in `part` that a second launch adds up.
template <bool ACOL, bool BCOL>
hipError_t launch_scaled(const ProductPlan &plan, const ProductArgs &p, float scale, int32_t dtype, void *out, float *part,
                         hipStream_t s);

// The partial sums alone, A by columns and B by rows; `add`: to what is in `part`.
hipError_t launch_partials(const ProductPlan &plan, const ProductArgs &p, float *part, int add, hipStream_t s);
// out[c] (dtype) = sum over r of part[r][c], r = 0 .. parts - 1
hipError_t launch_column_sums(const float *part, int parts, int width, int32_t dtype, void *out, hipStream_t s);
// zeros, by a kernel
hipError_t launch_zero(void *p, size_t bytes, hipStream_t s);
inline size_t partial_bytes(const ProductPlan &plan, long long m, long long n)
{
    return plan.splits > 1 ? (size_t)plan.splits * (size_t)n * (size_t)padded(m) * 4 : 0;
}

// ---- products with few rows: 16 lanes per row of W ---------------------------
// sums[f][r] += W[f] . x[r] for two rows of W per group of 16 lanes and R rows of x (`rows` of them exist); every lane of
// the group gets the sums.  Sums are in 32 bits, of the same bits in every kernel that forms them (their order and the fused
// multiply-adds are fixed here).  VEC: rows of W and x are whole aligned 16-byte pieces.
template <class T, int R, bool VEC>
__device__ __forceinline__ void few_rows_dot(const T *__restrict__ w0, const T *__restrict__ w1, const T *__restrict__ x,
                                             int rows, int k, float (&sum)[2][R])
{
    constexpr int V = VEC ? 16 / (int)sizeof(T) : 1;
    typedef T piece __attribute__((ext_vector_type(V)));
    const int lane = threadIdx.x & 15;
#pragma unroll 4
    for (int c = lane * V; c < k; c += 16 * V) {
        piece a, b, y[R];
        if constexpr (VEC) {
            a = *(const piece *)(w0 + c);
            b = *(const piece *)(w1 + c);
#pragma unroll
            for (int r = 0; r < R; ++r) y[r] = *(const piece *)(x + (long long)(r < rows ? r : 0) * k + c);
        } else {
            a[0] = w0[c];
            b[0] = w1[c];
#pragma unroll
            for (int r = 0; r < R; ++r) y[r][0] = x[(long long)(r < rows ? r : 0) * k + c];
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sum[0][r] = __builtin_fmaf((float)a[e], (float)y[r][e], sum[0][r]);
                sum[1][r] = __builtin_fmaf((float)b[e], (float)y[r][e], sum[1][r]);
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum[f][r] += __shfl_xor(sum[f][r], o, 16);
}

// part of the workspace: hands out 256-byte aligned pieces, or only counts them
struct Carver {
    char *base;
    size_t used = 0;
    void *take(size_t bytes)
    {
        void *r = base ? base + used : nullptr;
        used += (bytes + 255) & ~(size_t)255;
        return r;
    }
};

#define OPCHK(...)                            \
    do {                                      \
        if ((__VA_ARGS__) != hipSuccess) {    \
            (void)hipGetLastError();          \
            return LCN_ERR_DEVICE;            \
        }                                     \
    } while (0)

}  // namespace lcn
