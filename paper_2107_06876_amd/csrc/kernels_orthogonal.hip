// X -> X (a + b X^T X + c (X^T X)^2), so many times, from G / (|G| + eps): the singular vectors of G with singular values that
// such polynomials bring near 1, without a decomposition.
//
//   A = X X^T (or X^T X, where that is the smaller one),  B = a + b A + c A^2,  X <- B X (or X B)
//
// Every product is one of two planes of fp16 (product.h): the singular values are bounded by the polynomials, and with them every
// value of X, A and B, so that powers of two in front keep them in fp16's range.  Planes and sums are as exact as single precision,
// which is needed: what rounding adds in the first steps grows as the smallest singular values do, up to a per step.
#include "operators.h"

namespace lcn {

// The largest singular value of X that a step may leave, the largest of a + b t + c t^2 in its way, and what X, A and B are
// multiplied with: values up to 32 768 of fp16's 65 504.
constexpr double MOST_X = 4.0, MOST_POLY = 64.0;
constexpr float SCALE_X = 8192.f, SCALE_A = 2048.f, SCALE_B = 512.f;

typedef _Float16 f16;

// A matrix in two planes: rows of `ld` values, ld a multiple of 8, zeros behind a row's values
struct Planes {
    f16 *p;
    long long plane, ld;   // values from a plane to the next, from a row to the next
};

__device__ __forceinline__ void store_planes(const Planes &o, long long at, const f32x4 (&v)[2])
{
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[e >> 2][e & 3];
        hi[e] = (f16)x;
        lo[e] = (f16)(x - (float)hi[e]);
    }
    *(f16x8 *)(o.p + at) = hi;
    *(f16x8 *)(o.p + o.plane + at) = lo;
}

// planes of factor * the product (A, and X in between)
struct PlanesEpilogue {
    struct Args {
        Planes out;
        float factor;
    };
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0, int, char *lds,
                               int, int)
    {
        const int lane = threadIdx.x & 63;
        char *region = lds + (threadIdx.x >> 6) * RowRegion<TM>::BYTES;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) col[i] = acc[i][j] * e.factor;
            by_rows<TM>(
                region, col, lane, [](int, int) { return Nothing{}; },
                [&](int r, int c, f32x4 (&v)[2], Nothing) {
                    const long long n = n0 + j * 16 + r, m = m0 + c;
                    if (n < p.n && m < p.m) store_planes(e.out, n * e.out.ld + m, v);
                });
        }
    }
};

// planes of factor * the product + linear * A + constant on the diagonal (B)
struct PolynomialEpilogue {
    struct Args {
        Planes out, gram;
        float factor, linear, constant;
    };
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0, int, char *lds,
                               int, int)
    {
        const int lane = threadIdx.x & 63;
        char *region = lds + (threadIdx.x >> 6) * RowRegion<TM>::BYTES;
        struct Two {
            f16x8 hi, lo;
        };
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) col[i] = acc[i][j] * e.factor;
            by_rows<TM>(
                region, col, lane,
                [&](int r, int c) {
                    const long long n = n0 + j * 16 + r, m = m0 + c;
                    Two t{};
                    if (n < p.n && m < p.m) {
                        t.hi = *(const f16x8 *)(e.gram.p + n * e.gram.ld + m);
                        t.lo = *(const f16x8 *)(e.gram.p + e.gram.plane + n * e.gram.ld + m);
                    }
                    return t;
                },
                [&](int r, int c, f32x4 (&v)[2], const Two &t) {
                    const long long n = n0 + j * 16 + r, m = m0 + c;
                    if (n >= p.n || m >= p.m) return;
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        float x = v[u >> 2][u & 3] + e.linear * ((float)t.hi[u] + (float)t.lo[u]);
                        if (m + u == n) x += e.constant;
                        v[u >> 2][u & 3] = x;
                    }
                    store_planes(e.out, n * e.out.ld + m, v);
                });
        }
    }
};

// Partial sums of squares of a matrix (blockIdx.y), in 64 bits: squares of floats leave their own range.
constexpr int NORM_GROUPS = 64;
template <class T>
__global__ __launch_bounds__(256) void squares_kernel(const T *__restrict__ g, long long size, double *__restrict__ part)
{
    __shared__ double sums[4];
    const T *p = g + blockIdx.y * size;
    double v = 0.0;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < size; i += (long long)NORM_GROUPS * 256) {
        const double x = (double)(float)p[i];
        v += x * x;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.y * NORM_GROUPS + blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// X = SCALE_X G / (|G| + eps) in planes; matrix blockIdx.y
template <class T>
__global__ __launch_bounds__(256) void normalise_kernel(const T *__restrict__ g, const double *__restrict__ part, int rows, int cols,
                                                        float eps, int whole, Planes out)
{
    double sum = 0.0;
    for (int i = 0; i < NORM_GROUPS; ++i) sum += part[blockIdx.y * NORM_GROUPS + i];
    const double inv = (double)SCALE_X / (sqrt(sum) + (double)eps);
    const int per_row = (int)(out.ld / 8);
    const T *src = g + (long long)blockIdx.y * rows * cols;
    out.p += (long long)blockIdx.y * rows * out.ld;
    const long long pieces = (long long)rows * per_row;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < pieces; t += (long long)gridDim.x * 256) {
        const long long r = t / per_row;
        const int k = (int)(t - r * per_row) * 8;
        f32x4 v[2];
        load_eight(src + r * cols + k, cols - k, whole, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = k + e < cols ? (float)((double)v[e >> 2][e & 3] * inv) : 0.f;
        store_planes(out, t * 8, v);
    }
}

// ---- host ---------------------------------------------------------------------

static bool orthogonal_args_fit(int64_t count, int32_t rows, int32_t cols, int32_t dtype)
{
    const int32_t lo = rows < cols ? rows : cols;
    return count >= 0 && count <= (1 << 20) && rows >= 1 && cols >= 1 && rows <= MAX_WIDTH && cols <= MAX_WIDTH && lo <= 32768 &&
           (double)count * rows * cols <= (double)((int64_t)1 << 40) && (dtype == LCN_F32 || dtype == LCN_BF16);
}

// Whether every step keeps the singular values, which start at 1 or less, within the bounds above.
static bool coefficients_fit(int32_t steps, const float *c)
{
    double s = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double k[3] = {c[3 * i], c[3 * i + 1], c[3 * i + 2]}, top = s * s;
        double most = 0.0, poly = 0.0;
        auto at = [&](double t) {   // a singular value sqrt(t), if it can occur
            if (!(t >= 0.0) || t > top) return;
            const double q = __builtin_fabs(k[0] + t * (k[1] + t * k[2]));
            if (!(q <= poly)) poly = q;
            if (!(q * __builtin_sqrt(t) <= most)) most = q * __builtin_sqrt(t);
        };
        at(0.0);
        at(top);
        at(-k[1] / (2.0 * k[2]));
        // a + 3 b t + 5 c t^2 = 0: where the step's result is largest
        const double d = 9.0 * k[1] * k[1] - 20.0 * k[0] * k[2];
        if (d >= 0.0) {
            at((-3.0 * k[1] + __builtin_sqrt(d)) / (10.0 * k[2]));
            at((-3.0 * k[1] - __builtin_sqrt(d)) / (10.0 * k[2]));
        }
        at(-k[0] / (3.0 * k[1]));   // the same without c
        if (!(most <= MOST_X) || !(poly <= MOST_POLY)) return false;
        s = most;
    }
    return true;
}

struct OrthogonalSpace {
    f16 *x[2], *gram, *poly;
    double *part;
    long long size, ld, lo, ldg;   // values of a plane of X and its row; of A and its row
    size_t bytes;
};
static OrthogonalSpace orthogonal_space(char *ws, int64_t count, int32_t rows, int32_t cols)
{
    Carver c{ws};
    OrthogonalSpace o;
    o.ld = padded(cols);
    o.size = count * rows * o.ld;
    o.lo = rows < cols ? rows : cols;
    o.ldg = padded(o.lo);
    for (int i = 0; i < 2; ++i) o.x[i] = (f16 *)c.take((size_t)o.size * 4);
    o.gram = (f16 *)c.take((size_t)(count * o.lo * o.ldg) * 4);
    o.poly = (f16 *)c.take((size_t)(count * o.lo * o.ldg) * 4);
    o.part = (double *)c.take((size_t)count * NORM_GROUPS * 8);
    o.bytes = c.used;
    return o;
}

template <bool ACOL, bool BCOL, class Epi>
static hipError_t launch_pair(ProductArgs p, const typename Epi::Args &e, hipStream_t s)
{
    p.planes = 2;
    p.splits = 1;
    p.n_first = 0;
    p.n_last = p.n;
    const long long large = ((p.m + 255LL) / 256) * ((p.n + 255) / 256), mid = ((p.m + 127LL) / 128) * ((p.n + 127) / 128);
    if (large >= 256) return launch_product<256, 256, 32, 2, 4, 2, ACOL, BCOL, Epi>(p, e, s);
    if (mid >= 256) return launch_product<128, 128, 32, 2, 2, 2, ACOL, BCOL, Epi>(p, e, s);
    return launch_product<64, 64, 32, 2, 2, 2, ACOL, BCOL, Epi>(p, e, s);
}

template <class T>
static lcn_status orthogonal_as(const T *g, int64_t count, int32_t rows, int32_t cols, int32_t steps, const float *c, float eps,
                                float scale, T *out, char *ws, size_t ws_bytes, hipStream_t s)
{
    OrthogonalSpace o = orthogonal_space(ws, count, rows, cols);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < o.bytes) return LCN_ERR_ALLOC;
    const bool wide = rows <= cols;
    const int n = (int)o.lo;
    Planes x[2] = {{o.x[0], o.size, o.ld}, {o.x[1], o.size, o.ld}};
    const Planes gram{o.gram, count * n * o.ldg, o.ldg}, poly{o.poly, count * n * o.ldg, o.ldg};
    const long long groups = ((long long)rows * (o.ld / 8) + 255) / 256;
    for (int64_t first = 0; first < count; first += 32768) {   // a grid's second dimension
        const unsigned some = (unsigned)(count - first < 32768 ? count - first : 32768);
        hipLaunchKernelGGL(squares_kernel<T>, dim3(NORM_GROUPS, some), dim3(256), 0, s, g + first * rows * cols, (long long)rows * cols,
                           o.part + first * NORM_GROUPS);
        OPCHK(hipGetLastError());
        Planes to = x[0];
        to.p += first * rows * o.ld;
        hipLaunchKernelGGL(normalise_kernel<T>, dim3((unsigned)(groups < 1024 ? groups : 1024), some), dim3(256), 0, s,
                           g + first * rows * cols, o.part + first * NORM_GROUPS, rows, cols, eps, whole_rows<T>(g, cols), to);
        OPCHK(hipGetLastError());
    }
    auto operand = [](const Planes &m, long long at) { return Operand{m.p + at, m.plane * 2, m.ld}; };
    auto from = [](Planes m, long long at) {
        m.p += at;
        return m;
    };
    for (int i = 0; i < steps; ++i) {
        const float a = c[3 * i], b = c[3 * i + 1], k = c[3 * i + 2];
        for (int64_t u = 0; u < count; ++u) {
            const long long ax = u * rows * o.ld, ag = u * n * o.ldg;
            ProductArgs p{};
            p.a = p.b = operand(x[0], ax);
            p.m = p.n = n;
            p.k = wide ? cols : rows;
            const PlanesEpilogue::Args ga{from(gram, ag), SCALE_A / (SCALE_X * SCALE_X)};
            OPCHK(wide ? launch_pair<false, false, PlanesEpilogue>(p, ga, s) : launch_pair<true, true, PlanesEpilogue>(p, ga, s));
            p.a = p.b = operand(gram, ag);
            p.k = n;
            OPCHK(launch_pair<false, false, PolynomialEpilogue>(
                p, {from(poly, ag), from(gram, ag), SCALE_B * k / (SCALE_A * SCALE_A), SCALE_B * b / SCALE_A, SCALE_B * a}, s));
            // wide: out[r][c] = sum over k of X[k][c] B[r][k];  tall: sum over k of B[c][k] X[r][k]
            p.m = cols;
            p.n = rows;
            p.a = wide ? operand(x[0], ax) : operand(poly, ag);
            p.b = wide ? operand(poly, ag) : operand(x[0], ax);
            if (i + 1 < steps) {
                const PlanesEpilogue::Args xa{from(x[1], ax), 1.f / SCALE_B};
                OPCHK(wide ? launch_pair<true, false, PlanesEpilogue>(p, xa, s) : launch_pair<false, false, PlanesEpilogue>(p, xa, s));
            } else {
                const typename ScaledEpilogue<T>::Args xa{out + u * rows * cols, cols, scale / (SCALE_B * SCALE_X), whole_rows<T>(out, cols)};
                OPCHK(wide ? launch_pair<true, false, ScaledEpilogue<T>>(p, xa, s) : launch_pair<false, false, ScaledEpilogue<T>>(p, xa, s));
            }
        }
        const Planes t = x[0];
        x[0] = x[1];
        x[1] = t;
    }
    return LCN_OK;
}

}  // namespace lcn

using namespace lcn;

extern "C" {

lcn_status lcn_orthogonalise_workspace_bytes(int64_t count, int32_t rows, int32_t cols, int32_t dtype, size_t *bytes)
{
    if (!bytes || !orthogonal_args_fit(count, rows, cols, dtype)) return LCN_ERR_INVALID_ARG;
    *bytes = count == 0 ? 0 : orthogonal_space(nullptr, count, rows, cols).bytes;
    return LCN_OK;
}

lcn_status lcn_orthogonalise(const void *g, int64_t count, int32_t rows, int32_t cols, int32_t dtype, int32_t steps,
                             const float *coefficients, float eps, float scale, void *out, void *workspace, size_t workspace_bytes,
                             void *hip_stream)
{
    if (!orthogonal_args_fit(count, rows, cols, dtype) || steps < 1 || steps > 64 || !coefficients || !(eps >= 0.f) || eps > 3.4e38f ||
        !(__builtin_fabsf(scale) <= 3.4e38f) || !coefficients_fit(steps, coefficients))
        return LCN_ERR_INVALID_ARG;
    if (count == 0) return LCN_OK;
    if (!g || !out) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return orthogonal_as((const float *)g, count, rows, cols, steps, coefficients, eps, scale, (float *)out, (char *)workspace,
                             workspace_bytes, (hipStream_t)hip_stream);
    return orthogonal_as((const __bf16 *)g, count, rows, cols, steps, coefficients, eps, scale, (__bf16 *)out, (char *)workspace,
                         workspace_bytes, (hipStream_t)hip_stream);
}

}  // extern "C"
