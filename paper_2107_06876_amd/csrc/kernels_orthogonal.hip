// X -> X (a + b X^T X + c (X^T X)^2), so many times, from G / (|G| + eps): the singular vectors of G with singular values that
// such polynomials bring near 1, without a decomposition.
//
//   A = X X^T (or X^T X, where that is the smaller one),  B = a + b A + c A^2,  X <- B X (or X B)
//
// Every product is one of two planes of fp16 (product.h): the singular values are bounded by the polynomials, and with them every
// value of X, A and B, so that powers of two in front keep them in fp16's range.  Planes and sums are as exact as single precision,
// which is needed: what rounding adds in the first steps grows as the smallest singular values do, up to a per step.  bf16 matrices
// are one plane in the first step.
//
// Long bf16 matrices take several steps on A alone, which is small: with B_1, B_2, ... as they come, A <- A B^2 and X <- B_r .. B_1 X
// at the end of such a stage.  A then has to tell sigma^2 from the largest one's rounding, 2^-24, where X tells sigma: a stage's
// polynomials grow by 64 at most, so that a singular value whose result they decide is 1/64 of the largest at least, its square
// off by 64^2 2^-24 = 2^-12 of itself in the worst case, which a bf16 result has room for.  4 matrices of 8192 x 1024, 5 steps: 14
// products of 1024^3 at 33 us in place of three of A and of X, at 130 and 170.
//
// A and B are symmetric, and so are the products of two polynomials of one A: tiles on and below the diagonal are computed, and
// written twice.  A is a product with a long k and few tiles: k is split over workgroups, whose sums a second launch adds.
#include "orthogonal.h"

namespace lcn {

// Partial sums of squares of a matrix (blockIdx.y), in 64 bits: squares of floats leave their own range.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void squares_kernel(const T *__restrict__ g, long long size, double *__restrict__ part)
{
    constexpr int V = VEC ? 16 / (int)sizeof(T) : 1;
    typedef T piece __attribute__((ext_vector_type(V)));
    __shared__ double sums[4];
    const piece *p = (const piece *)(g + blockIdx.y * size);
    const long long pieces = size / V;
    double v = 0.0;
#pragma unroll 4
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (long long)NORM_GROUPS * 256) {
        const piece x = p[i];
#pragma unroll
        for (int e = 0; e < V; ++e) v = __builtin_fma((double)(float)x[e], (double)(float)x[e], v);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.y * NORM_GROUPS + blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// Matrix blockIdx.y.  float: SCALE_X G / (|G| + eps) in two planes.  bf16: G times the power of two that brings |G| to between
// SCALE_X / 2 and SCALE_X, in one plane, which holds it (values below 2^-30 |G| to 2^-38 |G|), and what is left of the factor in `ratio`.
template <class T>
__global__ __launch_bounds__(256) void normalise_kernel(const T *__restrict__ g, const double *__restrict__ part, int rows, int cols,
                                                        float eps, Planes out, float *__restrict__ ratio)
{
    double sum = 0.0;
    for (int i = 0; i < NORM_GROUPS; ++i) sum += part[blockIdx.y * NORM_GROUPS + i];
    const double norm = sqrt(sum), inv = (double)SCALE_X / (norm + (double)eps);
    int shift = 0;
    if (sizeof(T) == 2 && norm > 0.0 && norm < __builtin_huge_val()) {
        int e;
        (void)frexp(norm, &e);   // norm = 0.5 .. 1 times 2^e
        shift = 13 - e;
    }
    if (sizeof(T) == 2 && blockIdx.x == 0 && threadIdx.x == 0) ratio[blockIdx.y] = (float)ldexp(inv, -shift);
    const int per_row = (int)(out.ld / 8);
    const T *src = g + (long long)blockIdx.y * rows * cols;
    f16 *dst = out.p + (long long)blockIdx.y * rows * out.ld;
    const long long pieces = (long long)rows * per_row;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < pieces; t += (long long)gridDim.x * 256) {
        const long long r = t / per_row;
        const int k = (int)(t - r * per_row) * 8;
        f32x4 v[2];
        load_eight(src + r * cols + k, cols - k, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = v[e >> 2][e & 3];
            v[e >> 2][e & 3] = k + e >= cols ? 0.f : sizeof(T) == 2 ? __builtin_ldexpf(x, shift) : (float)((double)x * inv);
        }
        if (sizeof(T) == 2) {
            f16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (f16)v[e >> 2][e & 3];
            *(f16x8 *)(dst + t * 8) = o;
        } else {
            store_planes(Planes{dst, out.plane, out.ld}, t * 8, v);
        }
    }
}

// ---- small matrices --------------------------------------------------------------
// All steps of a matrix in one workgroup, X, A and B in planes in LDS.  X lies with its longer side as rows, and results are turned
// so that a lane writes four neighbours.  Bound by the chain of its products and barriers: 8 matrices of 96 x 32, 5 steps, 9.5 us,
// 3.6 of them start, loads and stores (on the float instruction 14.3); 8 of 256 x 64, 30 us (75).
template <class T, int D, int ROWS>
__global__ __launch_bounds__(512) void orthogonal_small_kernel(const T *__restrict__ g, int rows, int cols, int steps, SmallSteps c,
                                                               float eps, float scale, T *out)   // out may be g
{
    typedef Tile<__bf16, D> L;   // of any 16-bit values
    constexpr int N = D / 16;
    __shared__ __align__(1024) char xs[2][ROWS * D * 2];
    __shared__ __align__(1024) char as[2][D * D * 2];
    __shared__ __align__(1024) char bs[2][D * D * 2];
    __shared__ double sums[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = lane >> 4, l = lane & 15;
    const bool wide = rows < cols;
    const int hi = wide ? cols : rows, lo = wide ? rows : cols, blocks = (hi + 31) / 32 * 2;   // of 16 rows, whole chunks of 32 for A
    const T *src = g + (long long)blockIdx.x * rows * cols;
    auto place = [](int r, int k) { return L::place(r, k >> 3) + (k & 7) * 2; };
    auto store = [&](char (*to)[D * D * 2], int r, int k, f32x4 v) {
        f16x4 h, s;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = (f16)v[e];
            s[e] = (f16)(v[e] - (float)h[e]);
        }
        *(f16x4 *)(to[0] + place(r, k)) = h;
        *(f16x4 *)(to[1] + place(r, k)) = s;
    };
    // a product of two planes each: the small ones in `low`
    auto multiply = [](f32x4 &sum, f32x4 &low, const bf16x8(&a)[2], const bf16x8(&b)[2]) {
        low = mfma_f16(a[1], b[0], low);
        sum = mfma_f16(a[0], b[0], sum);
        low = mfma_f16(a[0], b[1], low);
    };
    const f32x4 none = {0.f, 0.f, 0.f, 0.f};
    // Pieces of eight neighbours in memory: of a row of X, or of a column of it where G is wide; X[r][k] is the first of them.
    constexpr int ROW = D / 8, COLUMN = ROWS / 8;
    const int limit = wide ? lo * COLUMN : blocks * 16 * ROW;
    auto row_of = [&](int i) { return wide ? i % COLUMN * 8 : i / ROW; };
    auto col_of = [&](int i) { return wide ? i / COLUMN : i % ROW * 8; };
    auto left_of = [&](int i) { return wide ? hi - row_of(i) : row_of(i) < hi ? lo - col_of(i) : 0; };
    auto index_of = [&](int i) { return wide ? col_of(i) * cols + row_of(i) : row_of(i) * cols + col_of(i); };
    double sum = 0.0;
    for (int i = tid; i < limit; i += 512) {
        f32x4 v[2];
        load_eight(src + index_of(i), left_of(i), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fma((double)v[e >> 2][e & 3], (double)v[e >> 2][e & 3], sum);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = ((sums[0] + sums[1]) + (sums[2] + sums[3])) + ((sums[4] + sums[5]) + (sums[6] + sums[7]));
    const double inv = (double)SCALE_X / (sqrt(sum) + (double)eps);
    const float factor = (float)inv;
    const bool plain = inv > 1e-30 && inv < 1e30;   // neither it nor a value times it leaves a float's range
    if (wide)   // what no piece below fills
        for (int i = tid; i < blocks * 16 * ROW; i += 512)
#pragma unroll
            for (int u = 0; u < 2; ++u) *(f16x8 *)(xs[u] + L::place(i / ROW, i % ROW)) = f16x8{};
    __syncthreads();
    for (int i = tid; i < limit; i += 512) {
        const int r = row_of(i), k = col_of(i);
        f32x4 v[2];
        f16x8 h, q;
        load_eight(src + index_of(i), left_of(i), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = v[e >> 2][e & 3], y = plain ? x * factor : (float)((double)x * inv);
            h[e] = (f16)y;
            q[e] = (f16)(y - (float)h[e]);
        }
        if (!wide) {
            *(f16x8 *)(xs[0] + place(r, k)) = h;
            *(f16x8 *)(xs[1] + place(r, k)) = q;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (r + e < hi) {
                    *(f16 *)(xs[0] + place(r + e, k)) = h[e];
                    *(f16 *)(xs[1] + place(r + e, k)) = q[e];
                }
        }
    }
    for (int s = 0; s < steps; ++s) {
        __syncthreads();
        for (int b = wave; b < N * N; b += 8) {   // A[i][j]: sum over the rows of X
            const int i = b / N * 16, j = b % N * 16;
            f32x4 acc = none, low = none;
            for (int r = 0; r < blocks * 16; r += 32) {
                bf16x8 x[2], y[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    x[u] = L::columns(xs[u], r, i, lane);
                    y[u] = L::columns(xs[u], r, j, lane);
                }
                multiply(acc, low, x, y);
            }
            store(as, j + l, i + 4 * grp, (acc + low) * (SCALE_A / (SCALE_X * SCALE_X)));
        }
        __syncthreads();
        const float square = SCALE_B * c.c[s][2] / (SCALE_A * SCALE_A), linear = SCALE_B * c.c[s][1] / SCALE_A;
        for (int b = wave; b < N * N; b += 8) {   // B = a + b A + c A A
            const int i = b / N * 16, j = b % N * 16;
            f32x4 acc = none, low = none;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                bf16x8 x[2], y[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    x[u] = L::rows(as[u], i, k, lane);
                    y[u] = L::rows(as[u], j, k, lane);
                }
                multiply(acc, low, x, y);
            }
            const int n = j + l, m = i + 4 * grp;
            const f16x4 h = *(const f16x4 *)(as[0] + place(n, m)), q = *(const f16x4 *)(as[1] + place(n, m));
            f32x4 v = (acc + low) * square;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += linear * ((float)h[e] + (float)q[e]) + (m + e == n ? SCALE_B * c.c[s][0] : 0.f);
            store(bs, n, m, v);
        }
        __syncthreads();
        for (int b = wave; b < blocks; b += 8) {   // X <- X B, 16 rows of a wavefront's own
            f32x4 acc[N], low[N];
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] = low[j] = none;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                bf16x8 x[2], y[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) x[u] = L::rows(xs[u], b * 16, k, lane);
#pragma unroll
                for (int j = 0; j < N; ++j) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) y[u] = L::rows(bs[u], j * 16, k, lane);
                    multiply(acc[j], low[j], y, x);
                }
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const f32x4 v = (acc[j] + low[j]) * (1.f / SCALE_B);
                f16x4 h, q;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    h[e] = (f16)v[e];
                    q[e] = (f16)(v[e] - (float)h[e]);
                }
                *(f16x4 *)(xs[0] + place(b * 16 + l, j * 16 + 4 * grp)) = h;
                *(f16x4 *)(xs[1] + place(b * 16 + l, j * 16 + 4 * grp)) = q;
            }
        }
    }
    __syncthreads();
    T *dst = out + (long long)blockIdx.x * rows * cols;
    for (int i = tid; i < limit; i += 512) {
        const int r = row_of(i), k = col_of(i);
        f16x8 h, q;
        if (!wide) {
            h = *(const f16x8 *)(xs[0] + place(r, k));
            q = *(const f16x8 *)(xs[1] + place(r, k));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (r + e < hi) {
                    h[e] = *(const f16 *)(xs[0] + place(r + e, k));
                    q[e] = *(const f16 *)(xs[1] + place(r + e, k));
                }
        }
        f32x4 v[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = ((float)h[e] + (float)q[e]) * (scale / SCALE_X);
        store_eight(dst + index_of(i), v, left_of(i));
    }
}

// ---- host ---------------------------------------------------------------------

static bool orthogonal_args_fit(int64_t count, int32_t rows, int32_t cols, int32_t dtype)
{
    const int32_t lo = rows < cols ? rows : cols;
    return count >= 0 && count <= (1 << 20) && rows >= 1 && cols >= 1 && rows <= MAX_WIDTH && cols <= MAX_WIDTH && lo <= 32768 &&
           (double)count * rows * cols <= (double)((int64_t)1 << 40) &&
           count * ((rows + 63) / 64) * ((cols + 63) / 64) < (int64_t)1 << 31 &&   // a product's tiles are numbered in 31 bits
           (dtype == LCN_F32 || dtype == LCN_BF16);
}

// Whether every step keeps the singular values, which start at 1 or less, within the bounds of orthogonal.h; poly: the largest
// value of every step's polynomial on the way.
static bool coefficients_fit(int32_t steps, const float *c, double *poly)
{
    double s = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double k[3] = {c[3 * i], c[3 * i + 1], c[3 * i + 2]}, top = s * s;
        double most = 0.0;
        poly[i] = 0.0;
        auto at = [&](double t) {   // a singular value sqrt(t), if it can occur
            if (!(t >= 0.0) || t > top) return;
            const double q = __builtin_fabs(k[0] + t * (k[1] + t * k[2]));
            if (!(q <= poly[i])) poly[i] = q;
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
        if (!(most <= MOST_X) || !(poly[i] <= MOST_POLY)) return false;
        s = most;
    }
    return true;
}

static bool small(int32_t rows, int32_t cols)
{
    const int32_t lo = rows < cols ? rows : cols, hi = rows < cols ? cols : rows;
    return (lo <= 32 && hi <= 512) || (lo <= 64 && hi <= 256);
}

template <class T>
static lcn_status small_as(const T *g, int64_t count, int32_t rows, int32_t cols, int32_t steps, const float *c, float eps, float scale,
                           T *out, hipStream_t s)
{
    SmallSteps k{};
    for (int i = 0; i < steps; ++i)
        for (int e = 0; e < 3; ++e) k.c[i][e] = c[3 * i + e];
    const int32_t lo = rows < cols ? rows : cols;
    if (lo <= 32)
        hipLaunchKernelGGL((orthogonal_small_kernel<T, 32, 512>), dim3((unsigned)count), dim3(512), 0, s, g, rows, cols, steps, k, eps,
                           scale, out);
    else
        hipLaunchKernelGGL((orthogonal_small_kernel<T, 64, 256>), dim3((unsigned)count), dim3(512), 0, s, g, rows, cols, steps, k, eps,
                           scale, out);
    OPCHK(hipGetLastError());
    return LCN_OK;
}

// Whether steps are taken on A alone.
static bool by_stages(int32_t rows, int32_t cols, int32_t dtype)
{
    const int64_t lo = rows < cols ? rows : cols, hi = rows < cols ? cols : rows;
    return dtype == LCN_BF16 && hi >= 4 * lo;
}

struct OrthogonalSpace {
    f16 *x[2], *gram, *next, *poly[3];   // next, poly[1 ..]: by stages
    double *part;
    float *ratio, *sums;
    long long size, ld, lo, ldg;   // values of a plane of X and its row; of A and its row
    PairPlan plan_gram, plan_poly, plan_apply;
    size_t bytes;
};
static OrthogonalSpace orthogonal_space(char *ws, int64_t count, int32_t rows, int32_t cols, int32_t dtype)
{
    Carver c{ws};
    OrthogonalSpace o;
    const bool bf16 = dtype == LCN_BF16;
    const int32_t hi = rows < cols ? cols : rows;
    o.ld = padded(cols);
    o.size = count * rows * o.ld;
    o.lo = rows < cols ? rows : cols;
    o.ldg = padded(o.lo);
    o.plan_gram = plan_pair(o.lo, o.lo, hi, count, true, bf16);
    o.plan_poly = plan_pair(o.lo, o.lo, o.lo, count, true, bf16);
    o.plan_apply = plan_pair(cols, rows, o.lo, count, false, bf16);
    for (int i = 0; i < 2; ++i) o.x[i] = (f16 *)c.take((size_t)o.size * 4);
    const size_t square = (size_t)(count * o.lo * o.ldg) * 4;
    const bool more = by_stages(rows, cols, dtype);
    o.gram = (f16 *)c.take(square);
    for (int i = 0; i < 3; ++i) o.poly[i] = i == 0 || more ? (f16 *)c.take(square) : nullptr;
    o.next = more ? (f16 *)c.take(square) : nullptr;
    o.part = (double *)c.take((size_t)count * NORM_GROUPS * 8);
    o.ratio = (float *)c.take((size_t)count * 4);
    const size_t one = pair_part_bytes(o.plan_gram, o.lo, count), two = pair_part_bytes(o.plan_poly, o.lo, count);
    o.sums = (float *)c.take(one > two ? one : two);
    o.bytes = c.used;
    return o;
}

template <class T>
static lcn_status orthogonal_as(const T *g, int64_t count, int32_t rows, int32_t cols, int32_t dtype, int32_t steps, const float *c,
                                const double *most, float eps, float scale, T *out, char *ws, size_t ws_bytes, hipStream_t s)
{
    const OrthogonalSpace o = orthogonal_space(ws, count, rows, cols, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < o.bytes) return LCN_ERR_ALLOC;
    const int n = (int)o.lo;
    Planes x[2] = {{o.x[0], o.size, o.ld}, {o.x[1], o.size, o.ld}};
    auto square = [&](f16 *p) { return Planes{p, count * n * o.ldg, o.ldg}; };
    const long long groups = ((long long)rows * (o.ld / 8) + 255) / 256, size = (long long)rows * cols;
    const bool vec = ((uintptr_t)g & 15) == 0 && size % (16 / (int)sizeof(T)) == 0;
    for (int64_t first = 0; first < count; first += 32768) {   // a grid's second dimension
        const unsigned some = (unsigned)(count - first < 32768 ? count - first : 32768);
        if (vec)
            hipLaunchKernelGGL((squares_kernel<T, true>), dim3(NORM_GROUPS, some), dim3(256), 0, s, g + first * size, size,
                               o.part + first * NORM_GROUPS);
        else
            hipLaunchKernelGGL((squares_kernel<T, false>), dim3(NORM_GROUPS, some), dim3(256), 0, s, g + first * size, size,
                               o.part + first * NORM_GROUPS);
        OPCHK(hipGetLastError());
        Planes to = x[0];
        to.p += first * rows * o.ld;
        hipLaunchKernelGGL(normalise_kernel<T>, dim3((unsigned)(groups < 1024 ? groups : 1024), some), dim3(256), 0, s, g + first * size,
                           o.part + first * NORM_GROUPS, rows, cols, eps, to, o.ratio + first);
        OPCHK(hipGetLastError());
    }
    auto operand = [](const Planes &m) { return Operand{m.p, m.plane * 2, m.ld}; };
    const long long x_batch = rows * o.ld, g_batch = n * o.ldg;
    const bool wide = rows <= cols;
    constexpr int FULL = sizeof(T) == 2 ? PAIR_TWO : PAIR_FLOAT;
    // out = factor * product (+ linear * gram + constant), of symmetric matrices
    auto multiply = [&](f16 *left, f16 *right, f16 *out, float factor, f16 *gram, float linear, float constant) {
        PairArgs p{};
        p.batches = (int)count;
        p.part = o.sums;
        p.a = operand(square(left));
        p.b = operand(square(right));
        p.a_batch = p.b_batch = g_batch * 2;
        p.m = p.n = p.k = n;
        return launch_gram(o.plan_poly, p, {square(out), g_batch, square(gram), factor, linear, constant, nullptr}, true, FULL, s);
    };
    for (int i = 0; i < steps;) {
        // the steps of this stage: as many as the polynomials' growth allows
        int stage = 1;
        if (by_stages(rows, cols, dtype))
            for (double growth = most[i]; i + stage < steps && growth * most[i + stage] <= MOST_POLY; ++stage) growth *= most[i + stage];
        const bool first = sizeof(T) == 2 && i == 0;   // X is one plane, and lacks its ratio
        const float *ratio = first ? o.ratio : nullptr;
        PairArgs p{};
        p.batches = (int)count;
        p.part = o.sums;
        p.a = p.b = operand(x[0]);
        p.a_batch = p.b_batch = x_batch * 2;
        p.m = p.n = n;
        p.k = wide ? cols : rows;
        OPCHK(launch_gram(o.plan_gram, p, {square(o.gram), g_batch, Planes{}, SCALE_A / (SCALE_X * SCALE_X), 0.f, 0.f, ratio}, wide,
                          first ? PAIR_ONE : FULL, s));
        int now = 0, all = 0;   // of o.poly: this step's B, and the product of the stage's
        for (int r = 0; r < stage; ++r) {
            const float *k = c + 3 * (i + r);
            if (r) {   // A <- A B B
                OPCHK(multiply(o.gram, o.poly[now], o.next, 1.f / SCALE_B, nullptr, 0.f, 0.f));
                OPCHK(multiply(o.next, o.poly[now], o.gram, 1.f / SCALE_B, nullptr, 0.f, 0.f));
            }
            int to = 0;
            while (r && (to == now || to == all)) ++to;
            OPCHK(multiply(o.gram, o.gram, o.poly[to], SCALE_B * k[2] / (SCALE_A * SCALE_A), o.gram, SCALE_B * k[1] / SCALE_A, SCALE_B * k[0]));
            if (r) {
                const int together = 3 - to - all;   // neither of them; the last step's B is no longer needed
                OPCHK(multiply(o.poly[to], o.poly[all], o.poly[together], 1.f / SCALE_B, nullptr, 0.f, 0.f));
                all = together;
            }
            now = to;
        }
        // wide: out[r][c] = sum over k of X[k][c] B[r][k];  tall: sum over k of B[c][k] X[r][k]
        const Operand poly = operand(square(o.poly[all]));
        p.m = cols;
        p.n = rows;
        p.k = n;
        p.a = wide ? operand(x[0]) : poly;
        p.b = wide ? poly : operand(x[0]);
        p.a_batch = (wide ? x_batch : g_batch) * 2;
        p.b_batch = (wide ? g_batch : x_batch) * 2;
        const int how = first ? PAIR_ONE : FULL;
        i += stage;
        if (i < steps)
            OPCHK(launch_apply(o.plan_apply, p, {x[1], x_batch, 1.f / SCALE_B, ratio}, wide, how, s));
        else
            OPCHK(launch_apply_last(o.plan_apply, p, {out, size, cols, scale / (SCALE_B * SCALE_X), ratio},
                                    wide, how, s));
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
    *bytes = count == 0 || small(rows, cols) ? 0 : orthogonal_space(nullptr, count, rows, cols, dtype).bytes;
    return LCN_OK;
}

lcn_status lcn_orthogonalise(const void *g, int64_t count, int32_t rows, int32_t cols, int32_t dtype, int32_t steps,
                             const float *coefficients, float eps, float scale, void *out, void *workspace, size_t workspace_bytes,
                             void *hip_stream)
{
    double poly[MOST_STEPS];
    if (!orthogonal_args_fit(count, rows, cols, dtype) || steps < 1 || steps > MOST_STEPS || !coefficients || !(eps >= 0.f) || eps > 3.4e38f ||
        !(__builtin_fabsf(scale) <= 3.4e38f) || !coefficients_fit(steps, coefficients, poly))
        return LCN_ERR_INVALID_ARG;
    if (count == 0) return LCN_OK;
    if (!g || !out) return LCN_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)hip_stream;
    if (small(rows, cols)) {
        if (dtype == LCN_F32)
            return small_as((const float *)g, count, rows, cols, steps, coefficients, eps, scale, (float *)out, s);
        return small_as((const __bf16 *)g, count, rows, cols, steps, coefficients, eps, scale, (__bf16 *)out, s);
    }
    if (dtype == LCN_F32)
        return orthogonal_as((const float *)g, count, rows, cols, dtype, steps, coefficients, poly, eps, scale, (float *)out,
                             (char *)workspace, workspace_bytes, s);
    return orthogonal_as((const __bf16 *)g, count, rows, cols, dtype, steps, coefficients, poly, eps, scale, (__bf16 *)out, (char *)workspace,
                         workspace_bytes, s);
}

}  // extern "C"
