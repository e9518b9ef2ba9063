// y = act(g) u with g = x Wg^T + bg and u = x Wu^T + bu, Wg above Wu in one matrix, and its gradients.
//
// Backward: dz = [dy u act'(g) | dy act(g)] once (as planes of bf16, with the column sums that are the biases' gradients), then
// dx = dz W and dW = dz^T x, which are two products because g's and u's halves lie in one matrix.
//
// Bound by the matrix instruction on many rows (16 391 rows, 1024 -> 4096, bf16: 337 us, of it some 60 of epilogue; backward dz 137, at
// the rate of a copy, dx 257, dW 289) and by reading W on few (one row, 2048 -> 8192, bf16: 11 us for 67 MB).
//
// Rounding: g, u, sums and activations are in 32 bits; with bf16 tensors y, dz, dx, dW and db are rounded once each.  What is
// kept of g and u for the backward pass is 16 bits a value for bf16 tensors, 11 of significand (gated.h); as bf16 each would add
// an error to dz of the size of dz's own rounding, as floats they are half of what moves.
#include "gated.h"

namespace lcn {

// eight outputs from g and u, which have their biases: at row n, column m (a multiple of 8)
template <class T, int ACT>
__device__ __forceinline__ void gated_finish(const GatedArgs<T> &e, f32x4 (&g)[2], const f32x4 (&u)[2], long long n, int m, int width)
{
    if (e.kept) {
        const long long dp = padded(width);
        Keep<T>::store(e.kept + n * 2 * dp + m, g);
        Keep<T>::store(e.kept + (n * 2 + 1) * dp + m, u);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i >> 2][i & 3] = gate<T, ACT>(g[i >> 2][i & 3]) * u[i >> 2][i & 3];
    store_eight(e.y + n * width + m, g, width - m);
}

// The product's epilogue: subtiles of 16 rows are g's and u's in turn.  A wavefront's 16 columns n go through LDS row by row, as in
// by_rows, and a lane takes up eight consecutive values of g and the eight of u that belong to them.
template <class T, int ACT>
struct GatedEpilogue {
    typedef GatedArgs<T> Args;
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0, int,
                               char *lds, int, int)
    {
        static_assert(TM % 2 == 0, "whole pairs");
        constexpr int PITCH = RowRegion<TM>::PITCH;
        const int lane = threadIdx.x & 63;
        float *f = (float *)(lds + (threadIdx.x >> 6) * RowRegion<TM>::BYTES);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
#pragma unroll
            for (int i = 0; i < TM; ++i) *(f32x4 *)(f + (lane & 15) * PITCH + i * 16 + 4 * (lane >> 4)) = acc[i][j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // LDS serves a wavefront in order
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (int q = lane; q < 16 * TM; q += 64) {
                const int r = q / TM, c = q % TM * 8, m = (int)m0 + c;
                const long long n = n0 + j * 16 + r;
                if (n >= p.n || m >= p.m) continue;
                const float *at = f + r * PITCH + (c >> 4) * 32 + (c & 15);
                f32x4 g[2], u[2], b[2];
                g[0] = *(const f32x4 *)at;
                g[1] = *(const f32x4 *)(at + 4);
                u[0] = *(const f32x4 *)(at + 16);
                u[1] = *(const f32x4 *)(at + 20);
                if (e.bias) {
                    load_eight(e.bias + m, p.m - m, b);
                    g[0] += b[0];
                    g[1] += b[1];
                    load_eight(e.bias + p.m + m, p.m - m, b);
                    u[0] += b[0];
                    u[1] += b[1];
                }
                gated_finish<T, ACT>(e, g, u, n, m, p.m);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
};
template <class T, int ACT>
constexpr bool paired_rows<GatedEpilogue<T, ACT>> = true;

// from the sums of [g | u] in memory, `splits` partial ones each
template <class T, int ACT>
__global__ __launch_bounds__(256) void gated_finish_kernel(GatedArgs<T> e, const float *__restrict__ part, int splits,
                                                           long long stride, long long rows, int width, long long ldp)
{
    const int per_row = (width + 7) / 8;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < rows * per_row; t += (long long)gridDim.x * 256) {
        const long long n = t / per_row;
        const int m = (int)(t - n * per_row) * 8, left = width - m;
        f32x4 z[2][2], v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float *p = part + n * ldp + h * width + m;
            load_eight(p, left, z[h]);
            for (int s = 1; s < splits; ++s) {
                load_eight(p + s * stride, left, v);
                z[h][0] += v[0];
                z[h][1] += v[1];
            }
            if (e.bias) {
                load_eight(e.bias + h * width + m, left, v);
                z[h][0] += v[0];
                z[h][1] += v[1];
            }
        }
        gated_finish<T, ACT>(e, z[0], z[1], n, m, width);
    }
}

template <int N>
struct Number {
    static constexpr int value = N;
};
// The dot products of rows w0 and w1 with R rows of x (`rows` of them exist), shared by 16 lanes, in each of them: in pieces of 16
// bytes wherever rows lie, several of them requested before the first is worked on.  One row, 4096 -> 2 x 4096 bf16, 16 us with a
// compiler's order of the loads, 11.5 so; eight 26 and 23; one, 2047 -> 2 x 8191, 24 value by value and 13.
template <class T, int R>
__device__ __forceinline__ void dot_of_rows(const T *__restrict__ w0, const T *__restrict__ w1, const T *__restrict__ x, int rows, int k,
                                            float (&sum)[2][R])
{
    constexpr int V = 16 / (int)sizeof(T), AHEAD = R <= 2 ? 4 : 2;
    typedef T piece __attribute__((ext_vector_type(V)));
    typedef T any __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    const int lane = threadIdx.x & 15, whole = k - k % V;
    auto add = [&](int c, auto count) {
        constexpr int U = decltype(count)::value;
        piece a[U], b[U], y[U][R];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            a[u] = *(const any *)(w0 + c + u * 16 * V);
            b[u] = *(const any *)(w1 + c + u * 16 * V);
#pragma unroll
            for (int r = 0; r < R; ++r) y[u][r] = *(const any *)(x + (long long)(r < rows ? r : 0) * k + c + u * 16 * V);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    sum[0][r] = __builtin_fmaf((float)a[u][e], (float)y[u][r][e], sum[0][r]);
                    sum[1][r] = __builtin_fmaf((float)b[u][e], (float)y[u][r][e], sum[1][r]);
                }
    };
    int c = lane * V;
    for (; c + (AHEAD - 1) * 16 * V < whole; c += AHEAD * 16 * V) add(c, Number<AHEAD>());
    for (; c < whole; c += 16 * V) add(c, Number<1>());
    if (whole + lane < k) {   // behind the last whole piece
        const float a = (float)w0[whole + lane], b = (float)w1[whole + lane];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float y = (float)x[(long long)(r < rows ? r : 0) * k + whole + lane];
            sum[0][r] = __builtin_fmaf(a, y, sum[0][r]);
            sum[1][r] = __builtin_fmaf(b, y, sum[1][r]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum[f][r] += __shfl_xor(sum[f][r], o, 16);
}

// Few rows: bound by reading W once; 16 lanes read a row of Wg and the one of Wu that belongs to it, a workgroup has 16 outputs.
template <class T, int R>
__global__ __launch_bounds__(256) void gated_few_kernel(GatedArgs<T> e, const T *__restrict__ x, const T *__restrict__ w, int rows,
                                                        int k, int width)
{
    __shared__ float z[R][2][16];
    const int group = threadIdx.x >> 4, f = (int)blockIdx.x * 16 + group, lane = threadIdx.x & 15;
    const int fr = f < width ? f : width - 1;
    float sum[2][R];
#pragma unroll
    for (int r = 0; r < R; ++r) sum[0][r] = sum[1][r] = 0.f;
    dot_of_rows<T, R>(w + (long long)fr * k, w + (long long)(width + fr) * k, x, rows, k, sum);
    float g = 0.f, u = 0.f;   // lane r finishes one value
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i == lane) {
            g = sum[0][i];
            u = sum[1][i];
        }
    if (e.bias) {
        g += (float)e.bias[fr];
        u += (float)e.bias[width + fr];
    }
    if (e.kept && lane < R) {
        z[lane][0][group] = f < width ? g : 0.f;
        z[lane][1][group] = f < width ? u : 0.f;
    }
    if (lane < rows && f < width) {
        switch (e.act) {
        case LCN_ACT_TANH: g = gate<T, LCN_ACT_TANH>(g); break;
        case LCN_ACT_RELU: g = gate<T, LCN_ACT_RELU>(g); break;
        case LCN_ACT_GELU: g = gate<T, LCN_ACT_GELU>(g); break;
        case LCN_ACT_SILU: g = gate<T, LCN_ACT_SILU>(g); break;
        }
        e.y[(long long)lane * width + f] = (T)(g * u);
    }
    if (!e.kept) return;
    __syncthreads();
    // two pieces of g and two of u for every row
    const int r = threadIdx.x >> 2, half = threadIdx.x >> 1 & 1, m = (int)blockIdx.x * 16 + (threadIdx.x & 1) * 8;
    if (r >= rows || m >= width) return;
    f32x4 v[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = z[r][half][(threadIdx.x & 1) * 8 + i];
    Keep<T>::store(e.kept + ((long long)r * 2 + half) * padded(width) + m, v);
}

template <class T, int R>
static hipError_t launch_few(const GatedArgs<T> &e, const T *x, const T *w, int rows, int k, int width, hipStream_t s)
{
    const unsigned grid = (unsigned)((width + 15) / 16);
    hipLaunchKernelGGL((gated_few_kernel<T, R>), dim3(grid), dim3(256), 0, s, e, x, w, rows, k, width);
    return hipGetLastError();
}

// dz as planes (dst: nullable; rows of dp values, zero behind 2 width), and the sums over this workgroup's rows for every column
// (part: nullable).  C pieces of eight columns of either half x 256 / C rows at a time.
template <class T, int ACT, int C, int PLANES>
__global__ __launch_bounds__(256) void gated_slope_kernel(const T *__restrict__ dy, const typename Keep<T>::type *__restrict__ kept,
                                                          long long rows, int width, int dp, int rows_each,
                                                          __bf16 *__restrict__ dst, float *__restrict__ part)
{
    constexpr int R = 256 / C;
    __shared__ float sums[R][C][17];
    const int c = threadIdx.x % C, q = threadIdx.x / C, k = ((int)blockIdx.x * C + c) * 8, left = width - k, wp = (int)padded(width);
    const long long plane = rows * dp, r0 = (long long)blockIdx.y * rows_each;
    float total[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) total[0][e] = total[1][e] = 0.f;
    if (k < width)
        for (long long r = r0 + q; r < r0 + rows_each && r < rows; r += R) {
            f32x4 d[2], z[2][2];
            load_eight(dy + r * width + k, left, d);
            Keep<T>::load(kept + r * 2 * wp + k, z[0]);
            Keep<T>::load(kept + (r * 2 + 1) * wp + k, z[1]);
            bf16x8 o[2][PLANES];
#pragma unroll
            for (int e = 0; e < 8; ++e) {   // what is behind a row's end is zero in dy and kept
                const float v = d[e >> 2][e & 3];
                float a, slope;
                gate_and_slope<T, ACT>(z[0][e >> 2][e & 3], a, slope);
                const float y[2] = {v * z[1][e >> 2][e & 3] * slope, v * a};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    total[h][e] += y[h];
                    if constexpr (PLANES == 1) {
                        o[h][0][e] = (__bf16)y[h];
                    } else {
                        __bf16 p[3];
                        split_planes(y[h], p[0], p[1], p[2]);
#pragma unroll
                        for (int u = 0; u < PLANES; ++u) o[h][u][e] = p[u];
                    }
                }
            }
            if (dst) {
#pragma unroll
                for (int p = 0; p < PLANES; ++p) {
                    __bf16 *first = dst + p * plane + r * dp + k;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (left >= 8) {
                            typedef bf16x8 any __attribute__((aligned(2)));
                            *(any *)(first + h * width) = o[h][p];
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (e < left) first[h * width + e] = o[h][p][e];
                            if (h && left < 8)   // the last piece of a row: what is behind it becomes zero
                                for (int e = left; e < dp - width - k; ++e) first[width + e] = (__bf16)0.f;
                        }
                    }
                }
            }
        }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sums[q][c][e] = total[0][e];
        sums[q][c][8 + e] = total[1][e];
    }
    __syncthreads();
    // a thread adds up a column of either half
    for (int i = threadIdx.x; i < C * 16; i += 256) {
        const int h = i / (C * 8), cc = i % (C * 8) >> 3, e = i & 7, col = (int)blockIdx.x * C * 8 + i % (C * 8);
        float v = 0.f;
#pragma unroll
        for (int u = 0; u < R; ++u) v += sums[u][cc][h * 8 + e];
        if (col < width) part[((long long)blockIdx.y * 2 + h) * width + col] = v;
    }
}

// ---- host ---------------------------------------------------------------------

static bool gated_args_fit(int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    return rows >= 0 && rows <= MAX_ROWS && d_in >= 1 && d_in <= MAX_WIDTH && d_out >= 1 && d_out <= MAX_WIDTH / 2 &&
           sizes_fit(rows, d_in) && sizes_fit(rows, 2 * (int64_t)d_out) && (dtype == LCN_F32 || dtype == LCN_BF16);
}

// A product in two launches where that is estimated to be faster: whole rounds of workgroups of one shape, and the columns behind
// them by another, whose k may be split.  20 000 float rows: 1024 -> 300, 111 us by 64 x 64 tiles in three rounds, 105 as one round of
// 320 x 64 and the rest; 16391 bf16 rows, 8192 -> 1024: the 7 rows behind 16384 took 64 us in one piece of k, 12 in 32.
// More than 640 tiles of 64 x 64 are taken as 15 % slower than product_us says (with the gates' epilogue, and on rows that are no whole
// lines): by them / by larger ones, us, dx of 4000 rows, 4006 -> 1001 bf16, 72 / 57, of 2048, 4096 -> 2048, 58 / 49; y of 9001, 517 -> 301
// float 66 / 52; of 512 tiles, dz and dx of 2048, 2048 -> 1024 bf16, 31 / 35.
struct Columns {
    ProductPlan main, rest;
    long long whole, n;
    float *part, *part_rest;
};
static Columns plan_columns(Carver &c, long long m, long long n, long long k, int planes, bool may_320)
{
    Columns r{};
    r.main = plan_product(m, n, k, planes, true, false, may_320);
    r.n = r.whole = n;
    auto weighed = [&](int t, double us, long long columns) {
        return t == TILE_64 && (m + 63) / 64 * ((columns + 63) / 64) > 640 ? 1.15 * us : us;
    };
    double least = weighed(r.main.tile, r.main.us, n);
    for (int t = 0; t < TILE_COUNT; ++t) {
        if (t == TILE_320 && !may_320) continue;
        const double alone = weighed(t, product_us(t, m, n, k, planes, 1), n);
        if (alone < least) {
            least = alone;
            r.main = ProductPlan{t, 1, false, alone};
            r.whole = n;
        }
        const long long across = (m + tile_m(t) - 1) / tile_m(t), round = product_room(t, planes) / across * tile_n(t, planes);
        const long long tiles = n - n % tile_n(t, planes);   // whole tiles, and whole rounds of them
        for (long long whole : {tiles, round > 0 ? n - n % round : 0}) {
            if (whole <= 0 || whole >= n) continue;
            const ProductPlan rest = plan_product(m, n - whole, k, planes, true, false, may_320);
            const double us = weighed(t, product_us(t, m, whole, k, planes, 1), whole) + 3.0 + rest.us;
            if (us < least) {
                least = us;
                r.main = ProductPlan{t, 1, false, us};
                r.rest = rest;
                r.whole = whole;
            }
        }
    }
    r.part = (float *)c.take(partial_bytes(r.main, m, r.whole));
    r.part_rest = r.whole < n ? (float *)c.take(partial_bytes(r.rest, m, n - r.whole)) : nullptr;
    return r;
}
// calls f(first column, columns, plan, partial sums) for both
template <class F>
static hipError_t by_columns(const Columns &c, F f)
{
    const hipError_t st = f((long long)0, (int)c.whole, c.main, c.part);
    return st != hipSuccess || c.whole == c.n ? st : f(c.whole, (int)(c.n - c.whole), c.rest, c.part_rest);
}
static Operand from_column(Operand o, long long n)
{
    o.p = (const char *)o.p + n * o.ld * 2;
    return o;
}

struct GatedForward {
    void *xp, *wp;
    Columns y;
    size_t bytes;
};
static GatedForward gated_forward_space(char *ws, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    Carver c{ws};
    GatedForward f;
    f.xp = c.take(planes_bytes(rows, d_in, planes_of(dtype)));
    f.wp = c.take(planes_bytes(2 * d_out, d_in, planes_of(dtype)));
    f.y = plan_columns(c, 2 * d_out, rows, d_in, planes_of(dtype), false);
    f.bytes = c.used;
    return f;
}

struct GatedBackward {
    void *xp, *wp, *dz;
    float *sums, *narrow;
    Columns dx, dw;
    int planes, groups, rows_each;   // planes of dz
    size_t bytes;
};
static GatedBackward gated_backward_space(char *ws, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    Carver c{ws};
    GatedBackward b;
    const int32_t wide = 2 * d_out;
    b.planes = gradient_planes(rows, dtype);
    // workgroups of dz: 256 columns each, and so many rows that there are some ten to a compute unit, with up to 512 partial sums per
    // column (13 502 rows of 211 in bf16: 211 workgroups 25 us, 422 16; 2000 of 512 floats, 126 13, 500 8; 16 391 of 4096 in bf16, 2736 138,
    // 3648 144)
    const int64_t blocks = (d_out + 255) / 256, most = blocks > 20 ? 128 : blocks > 5 ? 2720 / blocks : 512;
    const int64_t unit = d_out <= 64 ? 32 : d_out <= 128 ? 16 : 8;   // rows at a time
    b.rows_each = (int)(((rows + most - 1) / most + unit - 1) / unit * unit);
    b.groups = (int)((rows + b.rows_each - 1) / b.rows_each);
    b.xp = c.take(planes_bytes(rows, d_in, planes_of(dtype)));
    b.wp = c.take(planes_bytes(wide, d_in, planes_of(dtype)));
    b.dz = c.take(planes_bytes(rows, wide, b.planes));
    b.dx = plan_columns(c, d_in, rows, wide, b.planes, true);
    b.dw = plan_columns(c, d_in, wide, rows, b.planes, true);
    b.sums = (float *)c.take((size_t)b.groups * wide * 4);
    b.narrow = (float *)b.xp;   // in place of all others
    const size_t sums = gated_narrow(rows, d_in, d_out) ? (size_t)gated_narrow_groups(rows) * wide * (d_in + 1) * 4 : 0;
    b.bytes = c.used > sums ? c.used : sums;
    return b;
}

template <class T>
static lcn_status gated_as(const T *x, const T *w, const T *bias, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype,
                           int32_t act, T *y, typename Keep<T>::type *kept, char *ws, size_t ws_bytes, hipStream_t s)
{
    GatedArgs<T> e{bias, y, kept, act};
    if (rows <= FEW_ROWS) {
        const int r = (int)rows;
        OPCHK(r == 1   ? launch_few<T, 1>(e, x, w, r, d_in, d_out, s)
              : r == 2 ? launch_few<T, 2>(e, x, w, r, d_in, d_out, s)
              : r <= 4 ? launch_few<T, 4>(e, x, w, r, d_in, d_out, s)
                       : launch_few<T, 8>(e, x, w, r, d_in, d_out, s));
        return LCN_OK;
    }
    if constexpr (sizeof(T) == 4)
        if (gated_some(rows, d_in, dtype)) {
            OPCHK(launch_gated_some(e, x, w, (int)rows, d_in, d_out, s));
            return LCN_OK;
        }
    if (gated_narrow(rows, d_in, d_out)) {
        OPCHK(launch_gated_narrow(e, x, w, rows, d_in, d_out, s));
        return LCN_OK;
    }
    const GatedForward f = gated_forward_space(ws, rows, d_in, d_out, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < f.bytes) return LCN_ERR_ALLOC;
    ProductArgs p{};
    PlaneJobs jobs;
    p.a = add_operand(jobs, w, 2 * d_out, d_in, dtype, f.wp);
    p.b = add_operand(jobs, x, rows, d_in, dtype, f.xp);
    OPCHK(launch_planes(jobs, dtype, s));
    p.k = d_in;
    p.planes = planes_of(dtype);
    OPCHK(by_columns(f.y, [&](long long first, int n, const ProductPlan &plan, float *part) {
        constexpr int NP = sizeof(T) == 4 ? 3 : 1;
        ProductArgs q = p;
        GatedArgs<T> to = e;
        q.b = from_column(p.b, first);
        q.n = n;
        to.y += first * d_out;
        if (to.kept) to.kept += first * 2 * padded(d_out);
        if (plan.splits == 1) {
            q.m = d_out;
            return by_activation(act, [&](auto a) {
                return launch_planned<NP, false, false, GatedEpilogue<T, decltype(a)::value>>(plan, q, to, s);
            });
        }
        q.m = 2 * d_out;
        const long long ldp = padded(2 * d_out), groups = ((long long)n * ((d_out + 7) / 8) + 255) / 256;
        const hipError_t st = launch_planned<NP, false, false, PartialEpilogue>(plan, q, {part, ldp, n * ldp, 0}, s);
        if (st != hipSuccess) return st;
        return by_activation(act, [&](auto a) {
            hipLaunchKernelGGL((gated_finish_kernel<T, decltype(a)::value>), dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256),
                               0, s, to, part, plan.splits, n * ldp, (long long)n, d_out, ldp);
            return hipGetLastError();
        });
    }));
    return LCN_OK;
}

template <class T>
static lcn_status gated_backward_as(const T *x, const T *w, const typename Keep<T>::type *kept, const T *dy, int64_t rows, int32_t d_in, int32_t d_out,
                                    int32_t dtype, int32_t act, T *dx, T *dw, T *dbias, char *ws, size_t ws_bytes, hipStream_t s)
{
    const GatedBackward b = gated_backward_space(ws, rows, d_in, d_out, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < b.bytes) return LCN_ERR_ALLOC;
    if (gated_narrow(rows, d_in, d_out) && x && w) {
        OPCHK(launch_gated_narrow_backward(x, w, kept, dy, rows, d_in, d_out, act, dx, dw, dbias, b.narrow, s));
        return LCN_OK;
    }
    const int32_t wide = 2 * d_out;
    const int dp = (int)padded(wide);
    OPCHK(by_activation(act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        auto launch = [&](auto kernel, int pieces) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((d_out + pieces * 8 - 1) / (pieces * 8)), (unsigned)b.groups), dim3(256), 0, s, dy,
                               kept, (long long)rows, d_out, dp, b.rows_each,
                               dx || dw ? (__bf16 *)b.dz : nullptr, dbias ? b.sums : nullptr);
            return hipGetLastError();
        };
        constexpr int MOST = sizeof(T) == 4 ? 3 : 2;
        if constexpr (MOST == 2)
            if (b.planes == 1)
                return d_out <= 64    ? launch(gated_slope_kernel<T, ACT, 8, 1>, 8)
                       : d_out <= 128 ? launch(gated_slope_kernel<T, ACT, 16, 1>, 16)
                                      : launch(gated_slope_kernel<T, ACT, 32, 1>, 32);
        return d_out <= 64    ? launch(gated_slope_kernel<T, ACT, 8, MOST>, 8)
               : d_out <= 128 ? launch(gated_slope_kernel<T, ACT, 16, MOST>, 16)
                              : launch(gated_slope_kernel<T, ACT, 32, MOST>, 32);
    }));
    if (dbias) OPCHK(launch_column_sums(b.sums, b.groups, wide, dtype, dbias, s));
    ProductArgs p{};
    PlaneJobs jobs;
    Operand xo{}, wo{};
    if (dx) wo = add_operand(jobs, w, wide, d_in, dtype, b.wp);
    if (dw) xo = add_operand(jobs, x, rows, d_in, dtype, b.xp);
    OPCHK(launch_planes(jobs, dtype, s));
    p.planes = b.planes;
    p.m = d_in;
    const Operand dz = plane_operand(b.dz, rows, wide);
    if (dx) {
        p.a = wo;
        p.k = wide;
        OPCHK(by_columns(b.dx, [&](long long first, int n, const ProductPlan &plan, float *part) {
            p.b = from_column(dz, first);
            p.n = n;
            return launch_scaled<true, false>(plan, p, 1.f, dtype, dx + first * d_in, part, s);
        }));
    }
    if (dw) {
        p.a = xo;
        p.k = (int)rows;
        OPCHK(by_columns(b.dw, [&](long long first, int n, const ProductPlan &plan, float *part) {
            p.b = dz;   // its columns are the result's
            p.b.p = (const char *)p.b.p + first * 2;
            p.n = n;
            return launch_scaled<true, true>(plan, p, 1.f, dtype, dw + first * d_in, part, s);
        }));
    }
    return LCN_OK;
}

}  // namespace lcn

using namespace lcn;

extern "C" {

lcn_status lcn_gated_linear_kept_bytes(int64_t rows, int32_t d_out, int32_t dtype, size_t *bytes)
{
    if (!bytes || !gated_args_fit(rows, 1, d_out, dtype)) return LCN_ERR_INVALID_ARG;
    *bytes = (size_t)rows * 2 * (size_t)padded(d_out) * (dtype == LCN_F32 ? 4 : 2);
    return LCN_OK;
}

lcn_status lcn_gated_linear_workspace_bytes(int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype, int32_t backward,
                                            size_t *bytes)
{
    if (!bytes || !gated_args_fit(rows, d_in, d_out, dtype)) return LCN_ERR_INVALID_ARG;
    *bytes = 0;
    if (rows == 0 || (!backward && (rows <= FEW_ROWS || gated_some(rows, d_in, dtype) || gated_narrow(rows, d_in, d_out)))) return LCN_OK;
    *bytes = backward ? gated_backward_space(nullptr, rows, d_in, d_out, dtype).bytes
                      : gated_forward_space(nullptr, rows, d_in, d_out, dtype).bytes;
    return LCN_OK;
}

lcn_status lcn_gated_linear(const void *x, const void *W, const void *bias, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype,
                            int32_t activation, void *y, void *kept, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!gated_args_fit(rows, d_in, d_out, dtype) || activation < LCN_ACT_NONE || activation > LCN_ACT_SILU)
        return LCN_ERR_INVALID_ARG;
    if (rows == 0) return LCN_OK;
    if (!x || !W || !y || ((uintptr_t)kept & 15)) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return gated_as((const float *)x, (const float *)W, (const float *)bias, rows, d_in, d_out, dtype, activation, (float *)y,
                        (float *)kept, (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
    return gated_as((const __bf16 *)x, (const __bf16 *)W, (const __bf16 *)bias, rows, d_in, d_out, dtype, activation, (__bf16 *)y,
                    (unsigned short *)kept, (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
}

lcn_status lcn_gated_linear_backward(const void *x, const void *W, const void *kept, const void *dy, int64_t rows, int32_t d_in,
                                     int32_t d_out, int32_t dtype, int32_t activation, void *dx, void *dW, void *dbias,
                                     void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!gated_args_fit(rows, d_in, d_out, dtype) || activation < LCN_ACT_NONE || activation > LCN_ACT_SILU)
        return LCN_ERR_INVALID_ARG;
    if (!dx && !dW && !dbias) return LCN_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    const size_t e = dtype == LCN_F32 ? 4 : 2;
    if (rows == 0) {   // no rows: the parameters' gradients are zero
        if (dW) OPCHK(launch_zero(dW, (size_t)d_in * 2 * d_out * e, s));
        if (dbias) OPCHK(launch_zero(dbias, (size_t)2 * d_out * e, s));
        return LCN_OK;
    }
    if (!dy || !kept || ((uintptr_t)kept & 15) || (dx && !W) || (dW && !x)) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return gated_backward_as((const float *)x, (const float *)W, (const float *)kept, (const float *)dy, rows, d_in, d_out, dtype, activation,
                                 (float *)dx, (float *)dW, (float *)dbias, (char *)workspace, workspace_bytes, s);
    return gated_backward_as((const __bf16 *)x, (const __bf16 *)W, (const unsigned short *)kept, (const __bf16 *)dy, rows, d_in, d_out, dtype, activation,
                             (__bf16 *)dx, (__bf16 *)dW, (__bf16 *)dbias, (char *)workspace, workspace_bytes, s);
}

}  // extern "C"
