// y = act(x W^T + b) + r and its gradients.
//
// One product on the matrix instruction with everything else in its epilogue; the backward pass forms
// dz = dy act'(z) once (as planes of bf16, with the column sums that are db), then dx = dz W and dW = dz^T x, whose operands
// are read as they lie: a product takes either index of an operand as the contiguous one.  16391 rows, 1024 -> 4096, bf16,
// GELU, residual, z kept: forward 295 us (the product alone 160; 536 MB of z, residual and y at the rate of a copy 123),
// backward 131 for dz and its sums, 162 for dx, 157 for dW, 9 for the sums' last step.
//
// Rounding: z, sums and activations are in 32 bits; with bf16 tensors y, dz, dx, dW and db are rounded once each, the kept
// z is not (as bf16 it would add an error to dz of the size of dz's own rounding).
#include "fragments.h"

namespace lcn {

template <class T>
struct LinearArgs {
    const T *bias, *residual;
    T *y;
    float *pre;
    int act, whole;   // whole: rows of y, residual, bias and pre are whole 16-byte pieces
};

template <class T, int ACT>
__device__ __forceinline__ void linear_finish(const LinearArgs<T> &e, f32x4 (&z)[2], const Eight<T> &residual, long long at,
                                              int left)
{
    if (e.pre) store_eight(e.pre + at, z, left, e.whole);
#pragma unroll
    for (int u = 0; u < 8; ++u) z[u >> 2][u & 3] = activate<ACT>(z[u >> 2][u & 3]);
    if (e.residual) {
#pragma unroll
        for (int u = 0; u < 8; ++u) z[u >> 2][u & 3] += (float)residual.v[u];
    }
    store_eight(e.y + at, z, left, e.whole);
}

template <class T, int ACT>
struct LinearEpilogue {
    typedef LinearArgs<T> Args;
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0, int,
                               char *lds, int, int)
    {
        const int lane = threadIdx.x & 63;
        char *region = lds + (threadIdx.x >> 6) * RowRegion<TM>::BYTES;
        f32x4 bias[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const long long m = m0 + i * 16 + 4 * (lane >> 4);
            bias[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (e.bias && m < p.m) bias[i] = load_four(e.bias + m, (int)(p.m - m), e.whole);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) col[i] = acc[i][j] + bias[i];
            by_rows<TM>(
                region, col, lane,
                [&](int r, int c) {
                    const long long n = n0 + j * 16 + r, m = m0 + c;
                    return e.residual && n < p.n && m < p.m ? read_eight(e.residual + n * p.m + m, (int)(p.m - m), e.whole) : Eight<T>{};
                },
                [&](int r, int c, f32x4 (&v)[2], const Eight<T> &o) {
                    const long long n = n0 + j * 16 + r, m = m0 + c;
                    if (n < p.n && m < p.m) linear_finish<T, ACT>(e, v, o, n * p.m + m, (int)(p.m - m));
                });
        }
    }
};

// the epilogue of a product whose k was shared by workgroups
template <class T, int ACT>
__global__ __launch_bounds__(256) void linear_finish_kernel(LinearArgs<T> e, const float *__restrict__ part, int splits,
                                                            long long stride, long long rows, int width, long long ldp)
{
    const int per_row = (width + 7) / 8;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < rows * per_row; t += (long long)gridDim.x * 256) {
        const long long n = t / per_row;
        const int m = (int)(t - n * per_row) * 8, left = width - m;
        f32x4 z[2], v[2];
        Eight<T> r{};
        load_eight(part + n * ldp + m, 8, true, z);
        for (int u = 1; u < splits; ++u) {
            load_eight(part + u * stride + n * ldp + m, 8, true, v);
            z[0] += v[0];
            z[1] += v[1];
        }
        if (e.bias) {
            load_eight(e.bias + m, left, e.whole, v);
            z[0] += v[0];
            z[1] += v[1];
        }
        if (e.residual) r = read_eight(e.residual + n * width + m, left, e.whole);
        linear_finish<T, ACT>(e, z, r, n * width + m, left);
    }
}

// Few rows: bound by reading W once; 16 lanes read a row of W, a wavefront eight rows.  One row, 2048 -> 8192 in bf16: 9.0 us, 3.7 TB/s
// (launch and one trip to memory included; the floor of 33.6 MB is 5.6 us).  Rows 4 / 8, 1024 -> 4096, here and as a product:
// float 8 / 12 and 27 / 26 us, bf16 5 / 7 and 6 / 6.
template <class T, int R, bool VEC>
__global__ __launch_bounds__(256) void linear_few_kernel(LinearArgs<T> e, const T *__restrict__ x, const T *__restrict__ w,
                                                         int rows, int k, int width)
{
    const int group = (int)(blockIdx.x * 16 + (threadIdx.x >> 4)), f = group * 2;
    if (f >= width) return;
    const int f1 = f + 1 < width ? f + 1 : f;
    float sum[2][R];
#pragma unroll
    for (int r = 0; r < R; ++r) sum[0][r] = sum[1][r] = 0.f;
    few_rows_dot<T, R, VEC>(w + (long long)f * k, w + (long long)f1 * k, x, rows, k, sum);
    // lane r * 2 + (which of the two rows of W) finishes one value
    const int lane = threadIdx.x & 15, r = lane >> 1, which = lane & 1;
    if (r >= rows || f + which >= width) return;
    float z = 0.f;
#pragma unroll
    for (int u = 0; u < R; ++u)
        if (u == r) z = which ? sum[1][u] : sum[0][u];
    const long long at = (long long)r * width + f + which;
    if (e.bias) z += (float)e.bias[f + which];
    if (e.pre) e.pre[at] = z;
    switch (e.act) {
    case LCN_ACT_TANH: z = activate<LCN_ACT_TANH>(z); break;
    case LCN_ACT_RELU: z = activate<LCN_ACT_RELU>(z); break;
    case LCN_ACT_GELU: z = activate<LCN_ACT_GELU>(z); break;
    case LCN_ACT_SILU: z = activate<LCN_ACT_SILU>(z); break;
    }
    if (e.residual) z += (float)e.residual[at];
    e.y[at] = (T)z;
}

template <class T, int R>
static hipError_t launch_few(const LinearArgs<T> &e, const T *x, const T *w, int rows, int k, int width, hipStream_t s)
{
    const unsigned grid = (unsigned)((width + 31) / 32);
    if (k % (16 / (int)sizeof(T)) == 0 && (((uintptr_t)x | (uintptr_t)w) & 15) == 0)
        hipLaunchKernelGGL((linear_few_kernel<T, R, true>), dim3(grid), dim3(256), 0, s, e, x, w, rows, k, width);
    else
        hipLaunchKernelGGL((linear_few_kernel<T, R, false>), dim3(grid), dim3(256), 0, s, e, x, w, rows, k, width);
    return hipGetLastError();
}

// Narrow layers (few inputs and outputs) on many rows: bound by reading x and writing y, so nothing is laid out first.
// A workgroup has 64 outputs, their weights in registers, and a wavefront goes over rows 16 at a time, straight from
// memory into the matrix instruction (float: the float one, whose rate suffices here).  40 961 float rows, 32 -> 32 with tanh: 8 us,
// 1.3 TB/s; the launch and the chain row, product, tanh, store are most of it.
template <class T, int KP, int ACT, bool VEC>
__global__ __launch_bounds__(256) void linear_narrow_kernel(LinearArgs<T> e, const T *__restrict__ x, const T *__restrict__ w,
                                                            long long rows, int k, int width)
{
    constexpr int C = KP / 32;
    const int lane = threadIdx.x & 63, g = lane >> 4, m0 = (int)blockIdx.y * 64;
    typename Frag<T>::type fw[4][C];
    f32x4 bias[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + i * 16 + (lane & 15), mb = m0 + i * 16 + 4 * g;
#pragma unroll
        for (int c = 0; c < C; ++c) fw[i][c] = read_fragment<T, VEC>(m < width ? w + (long long)m * k : nullptr, 32 * c + 8 * g, k);
        bias[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (e.bias && mb < width) bias[i] = load_four(e.bias + mb, width - mb, e.whole);
    }
    const long long tiles = (rows + 15) / 16, step = (long long)gridDim.x * 4;
    for (long long t = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); t < tiles; t += step) {
        const long long n = t * 16 + (lane & 15);
        const T *row = n < rows ? x + n * k : nullptr;
        f32x4 acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = bias[i];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const typename Frag<T>::type fx = read_fragment<T, VEC>(row, 32 * c + 8 * g, k);
#pragma unroll
            for (int i = 0; i < 4; ++i) mma(acc[i], fw[i][c], fx);
        }
        if (n >= rows) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = m0 + i * 16 + 4 * g;
            if (m >= width) continue;
            const long long at = n * width + m;
            if (e.pre) store_four(e.pre + at, acc[i], width - m, e.whole);
            f32x4 y;
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = activate<ACT>(acc[i][u]);
            if (e.residual) y += load_four(e.residual + at, width - m, e.whole);
            store_four(e.y + at, y, width - m, e.whole);
        }
    }
}

// dz = dy act'(z) as planes (dst: nullable), and the sums over this workgroup's rows for every column (part: nullable).
// 32 pieces of eight columns x 8 rows at a time.  Bound by memory: 16391 x 4096, bf16, GELU: 130 us, 4.1 TB/s (a copy: 4.4).
template <class T, int ACT>
__global__ __launch_bounds__(256) void slope_kernel(const T *__restrict__ dy, const float *__restrict__ pre, long long rows,
                                                    int width, int dp, int rows_each, int whole,
                                                    int planes, __bf16 *__restrict__ dst, float *__restrict__ part)
{
    __shared__ float sums[8][32][9];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5, k = ((int)blockIdx.x * 32 + c) * 8;
    const long long plane = rows * dp, r0 = (long long)blockIdx.y * rows_each;
    float total[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) total[e] = 0.f;
    if (k < dp)
        for (long long r = r0 + q; r < r0 + rows_each && r < rows; r += 8) {
            f32x4 v[2];
            load_eight(dy + r * width + k, width - k, whole, v);
            if constexpr (ACT != LCN_ACT_NONE) {
                f32x4 z[2];
                load_eight(pre + r * width + k, width - k, whole, z);
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u >> 2][u & 3] *= activate_slope<ACT>(z[u >> 2][u & 3]);
            }
            bf16x8 o[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __bf16 a, b, d;
                const float y = k + e < width ? v[e >> 2][e & 3] : 0.f;
                total[e] += y;
                split_planes(y, a, b, d);
                o[0][e] = a;
                o[1][e] = b;
                o[2][e] = d;
            }
            if (dst) {
                *(bf16x8 *)(dst + r * dp + k) = o[0];
                if (planes > 1) *(bf16x8 *)(dst + plane + r * dp + k) = o[1];
                if (planes > 2) *(bf16x8 *)(dst + 2 * plane + r * dp + k) = o[2];
            }
        }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[q][c][e] = total[e];
    __syncthreads();
    // thread: column threadIdx.x of the 256
    const int cc = threadIdx.x >> 3, e = threadIdx.x & 7, col = (int)blockIdx.x * 256 + threadIdx.x;
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) v += sums[u][cc][e];
    if (col < width) part[(long long)blockIdx.y * width + col] = v;
}

// ---- host ---------------------------------------------------------------------

constexpr int FEW_ROWS = 8;

template <int ACT>
struct Activation {
    static constexpr int value = ACT;
};
// calls f with the activation as a type
template <class F>
static hipError_t by_activation(int act, F f)
{
    switch (act) {
    case LCN_ACT_TANH: return f(Activation<LCN_ACT_TANH>());
    case LCN_ACT_RELU: return f(Activation<LCN_ACT_RELU>());
    case LCN_ACT_GELU: return f(Activation<LCN_ACT_GELU>());
    case LCN_ACT_SILU: return f(Activation<LCN_ACT_SILU>());
    default: return f(Activation<LCN_ACT_NONE>());
    }
}

// Where that is faster than the product of planes (us for 40 000 rows, narrow / product): float 64 -> 256 35 / 36, 32 -> 512
// 39 / 49, 128 -> 64 23 / 28, 128 -> 128 37 / 32; bf16 64 -> 256 20 / 23, 32 -> 512 22 / 32, 128 -> 64 11 / 7; rows that are
// not whole pieces, 50 -> 64, 26 / 21 and 21 / 12.
static bool narrow(int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    if (rows < 128 || d_in % (dtype == LCN_F32 ? 4 : 8)) return false;
    return (d_in <= 64 && d_in * (int64_t)d_out <= 64 * 256) || (dtype == LCN_F32 && d_in <= 128 && d_out <= 64);
}

template <class T, int KP, bool VEC>
static hipError_t launch_narrow(const LinearArgs<T> &e, const T *x, const T *w, int64_t rows, int k, int width, hipStream_t s)
{
    const long long groups = (rows + 63) / 64, tiles = (width + 63) / 64, most = 2048 / tiles;
    return by_activation(e.act, [&](auto a) {
        hipLaunchKernelGGL((linear_narrow_kernel<T, KP, decltype(a)::value, VEC>),
                           dim3((unsigned)(groups < most ? groups : most), (unsigned)tiles), dim3(256), 0, s, e, x, w,
                           (long long)rows, k, width);
        return hipGetLastError();
    });
}

static bool linear_args_fit(int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    return rows >= 0 && rows <= MAX_ROWS && d_in >= 1 && d_in <= MAX_WIDTH && d_out >= 1 && d_out <= MAX_WIDTH &&
           sizes_fit(rows, d_in) && sizes_fit(rows, d_out) && (dtype == LCN_F32 || dtype == LCN_BF16);
}

struct LinearForward {
    void *xp, *wp;
    float *part;
    ProductPlan plan;
    size_t bytes;
};
static LinearForward linear_forward_space(char *ws, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    Carver c{ws};
    LinearForward f;
    f.plan = plan_product(d_out, rows, d_in, planes_of(dtype), true, true);
    f.xp = c.take(planes_bytes(rows, d_in, planes_of(dtype)));
    f.wp = c.take(planes_bytes(d_out, d_in, planes_of(dtype)));
    f.part = (float *)c.take(partial_bytes(f.plan, d_out, rows));
    f.bytes = c.used;
    return f;
}

struct LinearBackward {
    void *xp, *wp, *dz;
    float *part_dx, *part_dw, *sums;
    ProductPlan dx, dw;
    int planes, groups, rows_each;   // planes of dz
    size_t bytes;
};
static LinearBackward linear_backward_space(char *ws, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    Carver c{ws};
    LinearBackward b;
    b.planes = gradient_planes(rows, dtype);
    b.dx = plan_product(d_in, rows, d_out, b.planes, true, true);
    b.dw = plan_product(d_in, d_out, rows, b.planes, true, true);
    // enough workgroups to fill the chip, at most 256 partial sums per column
    b.rows_each = (int)((((rows + 255) / 256) + 31) & ~31LL);
    b.groups = (int)((rows + b.rows_each - 1) / b.rows_each);
    b.xp = c.take(planes_bytes(rows, d_in, planes_of(dtype)));
    b.wp = c.take(planes_bytes(d_out, d_in, planes_of(dtype)));
    b.dz = c.take(planes_bytes(rows, d_out, b.planes));
    b.part_dx = (float *)c.take(partial_bytes(b.dx, d_in, rows));
    b.part_dw = (float *)c.take(partial_bytes(b.dw, d_in, d_out));
    b.sums = (float *)c.take((size_t)b.groups * d_out * 4);
    b.bytes = c.used;
    return b;
}

template <class T>
static lcn_status linear_as(const T *x, const T *w, const T *bias, const T *residual, int64_t rows, int32_t d_in,
                            int32_t d_out, int32_t dtype, int32_t act, T *y, float *pre, char *ws, size_t ws_bytes,
                            hipStream_t s)
{
    LinearArgs<T> e{bias, residual, y, pre, act, 0};
    if (rows <= FEW_ROWS) {
        const int r = (int)rows;
        hipError_t st = r == 1   ? launch_few<T, 1>(e, x, w, r, d_in, d_out, s)
                        : r == 2 ? launch_few<T, 2>(e, x, w, r, d_in, d_out, s)
                        : r <= 4 ? launch_few<T, 4>(e, x, w, r, d_in, d_out, s)
                                 : launch_few<T, 8>(e, x, w, r, d_in, d_out, s);
        OPCHK(st);
        return LCN_OK;
    }
    e.whole = whole_rows<T>((const void *)((uintptr_t)y | (uintptr_t)bias | (uintptr_t)residual | (uintptr_t)pre), d_out);
    if (narrow(rows, d_in, d_out, dtype)) {
        const bool vec = whole_rows<T>((const void *)((uintptr_t)x | (uintptr_t)w), d_in);
        constexpr int MOST = sizeof(T) == 4 ? 128 : 64;
        OPCHK(!vec          ? launch_narrow<T, MOST, false>(e, x, w, rows, d_in, d_out, s)   // x or W not aligned
              : d_in <= 32 ? launch_narrow<T, 32, true>(e, x, w, rows, d_in, d_out, s)
              : d_in <= 64 ? launch_narrow<T, 64, true>(e, x, w, rows, d_in, d_out, s)
                           : launch_narrow<T, MOST, true>(e, x, w, rows, d_in, d_out, s));
        return LCN_OK;
    }
    const LinearForward f = linear_forward_space(ws, rows, d_in, d_out, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < f.bytes) return LCN_ERR_ALLOC;
    ProductArgs p{};
    PlaneJobs jobs;
    p.a = add_operand(jobs, w, d_out, d_in, dtype, f.wp);
    p.b = add_operand(jobs, x, rows, d_in, dtype, f.xp);
    OPCHK(launch_planes(jobs, dtype, s));
    p.m = d_out;
    p.n = (int)rows;
    p.k = d_in;
    p.planes = planes_of(dtype);
    if (f.plan.splits > 1) {
        const long long ldp = padded(d_out), groups = (rows * (ldp / 8) + 255) / 256;
        OPCHK((launch_planned<sizeof(T) == 4 ? 3 : 1, false, false, PartialEpilogue>(f.plan, p, {f.part, ldp, rows * ldp, 0}, s)));
        OPCHK(by_activation(act, [&](auto a) {
            hipLaunchKernelGGL((linear_finish_kernel<T, decltype(a)::value>), dim3((unsigned)(groups < 8192 ? groups : 8192)),
                               dim3(256), 0, s, e, f.part, f.plan.splits, rows * ldp, (long long)rows, d_out, ldp);
            return hipGetLastError();
        }));
        return LCN_OK;
    }
    OPCHK(by_activation(act, [&](auto a) {
        return launch_planned<sizeof(T) == 4 ? 3 : 1, false, false, LinearEpilogue<T, decltype(a)::value>>(f.plan, p, e, s);
    }));
    return LCN_OK;
}

template <class T>
static lcn_status linear_backward_as(const T *x, const T *w, const float *pre, const T *dy, int64_t rows, int32_t d_in,
                                     int32_t d_out, int32_t dtype, int32_t act, T *dx, T *dw, T *dbias, char *ws,
                                     size_t ws_bytes, hipStream_t s)
{
    const LinearBackward b = linear_backward_space(ws, rows, d_in, d_out, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < b.bytes) return LCN_ERR_ALLOC;
    Operand dz = plane_operand(b.dz, rows, d_out);
    const bool as_is = act == LCN_ACT_NONE && in_place(dy, d_out, dtype);
    int planes = b.planes;
    if (as_is) {   // dy itself: nothing is rounded
        dz = Operand{dy, 0, d_out};
        planes = 1;
    }
    if (!as_is || dbias) {
        const int dp = (int)padded(d_out);
        const int whole = whole_rows<T>((const void *)((uintptr_t)dy | (uintptr_t)pre), d_out);
        OPCHK(by_activation(act, [&](auto a) {
            hipLaunchKernelGGL((slope_kernel<T, decltype(a)::value>), dim3((unsigned)((dp + 255) / 256), (unsigned)b.groups),
                               dim3(256), 0, s, dy, pre, (long long)rows, d_out, dp, b.rows_each, whole, b.planes,
                               as_is ? nullptr : (__bf16 *)b.dz, dbias ? b.sums : nullptr);
            return hipGetLastError();
        }));
        if (dbias) OPCHK(launch_column_sums(b.sums, b.groups, d_out, dtype, dbias, s));
    }
    ProductArgs p{};
    PlaneJobs jobs;
    Operand xo{}, wo{};
    if (dx) wo = add_operand(jobs, w, d_out, d_in, dtype, b.wp);
    if (dw) xo = add_operand(jobs, x, rows, d_in, dtype, b.xp);
    OPCHK(launch_planes(jobs, dtype, s));
    p.planes = planes;
    p.m = d_in;
    if (dx) {
        p.a = wo;
        p.b = dz;
        p.n = (int)rows;
        p.k = d_out;
        OPCHK((launch_scaled<true, false>(b.dx, p, 1.f, dtype, dx, b.part_dx, s)));
    }
    if (dw) {
        p.a = xo;
        p.b = dz;
        p.n = d_out;
        p.k = (int)rows;
        OPCHK((launch_scaled<true, true>(b.dw, p, 1.f, dtype, dw, b.part_dw, s)));
    }
    return LCN_OK;
}

}  // namespace lcn

using namespace lcn;

extern "C" {

lcn_status lcn_linear_workspace_bytes(int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype, int32_t backward,
                                      size_t *bytes)
{
    if (!bytes || !linear_args_fit(rows, d_in, d_out, dtype)) return LCN_ERR_INVALID_ARG;
    *bytes = 0;
    if (rows == 0 || (!backward && (rows <= FEW_ROWS || narrow(rows, d_in, d_out, dtype)))) return LCN_OK;
    *bytes = backward ? linear_backward_space(nullptr, rows, d_in, d_out, dtype).bytes
                      : linear_forward_space(nullptr, rows, d_in, d_out, dtype).bytes;
    return LCN_OK;
}

lcn_status lcn_linear(const void *x, const void *W, const void *bias, const void *residual, int64_t rows, int32_t d_in,
                      int32_t d_out, int32_t dtype, int32_t activation, void *y, float *pre, void *workspace,
                      size_t workspace_bytes, void *hip_stream)
{
    if (!linear_args_fit(rows, d_in, d_out, dtype) || activation < LCN_ACT_NONE || activation > LCN_ACT_SILU)
        return LCN_ERR_INVALID_ARG;
    if (rows == 0) return LCN_OK;
    if (!x || !W || !y) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return linear_as((const float *)x, (const float *)W, (const float *)bias, (const float *)residual, rows, d_in, d_out,
                         dtype, activation, (float *)y, pre, (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
    return linear_as((const __bf16 *)x, (const __bf16 *)W, (const __bf16 *)bias, (const __bf16 *)residual, rows, d_in, d_out,
                     dtype, activation, (__bf16 *)y, pre, (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
}

lcn_status lcn_linear_backward(const void *x, const void *W, const float *pre, const void *dy, int64_t rows, int32_t d_in,
                               int32_t d_out, int32_t dtype, int32_t activation, void *dx, void *dW, void *dbias,
                               void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!linear_args_fit(rows, d_in, d_out, dtype) || activation < LCN_ACT_NONE || activation > LCN_ACT_SILU)
        return LCN_ERR_INVALID_ARG;
    if (!dx && !dW && !dbias) return LCN_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    const size_t e = dtype == LCN_F32 ? 4 : 2;
    if (rows == 0) {   // no rows: the parameters' gradients are zero
        if (dW) OPCHK(launch_zero(dW, (size_t)d_in * d_out * e, s));
        if (dbias) OPCHK(launch_zero(dbias, (size_t)d_out * e, s));
        return LCN_OK;
    }
    if (!dy || (activation != LCN_ACT_NONE && !pre) || (dx && !W) || (dW && !x)) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return linear_backward_as((const float *)x, (const float *)W, pre, (const float *)dy, rows, d_in, d_out, dtype,
                                  activation, (float *)dx, (float *)dW, (float *)dbias, (char *)workspace, workspace_bytes, s);
    return linear_backward_as((const __bf16 *)x, (const __bf16 *)W, pre, (const __bf16 *)dy, rows, d_in, d_out, dtype,
                              activation, (__bf16 *)dx, (__bf16 *)dW, (__bf16 *)dbias, (char *)workspace, workspace_bytes, s);
}

}  // extern "C"
