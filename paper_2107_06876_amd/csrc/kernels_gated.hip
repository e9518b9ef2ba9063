// y = act(g) u with g = x Wg^T + bg and u = x Wu^T + bu, Wg above Wu in one matrix, and its gradients.
//
// Backward: dz = [dy u act'(g) | dy act(g)] once (as planes of bf16, with the column sums that are the biases' gradients), then
// dx = dz W and dW = dz^T x, which are two products because g's and u's halves lie in one matrix.
//
// Rounding: g, u, sums and activations are in 32 bits; with bf16 tensors y, dz, dx, dW and db are rounded once each, the kept g
// and u are not (as bf16 each would add an error to dz of the size of dz's own rounding).
#include "operators.h"

namespace lcn {

template <class T>
struct GatedArgs {
    const T *bias;   // 2 width
    T *y;
    float *pre;      // rows x 2 width, nullable
    int act, whole;  // whole: rows of y, bias and pre, and their halves, are whole 16-byte pieces
};

// eight outputs from g and u, which have their biases: y and pre at row n, column m
template <class T, int ACT>
__device__ __forceinline__ void gated_finish(const GatedArgs<T> &e, f32x4 (&g)[2], const f32x4 (&u)[2], long long n, int m, int width)
{
    const int left = width - m;
    if (e.pre) {
        store_eight(e.pre + n * 2 * width + m, g, left, e.whole);
        store_eight(e.pre + (n * 2 + 1) * width + m, u, left, e.whole);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i >> 2][i & 3] = activate<ACT>(g[i >> 2][i & 3]) * u[i >> 2][i & 3];
    store_eight(e.y + n * width + m, g, left, e.whole);
}

// from the sums of [g | u] in memory, `splits` partial ones each
template <class T, int ACT>
__global__ __launch_bounds__(256) void gated_finish_kernel(GatedArgs<T> e, const float *__restrict__ part, int splits,
                                                           long long stride, long long rows, int width, long long ldp)
{
    const int per_row = (width + 7) / 8, whole_half = width % 4 == 0;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < rows * per_row; t += (long long)gridDim.x * 256) {
        const long long n = t / per_row;
        const int m = (int)(t - n * per_row) * 8, left = width - m;
        f32x4 z[2][2], v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float *p = part + n * ldp + h * width + m;
            load_eight(p, left, whole_half, z[h]);
            for (int s = 1; s < splits; ++s) {
                load_eight(p + s * stride, left, whole_half, v);
                z[h][0] += v[0];
                z[h][1] += v[1];
            }
            if (e.bias) {
                load_eight(e.bias + h * width + m, left, e.whole, v);
                z[h][0] += v[0];
                z[h][1] += v[1];
            }
        }
        gated_finish<T, ACT>(e, z[0], z[1], n, m, width);
    }
}

// Few rows: bound by reading W once; 16 lanes read a row of Wg and the one of Wu that belongs to it.
template <class T, int R, bool VEC>
__global__ __launch_bounds__(256) void gated_few_kernel(GatedArgs<T> e, const T *__restrict__ x, const T *__restrict__ w, int rows,
                                                        int k, int width)
{
    const int f = (int)(blockIdx.x * 16 + (threadIdx.x >> 4));
    if (f >= width) return;
    float sum[2][R];
#pragma unroll
    for (int r = 0; r < R; ++r) sum[0][r] = sum[1][r] = 0.f;
    few_rows_dot<T, R, VEC>(w + (long long)f * k, w + (long long)(width + f) * k, x, rows, k, sum);
    const int r = threadIdx.x & 15;   // lane r finishes one value
    if (r >= rows) return;
    float g = 0.f, u = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i == r) {
            g = sum[0][i];
            u = sum[1][i];
        }
    if (e.bias) {
        g += (float)e.bias[f];
        u += (float)e.bias[width + f];
    }
    if (e.pre) {
        e.pre[(long long)r * 2 * width + f] = g;
        e.pre[((long long)r * 2 + 1) * width + f] = u;
    }
    switch (e.act) {
    case LCN_ACT_TANH: g = activate<LCN_ACT_TANH>(g); break;
    case LCN_ACT_RELU: g = activate<LCN_ACT_RELU>(g); break;
    case LCN_ACT_GELU: g = activate<LCN_ACT_GELU>(g); break;
    case LCN_ACT_SILU: g = activate<LCN_ACT_SILU>(g); break;
    }
    e.y[(long long)r * width + f] = (T)(g * u);
}

template <class T, int R>
static hipError_t launch_few(const GatedArgs<T> &e, const T *x, const T *w, int rows, int k, int width, hipStream_t s)
{
    const unsigned grid = (unsigned)((width + 15) / 16);
    if (k % (16 / (int)sizeof(T)) == 0 && (((uintptr_t)x | (uintptr_t)w) & 15) == 0)
        hipLaunchKernelGGL((gated_few_kernel<T, R, true>), dim3(grid), dim3(256), 0, s, e, x, w, rows, k, width);
    else
        hipLaunchKernelGGL((gated_few_kernel<T, R, false>), dim3(grid), dim3(256), 0, s, e, x, w, rows, k, width);
    return hipGetLastError();
}

// dz as planes (dst: nullable; rows of dp values, zero behind 2 width), and the sums over this workgroup's rows for every column
// (part: nullable).  32 pieces of eight columns of either half x 8 rows at a time.
template <class T, int ACT>
__global__ __launch_bounds__(256) void gated_slope_kernel(const T *__restrict__ dy, const float *__restrict__ pre, long long rows,
                                                          int width, int dp, int rows_each, int whole, int planes,
                                                          __bf16 *__restrict__ dst, float *__restrict__ part)
{
    __shared__ float sums[8][32][17];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5, k = ((int)blockIdx.x * 32 + c) * 8, left = width - k;
    const long long plane = rows * dp, r0 = (long long)blockIdx.y * rows_each;
    float total[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) total[0][e] = total[1][e] = 0.f;
    if (k < width)
        for (long long r = r0 + q; r < r0 + rows_each && r < rows; r += 8) {
            f32x4 d[2], z[2][2];
            load_eight(dy + r * width + k, left, whole, d);
            load_eight(pre + r * 2 * width + k, left, whole, z[0]);
            load_eight(pre + (r * 2 + 1) * width + k, left, whole, z[1]);
            bf16x8 o[2][3];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = d[e >> 2][e & 3], g = z[0][e >> 2][e & 3];
                const float y[2] = {e < left ? v * z[1][e >> 2][e & 3] * activate_slope<ACT>(g) : 0.f, e < left ? v * activate<ACT>(g) : 0.f};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    __bf16 a, b, f;
                    total[h][e] += y[h];
                    split_planes(y[h], a, b, f);
                    o[h][0][e] = a;
                    o[h][1][e] = b;
                    o[h][2][e] = f;
                }
            }
            if (dst) {
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    if (p >= planes) break;
                    __bf16 *first = dst + p * plane + r * dp + k;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (width % 8 == 0) {
                            *(bf16x8 *)(first + h * width) = o[h][p];
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
    // thread: column threadIdx.x of the 256, in both halves
    const int cc = threadIdx.x >> 3, e = threadIdx.x & 7, col = (int)blockIdx.x * 256 + threadIdx.x;
    float v[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        v[0] += sums[u][cc][e];
        v[1] += sums[u][cc][8 + e];
    }
    if (col < width) {
        part[(long long)blockIdx.y * 2 * width + col] = v[0];
        part[((long long)blockIdx.y * 2 + 1) * width + col] = v[1];
    }
}

// ---- host ---------------------------------------------------------------------

static bool gated_args_fit(int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    return rows >= 0 && rows <= MAX_ROWS && d_in >= 1 && d_in <= MAX_WIDTH && d_out >= 1 && d_out <= MAX_WIDTH / 2 &&
           sizes_fit(rows, d_in) && sizes_fit(rows, 2 * (int64_t)d_out) && (dtype == LCN_F32 || dtype == LCN_BF16);
}

struct GatedForward {
    void *xp, *wp;
    float *part;
    ProductPlan plan;
    size_t bytes;
};
static GatedForward gated_forward_space(char *ws, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    Carver c{ws};
    GatedForward f;
    f.plan = plan_product(2 * d_out, rows, d_in, planes_of(dtype), true, true);
    f.xp = c.take(planes_bytes(rows, d_in, planes_of(dtype)));
    f.wp = c.take(planes_bytes(2 * d_out, d_in, planes_of(dtype)));
    f.part = (float *)c.take((size_t)f.plan.splits * (size_t)rows * (size_t)padded(2 * d_out) * 4);
    f.bytes = c.used;
    return f;
}

struct GatedBackward {
    void *xp, *wp, *dz;
    float *part_dx, *part_dw, *sums;
    ProductPlan dx, dw;
    int planes, groups, rows_each;   // planes of dz
    size_t bytes;
};
static GatedBackward gated_backward_space(char *ws, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype)
{
    Carver c{ws};
    GatedBackward b;
    const int32_t wide = 2 * d_out;
    b.planes = gradient_planes(rows, dtype);
    b.dx = plan_product(d_in, rows, wide, b.planes, true, true);
    b.dw = plan_product(d_in, wide, rows, b.planes, true, true);
    // enough workgroups to fill the chip, at most 256 partial sums per column
    b.rows_each = (int)((((rows + 255) / 256) + 31) & ~31LL);
    b.groups = (int)((rows + b.rows_each - 1) / b.rows_each);
    b.xp = c.take(planes_bytes(rows, d_in, planes_of(dtype)));
    b.wp = c.take(planes_bytes(wide, d_in, planes_of(dtype)));
    b.dz = c.take(planes_bytes(rows, wide, b.planes));
    b.part_dx = (float *)c.take(partial_bytes(b.dx, d_in, rows));
    b.part_dw = (float *)c.take(partial_bytes(b.dw, d_in, wide));
    b.sums = (float *)c.take((size_t)b.groups * wide * 4);
    b.bytes = c.used;
    return b;
}

template <class T>
static lcn_status gated_as(const T *x, const T *w, const T *bias, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype,
                           int32_t act, T *y, float *pre, char *ws, size_t ws_bytes, hipStream_t s)
{
    GatedArgs<T> e{bias, y, pre, act, 0};
    if (rows <= FEW_ROWS) {
        const int r = (int)rows;
        OPCHK(r == 1   ? launch_few<T, 1>(e, x, w, r, d_in, d_out, s)
              : r == 2 ? launch_few<T, 2>(e, x, w, r, d_in, d_out, s)
              : r <= 4 ? launch_few<T, 4>(e, x, w, r, d_in, d_out, s)
                       : launch_few<T, 8>(e, x, w, r, d_in, d_out, s));
        return LCN_OK;
    }
    e.whole = whole_rows<T>((const void *)((uintptr_t)y | (uintptr_t)bias | (uintptr_t)pre), d_out);
    const GatedForward f = gated_forward_space(ws, rows, d_in, d_out, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < f.bytes) return LCN_ERR_ALLOC;
    ProductArgs p{};
    PlaneJobs jobs;
    p.a = add_operand(jobs, w, 2 * d_out, d_in, dtype, f.wp);
    p.b = add_operand(jobs, x, rows, d_in, dtype, f.xp);
    OPCHK(launch_planes(jobs, dtype, s));
    p.m = 2 * d_out;
    p.n = (int)rows;
    p.k = d_in;
    p.planes = planes_of(dtype);
    const long long ldp = padded(2 * d_out), groups = (rows * ((d_out + 7) / 8) + 255) / 256;
    OPCHK((launch_planned<sizeof(T) == 4 ? 3 : 1, false, false, PartialEpilogue>(f.plan, p, {f.part, ldp, rows * ldp, 0}, s)));
    OPCHK(by_activation(act, [&](auto a) {
        hipLaunchKernelGGL((gated_finish_kernel<T, decltype(a)::value>), dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0,
                           s, e, f.part, f.plan.splits, rows * ldp, (long long)rows, d_out, ldp);
        return hipGetLastError();
    }));
    return LCN_OK;
}

template <class T>
static lcn_status gated_backward_as(const T *x, const T *w, const float *pre, const T *dy, int64_t rows, int32_t d_in, int32_t d_out,
                                    int32_t dtype, int32_t act, T *dx, T *dw, T *dbias, char *ws, size_t ws_bytes, hipStream_t s)
{
    const GatedBackward b = gated_backward_space(ws, rows, d_in, d_out, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < b.bytes) return LCN_ERR_ALLOC;
    const int32_t wide = 2 * d_out;
    const int dp = (int)padded(wide), whole = whole_rows<T>((const void *)((uintptr_t)dy | (uintptr_t)pre), d_out);
    OPCHK(by_activation(act, [&](auto a) {
        hipLaunchKernelGGL((gated_slope_kernel<T, decltype(a)::value>), dim3((unsigned)((d_out + 255) / 256), (unsigned)b.groups),
                           dim3(256), 0, s, dy, pre, (long long)rows, d_out, dp, b.rows_each, whole, b.planes,
                           dx || dw ? (__bf16 *)b.dz : nullptr, dbias ? b.sums : nullptr);
        return hipGetLastError();
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
    p.b = plane_operand(b.dz, rows, wide);
    if (dx) {
        p.a = wo;
        p.n = (int)rows;
        p.k = wide;
        OPCHK((launch_scaled<true, false>(b.dx, p, 1.f, dtype, dx, b.part_dx, s)));
    }
    if (dw) {
        p.a = xo;
        p.n = wide;
        p.k = (int)rows;
        OPCHK((launch_scaled<true, true>(b.dw, p, 1.f, dtype, dw, b.part_dw, s)));
    }
    return LCN_OK;
}

}  // namespace lcn

using namespace lcn;

extern "C" {

lcn_status lcn_gated_linear_workspace_bytes(int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype, int32_t backward,
                                            size_t *bytes)
{
    if (!bytes || !gated_args_fit(rows, d_in, d_out, dtype)) return LCN_ERR_INVALID_ARG;
    *bytes = 0;
    if (rows == 0 || (!backward && rows <= FEW_ROWS)) return LCN_OK;
    *bytes = backward ? gated_backward_space(nullptr, rows, d_in, d_out, dtype).bytes
                      : gated_forward_space(nullptr, rows, d_in, d_out, dtype).bytes;
    return LCN_OK;
}

lcn_status lcn_gated_linear(const void *x, const void *W, const void *bias, int64_t rows, int32_t d_in, int32_t d_out, int32_t dtype,
                            int32_t activation, void *y, float *pre, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!gated_args_fit(rows, d_in, d_out, dtype) || activation < LCN_ACT_NONE || activation > LCN_ACT_SILU)
        return LCN_ERR_INVALID_ARG;
    if (rows == 0) return LCN_OK;
    if (!x || !W || !y) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return gated_as((const float *)x, (const float *)W, (const float *)bias, rows, d_in, d_out, dtype, activation, (float *)y, pre,
                        (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
    return gated_as((const __bf16 *)x, (const __bf16 *)W, (const __bf16 *)bias, rows, d_in, d_out, dtype, activation, (__bf16 *)y, pre,
                    (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
}

lcn_status lcn_gated_linear_backward(const void *x, const void *W, const float *pre, const void *dy, int64_t rows, int32_t d_in,
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
    if (!dy || !pre || (dx && !W) || (dW && !x)) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return gated_backward_as((const float *)x, (const float *)W, pre, (const float *)dy, rows, d_in, d_out, dtype, activation,
                                 (float *)dx, (float *)dW, (float *)dbias, (char *)workspace, workspace_bytes, s);
    return gated_backward_as((const __bf16 *)x, (const __bf16 *)W, pre, (const __bf16 *)dy, rows, d_in, d_out, dtype, activation,
                             (__bf16 *)dx, (__bf16 *)dW, (__bf16 *)dbias, (char *)workspace, workspace_bytes, s);
}

}  // extern "C"
