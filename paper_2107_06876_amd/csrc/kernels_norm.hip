// Layer norm of rows and its gradients.
//
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(mean of (x - mean)^2 + eps)
//   dx = rstd (g - mean of g - xhat mean of (g xhat)) + around,  g = dy w,  xhat = (x - mean) rstd
//   dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// A workgroup per row, which reads it three times (the variance is formed from differences to the mean); the sums over
// rows by a kernel of their own.
#include "operators.h"

namespace lcn {

template <class T, int V>
struct Piece {
    typedef T type __attribute__((ext_vector_type(V)));
};

// The sums of a and b over the workgroup, in every thread.
__device__ __forceinline__ void sum_over_group(float &a, float &b, float (*lds)[2])
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        a += __shfl_xor(a, o);
        b += __shfl_xor(b, o);
    }
    __syncthreads();   // whoever reads the sums before
    if ((threadIdx.x & 63) == 0) {
        lds[threadIdx.x >> 6][0] = a;
        lds[threadIdx.x >> 6][1] = b;
    }
    __syncthreads();
    a = b = 0.f;
    for (unsigned u = 0; u < blockDim.x / 64; ++u) {
        a += lds[u][0];
        b += lds[u][1];
    }
}

template <class T, int V>
__global__ __launch_bounds__(256) void norm_kernel(const T *x, const T *__restrict__ w, const T *__restrict__ b,
                                                   long long rows, int dim, float eps, T *y,   // y may be x
                                                   float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    typedef typename Piece<T, V>::type piece;
    __shared__ float lds[4][2];
    const long long r = group_number();
    if (r >= rows) return;
    const int units = dim / V;
    const piece *row = (const piece *)(x + r * dim);
    float sum = 0.f, none = 0.f;
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece p = row[u];
#pragma unroll
        for (int e = 0; e < V; ++e) sum += (float)p[e];
    }
    sum_over_group(sum, none, lds);
    const float mean = sum / (float)dim;
    float square = 0.f;
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece p = row[u];
#pragma unroll
        for (int e = 0; e < V; ++e) square += ((float)p[e] - mean) * ((float)p[e] - mean);
    }
    sum_over_group(square, none, lds);
    const float rstd = 1.f / sqrtf(square / (float)dim + eps);
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece p = row[u];
        piece o, pw, pb;
        if (w) pw = ((const piece *)w)[u];
        if (b) pb = ((const piece *)b)[u];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float v = ((float)p[e] - mean) * rstd;
            if (w) v *= (float)pw[e];
            if (b) v += (float)pb[e];
            o[e] = (T)v;
        }
        ((piece *)(y + r * dim))[u] = o;
    }
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[r] = mean;
        if (rstd_out) rstd_out[r] = rstd;
    }
}

template <class T, int V>
__global__ __launch_bounds__(256) void norm_dx_kernel(const T *__restrict__ x, const T *__restrict__ w,
                                                      const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
                                                      const T *__restrict__ dy, const T *around, long long rows,
                                                      int dim, T *dx)   // dx may be around
{
    typedef typename Piece<T, V>::type piece;
    __shared__ float lds[4][2];
    const long long r = group_number();
    if (r >= rows) return;
    const int units = dim / V;
    const piece *px = (const piece *)(x + r * dim), *pd = (const piece *)(dy + r * dim), *pw = (const piece *)w;
    const piece *pa = (const piece *)(around + r * dim);
    const float mean = mean_in[r], rstd = rstd_in[r];
    float s1 = 0.f, s2 = 0.f;
    for (int u = threadIdx.x; u < units; u += 256)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float g = (float)pd[u][e] * (w ? (float)pw[u][e] : 1.f);
            s1 += g;
            s2 += g * (((float)px[u][e] - mean) * rstd);
        }
    sum_over_group(s1, s2, lds);
    s1 /= (float)dim;
    s2 /= (float)dim;
    for (int u = threadIdx.x; u < units; u += 256) {
        piece o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float g = (float)pd[u][e] * (w ? (float)pw[u][e] : 1.f);
            float v = rstd * (g - s1 - ((float)px[u][e] - mean) * rstd * s2);
            if (around) v += (float)pa[u][e];
            o[e] = (T)v;
        }
        ((piece *)(dx + r * dim))[u] = o;
    }
}

// part[g][0][c], part[g][1][c]: the sums of dy xhat and of dy over the rows r = g, g + gridDim.y, ...; a thread has V columns
template <class T, int V>
__global__ __launch_bounds__(256) void norm_columns_kernel(const T *__restrict__ x, const float *__restrict__ mean,
                                                           const float *__restrict__ rstd, const T *__restrict__ dy,
                                                           long long rows, int dim, float *__restrict__ part)
{
    typedef typename Piece<T, V>::type piece;
    const int u = (int)(blockIdx.x * 256 + threadIdx.x);
    if (u >= dim / V) return;
    float dw[V], db[V];
#pragma unroll
    for (int e = 0; e < V; ++e) dw[e] = db[e] = 0.f;
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        const piece px = ((const piece *)(x + r * dim))[u], pd = ((const piece *)(dy + r * dim))[u];
        const float m = mean[r], s = rstd[r];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dw[e] += (float)pd[e] * (((float)px[e] - m) * s);
            db[e] += (float)pd[e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        part[((long long)blockIdx.y * 2) * dim + u * V + e] = dw[e];
        part[((long long)blockIdx.y * 2 + 1) * dim + u * V + e] = db[e];
    }
}

// Adds up the partial sums of dw (columns 0 .. dim - 1) and db (the dim behind): 32 columns per workgroup, 8 threads each,
// in a fixed order.
template <class T>
__global__ __launch_bounds__(256) void norm_join_kernel(const float *__restrict__ part, int parts, int dim, T *__restrict__ dw,
                                                        T *__restrict__ db)
{
    __shared__ float sums[8][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), q = threadIdx.x >> 5, width = 2 * dim;
    float v = 0.f;
    if (c < width)
        for (int r = q; r < parts; r += 8) v += part[(long long)r * width + c];
    sums[q][threadIdx.x & 31] = v;
    __syncthreads();
    if (q || c >= width) return;
#pragma unroll
    for (int u = 1; u < 8; ++u) v += sums[u][threadIdx.x];
    if (c < dim) {
        if (dw) dw[c] = (T)v;
    } else if (db) {
        db[c - dim] = (T)v;
    }
}

// ---- host ---------------------------------------------------------------------

static bool norm_args_fit(int64_t rows, int32_t dim, int32_t dtype)
{
    return rows >= 0 && rows <= MAX_ROWS && dim >= 1 && dim <= MAX_WIDTH && sizes_fit(rows, dim) &&
           (dtype == LCN_F32 || dtype == LCN_BF16);
}

// Workgroups that share the rows of the sums of dw and db, each with partial sums of its own.
static int norm_groups(int64_t rows) { return (int)(rows < 256 ? rows : 256); }
static size_t norm_backward_space(int64_t rows, int32_t dim)
{
    return ((size_t)norm_groups(rows) * 2 * dim * 4 + 255) & ~(size_t)255;
}

// calls f with the values of a load as a type: 16 bytes, 8 (bf16) or one value, as `addresses` and dim allow
template <int V>
struct Width {
    static constexpr int value = V;
};
template <class T, class F>
static hipError_t by_width(uintptr_t addresses, int32_t dim, F f)
{
    constexpr int MOST = 16 / (int)sizeof(T);
    if (dim % MOST == 0 && addresses % 16 == 0) return f(Width<MOST>());
    if (MOST == 8 && dim % 4 == 0 && addresses % 8 == 0) return f(Width<4>());
    return f(Width<1>());
}

template <class T>
static lcn_status norm_as(const T *x, const T *w, const T *b, int64_t rows, int32_t dim, float eps, T *y, float *mean,
                          float *rstd, hipStream_t s)
{
    OPCHK(by_width<T>((uintptr_t)x | (uintptr_t)w | (uintptr_t)b | (uintptr_t)y, dim, [&](auto v) {
        hipLaunchKernelGGL((norm_kernel<T, decltype(v)::value>), grid_of(rows), dim3(256), 0, s, x, w, b, (long long)rows, dim, eps,
                           y, mean, rstd);
        return hipGetLastError();
    }));
    return LCN_OK;
}

template <class T>
static lcn_status norm_backward_as(const T *x, const T *w, const float *mean, const float *rstd, const T *dy, const T *around,
                                   int64_t rows, int32_t dim, T *dx, T *dw, T *db, float *part, hipStream_t s)
{
    const uintptr_t all = (uintptr_t)x | (uintptr_t)w | (uintptr_t)dy | (uintptr_t)around | (uintptr_t)dx;
    if (dx)
        OPCHK(by_width<T>(all, dim, [&](auto v) {
            hipLaunchKernelGGL((norm_dx_kernel<T, decltype(v)::value>), grid_of(rows), dim3(256), 0, s, x, w, mean, rstd, dy, around,
                               (long long)rows, dim, dx);
            return hipGetLastError();
        }));
    if (!dw && !db) return LCN_OK;
    const int groups = norm_groups(rows);
    OPCHK(by_width<T>((uintptr_t)x | (uintptr_t)dy, dim, [&](auto v) {
        constexpr int V = decltype(v)::value;
        hipLaunchKernelGGL((norm_columns_kernel<T, V>), dim3((unsigned)((dim / V + 255) / 256), (unsigned)groups), dim3(256), 0, s, x,
                           mean, rstd, dy, (long long)rows, dim, part);
        return hipGetLastError();
    }));
    hipLaunchKernelGGL(norm_join_kernel<T>, dim3((unsigned)((2 * dim + 31) / 32)), dim3(256), 0, s, part, groups, dim, dw, db);
    OPCHK(hipGetLastError());
    return LCN_OK;
}

}  // namespace lcn

using namespace lcn;

extern "C" {

lcn_status lcn_layer_norm(const void *x, const void *weight, const void *bias, int64_t rows, int32_t dim, int32_t dtype, float eps,
                          void *y, float *mean, float *rstd, void *hip_stream)
{
    if (!norm_args_fit(rows, dim, dtype) || !(eps >= 0.f) || eps > 3.4e38f) return LCN_ERR_INVALID_ARG;
    if (rows == 0) return LCN_OK;
    if (!x || !y) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return norm_as((const float *)x, (const float *)weight, (const float *)bias, rows, dim, eps, (float *)y, mean, rstd,
                       (hipStream_t)hip_stream);
    return norm_as((const __bf16 *)x, (const __bf16 *)weight, (const __bf16 *)bias, rows, dim, eps, (__bf16 *)y, mean, rstd,
                   (hipStream_t)hip_stream);
}

lcn_status lcn_layer_norm_workspace_bytes(int64_t rows, int32_t dim, int32_t dtype, size_t *bytes)
{
    if (!bytes || !norm_args_fit(rows, dim, dtype)) return LCN_ERR_INVALID_ARG;
    *bytes = rows == 0 ? 0 : norm_backward_space(rows, dim);
    return LCN_OK;
}

lcn_status lcn_layer_norm_backward(const void *x, const void *weight, const float *mean, const float *rstd, const void *dy,
                                   const void *around, int64_t rows, int32_t dim, int32_t dtype, void *dx, void *dweight,
                                   void *dbias, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!norm_args_fit(rows, dim, dtype)) return LCN_ERR_INVALID_ARG;
    if (!dx && !dweight && !dbias) return LCN_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    const size_t e = dtype == LCN_F32 ? 4 : 2;
    if (rows == 0) {   // no rows: the parameters' gradients are zero
        if (dweight) OPCHK(launch_zero(dweight, (size_t)dim * e, s));
        if (dbias) OPCHK(launch_zero(dbias, (size_t)dim * e, s));
        return LCN_OK;
    }
    if (!x || !mean || !rstd || !dy) return LCN_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < norm_backward_space(rows, dim)) return LCN_ERR_ALLOC;
    if (dtype == LCN_F32)
        return norm_backward_as((const float *)x, (const float *)weight, mean, rstd, (const float *)dy, (const float *)around, rows,
                                dim, (float *)dx, (float *)dweight, (float *)dbias, (float *)workspace, s);
    return norm_backward_as((const __bf16 *)x, (const __bf16 *)weight, mean, rstd, (const __bf16 *)dy, (const __bf16 *)around, rows,
                            dim, (__bf16 *)dx, (__bf16 *)dweight, (__bf16 *)dbias, (float *)workspace, s);
}

}  // extern "C"
