// Operands of the matrix products in planes of bf16, partial sums, and the choice of a product's tile.
#include "operators.h"

namespace lcn {

// A thread writes 8 values of every plane.  Bound by memory; VEC: source rows are aligned to four values.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void planes_kernel(const T *__restrict__ src, long long rows, int d, int dp,
                                                     const int64_t *__restrict__ target, __bf16 *__restrict__ dst)
{
    const int per_row = dp / 8;
    const long long pieces = rows * per_row, plane = rows * dp;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < pieces; t += (long long)gridDim.x * 256) {
        const long long r = t / per_row;
        const int k = (int)(t - r * per_row) * 8;
        const T *p = src + r * d + k;
        f32x4 v[2];
        v[0] = load_four(p, d - k, VEC);
        v[1] = load_four(p + 4, d - k - 4, VEC);
        if (target && target[r] < 0) v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f};
        bf16x8 o[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            __bf16 a, b, c;
            split_planes(v[e >> 2][e & 3], a, b, c);
            o[0][e] = a;
            o[1][e] = b;
            o[2][e] = c;
        }
        *(bf16x8 *)(dst + t * 8) = o[0];
        if (sizeof(T) == 4) {
            *(bf16x8 *)(dst + plane + t * 8) = o[1];
            *(bf16x8 *)(dst + 2 * plane + t * 8) = o[2];
        }
    }
}

template <class T>
static hipError_t planes_as(const T *src, long long rows, int d, const int64_t *target, void *dst, hipStream_t s)
{
    const int dp = (int)padded(d);
    const long long groups = (rows * (dp / 8) + 255) / 256;
    const unsigned grid = (unsigned)(groups < 8192 ? groups : 8192);
    if (d % 4 == 0 && ((uintptr_t)src & (4 * sizeof(T) - 1)) == 0)
        hipLaunchKernelGGL((planes_kernel<T, true>), dim3(grid), dim3(256), 0, s, src, rows, d, dp, target, (__bf16 *)dst);
    else
        hipLaunchKernelGGL((planes_kernel<T, false>), dim3(grid), dim3(256), 0, s, src, rows, d, dp, target, (__bf16 *)dst);
    return hipGetLastError();
}

hipError_t launch_planes(const void *src, long long rows, int d, int32_t dtype, const int64_t *target, void *dst,
                         hipStream_t s)
{
    if (dtype == LCN_F32) return planes_as((const float *)src, rows, d, target, dst, s);
    return planes_as((const __bf16 *)src, rows, d, target, dst, s);
}

Operand plane_operand(const void *dst, long long rows, long long d)
{
    return Operand{dst, rows * padded(d) * 2, padded(d)};
}

// A thread adds four values of a row over all splits, in their order.
template <class T>
__global__ __launch_bounds__(256) void add_partials_kernel(const float *__restrict__ part, int splits, long long stride,
                                                           long long n, int m, long long ldp, float scale,
                                                           T *__restrict__ out, int whole)
{
    const int per_row = (m + 3) / 4;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < n * per_row; t += (long long)gridDim.x * 256) {
        const long long r = t / per_row;
        const int c = (int)(t - r * per_row) * 4;
        f32x4 v = *(const f32x4 *)(part + r * ldp + c);
        for (int u = 1; u < splits; ++u) v += *(const f32x4 *)(part + u * stride + r * ldp + c);
        store_four(out + r * m + c, v * scale, m - c, whole);
    }
}

hipError_t launch_add_partials(const float *part, int splits, long long n, int m, long long ldp, float scale, int32_t dtype,
                               void *out, hipStream_t s)
{
    const long long groups = (n * ((m + 3) / 4) + 255) / 256;
    const unsigned grid = (unsigned)(groups < 8192 ? groups : 8192);
    const size_t e = dtype == LCN_F32 ? 4 : 2;
    const int whole = m % 4 == 0 && ((uintptr_t)out & (4 * e - 1)) == 0;
    if (dtype == LCN_F32)
        hipLaunchKernelGGL(add_partials_kernel<float>, dim3(grid), dim3(256), 0, s, part, splits, n * ldp, n, m, ldp, scale,
                           (float *)out, whole);
    else
        hipLaunchKernelGGL(add_partials_kernel<__bf16>, dim3(grid), dim3(256), 0, s, part, splits, n * ldp, n, m, ldp, scale,
                           (__bf16 *)out, whole);
    return hipGetLastError();
}

// The tile shape and the split with the least estimated time.  A workgroup's step costs its tile's area at the rate
// that the shape reaches (256 x 256: 1.2 PFLOP/s on 8192^3, 128 x 128: 1.05, 64 x 64: 0.7); `overhead` steps stand for a
// workgroup's start and epilogue; the chip takes 256 workgroups of the large shapes at a time, 512 and 1024 of the
// small ones; the partial sums of a split are written and read once at the rate of memory.
ProductPlan plan_product(long long m, long long n, long long k, int planes, bool may_split)
{
    static const struct {
        int bm, bn, resident;
        double step_us;   // of one workgroup's 64 values of k with the chip full
    } shape[TILE_COUNT] = {{256, 256, 1, 1.8}, {128, 128, 2, 1.03}, {64, 64, 4, 0.77}, {320, 128, 1, 1.25}};
    const long long steps = (k + 63) / 64 * pairs_of(planes);
    ProductPlan best{TILE_256, 1};
    double least = 1e300;
    for (int t = 0; t < TILE_COUNT; ++t) {
        const long long tiles = ((m + shape[t].bm - 1) / shape[t].bm) * ((n + shape[t].bn - 1) / shape[t].bn);
        for (int splits = 1; splits <= 64; splits *= 2) {
            if (splits > 1 && (!may_split || steps / splits < 4)) break;
            const long long groups = tiles * splits, room = 256 * shape[t].resident;
            const double rounds = (double)((groups + room - 1) / room);
            double us = rounds * shape[t].step_us * ((double)((steps + splits - 1) / splits) + 2.0);
            if (groups < room) {   // fewer to share a compute unit with
                const double share = (double)((groups + 255) / 256) / shape[t].resident;
                us *= share > 0.5 ? share : 0.5 + 0.5 * share;
            }
            if (splits > 1) us += 3.0 + (double)splits * m * n * 8e-6 / 4.0;
            if (us < least) {
                least = us;
                best = ProductPlan{t, splits};
            }
        }
    }
    return best;
}

template <bool ACOL, bool BCOL>
hipError_t launch_scaled(const ProductPlan &plan, const ProductArgs &p, float scale, int32_t dtype, void *out, float *part,
                         hipStream_t s)
{
    if (plan.splits > 1) {
        const long long ldp = padded(p.m);
        const hipError_t e = launch_planned<ACOL, BCOL, PartialEpilogue>(plan, p, {part, ldp, p.n * ldp, 0}, s);
        if (e != hipSuccess) return e;
        return launch_add_partials(part, plan.splits, p.n, p.m, ldp, scale, dtype, out, s);
    }
    if (dtype == LCN_F32)
        return launch_planned<ACOL, BCOL, ScaledEpilogue<float>>(plan, p, {(float *)out, p.m, scale, whole_rows<float>(out, p.m)}, s);
    return launch_planned<ACOL, BCOL, ScaledEpilogue<__bf16>>(plan, p, {(__bf16 *)out, p.m, scale, whole_rows<__bf16>(out, p.m)}, s);
}
template hipError_t launch_scaled<true, false>(const ProductPlan &, const ProductArgs &, float, int32_t, void *, float *,
                                               hipStream_t);
template hipError_t launch_scaled<true, true>(const ProductPlan &, const ProductArgs &, float, int32_t, void *, float *,
                                              hipStream_t);
hipError_t launch_partials(const ProductPlan &plan, const ProductArgs &p, float *part, int add, hipStream_t s)
{
    const long long ldp = padded(p.m);
    return launch_planned<true, false, PartialEpilogue>(plan, p, {part, ldp, p.n * ldp, add}, s);
}

// column sums: part is [parts][width]; 32 columns per workgroup, 8 threads each, in a fixed order
template <class T>
__global__ __launch_bounds__(256) void column_sums_kernel(const float *__restrict__ part, int parts, int width, T *__restrict__ out)
{
    __shared__ float sums[8][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), q = threadIdx.x >> 5;
    float v = 0.f;
    if (c < width)
        for (int r = q; r < parts; r += 8) v += part[(long long)r * width + c];
    sums[q][threadIdx.x & 31] = v;
    __syncthreads();
    if (q == 0 && c < width) {
#pragma unroll
        for (int u = 1; u < 8; ++u) v += sums[u][threadIdx.x];
        out[c] = (T)v;
    }
}
hipError_t launch_column_sums(const float *part, int parts, int width, int32_t dtype, void *out, hipStream_t s)
{
    const unsigned grid = (unsigned)((width + 31) / 32);
    if (dtype == LCN_F32)
        hipLaunchKernelGGL(column_sums_kernel<float>, dim3(grid), dim3(256), 0, s, part, parts, width, (float *)out);
    else
        hipLaunchKernelGGL(column_sums_kernel<__bf16>, dim3(grid), dim3(256), 0, s, part, parts, width, (__bf16 *)out);
    return hipGetLastError();
}

// the operand of a matrix: as it lies, or its planes at `space`
hipError_t operand_of(const void *p, long long rows, int d, int32_t dtype, void *space, hipStream_t s, Operand *o)
{
    if (in_place(p, d, dtype)) {
        *o = Operand{p, 0, d};
        return hipSuccess;
    }
    *o = plane_operand(space, rows, d);
    return launch_planes(p, rows, d, dtype, nullptr, space, s);
}

// zeros by a kernel: a fill of memory that a caller may capture into a graph
__global__ __launch_bounds__(256) void zero_kernel(unsigned short *p, size_t halves)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < halves; i += (size_t)gridDim.x * 256) p[i] = 0;
}
hipError_t launch_zero(void *p, size_t bytes, hipStream_t s)
{
    const size_t groups = (bytes / 2 + 255) / 256;
    if (!groups) return hipSuccess;
    hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, (unsigned short *)p, bytes / 2);
    return hipGetLastError();
}

}  // namespace lcn
