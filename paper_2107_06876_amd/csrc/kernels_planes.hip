// Operands of the matrix products in planes of bf16, partial sums, and the choice of a product's tile.
#include "operators.h"

namespace lcn {

// A thread writes 8 values of every plane.  Bound by memory.
template <class T>
__global__ __launch_bounds__(256) void planes_kernel(PlaneJobs jobs)
{
    int at = 0;
    while (at + 1 < jobs.count && blockIdx.x >= jobs.job[at].end) ++at;
    const PlaneJobs::Job &j = jobs.job[at];
    const unsigned begin = at ? jobs.job[at - 1].end : 0, groups = j.end - begin;
    const int per_row = j.dp / 8;
    const long long pieces = j.rows * per_row, plane = j.rows * j.dp;
    __bf16 *dst = (__bf16 *)j.dst;
    for (long long t = (long long)(blockIdx.x - begin) * 256 + threadIdx.x; t < pieces; t += (long long)groups * 256) {
        const long long r = t / per_row;
        const int k = (int)(t - r * per_row) * 8;
        const T *p = (const T *)j.src + r * j.d + k;
        f32x4 v[2];
        v[0] = load_four(p, j.d - k, j.vec);
        v[1] = load_four(p + 4, j.d - k - 4, j.vec);
        if (j.target && j.target[r] < 0) v[0] = v[1] = f32x4{0.f, 0.f, 0.f, 0.f};
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

Operand add_masked(PlaneJobs &jobs, const void *p, long long rows, int d, int32_t dtype, const int64_t *target, void *space)
{
    const size_t e = dtype == LCN_F32 ? 4 : 2;
    const long long groups = (rows * (padded(d) / 8) + 255) / 256;
    PlaneJobs::Job &j = jobs.job[jobs.count];
    j.src = p;
    j.dst = space;
    j.target = target;
    j.rows = rows;
    j.d = d;
    j.dp = (int)padded(d);
    j.vec = d % 4 == 0 && ((uintptr_t)p & (4 * e - 1)) == 0;
    j.end = (jobs.count ? jobs.job[jobs.count - 1].end : 0) + (unsigned)(groups < 8192 ? groups : 8192);
    ++jobs.count;
    return plane_operand(space, rows, d);
}

Operand add_operand(PlaneJobs &jobs, const void *p, long long rows, int d, int32_t dtype, void *space)
{
    if (in_place(p, d, dtype)) return Operand{p, 0, d};
    return add_masked(jobs, p, rows, d, dtype, nullptr, space);
}

hipError_t launch_planes(const PlaneJobs &jobs, int32_t dtype, hipStream_t s)
{
    if (!jobs.count) return hipSuccess;
    const dim3 grid(jobs.job[jobs.count - 1].end);
    if (dtype == LCN_F32)
        hipLaunchKernelGGL(planes_kernel<float>, grid, dim3(256), 0, s, jobs);
    else
        hipLaunchKernelGGL(planes_kernel<__bf16>, grid, dim3(256), 0, s, jobs);
    return hipGetLastError();
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
// that the shape reaches on large products (bf16: 256 x 256 1.25 PFLOP/s, 128 x 128 1.1, 64 x 64 0.7; three planes, six
// products counted: 256 x 128 1.4, 320 x 64 1.1, 128 x 128 0.87, 64 x 64 1.0); two steps stand for a workgroup's start and epilogue,
// three where these are 256 x 128 in three planes; the chip takes 256 workgroups of the large shapes at a
// time and several times as many small ones; the partial sums of a split are written and read once at the rate of memory.
//
// Columns behind the last whole tile cost a tile's time, and often a round of them: where that is estimated to be more than
// 3 us and a launch of 64 x 64 tiles, they get that (a bf16 training step of 16391 rows, 1024 to 4096: 711 us, else 784).
ProductPlan plan_product(long long m, long long n, long long k, int planes, bool may_split, bool may_tail)
{
    struct Shape {
        int resident;
        double step_us;   // of one workgroup's step with the chip full: 64 values of k, or 32 in three planes
    };
    static const Shape one[TILE_COUNT] = {{1, 1.8}, {2, 1.03}, {4, 0.77}, {1, 1.25}};
    static const Shape three[TILE_COUNT] = {{1, 2.3}, {1, 1.85}, {3, 1.2}, {1, 1.81}};
    const Shape *shape = planes == 3 ? three : one;
    const long long steps = planes == 3 ? (k + 31) / 32 : (k + 63) / 64 * planes;
    auto launch_us = [&](int t, long long columns, int splits) {
        const int bm = tile_m(t), bn = tile_n(t, planes);
        const long long groups = ((m + bm - 1) / bm) * ((columns + bn - 1) / bn) * splits, room = 256 * shape[t].resident;
        const double rounds = (double)((groups + room - 1) / room);
        double us = rounds * shape[t].step_us * ((double)((steps + splits - 1) / splits) + (planes == 3 && t == TILE_256 ? 3.0 : 2.0));
        if (groups < room) {   // fewer to share a compute unit with
            const double share = (double)((groups + 255) / 256) / shape[t].resident;
            us *= share > 0.5 ? share : 0.5 + 0.5 * share;
        }
        return us;
    };
    ProductPlan best{TILE_256, 1, false};
    double least = 1e300;
    for (int t = 0; t < TILE_COUNT; ++t) {
        const long long rest = n % tile_n(t, planes);
        for (int splits = 1; splits <= 64; splits += splits < 16 ? 1 : 16) {
            if (splits > 1 && (!may_split || steps / splits < 4)) break;
            for (int tail = 0; tail <= (may_tail && t != TILE_64 && rest && n > rest ? 1 : 0); ++tail) {
                double us = tail ? launch_us(t, n - rest, splits) + 3.0 + launch_us(TILE_64, rest, splits) : launch_us(t, n, splits);
                if (splits > 1) us += 3.0 + (double)splits * m * n * 8e-6 / 4.0;
                if (us < least) {
                    least = us;
                    best = ProductPlan{t, splits, tail != 0};
                }
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
        const PartialEpilogue::Args a{part, ldp, p.n * ldp, 0};
        const hipError_t e = p.planes == 3 ? launch_planned<3, ACOL, BCOL, PartialEpilogue>(plan, p, a, s)
                                           : launch_planned<1, ACOL, BCOL, PartialEpilogue>(plan, p, a, s);
        if (e != hipSuccess) return e;
        return launch_add_partials(part, plan.splits, p.n, p.m, ldp, scale, dtype, out, s);
    }
    if (dtype == LCN_F32)
        return launch_planned<3, ACOL, BCOL, ScaledEpilogue<float>>(plan, p, {(float *)out, p.m, scale, whole_rows<float>(out, p.m)}, s);
    return launch_planned<1, ACOL, BCOL, ScaledEpilogue<__bf16>>(plan, p, {(__bf16 *)out, p.m, scale, whole_rows<__bf16>(out, p.m)}, s);
}
template hipError_t launch_scaled<true, false>(const ProductPlan &, const ProductArgs &, float, int32_t, void *, float *,
                                               hipStream_t);
template hipError_t launch_scaled<true, true>(const ProductPlan &, const ProductArgs &, float, int32_t, void *, float *,
                                              hipStream_t);
hipError_t launch_partials(const ProductPlan &plan, const ProductArgs &p, float *part, int add, hipStream_t s)
{
    const long long ldp = padded(p.m);
    const PartialEpilogue::Args a{part, ldp, p.n * ldp, add};
    return p.planes == 3 ? launch_planned<3, true, false, PartialEpilogue>(plan, p, a, s)
                         : launch_planned<1, true, false, PartialEpilogue>(plan, p, a, s);
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
