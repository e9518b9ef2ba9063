// The gated layer with few inputs and outputs on many rows: bound by reading rows and writing them, so nothing is laid out first.
//
// Forward, a workgroup has 32 outputs, their rows of Wg and Wu in registers, and a wavefront goes over rows 16 at a time, straight
// from memory into the matrix instruction.  Backward, all in one launch: a wavefront forms dz of 16 rows in the order that the
// instruction takes for dx = dz W, W from LDS, and turns it around in LDS for its part of dW = dz^T x, which stays in registers from
// row to row, as db does; a workgroup leaves its sums, which a second launch adds.  The float instruction serves bf16 tensors as
// well: dz and all sums are in 32 bits.  40 961 rows, 32 -> 64, float: 14 us and 29 + 4, where the products through planes took 73 in all
// and more than the 31 MB at a copy's rate, 7, what bounds it is the chain from a row's load over two products and LDS to its stores;
// a wavefront has 2.5 tiles of rows, so that W's and the sums' fixed parts count, and reads W's fragments from LDS anew for each.
#include "gated.h"

namespace lcn {

constexpr int NARROW = 64;   // inputs, outputs
constexpr int SOME_ROWS = 64;

// values d0 .. d0 + 7 of a row (nullptr: zeros)
template <class T>
__device__ __forceinline__ typename Frag<T>::type fragment_of(const T *row, int d0, int dim)
{
    typename Frag<T>::type f;
    Eight<T> v{};
    if (row && d0 < dim) v = read_eight(row + d0, dim - d0);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = v.v[e];
    return f;
}

template <class T, int KP, int ACT, bool KEPT>
__global__ __launch_bounds__(256) void gated_narrow_kernel(GatedArgs<T> e, const T *__restrict__ x, const T *__restrict__ w,
                                                           long long rows, int k, int width)
{
    constexpr int C = KP / 32;
    const int lane = threadIdx.x & 63, g = lane >> 4, m0 = (int)blockIdx.y * 32, wp = (int)padded(width);
    typename Frag<T>::type fw[2][2][C];   // of Wg and Wu
    f32x4 bias[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = m0 + i * 16 + (lane & 15), mb = m0 + i * 16 + 4 * g;
#pragma unroll
            for (int c = 0; c < C; ++c)
                fw[h][i][c] = fragment_of(m < width ? w + (long long)(h * width + m) * k : (const T *)nullptr, 32 * c + 8 * g, k);
            bias[h][i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (e.bias && mb < width) bias[h][i] = load_four(e.bias + h * width + mb, width - mb);
        }
    const long long tiles = (rows + 15) / 16, step = (long long)gridDim.x * 4;
    typename Frag<T>::type fx[C];
    auto read = [&](long long t) {
        const long long n = t * 16 + (lane & 15);
#pragma unroll
        for (int c = 0; c < C; ++c) fx[c] = fragment_of(n < rows ? x + n * k : (const T *)nullptr, 32 * c + 8 * g, k);
    };
    long long t = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    read(t);
    for (; t < tiles; t += step) {
        const long long n = t * 16 + (lane & 15);
        f32x4 z[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) z[h][i] = bias[h][i];
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) mma(z[h][i], fw[h][i][c], fx[c]);
        read(t + step);   // the next rows, while these are finished
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = m0 + i * 16 + 4 * g;   // four values; a piece of eight has those of the lane 16 before or behind as well
            if constexpr (KEPT) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (sizeof(T) == 4) {
                        if (n < rows && m < wp) *(f32x4 *)(e.kept + (n * 2 + h) * wp + m) = z[h][i];
                    } else {
                        f32x4 v[2], other;
#pragma unroll
                        for (int u = 0; u < 4; ++u) other[u] = __shfl_xor(z[h][i][u], 16);
                        v[0] = g & 1 ? other : z[h][i];
                        v[1] = g & 1 ? z[h][i] : other;
                        if (!(g & 1) && n < rows && m < wp) Keep<T>::store(e.kept + (n * 2 + h) * wp + m, v);
                    }
                }
            }
            if (n >= rows || m >= width) continue;
            f32x4 y;
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = gate<T, ACT>(z[0][i][u]) * z[1][i][u];
            store_four(e.y + n * width + m, y, width - m);
        }
    }
}

// Some rows, up to 16 N of floats: bound by reading W once, which through planes is read, written and read.  A workgroup has 16 outputs;
// its wavefronts share k, 32 values of it at a time straight from memory into the float instruction, and add up through LDS.  us, so /
// through planes: 16 rows, 576 -> 4096, 7 / 27, 64 15 / 27; 16, 4096 -> 1024, 32 / 41, 32 44 / 41; 64, 1024 -> 8192, 34 / 55, 2048 -> 2048 37 / 37.
template <int ACT, int N>
__global__ __launch_bounds__(256) void gated_some_kernel(GatedArgs<float> e, const float *__restrict__ x, const float *__restrict__ w,
                                                         int rows, int k, int width)
{
    __shared__ f32x4 sums[4][2][N][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4, m0 = (int)blockIdx.x * 16, wp = (int)padded(width);
    const float *rw[2], *rx[N];   // nullptr: a row of zeros
#pragma unroll
    for (int h = 0; h < 2; ++h) rw[h] = m0 + l < width ? w + (long long)(h * width + m0 + l) * k : nullptr;
#pragma unroll
    for (int t = 0; t < N; ++t) rx[t] = t * 16 + l < rows ? x + (long long)(t * 16 + l) * k : nullptr;
    struct Chunk {
        Frag<float>::type w[2], x[N];
    };
    auto read = [&](int c, Chunk &v) {
#pragma unroll
        for (int h = 0; h < 2; ++h) v.w[h] = fragment_of(rw[h], 32 * c + 8 * g, k);
#pragma unroll
        for (int t = 0; t < N; ++t) v.x[t] = fragment_of(rx[t], 32 * c + 8 * g, k);
    };
    f32x4 z[2][N];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < N; ++t) z[h][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int chunks = (k + 31) / 32;
    Chunk next;
    read(wave, next);   // zeros behind k
    for (int c = wave; c < chunks; c += 4) {
        const Chunk now = next;
        read(c + 4, next);   // while this one is worked on
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int t = 0; t < N; ++t) mma(z[h][t], now.w[h], now.x[t]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < N; ++t) sums[wave][h][t][lane] = z[h][t];
    __syncthreads();
    const int m = m0 + 4 * g;
    for (int t = wave; t < N; t += 4) {
        const int n = t * 16 + l;
        if (n >= rows || m >= wp) continue;
        f32x4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v[h] = (sums[0][h][t][lane] + sums[1][h][t][lane]) + (sums[2][h][t][lane] + sums[3][h][t][lane]);
            if (e.bias && m < width) v[h] += load_four(e.bias + h * width + m, width - m);
            if (e.kept) *(f32x4 *)(e.kept + (n * 2LL + h) * wp + m) = v[h];
        }
        if (m >= width) continue;
#pragma unroll
        for (int u = 0; u < 4; ++u) v[0][u] = gate<float, ACT>(v[0][u]) * v[1][u];
        store_four(e.y + (long long)n * width + m, v[0], width - m);
    }
}

// D tiles of 16 inputs, C chunks of 32 outputs
template <class T, int ACT, int D, int C>
__global__ __launch_bounds__(256) void gated_narrow_grad_kernel(const T *__restrict__ x, const T *__restrict__ w,
                                                                const typename Keep<T>::type *__restrict__ kept,
                                                                const T *__restrict__ dy, long long rows, int d_in, int width,
                                                                T *__restrict__ dx, float *__restrict__ part)
{
    // pitches: rows 8 (of W) and 1 (of dz) apart begin 16 banks apart
    constexpr int WP = D * 16 + 2, ZP = C * 64 + 16, K = C * 64;
    __shared__ __align__(16) float lds_w[K * WP];         // rows of Wg, then of Wu from C * 32 on
    __shared__ __align__(16) float lds_z[4 * 16 * ZP];    // a wavefront's dz
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, l = lane & 15, wp = (int)padded(width);
#pragma unroll
    for (int u = 0; u < K * D * 4 / 256; ++u) {
        const int i = u * 256 + tid, k = i / (D * 4), c = i % (D * 4) * 4, h = k / (C * 32), m = k % (C * 32);
        const f32x4 v = m < width ? load_four(w + (h * width + m) * d_in + c, d_in - c) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) lds_w[k * WP + c + e] = v[e];
    }
    __syncthreads();
    float *z = lds_z + wave * 16 * ZP;
    f32x4 dw[2 * C * 2][D];
    float db[2][C][8];
#pragma unroll
    for (int i = 0; i < 4 * C; ++i)
#pragma unroll
        for (int t = 0; t < D; ++t) dw[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int u = 0; u < 8; ++u) db[0][c][u] = db[1][c][u] = 0.f;
    const long long tiles = (rows + 15) / 16, step = (long long)gridDim.x * 4;
    struct Rows {
        f32x4 d[C][2], a[C][2], b[C][2];   // of row l: dy, g and u
        float x[4][D];                     // of rows 4 s + g, for dW
    };
    auto read = [&](long long tile, Rows &v) {
        const long long n = tile * 16 + l;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int m = 32 * c + 8 * g;
            v.d[c][0] = v.d[c][1] = v.a[c][0] = v.a[c][1] = v.b[c][0] = v.b[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (n < rows && m < width) {
                load_eight(dy + n * width + m, width - m, v.d[c]);
                Keep<T>::load(kept + n * 2 * wp + m, v.a[c]);
                Keep<T>::load(kept + (n * 2 + 1) * wp + m, v.b[c]);
            }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int t = 0; t < D; ++t) {
                const long long r = tile * 16 + 4 * s + g;
                v.x[s][t] = part && r < rows && t * 16 + l < d_in ? (float)x[r * d_in + t * 16 + l] : 0.f;
            }
    };
    long long tile = (long long)blockIdx.x * 4 + wave;
    Rows next;
    read(tile, next);
    for (; tile < tiles; tile += step) {
        const long long n = tile * 16 + l;
        const Rows now = next;
        read(tile + step, next);   // while these rows are worked on
        f32x4 out[D];
#pragma unroll
        for (int t = 0; t < D; ++t) out[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int m = 32 * c + 8 * g;
            Frag<float>::type f[2];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float v = now.d[c][u >> 2][u & 3];
                float act, slope;
                gate_and_slope<T, ACT>(now.a[c][u >> 2][u & 3], act, slope);
                f[0][u] = v * now.b[c][u >> 2][u & 3] * slope;
                f[1][u] = v * act;
                db[0][c][u] += f[0][u];
                db[1][c][u] += f[1][u];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k0 = h * C * 32 + m;
                if (dx)
#pragma unroll
                    for (int t = 0; t < D; ++t) {
                        Frag<float>::type fw;
#pragma unroll
                        for (int u = 0; u < 8; ++u) fw[u] = lds_w[(k0 + u) * WP + t * 16 + l];
                        mma(out[t], fw, f[h]);
                    }
#pragma unroll
                for (int u = 0; u < 8; u += 4) *(f32x4 *)(z + l * ZP + k0 + u) = f32x4{f[h][u], f[h][u + 1], f[h][u + 2], f[h][u + 3]};
            }
        }
        if (dx && n < rows)
#pragma unroll
            for (int t = 0; t < D; ++t)
                if (t * 16 + 4 * g < d_in) store_four(dx + n * d_in + t * 16 + 4 * g, out[t], d_in - t * 16 - 4 * g);
        if (!part) continue;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // LDS serves a wavefront in order
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4 * C; ++i)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const float v = z[(4 * s + g) * ZP + i * 16 + l];
#pragma unroll
                for (int t = 0; t < D; ++t) dw[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, now.x[s][t], dw[i][t], 0, 0, 0);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    if (!part) return;
    // dw[i][t]: row k = 16 i + 4 g + e, column 16 t + l.  Two wavefronts leave their sums in LDS, the other two add theirs.
    __shared__ float lds_b[2][K];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) db[h][c][u] += __shfl_xor(db[h][c][u], o, 16);
    static_assert(K * WP <= 4 * 16 * ZP, "a second place for dW's sums");
    float *sum = wave & 1 ? lds_z : lds_w;
    for (int turn = 0; turn < 2; ++turn) {
        __syncthreads();
        if (wave >> 1 != turn) continue;
#pragma unroll
        for (int i = 0; i < 4 * C; ++i)
#pragma unroll
            for (int t = 0; t < D; ++t)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float *at = sum + (16 * i + 4 * g + q) * WP + 16 * t + l;
                    *at = turn ? *at + dw[i][t][q] : dw[i][t][q];
                }
        if (l == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        float *at = lds_b[wave & 1] + h * C * 32 + 32 * c + 8 * g + u;
                        *at = turn ? *at + db[h][c][u] : db[h][c][u];
                    }
    }
    __syncthreads();
    // rows of dW as they lie in memory, without those that are padding
    float *to = part + (long long)blockIdx.x * 2 * width * (d_in + 1);
#pragma unroll 4
    for (int i = tid; i < K * D * 16; i += 256) {
        const int k = i / (D * 16), c = i % (D * 16), h = k / (C * 32), m = k % (C * 32);
        if (m < width && c < d_in) to[(h * width + m) * d_in + c] = lds_w[k * WP + c] + lds_z[k * WP + c];
    }
    for (int k = tid; k < K; k += 256) {
        const int h = k / (C * 32), m = k % (C * 32);
        if (m < width) to[2 * width * d_in + h * width + m] = lds_b[0][k] + lds_b[1][k];
    }
}

// adds up the workgroups' sums: values 0 .. first - 1 are dw, the others db; 16 values per workgroup, 16 threads each, in a fixed order
template <class T>
__global__ __launch_bounds__(256) void gated_narrow_join_kernel(const float *__restrict__ part, int parts, int first, int all,
                                                                T *__restrict__ dw, T *__restrict__ db)
{
    __shared__ float sums[16][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), q = threadIdx.x >> 4;
    float v = 0.f;
    if (c < all)
#pragma unroll 8
        for (int r = q; r < parts; r += 16) v += part[(long long)r * all + c];
    sums[q][threadIdx.x & 15] = v;
    __syncthreads();
    if (q || c >= all) return;
#pragma unroll
    for (int u = 1; u < 16; ++u) v += sums[u][threadIdx.x];
    if (c < first) {
        if (dw) dw[c] = (T)v;
    } else if (db) {
        db[c - first] = (T)v;
    }
}

// ---- host ---------------------------------------------------------------------

bool gated_some(int64_t rows, int32_t d_in, int32_t dtype)
{
    return dtype == LCN_F32 && rows <= SOME_ROWS && (rows <= 16 ? 1 : rows <= 32 ? 2 : 4) * (int64_t)d_in <= 4096;
}

hipError_t launch_gated_some(const GatedArgs<float> &e, const float *x, const float *w, int rows, int d_in, int d_out, hipStream_t s)
{
    return by_activation(e.act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((d_out + 15) / 16)), dim3(256), 0, s, e, x, w, rows, d_in, d_out);
            return hipGetLastError();
        };
        return rows <= 16 ? launch(gated_some_kernel<ACT, 1>) : rows <= 32 ? launch(gated_some_kernel<ACT, 2>) : launch(gated_some_kernel<ACT, 4>);
    });
}

bool gated_narrow(int64_t rows, int32_t d_in, int32_t d_out) { return rows >= 128 && d_in <= NARROW && d_out <= NARROW; }

int gated_narrow_groups(int64_t rows)
{
    const int64_t groups = (rows + 63) / 64;
    return (int)(groups < 256 ? groups : 256);   // one to a compute unit: 512 take 38 us instead of 31
}

template <class T>
hipError_t launch_gated_narrow(const GatedArgs<T> &e, const T *x, const T *w, int64_t rows, int32_t d_in, int32_t d_out, hipStream_t s)
{
    const long long groups = (rows + 63) / 64, tiles = (d_out + 31) / 32;
    // a wavefront has W's rows to bring first: 256, 512 and 2048 workgroups for 40 961 rows, 32 -> 64, float 14, 15 and 17 us, bf16 11, 9
    // and 10
    const long long most = (sizeof(T) == 4 ? 256 : 512) / tiles;
    const dim3 grid((unsigned)(groups < most ? groups : most), (unsigned)tiles);
    return by_activation(e.act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, e, x, w, (long long)rows, d_in, d_out);
            return hipGetLastError();
        };
        if (e.kept) return d_in <= 32 ? launch(gated_narrow_kernel<T, 32, ACT, true>) : launch(gated_narrow_kernel<T, 64, ACT, true>);
        return d_in <= 32 ? launch(gated_narrow_kernel<T, 32, ACT, false>) : launch(gated_narrow_kernel<T, 64, ACT, false>);
    });
}
template hipError_t launch_gated_narrow(const GatedArgs<float> &, const float *, const float *, int64_t, int32_t, int32_t, hipStream_t);
template hipError_t launch_gated_narrow(const GatedArgs<__bf16> &, const __bf16 *, const __bf16 *, int64_t, int32_t, int32_t, hipStream_t);

template <class T>
hipError_t launch_gated_narrow_backward(const T *x, const T *w, const typename Keep<T>::type *kept, const T *dy, int64_t rows, int32_t d_in,
                                        int32_t d_out, int32_t act, T *dx, T *dw, T *db, float *part, hipStream_t s)
{
    const int groups = gated_narrow_groups(rows), first = 2 * d_out * d_in, all = first + 2 * d_out;
    const bool sums = dw || db;
    const hipError_t st = by_activation(act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, s, x, w, kept, dy, (long long)rows, d_in, d_out, dx,
                               sums ? part : nullptr);
            return hipGetLastError();
        };
        if (d_out <= 32)
            return d_in <= 32 ? launch(gated_narrow_grad_kernel<T, ACT, 2, 1>) : launch(gated_narrow_grad_kernel<T, ACT, 4, 1>);
        return d_in <= 32 ? launch(gated_narrow_grad_kernel<T, ACT, 2, 2>) : launch(gated_narrow_grad_kernel<T, ACT, 4, 2>);
    });
    if (st != hipSuccess || !sums) return st;
    hipLaunchKernelGGL(gated_narrow_join_kernel<T>, dim3((unsigned)((all + 15) / 16)), dim3(256), 0, s, part, groups, first, all, dw, db);
    return hipGetLastError();
}
template hipError_t launch_gated_narrow_backward(const float *, const float *, const float *, const float *, int64_t, int32_t, int32_t,
                                                 int32_t, float *, float *, float *, float *, hipStream_t);
template hipError_t launch_gated_narrow_backward(const __bf16 *, const __bf16 *, const unsigned short *, const __bf16 *, int64_t, int32_t,
                                                 int32_t, int32_t, __bf16 *, __bf16 *, __bf16 *, float *, hipStream_t);

}  // namespace lcn
