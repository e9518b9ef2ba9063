// Layer norm of rows and its gradients.
//
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(mean of (x - mean)^2 + eps)
//   dx = rstd (g - mean of g - xhat mean of (g xhat)) + around,  g = dy w,  xhat = (x - mean) rstd
//   dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// Bound by memory: a row is read once and stays in registers (so its variance is formed from differences to its mean), by as
// many lanes as hold it in 16-byte pieces: 4 to 64, so that a wavefront has several narrow rows, or a workgroup.  Backward, a
// thread keeps its columns from row to row and adds up dw and db for them; a workgroup leaves one partial sum per column.
// 16 391 rows of 4096 bf16 values: forward 43 to 51 us (5.3 TB/s or more), backward 92 to 107 (5.0 TB/s: three streams in, one
// out) and 7 for the join; 40 961 rows of 32 floats 4.5 and 6.5 + 3, of which a launch
// is 2.5.  Rows too long for that are read by a workgroup in a loop, several times, with the sums over rows in a kernel of their own.
#include "operators.h"

namespace lcn {

// V neighbours of a row, from its value c on.  TAIL: wherever they lie, and of a row's last piece only those that exist.
template <class T, int V>
struct Piece {
    typedef T type __attribute__((ext_vector_type(V)));
    typedef T any __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <class T, int V, bool TAIL>
__device__ __forceinline__ typename Piece<T, V>::type load_piece(const T *row, int c, int dim)
{
    typedef typename Piece<T, V>::type piece;
    if constexpr (TAIL) {
        if (c + V > dim) {
            piece v{};
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (c + e < dim) v[e] = row[c + e];
            return v;
        }
        return *(const typename Piece<T, V>::any *)(row + c);
    }
    return *(const piece *)(row + c);
}
template <class T, int V, bool TAIL>
__device__ __forceinline__ void store_piece(T *p, int left, typename Piece<T, V>::type v)
{
    if constexpr (TAIL) {
        if (left < V) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < left) p[e] = v[e];
        } else {
            *(typename Piece<T, V>::any *)p = v;
        }
    } else {
        *(typename Piece<T, V>::type *)p = v;
    }
}

// Sums over the L lanes (or the workgroup's 256 threads) that share a row, in each of them.  `lds`: 4 values of the workgroup's
// own, others from one call to the next (whoever is late still reads the last call's).
template <int L>
__device__ __forceinline__ float sum_over(float a, float *lds)
{
    constexpr int W = L < 64 ? L : 64;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) a += __shfl_xor(a, o, W);
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
        __syncthreads();
        a = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    }
    return a;
}

// A power of two from 1 / (2 dim) on, below 1 / dim: a sum of `dim` finite values times it stays in a float's range, as their mean does.
__device__ __forceinline__ float share_of(int dim) { return __builtin_ldexpf(1.f, __builtin_clz(dim) - 32); }
// A power of two whose square times dim is from 1 / 8 on, below 1 / 2: differences times it have a sum of squares that stays in a
// float's range where the variance does, with no rounding of a factor's own (1 / sqrt(dim) is off by 1e-7 in the variance).
__device__ __forceinline__ float root_share_of(int dim) { return __builtin_ldexpf(1.f, -((34 - __builtin_clz(dim)) / 2)); }
// x - mean, halved, so that it stays in that range as well: what it is multiplied with is doubled, and the product has the same bits.
__device__ __forceinline__ float half_less(float x, float half_mean) { return __builtin_fmaf(x, 0.5f, -half_mean); }

// L lanes have a row, C pieces of V values each.
template <class T, int V, bool TAIL, int L, int C>
__global__ __launch_bounds__(256) void norm_kernel(const T *x, const T *__restrict__ w, const T *__restrict__ b, long long rows,
                                                   int dim, float eps, T *y,   // y may be x
                                                   float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    typedef typename Piece<T, V>::type piece;
    __shared__ float lds[2][4];
    const int lane = threadIdx.x % L, units = TAIL ? (dim + V - 1) / V : dim / V;
    const long long r = (long long)group_number() * (256 / L) + threadIdx.x / L;
    if (L > 64 && r >= rows) return;
    const bool here = r < rows;
    piece p[C];
    float sum = 0.f;
    const float part = share_of(dim);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int u = c * L + lane;
        p[c] = here && u < units ? load_piece<T, V, TAIL>(x + r * dim, u * V, dim) : piece{};
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < V; ++e) sum = __builtin_fmaf((float)p[c][e], part, sum);
    const float mean = sum_over<L>(sum, lds[0]) / ((float)dim * part), half = 0.5f * mean;
    float square = 0.f;
    const float root = root_share_of(dim), mean_part = mean * root;
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (c * L + lane < units)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = __builtin_fmaf((float)p[c][e], root, -mean_part);
                if (!TAIL || (c * L + lane) * V + e < dim) square += d * d;
            }
    const float rstd = 1.f / sqrtf(sum_over<L>(square, lds[1]) / ((float)dim * root * root) + eps), twice = 2.f * rstd;
    if (!here) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int u = c * L + lane;
        if (u >= units) break;
        piece o, pw, pb;
        if (w) pw = load_piece<T, V, TAIL>(w, u * V, dim);
        if (b) pb = load_piece<T, V, TAIL>(b, u * V, dim);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float v = half_less((float)p[c][e], half) * twice;
            if (w) v *= (float)pw[e];
            if (b) v += (float)pb[e];
            o[e] = (T)v;
        }
        store_piece<T, V, TAIL>(y + r * dim + u * V, dim - u * V, o);
    }
    if (lane == 0) {
        if (mean_out) mean_out[r] = mean;
        if (rstd_out) rstd_out[r] = rstd;
    }
}

// Rows g, g + gridDim.x, ... (256 / L at a time) for workgroup g: dx (nullable), and the workgroup's sums of dy xhat and dy for
// every column at part[g][0 .. 1] (nullable).  With one or two pieces per lane the next row is requested before this one is
// worked on.
template <class T, int V, bool TAIL, int L, int C>
__global__ __launch_bounds__(256) void norm_grad_kernel(const T *__restrict__ x, const T *__restrict__ w,
                                                        const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
                                                        const T *__restrict__ dy, const T *around, long long rows, int dim,
                                                        T *dx,   // dx may be around
                                                        float *__restrict__ part)
{
    typedef typename Piece<T, V>::type piece;
    constexpr int PER = 256 / L, WIDTH = L * C * V;
    constexpr bool AHEAD = C <= 2;
    __shared__ float lds[2][2][4];
    __shared__ float columns[L > 64 ? 1 : 4 * WIDTH];
    const int lane = threadIdx.x % L, units = TAIL ? (dim + V - 1) / V : dim / V;
    const long long step = (long long)gridDim.x * PER;
    struct Row {
        piece x[C], dy[C], around[C];
        float half, rstd;   // half of the mean
    };
    auto read = [&](long long r) {
        Row t;
        const bool here = r < rows;
        t.half = here ? 0.5f * mean_in[r] : 0.f;
        t.rstd = here ? rstd_in[r] : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int u = c * L + lane;
            const bool in = here && u < units;
            t.x[c] = in ? load_piece<T, V, TAIL>(x + r * dim, u * V, dim) : piece{};
            t.dy[c] = in ? load_piece<T, V, TAIL>(dy + r * dim, u * V, dim) : piece{};
            t.around[c] = in && around ? load_piece<T, V, TAIL>(around + r * dim, u * V, dim) : piece{};
        }
        return t;
    };
    piece pw[C];
    float dw[C][V], db[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        pw[c] = w && c * L + lane < units ? load_piece<T, V, TAIL>(w, (c * L + lane) * V, dim) : piece{};
#pragma unroll
        for (int e = 0; e < V; ++e) dw[c][e] = db[c][e] = 0.f;
    }
    // every thread makes the same number of rounds: the sums over a workgroup wait for all of it
    long long r = (long long)blockIdx.x * PER + threadIdx.x / L;
    int turn = 0;
    Row next{};
    if (AHEAD) next = read(r);
    for (long long first = (long long)blockIdx.x * PER; first < rows; first += step, r += step, turn ^= 1) {
        Row t = AHEAD ? next : read(r);
        if (AHEAD && first + step < rows) next = read(r + step);
        const float twice = 2.f * t.rstd;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = (float)t.dy[c][e], h = half_less((float)t.x[c][e], t.half) * twice, g = w ? d * (float)pw[c][e] : d;
                s1 += g;
                s2 += g * h;
                dw[c][e] += d * h;
                db[c][e] += d;
            }
        if (!dx) continue;
        s1 = sum_over<L>(s1, lds[turn][0]) / (float)dim;
        s2 = sum_over<L>(s2, lds[turn][1]) / (float)dim;
        if (r >= rows) continue;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int u = c * L + lane;
            if (u >= units) break;
            piece o;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = (float)t.dy[c][e], h = half_less((float)t.x[c][e], t.half) * twice, g = w ? d * (float)pw[c][e] : d;
                float v = t.rstd * (g - s1 - h * s2);
                if (around) v += (float)t.around[c][e];
                o[e] = (T)v;
            }
            store_piece<T, V, TAIL>(dx + r * dim + u * V, dim - u * V, o);
        }
    }
    if (!part) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&v)[C][V] = which ? db : dw;
        float *to = part + ((long long)blockIdx.x * 2 + which) * dim;
        if constexpr (L > 64) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (TAIL ? (c * L + lane) * V + e < dim : c * L + lane < units) to[(c * L + lane) * V + e] = v[c][e];
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < V; ++e)
#pragma unroll
                    for (int o = L; o < 64; o <<= 1) v[c][e] += __shfl_xor(v[c][e], o);
            __syncthreads();
            if ((threadIdx.x & 63) < L)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int e = 0; e < V; ++e) columns[(threadIdx.x >> 6) * WIDTH + (c * L + lane) * V + e] = v[c][e];
            __syncthreads();
            for (int i = threadIdx.x; i < dim; i += 256)
                to[i] = (columns[i] + columns[WIDTH + i]) + (columns[2 * WIDTH + i] + columns[3 * WIDTH + i]);
        }
    }
}

// ---- rows that no workgroup holds in registers ---------------------------------

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

template <class T, int V, bool TAIL>
__global__ __launch_bounds__(256) void norm_long_kernel(const T *x, const T *__restrict__ w, const T *__restrict__ b,
                                                   long long rows, int dim, float eps, T *y,   // y may be x
                                                   float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    typedef typename Piece<T, V>::type piece;
    __shared__ float lds[4][2];
    const long long r = group_number();
    if (r >= rows) return;
    const int units = TAIL ? (dim + V - 1) / V : dim / V;
    const T *row = x + r * dim;
    const float part = share_of(dim);
    float sum = 0.f, none = 0.f;
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece p = load_piece<T, V, TAIL>(row, u * V, dim);
#pragma unroll
        for (int e = 0; e < V; ++e) sum = __builtin_fmaf((float)p[e], part, sum);
    }
    sum_over_group(sum, none, lds);
    const float mean = sum / ((float)dim * part), half = 0.5f * mean;
    float square = 0.f;
    const float root = root_share_of(dim), mean_part = mean * root;
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece p = load_piece<T, V, TAIL>(row, u * V, dim);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = __builtin_fmaf((float)p[e], root, -mean_part);
            if (!TAIL || u * V + e < dim) square += d * d;
        }
    }
    sum_over_group(square, none, lds);
    const float rstd = 1.f / sqrtf(square / ((float)dim * root * root) + eps), twice = 2.f * rstd;
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece p = load_piece<T, V, TAIL>(row, u * V, dim);
        piece o, pw, pb;
        if (w) pw = load_piece<T, V, TAIL>(w, u * V, dim);
        if (b) pb = load_piece<T, V, TAIL>(b, u * V, dim);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float v = half_less((float)p[e], half) * twice;
            if (w) v *= (float)pw[e];
            if (b) v += (float)pb[e];
            o[e] = (T)v;
        }
        store_piece<T, V, TAIL>(y + r * dim + u * V, dim - u * V, o);
    }
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[r] = mean;
        if (rstd_out) rstd_out[r] = rstd;
    }
}

template <class T, int V, bool TAIL>
__global__ __launch_bounds__(256) void norm_long_dx_kernel(const T *__restrict__ x, const T *__restrict__ w,
                                                      const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
                                                      const T *__restrict__ dy, const T *around, long long rows,
                                                      int dim, T *dx)   // dx may be around
{
    typedef typename Piece<T, V>::type piece;
    __shared__ float lds[4][2];
    const long long r = group_number();
    if (r >= rows) return;
    const int units = TAIL ? (dim + V - 1) / V : dim / V;
    x += r * dim, dy += r * dim, dx += r * dim;
    if (around) around += r * dim;
    const float half = 0.5f * mean_in[r], rstd = rstd_in[r], twice = 2.f * rstd;
    float s1 = 0.f, s2 = 0.f;
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece px = load_piece<T, V, TAIL>(x, u * V, dim), pd = load_piece<T, V, TAIL>(dy, u * V, dim);
        piece pw;
        if (w) pw = load_piece<T, V, TAIL>(w, u * V, dim);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float g = (float)pd[e] * (w ? (float)pw[e] : 1.f);
            s1 += g;
            s2 += g * (half_less((float)px[e], half) * twice);
        }
    }
    sum_over_group(s1, s2, lds);
    s1 /= (float)dim;
    s2 /= (float)dim;
    for (int u = threadIdx.x; u < units; u += 256) {
        const piece px = load_piece<T, V, TAIL>(x, u * V, dim), pd = load_piece<T, V, TAIL>(dy, u * V, dim);
        piece pw, pa, o;
        if (w) pw = load_piece<T, V, TAIL>(w, u * V, dim);
        if (around) pa = load_piece<T, V, TAIL>(around, u * V, dim);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float g = (float)pd[e] * (w ? (float)pw[e] : 1.f);
            float v = rstd * (g - s1 - half_less((float)px[e], half) * twice * s2);
            if (around) v += (float)pa[e];
            o[e] = (T)v;
        }
        store_piece<T, V, TAIL>(dx + u * V, dim - u * V, o);
    }
}

// part[g][0][c], part[g][1][c]: the sums of dy xhat and of dy over the rows r = g, g + gridDim.y, ...; a thread has V columns
template <class T, int V, bool TAIL>
__global__ __launch_bounds__(256) void norm_columns_kernel(const T *__restrict__ x, const float *__restrict__ mean,
                                                           const float *__restrict__ rstd, const T *__restrict__ dy,
                                                           long long rows, int dim, float *__restrict__ part)
{
    typedef typename Piece<T, V>::type piece;
    const int u = (int)(blockIdx.x * 256 + threadIdx.x);
    if (u >= (TAIL ? (dim + V - 1) / V : dim / V)) return;
    float dw[V], db[V];
#pragma unroll
    for (int e = 0; e < V; ++e) dw[e] = db[e] = 0.f;
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        const piece px = load_piece<T, V, TAIL>(x + r * dim, u * V, dim), pd = load_piece<T, V, TAIL>(dy + r * dim, u * V, dim);
        const float half = 0.5f * mean[r], twice = 2.f * rstd[r];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dw[e] += (float)pd[e] * (half_less((float)px[e], half) * twice);
            db[e] += (float)pd[e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        if (TAIL && u * V + e >= dim) break;
        part[((long long)blockIdx.y * 2) * dim + u * V + e] = dw[e];
        part[((long long)blockIdx.y * 2 + 1) * dim + u * V + e] = db[e];
    }
}

// Adds up the partial sums of dw (columns 0 .. dim - 1) and db (the dim behind): 16 columns per workgroup, 16 threads each, in a
// fixed order: chains of up to 7, then in pairs (dw and db of 40 961 rows off by 1.0e-7; one chain of 32 and one of 16, 1.6e-7).
template <class T>
__global__ __launch_bounds__(256) void norm_join_kernel(const float *__restrict__ part, int parts, int dim, T *__restrict__ dw,
                                                        T *__restrict__ db)
{
    __shared__ float sums[16][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), q = threadIdx.x >> 4, width = 2 * dim;
    float t[16] = {};
    if (c < width) {
        int r = q;
        for (; r + 112 < parts; r += 128)
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] += part[(long long)(r + 16 * u) * width + c];
        for (; r < parts; r += 16) t[8] += part[(long long)r * width + c];
    }
    sums[q][threadIdx.x & 15] = (((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]))) + t[8];
    __syncthreads();
    if (q || c >= width) return;
#pragma unroll
    for (int u = 0; u < 16; ++u) t[u] = sums[u][threadIdx.x];
#pragma unroll
    for (int n = 8; n > 0; n >>= 1)
#pragma unroll
        for (int u = 0; u < n; ++u) t[u] += t[u + n];
    const float v = t[0];
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

// Partial sums of dw and db: one per workgroup that shares the rows.  As many workgroups as keep memory busy; more cost their
// sums' way through memory.
static int norm_groups(int64_t rows) { return (int)(rows < 512 ? rows : 512); }
static size_t norm_backward_space(int64_t rows, int32_t dim)
{
    return ((size_t)norm_groups(rows) * 2 * dim * 4 + 255) & ~(size_t)255;
}

// Calls f with the values of a load as a type: 16 bytes, or 8 (bf16), where rows are whole ones of those, aligned; else single
// values in short rows and 16 bytes wherever they lie in long ones.  us forward + backward, singly / in 16 bytes: 20 000 rows of 301,
// float 13 + 21 / 13 + 23, bf16 12 + 20 / 14 + 27; 40 000 of 75, float 11 + 16 / 12 + 24; 8000 of 1001, bf16 15 + 30 / 13 + 25; of 4097,
// bf16 48 + 363 / 31 + 89; of 2050, float 27 + 158 / 27 + 55.
template <int V, bool TAIL>
struct Width {
    static constexpr int value = V;
    static constexpr bool tail = TAIL;
};
template <class T, class F>
static hipError_t by_width(uintptr_t addresses, int32_t dim, F f)
{
    constexpr int MOST = 16 / (int)sizeof(T);
    if (dim % MOST == 0 && addresses % 16 == 0) return f(Width<MOST, false>());
    if (MOST == 8 && dim % 4 == 0 && addresses % 8 == 0) return f(Width<4, false>());
    return dim <= 512 ? f(Width<1, false>()) : f(Width<MOST, true>());
}

// Calls f with the lanes that share a row of `units` pieces and the pieces of each as a type; false: a row is too long for that.
// With many rows a row gets few lanes with several pieces each (more loads of a wavefront at once, sums over fewer lanes), as many
// slots as it has pieces or little more; with few rows it gets all the lanes that it can use.  20 000 rows of 300, forward and
// backward, us: 16 x 5 lanes x pieces float 9 + 19, bf16 7 + 14; 64 x 2 11 + 19, 9 + 19; of 301 (single values), 64 x 5 12 + 20 and
// 10 + 19, 256 x 2 22 + 45 and 21 + 45; 16 391 of 2048 in bf16, 64 x 4 23 + 39, 256 x 1 28 + 49; of 4096, 64 x 8 46 + 117,
// 256 x 2 43 + 83; 40 000 float rows of 256, 32 x 2 15 + 25, 64 x 1 16 + 25;
// backward, 4000 float rows of 4097, 256 x 6 52, 256 x 8 78; 8000 bf16 rows of 5000, 256 x 3 59, 256 x 4 62.
template <int L, int C>
struct Lanes {
    static constexpr int lanes = L, pieces = C;
};
constexpr int LONGEST = 2048;
template <int V, bool TAIL, class F>
static bool by_lanes(int units, int64_t rows, hipError_t &st, F f)
{
    const bool many = rows >= 2048;
    if constexpr (V == 1)   // up to 512 single values: a wavefront's registers hold them easily
        if (many && units > 256) {
            st = units <= 320 ? f(Lanes<64, 5>()) : f(Lanes<64, 8>());
            return true;
        }
    if constexpr (!TAIL) {   // with TAIL a row has more than 64 pieces
        if (many && units > 32 && units <= 64) {
            st = f(Lanes<32, 2>());
            return true;
        }
        if (units <= 64) {
            st = units <= 4    ? f(Lanes<4, 1>())
                 : units <= 8  ? f(Lanes<8, 1>())
                 : units <= 16 ? f(Lanes<16, 1>())
                 : units <= 32 ? f(Lanes<32, 1>())
                               : f(Lanes<64, 1>());
            return true;
        }
    }
    if (many && units <= 80) {
        st = f(Lanes<16, 5>());
    } else if (many && units <= 96) {
        st = f(Lanes<32, 3>());
    } else if (many && units > 128 && units <= 256) {
        st = f(Lanes<64, 4>());
    } else if (units <= 512) {
        st = units <= 128 ? f(Lanes<64, 2>()) : units <= 256 ? f(Lanes<256, 1>()) : f(Lanes<256, 2>());
    } else {
        if constexpr (V == 1) return false;   // none so long
        else if (units <= LONGEST)
            st = units <= 768    ? f(Lanes<256, 3>())
                 : units <= 1024 ? f(Lanes<256, 4>())
                 : units <= 1536 ? f(Lanes<256, 6>())
                                 : f(Lanes<256, 8>());
    }
    return units <= LONGEST;
}

template <class T>
static lcn_status norm_as(const T *x, const T *w, const T *b, int64_t rows, int32_t dim, float eps, T *y, float *mean,
                          float *rstd, hipStream_t s)
{
    OPCHK(by_width<T>((uintptr_t)x | (uintptr_t)w | (uintptr_t)b | (uintptr_t)y, dim, [&](auto v) {
        constexpr int V = decltype(v)::value;
        constexpr bool TAIL = decltype(v)::tail;
        hipError_t st;
        if (by_lanes<V, TAIL>((dim + V - 1) / V, rows, st, [&](auto l) {
                constexpr int L = decltype(l)::lanes, C = decltype(l)::pieces;
                hipLaunchKernelGGL((norm_kernel<T, V, TAIL, L, C>), grid_of((rows + 256 / L - 1) / (256 / L)), dim3(256), 0, s, x, w, b,
                                   (long long)rows, dim, eps, y, mean, rstd);
                return hipGetLastError();
            }))
            return st;
        if constexpr (V > 1)
            hipLaunchKernelGGL((norm_long_kernel<T, V, TAIL>), grid_of(rows), dim3(256), 0, s, x, w, b, (long long)rows, dim, eps, y, mean, rstd);
        return hipGetLastError();
    }));
    return LCN_OK;
}

template <class T>
static lcn_status norm_backward_as(const T *x, const T *w, const float *mean, const float *rstd, const T *dy, const T *around,
                                   int64_t rows, int32_t dim, T *dx, T *dw, T *db, float *part, hipStream_t s)
{
    const uintptr_t all = (uintptr_t)x | (uintptr_t)w | (uintptr_t)dy | (uintptr_t)around | (uintptr_t)dx;
    const int most = norm_groups(rows);
    const bool sums = dw || db;
    int groups = most;
    OPCHK(by_width<T>(all, dim, [&](auto v) {
        constexpr int V = decltype(v)::value;
        constexpr bool TAIL = decltype(v)::tail;
        hipError_t st;
        if (by_lanes<V, TAIL>((dim + V - 1) / V, rows, st, [&](auto l) {
                constexpr int L = decltype(l)::lanes, C = decltype(l)::pieces;
                const int64_t needed = (rows + 256 / L - 1) / (256 / L);
                groups = (int)(needed < most ? needed : most);
                hipLaunchKernelGGL((norm_grad_kernel<T, V, TAIL, L, C>), dim3((unsigned)groups), dim3(256), 0, s, x, w, mean, rstd, dy, around,
                                   (long long)rows, dim, dx, sums ? part : nullptr);
                return hipGetLastError();
            }))
            return st;
        if constexpr (V > 1) {
            if (dx) hipLaunchKernelGGL((norm_long_dx_kernel<T, V, TAIL>), grid_of(rows), dim3(256), 0, s, x, w, mean, rstd, dy, around,
                                       (long long)rows, dim, dx);
            st = hipGetLastError();
            if (st != hipSuccess || !sums) return st;
            hipLaunchKernelGGL((norm_columns_kernel<T, V, TAIL>), dim3((unsigned)(((dim + V - 1) / V + 255) / 256), (unsigned)groups), dim3(256), 0, s, x,
                               mean, rstd, dy, (long long)rows, dim, part);
        }
        return hipGetLastError();
    }));
    if (!sums) return LCN_OK;
    hipLaunchKernelGGL(norm_join_kernel<T>, dim3((unsigned)((2 * dim + 15) / 16)), dim3(256), 0, s, part, groups, dim, dw, db);
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
