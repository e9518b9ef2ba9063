// Softmax cross entropy of rows x against a vocabulary W, z = scale x W^T + b, without keeping z:
//   loss_n = lse_n - z_n,t(n),  lse_n = log sum_v exp z_nv;   G = g_n (exp(z_nv - lse_n) - [v = t(n)]),
//   dx = scale G W,  dW = scale G^T x,  db_v = sum_n G_nv.
//
// Forward: one product whose epilogue leaves the maximum and the sum of exponentials of its 256 (or fewer) words for
// every row; a second launch joins them.  Backward: for a piece of the vocabulary at a time the product is formed again,
// its epilogue writes G of the piece (planes of bf16) into the workspace, and two products read it from there, G by rows for
// dx and by columns for dW.  8 N V D operations, against 6 N V D with z kept at 4 bytes a value (N V values).
// Bound by the products, and with short rows by the epilogues behind them (an exponential per score, G's store).  bf16, 4099 rows,
// 50 021 words of 1024: forward 432 us (0.97 PFLOP/s), backward four pieces of 136 (G) + 118 (dx) + 110 (dW); 8192 rows,
// 200 000 words of 300: 1294 (0.76), 25 pieces of 82 + 53 + 47 + 9.  float, 5000 rows, 20 000 words of 300: 402 (149 TFLOP/s),
// five pieces of 111 + 78 + 74.
//
// Statistics, sums and z are in 32 bits; G is rounded to bf16 for bf16 tensors (its error is that of rounding the result
// once more) and kept as three planes for float ones.
#include "operators.h"

namespace lcn {

constexpr float LOG2E = 1.4426950408889634f;

// A score, and e^(z - m).  Forward and backward pass form scores by the same operations in the same order, and differences
// before they change the unit: a target with all the weight has z = m = lse, loss 0 and P = 1 to the last bit, where lse times
// log2(e) and back would leave 2^-24 of the score in either direction, a gradient without meaning.
__device__ __forceinline__ float score(float dot, float scale, float bias) { return __builtin_fmaf(dot, scale, bias); }
__device__ __forceinline__ float exp_of(float difference) { return exp2_fast(difference * LOG2E); }

struct EntropyRow {
    const float *bias;        // nullable
    const int64_t *target;
    float scale;
    int vocab;
};

// Joins (m, s) with another pair: the sum of exponentials relative to the larger maximum.  -inf: nothing yet.
__device__ __forceinline__ void join(float &m, float &s, float om, float os)
{
    const float top = fmaxf(m, om);
    const float a = m == top ? 1.f : exp_of(m - top), b = om == top ? 1.f : exp_of(om - top);
    s = s * a + os * b;
    m = top;
}

struct EntropyForward {
    struct Args {
        EntropyRow r;
        float2 *part;    // [tile][row]
        float *at_target;
    };
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0, int,
                               char *lds, int tm, int tn)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g4 = 4 * (lane >> 4);
        float2 *joined = (float2 *)lds;   // [WM][WN * TN * 16]
        f32x4 bias[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            bias[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (e.r.bias) bias[i] = load_four(e.r.bias + m0 + i * 16 + g4, (int)(p.m - (m0 + i * 16 + g4)));
        }
        const bool edge = m0 + TM * 16 > p.m;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const long long n = n0 + j * 16 + (lane & 15);
            const long long t = n < p.n ? e.r.target[n] - (m0 + g4) : -1;
            const bool mine = t >= 0 && t < TM * 16 && (t & 15) < 4 && t + m0 + g4 < p.m;
            float top = -__builtin_huge_valf();
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[i][j][u] = score(acc[i][j][u], e.r.scale, bias[i][u]);
            if (__any(mine)) {   // the target is among this lane's words
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (mine && t == i * 16 + u) e.at_target[n] = acc[i][j][u];
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                if (edge) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (m0 + i * 16 + g4 + u >= p.m) acc[i][j][u] = -__builtin_huge_valf();
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) top = fmaxf(top, acc[i][j][u]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            // a row without a finite score: its terms are exp(-inf) = 0, or not a number
            const float ref = top == -__builtin_huge_valf() ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u) sum += exp_of(acc[i][j][u] - ref);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (lane < 16) joined[(wave % WM) * (WN * TN * 16) + (wave / WM) * (TN * 16) + j * 16 + lane] = make_float2(top, sum);
        }
        __syncthreads();
        const int c = threadIdx.x;
        const long long n = (long long)tn * (WN * TN * 16) + c;
        if (c < WN * TN * 16 && n < p.n) {
            float2 v = joined[c];
#pragma unroll
            for (int w = 1; w < WM; ++w) {
                const float2 o = joined[w * (WN * TN * 16) + c];
                join(v.x, v.y, o.x, o.y);
            }
            e.part[(long long)tm * p.n + n] = v;
        }
    }
};

// One workgroup of `width` x `height` threads: a row per column of threads; joins the parts in a fixed order.
__global__ __launch_bounds__(256) void entropy_join_kernel(const float2 *__restrict__ part, int parts, long long rows,
                                                           EntropyRow r, const float *__restrict__ at_target,
                                                           float *__restrict__ loss, float *__restrict__ lse, int across)
{
    __shared__ float2 sums[256];
    const int c = threadIdx.x % across, q = threadIdx.x / across, down = 256 / across;
    const long long n = (long long)group_number() * across + c;
    float m = -__builtin_huge_valf(), s = 0.f;
    if (n < rows)
        for (int i = q; i < parts; i += down) {
            const float2 v = part[(long long)i * rows + n];
            join(m, s, v.x, v.y);
        }
    sums[threadIdx.x] = make_float2(m, s);
    for (int half = down / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (q < half) {
            const float2 o = sums[threadIdx.x + half * across];
            join(m, s, o.x, o.y);
            sums[threadIdx.x] = make_float2(m, s);
        }
    }
    if (q || n >= rows) return;
    const float rest = logf(s);
    const int64_t t = r.target[n];
    lse[n] = m + rest;
    // no target: no loss; a target outside the vocabulary: not a number; else without the rounding of lse
    loss[n] = t < 0 ? 0.f : t >= r.vocab ? __builtin_nanf("") : (m - at_target[n]) + rest;
}

// Few rows: bound by reading W once.  A workgroup goes over a share of the words and leaves one pair per row.  One row, 20 000 words
// of 300 in float: 5.9 us, 4.1 TB/s, and 3.2 for the join.  Eight rows, here / as a product: float 14 / 35 us, bf16 13 / 12.
template <class T, int R, bool VEC>
__global__ __launch_bounds__(256) void entropy_few_kernel(EntropyRow e, const T *__restrict__ x, const T *__restrict__ w,
                                                          int rows, int k, float2 *__restrict__ part,
                                                          float *__restrict__ at_target)
{
    __shared__ float2 joined[16][R];
    const int group = threadIdx.x >> 4;
    float m[R], s[R];
    long long t[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = -__builtin_huge_valf();
        s[r] = 0.f;
        t[r] = r < rows ? e.target[r] : -1;
    }
    for (long long f = ((long long)blockIdx.x * 16 + group) * 2; f < e.vocab; f += (long long)gridDim.x * 32) {
        const bool two = f + 1 < e.vocab;
        float sum[2][R];
#pragma unroll
        for (int r = 0; r < R; ++r) sum[0][r] = sum[1][r] = 0.f;
        few_rows_dot<T, R, VEC>(w + f * k, w + (two ? f + 1 : f) * k, x, rows, k, sum);
        const float b0 = e.bias ? e.bias[f] : 0.f, b1 = e.bias && two ? e.bias[f + 1] : 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float z0 = score(sum[0][r], e.scale, b0), z1 = two ? score(sum[1][r], e.scale, b1) : -__builtin_huge_valf();
            if ((threadIdx.x & 15) == 0 && r < rows) {
                if (t[r] == f) at_target[r] = z0;
                if (t[r] == f + 1 && two) at_target[r] = z1;
            }
            const float top = fmaxf(m[r], fmaxf(z0, z1)), ref = top == -__builtin_huge_valf() ? 0.f : top;
            s[r] = s[r] * exp_of(m[r] - ref) + exp_of(z0 - ref) + exp_of(z1 - ref);
            m[r] = top;
        }
    }
    if ((threadIdx.x & 15) == 0)
#pragma unroll
        for (int r = 0; r < R; ++r) joined[group][r] = make_float2(m[r], s[r]);
    __syncthreads();
    if ((int)threadIdx.x < rows) {
        float2 v = joined[0][threadIdx.x];
        for (int g = 1; g < 16; ++g) join(v.x, v.y, joined[g][threadIdx.x].x, joined[g][threadIdx.x].y);
        part[(long long)blockIdx.x * rows + threadIdx.x] = v;
    }
}

// G of a piece of the vocabulary, in planes; optionally the sums over this tile's rows.
template <int PLANES>
struct EntropyGradient {
    struct Args {
        EntropyRow r;        // bias: of this piece
        long long first;     // the piece's first word
        const float *lse, *grad;
        __bf16 *g;
        long long ldg, plane;   // elements
        float *sums;         // [tile of rows][word of the piece], nullable
        float *rest;         // [row]: what rounding takes from the target's G, nullable
    };
    template <int TM, int TN, int WM, int WN>
    static __device__ void run(const Args &e, const ProductArgs &p, f32x4 (&acc)[TM][TN], long long m0, long long n0, int,
                               char *lds, int tm, int tn)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g4 = 4 * (lane >> 4);
        constexpr int BM = WM * TM * 16;
        float *total = (float *)lds;   // [WN][BM]
        const long long wide = padded(p.m);   // G is read in pieces of eight words
        char *region = lds + wave * RowRegion<TM>::BYTES;
        const bool edge = m0 + TM * 16 > p.m;
        f32x4 bias[TM], sum[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const long long m = m0 + i * 16 + g4;
            bias[i] = sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (e.r.bias) bias[i] = load_four(e.r.bias + m, (int)(p.m - m));
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const long long n = n0 + j * 16 + (lane & 15);
            const bool in = n < p.n;
            const long long t = in ? e.r.target[n] : -1;
            const float lse = in ? e.lse[n] : 0.f;
            // a row without a target adds nothing, whatever it holds: min(x, NaN) is x, min(NaN, 0) is 0
            const bool none = t < 0;
            const float grad = none ? 0.f : t >= e.r.vocab ? __builtin_nanf("") : e.grad[n];   // >= vocab: no such word
            const float most = none ? 0.f : __builtin_nanf("");
            const long long here = none ? -1 : t - e.first - (m0 + g4);   // the target among this lane's words
            const int at = here >= 0 && here < TM * 16 ? (int)here : -1;
            f32x4 col[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                f32x4 v;
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = __builtin_fminf(exp_of(score(acc[i][j][u], e.r.scale, bias[i][u]) - lse), most);
                if (__any((unsigned)(at - i * 16) < 4u)) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (at == i * 16 + u) {
                            v[u] -= 1.f;
                            const float all = v[u] * grad;
                            if (PLANES == 1 && e.rest) e.rest[n] = all - (float)(__bf16)all;
                        }
                }
                v *= grad;
                if (edge) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (m0 + i * 16 + g4 + u >= p.m) v[u] = 0.f;
                }
                sum[i] += v;
                col[i] = v;
            }
            by_rows<TM>(
                region, col, lane, [](int, int) { return Nothing{}; },
                [&](int r, int c, f32x4 (&v)[2], Nothing) {
                    const long long row = n0 + j * 16 + r, m = m0 + c;
                    if (row >= p.n || m >= wide) return;
                    __bf16 *to = e.g + row * e.ldg + m;
                    bf16x8 o[3];
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const float x = v[u >> 2][u & 3];
                        __bf16 a = (__bf16)x, b = a, c3 = a;
                        if (PLANES == 2) b = (__bf16)(x - (float)a);
                        if (PLANES == 3) split_planes(x, a, b, c3);
                        o[0][u] = a;
                        o[1][u] = b;
                        o[2][u] = c3;
                    }
                    *(bf16x8 *)to = o[0];
                    if (PLANES > 1) *(bf16x8 *)(to + e.plane) = o[1];
                    if (PLANES > 2) *(bf16x8 *)(to + 2 * e.plane) = o[2];
                });
        }
        if (!e.sums) return;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) sum[i][u] += __shfl_xor(sum[i][u], o, 16);
                if ((lane & 15) == u) total[(wave / WM) * BM + (wave % WM) * (TM * 16) + i * 16 + g4 + u] = sum[i][u];
            }
        __syncthreads();
        const int c = threadIdx.x;
        const long long m = (long long)tm * BM + c;
        if (c < BM && m < p.m) {
            float v = total[c];
#pragma unroll
            for (int w = 1; w < WN; ++w) v += total[w * BM + c];
            e.sums[(long long)tn * p.m + m] = v;
        }
    }
};

// G of few rows, with the sums of entropy_few_kernel (a product's order of additions would give other scores than lse was
// formed of).  A wavefront has eight words at a time, lane 2 r + which of 16 finishes row r of one of its group's two.  Words up
// to `wide` are written, zeros behind the last.  Bound by reading W once; with both products behind it one row / eight rows, 20 000
// words of 300: float 58 / 63 us, bf16 58 / 64 (by a product of tiles 64 / 66, 57 / 59).
template <class T, int R, bool VEC>
__global__ __launch_bounds__(256) void entropy_few_gradient_kernel(EntropyRow e, long long first, int words, int wide,
                                                                   const T *__restrict__ x, const T *__restrict__ w, int rows,
                                                                   int k, const float *__restrict__ lse,
                                                                   const float *__restrict__ grad, __bf16 *__restrict__ g,
                                                                   long long plane, float *__restrict__ dbias)
{
    const int lane = threadIdx.x & 15, r = lane >> 1, which = lane & 1;
    const bool in = r < rows;
    const long long t = in ? e.target[r] : -1;
    // as in EntropyGradient: a row without a target adds nothing, a target behind the vocabulary is not a number
    const bool none = t < 0;
    const float own = none ? 0.f : t >= e.vocab ? __builtin_nanf("") : grad[r], most = none ? 0.f : __builtin_nanf("");
    const float sum_of_row = in ? lse[r] : 0.f;
    for (long long f = ((long long)blockIdx.x * 16 + (threadIdx.x >> 4)) * 2; f < wide; f += (long long)gridDim.x * 32) {
        const long long f0 = f < words ? f : words - 1, f1 = f + 1 < words ? f + 1 : words - 1;
        float sum[2][R];
#pragma unroll
        for (int u = 0; u < R; ++u) sum[0][u] = sum[1][u] = 0.f;
        few_rows_dot<T, R, VEC>(w + f0 * k, w + f1 * k, x, rows, k, sum);
        float dot = 0.f;
#pragma unroll
        for (int u = 0; u < R; ++u)
            if (u == r) dot = which ? sum[1][u] : sum[0][u];
        float v = 0.f;
        if (in && f + which < words) {
            v = __builtin_fminf(exp_of(score(dot, e.scale, e.bias ? e.bias[f + which] : 0.f) - sum_of_row), most);
            if (!none && t - first == f + which) v -= 1.f;
            v *= own;
        }
        float total = 0.f;
#pragma unroll
        for (int u = 0; u < R; ++u) total += __shfl(v, 2 * u + which, 16);
        if (dbias && r == 0 && f + which < words) dbias[f + which] = total;
        if (in) {
            __bf16 a, b, c;
            split_planes(v, a, b, c);
            __bf16 *to = g + r * (long long)wide + f + which;
            to[0] = a;
            to[plane] = b;
            if (sizeof(T) == 4) to[2 * plane] = c;
        }
    }
}

// dx = scale (the sums of G W + what rounding took from the target's G times its word).  The target's G is most of a row's: its
// rounding to bf16 would be as large in dx as that of dx itself, and the same for all of the row.
__global__ __launch_bounds__(256) void entropy_finish_kernel(const float *__restrict__ part, int splits, long long stride,
                                                             long long rows, int dim, long long ldp, float scale,
                                                             const float *__restrict__ rest, const int64_t *__restrict__ target,
                                                             const __bf16 *__restrict__ w, int vocab, __bf16 *__restrict__ out)
{
    const int per_row = (dim + 7) / 8;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < rows * per_row; t += (long long)gridDim.x * 256) {
        const long long n = t / per_row;
        const int c = (int)(t - n * per_row) * 8;
        f32x4 v[2], o[2];
        load_eight(part + n * ldp + c, 8, v);
        for (int s = 1; s < splits; ++s) {
            load_eight(part + s * stride + n * ldp + c, 8, o);
            v[0] += o[0];
            v[1] += o[1];
        }
        const int64_t at = target[n];
        if (at >= 0 && at < vocab) {
            load_eight(w + at * dim + c, dim - c, o);
            v[0] += o[0] * rest[n];
            v[1] += o[1] * rest[n];
        }
        v[0] *= scale;
        v[1] *= scale;
        store_eight(out + n * dim + c, v, dim - c);
    }
}

// ---- host ---------------------------------------------------------------------

constexpr int FEW_GROUPS = 1024;
// G of a piece of the vocabulary takes at most this much of the workspace: what is written stays in the last-level cache until
// both products have read it (8192 rows against 200 000 words: 6.11 ms; with 64 MiB 7.23, with 256 MiB 6.46, with 512 MiB 6.23)
constexpr size_t PIECE_BYTES = (size_t)128 << 20;

static bool entropy_args_fit(int64_t rows, int32_t vocab, int32_t dim, int32_t dtype)
{
    return rows >= 0 && rows <= MAX_ROWS && vocab >= 1 && vocab <= (int32_t)MAX_ROWS && dim >= 1 && dim <= MAX_WIDTH &&
           sizes_fit(rows, vocab) && sizes_fit(rows, dim) && sizes_fit(vocab, dim) && (dtype == LCN_F32 || dtype == LCN_BF16);
}
static int few_groups(int32_t vocab)
{
    const int g = (vocab + 31) / 32;
    return g < FEW_GROUPS ? g : FEW_GROUPS;
}

static int64_t row_tiles(const ProductPlan &plan, int64_t rows, int32_t dtype)
{
    const int bn = tile_n(plan.tile, planes_of(dtype));
    return (rows + bn - 1) / bn;
}

struct EntropySpace {
    ProductPlan plan;         // of the scores
    void *xp, *wp;
    float2 *part;
    float *at_target;
    size_t bytes;
};
static EntropySpace entropy_space(char *ws, int64_t rows, int32_t vocab, int32_t dim, int32_t dtype)
{
    Carver c{ws};
    EntropySpace f{};
    f.at_target = (float *)c.take((size_t)rows * 4);
    if (rows <= FEW_ROWS) {
        f.part = (float2 *)c.take((size_t)few_groups(vocab) * rows * 8);
    } else {
        f.plan = plan_product(vocab, rows, dim, planes_of(dtype), false, false);
        f.part = (float2 *)c.take((size_t)((vocab + tile_m(f.plan.tile) - 1) / tile_m(f.plan.tile)) * rows * 8);
        f.xp = c.take(planes_bytes(rows, dim, planes_of(dtype)));
        f.wp = c.take(planes_bytes(vocab, dim, planes_of(dtype)));
    }
    f.bytes = c.used;
    return f;
}

struct EntropyBackward {
    ProductPlan scores, dx, dw;   // for a piece
    int32_t piece;                // words
    int planes;                   // of G
    void *xp, *xz, *wp, *g;       // xz: x with zeros in the rows without a target
    float *part_dx, *part_dw, *sums, *rest;
    size_t bytes;
};
static EntropyBackward entropy_backward_space(char *ws, int64_t rows, int32_t vocab, int32_t dim, int32_t dtype)
{
    Carver c{ws};
    EntropyBackward b{};
    const int planes = b.planes = gradient_planes(rows, dtype);
    int64_t most = (int64_t)(PIECE_BYTES / ((size_t)rows * 2 * planes)) & ~(int64_t)255;
    if (most < 256) most = 256;
    const int64_t pieces = (vocab + most - 1) / most;
    int64_t piece = ((vocab + pieces - 1) / pieces + 255) & ~(int64_t)255;   // pieces of about one size
    if (piece > vocab) piece = vocab;
    b.piece = (int32_t)piece;
    b.scores = plan_product(piece, rows, dim, planes_of(dtype), false, false);
    b.dx = plan_product(dim, rows, piece, planes, true, true);
    b.dw = plan_product(dim, piece, rows, planes, true, true);
    b.xp = c.take(planes_bytes(rows, dim, planes_of(dtype)));
    b.xz = c.take(planes_bytes(rows, dim, planes_of(dtype)));
    b.wp = c.take(planes_bytes(vocab, dim, planes_of(dtype)));
    b.g = c.take(planes_bytes(rows, piece, b.planes));
    b.part_dx = (float *)c.take((size_t)b.dx.splits * rows * padded(dim) * 4);
    b.part_dw = (float *)c.take(partial_bytes(b.dw, dim, piece));
    b.sums = (float *)c.take((size_t)(row_tiles(b.scores, rows, dtype)) * piece * 4);
    b.rest = (float *)c.take(b.planes == 1 ? (size_t)rows * 4 : 0);
    b.bytes = c.used;
    return b;
}

template <class T, int R>
static hipError_t launch_few(const EntropyRow &e, const T *x, const T *w, int rows, int k, float2 *part, float *at_target,
                             hipStream_t s)
{
    const unsigned grid = (unsigned)few_groups(e.vocab);
    if (k % (16 / (int)sizeof(T)) == 0 && (((uintptr_t)x | (uintptr_t)w) & 15) == 0)
        hipLaunchKernelGGL((entropy_few_kernel<T, R, true>), dim3(grid), dim3(256), 0, s, e, x, w, rows, k, part, at_target);
    else
        hipLaunchKernelGGL((entropy_few_kernel<T, R, false>), dim3(grid), dim3(256), 0, s, e, x, w, rows, k, part, at_target);
    return hipGetLastError();
}

template <class T, int R>
static hipError_t launch_few_gradient(const EntropyRow &e, long long first, int words, const T *x, const T *w, int rows, int k,
                                      const float *lse, const float *grad, void *g, float *dbias, hipStream_t s)
{
    const int wide = (int)padded(words);
    const unsigned grid = (unsigned)few_groups(wide);
    if (k % (16 / (int)sizeof(T)) == 0 && (((uintptr_t)x | (uintptr_t)w) & 15) == 0)   // as launch_few
        hipLaunchKernelGGL((entropy_few_gradient_kernel<T, R, true>), dim3(grid), dim3(256), 0, s, e, first, words, wide, x, w, rows, k,
                           lse, grad, (__bf16 *)g, (long long)rows * wide, dbias);
    else
        hipLaunchKernelGGL((entropy_few_gradient_kernel<T, R, false>), dim3(grid), dim3(256), 0, s, e, first, words, wide, x, w, rows,
                           k, lse, grad, (__bf16 *)g, (long long)rows * wide, dbias);
    return hipGetLastError();
}
template <class T>
static hipError_t few_gradient(const EntropyRow &e, long long first, int words, const void *x, const void *w, int64_t rows, int k,
                               const float *lse, const float *grad, void *g, float *dbias, hipStream_t s)
{
    const T *xt = (const T *)x, *wt = (const T *)w + first * k;
    const int r = (int)rows;
    return r == 1   ? launch_few_gradient<T, 1>(e, first, words, xt, wt, r, k, lse, grad, g, dbias, s)
           : r == 2 ? launch_few_gradient<T, 2>(e, first, words, xt, wt, r, k, lse, grad, g, dbias, s)
           : r <= 4 ? launch_few_gradient<T, 4>(e, first, words, xt, wt, r, k, lse, grad, g, dbias, s)
                    : launch_few_gradient<T, 8>(e, first, words, xt, wt, r, k, lse, grad, g, dbias, s);
}

template <class T>
static lcn_status entropy_as(const T *x, const T *w, const float *bias, const int64_t *target, int64_t rows, int32_t vocab,
                             int32_t dim, int32_t dtype, float scale, float *loss, float *lse, char *ws, size_t ws_bytes,
                             hipStream_t s)
{
    const EntropySpace f = entropy_space(ws, rows, vocab, dim, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < f.bytes) return LCN_ERR_ALLOC;
    const EntropyRow e{bias, target, scale, vocab};
    int parts, across;
    if (rows <= FEW_ROWS) {
        const int r = (int)rows;
        hipError_t st = r == 1   ? launch_few<T, 1>(e, x, w, r, dim, f.part, f.at_target, s)
                        : r == 2 ? launch_few<T, 2>(e, x, w, r, dim, f.part, f.at_target, s)
                        : r <= 4 ? launch_few<T, 4>(e, x, w, r, dim, f.part, f.at_target, s)
                                 : launch_few<T, 8>(e, x, w, r, dim, f.part, f.at_target, s);
        OPCHK(st);
        parts = few_groups(vocab);
        across = 1;
    } else {
        ProductArgs p{};
        PlaneJobs jobs;
        p.a = add_operand(jobs, w, vocab, dim, dtype, f.wp);
        p.b = add_operand(jobs, x, rows, dim, dtype, f.xp);
        OPCHK(launch_planes(jobs, dtype, s));
        p.m = vocab;
        p.n = (int)rows;
        p.k = dim;
        p.planes = planes_of(dtype);
        OPCHK((launch_planned<sizeof(T) == 4 ? 3 : 1, false, false, EntropyForward>(f.plan, p, {e, f.part, f.at_target}, s)));
        parts = (vocab + tile_m(f.plan.tile) - 1) / tile_m(f.plan.tile);
        across = 16;
    }
    hipLaunchKernelGGL(entropy_join_kernel, grid_of((rows + across - 1) / across), dim3(256), 0, s, f.part, parts,
                       (long long)rows, e, f.at_target, loss, lse, across);
    OPCHK(hipGetLastError());
    return LCN_OK;
}

template <int PLANES>
static hipError_t launch_gradient(const ProductPlan &plan, const ProductArgs &p, const EntropyRow &r, long long first,
                                  const float *lse, const float *grad, void *g, long long ldg, float *sums, float *rest, hipStream_t s)
{
    return launch_planned<PLANES == 3 ? 3 : 1, false, false, EntropyGradient<PLANES>>(plan, p,
                                                                 {r, first, lse, grad, (__bf16 *)g, ldg, p.n * ldg, sums, rest}, s);
}

static lcn_status entropy_backward_as(const void *x, const void *w, const float *bias, const int64_t *target, const float *lse,
                                      const float *grad, int64_t rows, int32_t vocab, int32_t dim, int32_t dtype, float scale,
                                      void *dx, void *dw, float *dbias, char *ws, size_t ws_bytes, hipStream_t s)
{
    const EntropyBackward b = entropy_backward_space(ws, rows, vocab, dim, dtype);
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < b.bytes) return LCN_ERR_ALLOC;
    const size_t size = dtype == LCN_F32 ? 4 : 2;
    PlaneJobs jobs;
    const bool few = rows <= FEW_ROWS;
    Operand wo{}, xo{}, xz{};
    if (dx || !few) wo = add_operand(jobs, w, vocab, dim, dtype, b.wp);
    if (!few) xo = add_operand(jobs, x, rows, dim, dtype, b.xp);
    if (dw) xz = add_masked(jobs, x, rows, dim, dtype, target, b.xz);
    OPCHK(launch_planes(jobs, dtype, s));
    const bool rounded = dx && b.planes == 1, one = b.piece >= vocab && !rounded;
    float *rest = rounded ? b.rest : nullptr;
    if (rounded) OPCHK(launch_zero(rest, (size_t)rows * 4, s));
    for (int64_t first = 0; first < vocab; first += b.piece) {
        const int words = (int)(vocab - first < b.piece ? vocab - first : b.piece);
        const Operand here{(const char *)wo.p + first * wo.ld * 2, wo.plane, wo.ld};
        const Operand g = plane_operand(b.g, rows, words);
        const EntropyRow r{bias ? bias + first : nullptr, target, scale, vocab};
        ProductArgs p{};
        p.planes = planes_of(dtype);
        p.a = here;
        p.b = xo;
        p.m = words;
        p.n = (int)rows;
        p.k = dim;
        float *sums = dbias ? b.sums : nullptr;
        if (few)
            OPCHK(dtype == LCN_F32
                      ? few_gradient<float>(r, first, words, x, w, rows, dim, lse, grad, b.g, dbias ? dbias + first : nullptr, s)
                      : few_gradient<__bf16>(r, first, words, x, w, rows, dim, lse, grad, b.g, dbias ? dbias + first : nullptr, s));
        else
            OPCHK(b.planes == 3   ? launch_gradient<3>(b.scores, p, r, first, lse, grad, b.g, g.ld, sums, rest, s)
                  : b.planes == 2 ? launch_gradient<2>(b.scores, p, r, first, lse, grad, b.g, g.ld, sums, rest, s)
                                  : launch_gradient<1>(b.scores, p, r, first, lse, grad, b.g, g.ld, sums, rest, s));
        if (dbias && !few) {
            const int parts = (int)(row_tiles(b.scores, rows, dtype));
            OPCHK(launch_column_sums(sums, parts, words, LCN_F32, dbias + first, s));
        }
        p.m = dim;
        p.planes = b.planes;
        if (dx) {   // G by rows x W by columns
            p.a = here;
            p.b = g;
            p.n = (int)rows;
            p.k = words;
            if (one)
                OPCHK((launch_scaled<true, false>(b.dx, p, scale, dtype, dx, b.part_dx, s)));
            else
                OPCHK(launch_partials(b.dx, p, b.part_dx, first > 0, s));
        }
        if (dw) {   // G by columns x x by columns
            p.a = xz;
            p.b = g;
            p.n = words;
            p.k = (int)rows;
            OPCHK((launch_scaled<true, true>(b.dw, p, scale, dtype, (char *)dw + (size_t)first * dim * size, b.part_dw, s)));
        }
    }
    if (rounded) {
        const long long groups = (rows * ((dim + 7) / 8) + 255) / 256, ldp = padded(dim);
        hipLaunchKernelGGL(entropy_finish_kernel, dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0, s, b.part_dx,
                           b.dx.splits, rows * ldp, (long long)rows, dim, ldp, scale, rest, target, (const __bf16 *)w, vocab,
                           (__bf16 *)dx);
        OPCHK(hipGetLastError());
    } else if (dx && !one)
        OPCHK(launch_add_partials(b.part_dx, b.dx.splits, rows, dim, padded(dim), scale, dtype, dx, s));
    return LCN_OK;
}

}  // namespace lcn

using namespace lcn;

extern "C" {

lcn_status lcn_cross_entropy_workspace_bytes(int64_t rows, int32_t vocab, int32_t dim, int32_t dtype, int32_t backward,
                                             size_t *bytes)
{
    if (!bytes || !entropy_args_fit(rows, vocab, dim, dtype)) return LCN_ERR_INVALID_ARG;
    *bytes = 0;
    if (rows == 0) return LCN_OK;
    *bytes = backward ? entropy_backward_space(nullptr, rows, vocab, dim, dtype).bytes
                      : entropy_space(nullptr, rows, vocab, dim, dtype).bytes;
    return LCN_OK;
}

lcn_status lcn_cross_entropy(const void *x, const void *W, const float *bias, const int64_t *target, int64_t rows,
                             int32_t vocab, int32_t dim, int32_t dtype, float scale, float *loss, float *lse, void *workspace,
                             size_t workspace_bytes, void *hip_stream)
{
    if (!entropy_args_fit(rows, vocab, dim, dtype) || !(scale - scale == 0.f)) return LCN_ERR_INVALID_ARG;
    if (rows == 0) return LCN_OK;
    if (!x || !W || !target || !loss || !lse) return LCN_ERR_INVALID_ARG;
    if (dtype == LCN_F32)
        return entropy_as((const float *)x, (const float *)W, bias, target, rows, vocab, dim, dtype, scale, loss, lse,
                          (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
    return entropy_as((const __bf16 *)x, (const __bf16 *)W, bias, target, rows, vocab, dim, dtype, scale, loss, lse,
                      (char *)workspace, workspace_bytes, (hipStream_t)hip_stream);
}

lcn_status lcn_cross_entropy_backward(const void *x, const void *W, const float *bias, const int64_t *target, const float *lse,
                                      const float *grad_loss, int64_t rows, int32_t vocab, int32_t dim, int32_t dtype,
                                      float scale, void *dx, void *dW, float *dbias, void *workspace, size_t workspace_bytes,
                                      void *hip_stream)
{
    if (!entropy_args_fit(rows, vocab, dim, dtype) || !(scale - scale == 0.f)) return LCN_ERR_INVALID_ARG;
    if (!dx && !dW && !dbias) return LCN_OK;
    hipStream_t s = (hipStream_t)hip_stream;
    if (rows == 0) {   // no rows: the parameters' gradients are zero
        if (dW) OPCHK(launch_zero(dW, (size_t)vocab * dim * (dtype == LCN_F32 ? 4 : 2), s));
        if (dbias) OPCHK(launch_zero(dbias, (size_t)vocab * 4, s));
        return LCN_OK;
    }
    if (!x || !W || !target || !lse || !grad_loss) return LCN_ERR_INVALID_ARG;
    return entropy_backward_as(x, W, bias, target, lse, grad_loss, rows, vocab, dim, dtype, scale, dx, dW, dbias,
                               (char *)workspace, workspace_bytes, s);
}

}  // extern "C"
