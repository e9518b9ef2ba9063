// Attention inside the sets of a ragged batch: forward, and the gradients of q, k and v.
//
// For query i and key j of a set (nq queries, nk keys; a query's position is i + nk - nq, so the last query stands at the
// last key):  z = scale q_i . k_j;  with a cap c: z = c tanh(z / c);  with a slope of the head: z -= slope |position - j|;
// causal: only j <= position, or j < prefix.  o_i = sum_j softmax(z)_ij v_j,  lse_i = log sum_j exp z_ij.
//
// Layout: the matrix instruction's accumulator has its column in lane % 16 and rows 4 (lane / 16) + 0 .. 3.  Scores are formed
// with keys as rows (forward, dq) or queries as rows (dk, dv), so that two accumulators, converted, ARE the right-hand
// operand of the next product: the 32 values of its k are keys 4 g + 0 .. 3 and 16 + 4 g + 0 .. 3 in lane group g, and the
// left-hand operand is read from LDS in the same order, transposed by the reads.  Scores never pass through LDS, and a
// query's maximum and sum are in its own lanes.
//
// bf16 tensors use the 16x16x32 bf16 instruction, float ones eight 16x16x4 float instructions on the same registers.
// Scores, statistics, sums and dS are in 32 bits; P and dS are rounded to the tensors' type where they enter a product.
#pragma once

#include "fragments.h"

namespace lcn {

struct AttentionArgs {
    const void *q, *k, *v;
    const int64_t *q_off, *k_off;
    const int32_t *prefix;      // nullable
    const float *slopes;        // nullable
    long long q_token, q_head, k_token, k_head, v_token, v_head;   // strides in elements
    long long total_q, total_k;
    int sets, heads, kv_heads, dim;
    int causal;
    float scale, cap;
    int tiles;                  // of queries (forward, dq) or keys (dk, dv), over all sets
    unsigned groups;            // workgroups with work, see group_number(); where `clear` is set CLEARERS more follow
    int clear;                  // tokens in no set: 0: not written, 1: zeros
    // forward
    void *o;                    // read in the backward pass
    float *lse;                 // [head][query]
    // keys split over workgroups: chunks of `chunk` keys, `rows` = max_q * (heads / kv_heads)
    int chunk, rows;            // part: [chunk][key head][row][dim], part_top: [chunk][key head][row]
    // backward
    const void *d_o;
    const float *lse_in;
    float *delta;               // [head][query]
    void *dq, *dk, *dv;         // dq: nullable, delta alone is formed then
    // sums shared by several workgroups, where there are few tiles, and joined by a second launch
    int key_splits;             // of a query tile's keys (forward, dq)
    int splits;                 // of a key tile's queries (dk, dv)
    float *part;                // forward, dq: [split][query][head][dim]; dk, dv: [split][dk, dv][key][key head][dim]
    float2 *part_top;           // forward: [split][query][head], maximum (times log2(e)) and sum
};

// The last set p of `sets` with below(p), which holds for the first ones; 0 where it holds for none.  All lanes search.
template <class Below>
__device__ __forceinline__ int last_set(int sets, Below is_below)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = sets;
    while (n > 1) {
        const int step = (n + 63) >> 6, p = lo + lane * step;
        const bool below = p < lo + n && is_below(p);
        const int count = __popcll(__ballot(below));
        const int end = lo + n;
        lo += (count > 0 ? count - 1 : 0) * step;
        n = end - lo < step ? end - lo : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
// The set that a tile of B tokens belongs to: set p's tiles are numbered from off[p] / B + p on.
__device__ __forceinline__ int set_of_tile(const int64_t *off, int sets, int B, long long tile)
{
    return last_set(sets, [&](int p) { return off[p] / B + p <= tile; });
}

struct SetRange {
    long long q0, k0;
    int nq, nk;
};
// A set's tokens; offsets that are not in order or outside the tensors are cut to what exists.
__device__ __forceinline__ SetRange range_of(const AttentionArgs &a, int p)
{
    auto cut = [](long long v, long long lo, long long hi) { return v < lo ? lo : v > hi ? hi : v; };
    SetRange r;
    r.q0 = cut(a.q_off[p], 0, a.total_q);
    r.k0 = cut(a.k_off[p], 0, a.total_k);
    r.nq = (int)(cut(a.q_off[p + 1], r.q0, a.total_q) - r.q0);
    r.nk = (int)(cut(a.k_off[p + 1], r.k0, a.total_k) - r.k0);
    return r;
}

constexpr float LOG2_E = 1.4426950408889634f, LN_2 = 0.6931471805599453f;

// log(2^m s), m times a log(2) in two parts
__device__ __forceinline__ float natural_log(float m, float s)
{
    if (m == -__builtin_huge_valf()) return s == s ? m : s;   // no key; or scores that are not numbers
    return __builtin_fmaf(m, LN_2, __builtin_fmaf(m, -1.9046542e-9f, logf(s)));
}

// How q . k becomes a score.  PLAIN: a positive multiple.  CAPPED (bf16 tensors, scale > 0, cap up to MOST_CAP, no slopes):
// cap tanh(scale q.k / cap) = cap - 2 cap r with r = 1 / (e^(2 scale q.k / cap) + 1), off by about 2^-23 of the cap, far
// below the rounding of P; a score is between -cap and cap, so the exponentials need no running maximum: with 0 as their
// reference P' is between 2^-58 and 2^58, and its products with small v and its sums over 2^30 keys keep their bits (with the cap
// as reference it was down to 2^-116).  The cap's derivative is 4 r (1 - r).  SHAPED: anything, by tanhf.
enum Shape { PLAIN = 0, CAPPED = 1, SHAPED = 2 };
constexpr float MOST_CAP = 40.f;

// Four scores at a time, times log2(e); PLAIN: not yet scaled, `unit` scales them.
template <class T, int SHAPE>
struct Scores {
    float unit, natural, scale, cap, inv_cap, slope;
    __device__ __forceinline__ void init(const AttentionArgs &a, int head)
    {
        unit = SHAPE == PLAIN ? a.scale * LOG2_E : 1.f;
        natural = a.scale;
        scale = a.scale * LOG2_E;
        cap = a.cap * LOG2_E;
        inv_cap = SHAPE == CAPPED ? 2.f * LOG2_E * a.scale / a.cap : SHAPE == SHAPED && a.cap > 0.f ? a.scale / a.cap : 0.f;
        slope = SHAPE == SHAPED && a.slopes ? a.slopes[head] * LOG2_E : 0.f;
    }
    // CAPPED: r of q . k; the score is cap - 2 cap r
    __device__ __forceinline__ float under(float dot) const { return __builtin_amdgcn_rcpf(exp2_fast(dot * inv_cap) + 1.f); }
    // z: q . k of a query and four keys (STEP = -1) or a key and four queries (STEP = 1), `ahead`: how far the first query
    // is ahead of the first key; cut: the cap's derivative, where not nullptr
    template <int STEP>
    __device__ __forceinline__ void shape(f32x4 &z, int ahead, f32x4 *cut) const
    {
        if constexpr (SHAPE == SHAPED) {
            if (cap > 0.f) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float t = tanhf(z[e] * inv_cap);
                    z[e] = cap * t;
                    if (cut) (*cut)[e] = 1.f - t * t;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] *= scale;
                if (cut) *cut = f32x4{1.f, 1.f, 1.f, 1.f};
            }
            const float far = (float)ahead;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] -= slope * __builtin_fabsf(far + (float)(STEP * e));
        }
    }
    // P of four q . k for a query (key) with lse (by lse_in()), and the factor of the cap in dS (CAPPED: without its 4)
    template <int STEP>
    __device__ __forceinline__ void weigh(f32x4 &z, int ahead, f32x4 lse, f32x4 &cut) const
    {
        if constexpr (SHAPE == CAPPED) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float r = under(z[e]);
                z[e] = exp2_fast(__builtin_fmaf(r, -2.f * cap, cap - lse[e]));
                cut[e] = __builtin_fmaf(-r, r, r);
            }
        } else {
            shape<STEP>(z, ahead, &cut);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = weight(z[e], lse[e]);
        }
    }
    // e^(score - lse), lse in the units of lse_in(): float tensors take the difference before they change its unit, so that
    // it is rounded at its own size and not at that of lse times log2(e)
    static __device__ __forceinline__ float lse_in(float lse) { return sizeof(T) == 4 ? lse : lse * LOG2_E; }
    __device__ __forceinline__ float weight(float z, float lse) const
    {
        if constexpr (sizeof(T) == 4)
            return exp2_fast((SHAPE == PLAIN ? __builtin_fmaf(z, natural, -lse) : __builtin_fmaf(z, LN_2, -lse)) * LOG2_E);
        else
            return exp2_fast(z * unit - lse);
    }
    // what dS is still to be multiplied with
    __device__ __forceinline__ float rest(const AttentionArgs &a) const { return SHAPE == CAPPED ? 4.f * a.scale : a.scale; }
};

template <int N>
struct Buffer {
    static constexpr int value = N;
};

__device__ __forceinline__ float minus_infinity() { return -__builtin_huge_valf(); }

// The accumulators are in general registers from here on.  Without, the compiler (AMD clang 22, ROCm 7.2) has left out the wait between the
// last matrix instruction and a read of its result behind a branch (attention_chunk_kernel: a wait of 1 to 6 cycles
// where 8 are due, wrong scores); in one stretch of code it puts it in.
template <int N>
__device__ __forceinline__ void settle(f32x4 (&z)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(z[i]));
}
template <int N, int M>
__device__ __forceinline__ void settle(f32x4 (&z)[N][M])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < M; ++j) asm volatile("" : "+v"(z[i][j]));
}

// The same behind a loop whose last instructions are matrix instructions.
__device__ __forceinline__ void settle_loop()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15");
    __builtin_amdgcn_sched_barrier(0);
}

// Workgroups are dealt to the eight dies in turn; a die gets a run of neighbours, which share keys or queries.
__device__ __forceinline__ long long die_run(long long id, long long total)
{
    const long long base = total / 8, more = total % 8, die = id % 8, nth = id / 8;
    return die * base + (die < more ? die : more) + nth;
}

// What a workgroup of the forward and dq kernels works on: a tile of BQ queries of a set, for one head.
struct QueryTile {
    SetRange s;
    int head, kv, first, shift, prefix, last;   // last: behind the last key that any query of the tile sees
    int split;
    bool any;
    // this workgroup's steps of BK keys
    template <int BK>
    __device__ __forceinline__ int step(const AttentionArgs &a, int which) const
    {
        return (int)((long long)((last + BK - 1) / BK) * which / a.key_splits);
    }
};
template <int BQ>
__device__ __forceinline__ QueryTile query_tile(const AttentionArgs &a)
{
    QueryTile w;
    const int group = a.heads / a.kv_heads;
    // Heads are numbered fastest: workgroups are dealt to the eight dies in turn, so a die has the same heads of all tiles, and
    // their keys in its cache, and long and short tiles alike.
    const unsigned id = group_number();
    w.any = false;
    if (id >= a.groups) return w;
    w.head = (int)(id % a.heads);
    w.kv = w.head / group;
    w.split = (int)(id / a.heads % a.key_splits);
    const long long tile = a.tiles - 1 - (long long)(id / a.heads / a.key_splits);   // causal: the long ones first
    const int p = set_of_tile(a.q_off, a.sets, BQ, tile);
    w.s = range_of(a, p);
    const long long b0 = (tile - (w.s.q0 / BQ + p)) * BQ;
    w.any = b0 >= 0 && b0 < w.s.nq;
    w.first = (int)b0;
    w.shift = w.s.nk - w.s.nq;
    w.prefix = a.causal && a.prefix ? a.prefix[p] : 0;
    w.last = w.s.nk;
    if (a.causal) {
        const int reach = (w.first + BQ < w.s.nq ? w.first + BQ : w.s.nq) + w.shift;
        w.last = reach > w.prefix ? reach : w.prefix;
        w.last = w.last < w.s.nk ? w.last : w.s.nk;
    }
    return w;
}

// Steps begin .. end - 1 with two buffers in turn: step t + 1 is on its way while t is worked on.  fetch(t, which),
// landed(t, which): what is left to do when step t's loads have arrived (before all wavefronts meet), work(t, which).
template <class Fetch, class Landed, class Work>
__device__ __forceinline__ void two_buffers(int begin, int end, Fetch fetch, Landed landed, Work work)
{
    auto arrived = [&](int t, auto which) {
        __builtin_amdgcn_s_waitcnt(0x0f70);
        landed(t, which);
        __syncthreads();
    };
    if (begin >= end) return;
    fetch(begin, Buffer<0>());
    int t = begin;
    for (; t + 2 <= end; t += 2) {
        arrived(t, Buffer<0>());
        fetch(t + 1, Buffer<1>());
        work(t, Buffer<0>());
        arrived(t + 1, Buffer<1>());
        if (t + 2 < end) fetch(t + 2, Buffer<0>());
        work(t + 1, Buffer<1>());
    }
    if (t < end) {
        arrived(t, Buffer<0>());
        work(t, Buffer<0>());
    }
}

// What stands in for tokens before the first and behind the last set: zeros in rows of `width` values, -inf in lse.  The workgroups
// behind those with work share it; where every token is in a set there is nothing to do.  These lines cost the kernels of the small
// float sets 4 us of 173 altogether, a launch of their own as much, and 5 to 10 in longer calls.
constexpr unsigned CLEARERS = 64;
template <class T, bool VEC>
__device__ __forceinline__ void clear_others(const AttentionArgs &a, const int64_t *off, long long tokens, long long width, T *out0,
                                             T *out1, float *lse)
{
    const unsigned nth = group_number() - a.groups;   // wraps around for those with work
    if (!a.clear || !out0 || nth >= CLEARERS) return;
    const long long first = off[0], last = off[a.sets];
    const long long begin = first < 0 ? 0 : first < tokens ? first : tokens, end = last < begin ? begin : last < tokens ? last : tokens;
    const long long others = begin + tokens - end;
    constexpr int EACH = VEC ? 16 / (int)sizeof(T) : 1;
    typedef T piece __attribute__((ext_vector_type(EACH)));
    const long long step = CLEARERS * blockDim.x, mine = (long long)nth * blockDim.x + threadIdx.x, per_row = width / EACH;
    for (long long t = mine; t < others * per_row; t += step) {
        const long long at = (t < begin * per_row ? t : t + (end - begin) * per_row) * EACH;
        *(piece *)(out0 + at) = piece{};
        if (out1) *(piece *)(out1 + at) = piece{};
    }
    if (lse)
        for (long long t = mine; t < others * a.heads; t += step) {
            const long long n = t % others;
            lse[t / others * tokens + (n < begin ? n : n + end - begin)] = minus_infinity();
        }
}

// ---- forward -------------------------------------------------------------------
// Four wavefronts of 16 QT queries each go over the set's keys, 64 at a time.  Bound by the vector instructions beside the
// matrix ones: an exponential, a maximum and two conversions per score.  bf16, two sets of 8192, 16 heads of 64: 803 us,
// 0.68 PFLOP/s; packed documents of 500 to 5000 tokens, causal, capped, 16 heads of 128 on 4: 320 us, 0.56.  Float, 1024 sets of 16 to
// 64 tokens, 4 heads of 32, slopes: 48 us.  With few tiles the keys are dealt to a.key_splits workgroups.
template <class T, int DP, int QT, bool VEC, int SHAPE>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attention_forward_kernel(AttentionArgs a)
{
    constexpr int BQ = 64 * QT, BK = 64, C = DP / 32, DT = DP / 16;
    typedef Tile<T, DP> L;
    __shared__ __align__(1024) char lds0[2 * BK * L::PITCH];
    __shared__ __align__(1024) char lds1[2 * BK * L::PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
    const QueryTile w = query_tile<BQ>(a);
    if (!w.any) return clear_others<T, VEC>(a, a.q_off, a.total_q, (long long)a.heads * a.dim, (T *)a.o, nullptr, a.lse);
    const SetRange s = w.s;
    Scores<T, SHAPE> score;
    score.init(a, w.head);

    const T *qp = (const T *)a.q + s.q0 * a.q_token + w.head * a.q_head;
    const T *kp = (const T *)a.k + s.k0 * a.k_token + w.kv * a.k_head;
    const T *vp = (const T *)a.v + s.k0 * a.v_token + w.kv * a.v_head;
    typename Frag<T>::type fq[QT][C];
    int qi[QT];
    f32x4 o[DT][QT];
    // top: the maximum, in the score's units; ref: the same times log2(e), rounded once, what the exponentials are taken against.
    // A query whose maximum stays is scaled by 2^(ref - ref) = 1, whatever the other queries do.
    float top[QT], ref[QT], sum[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        qi[u] = w.first + (wave * QT + u) * 16 + (lane & 15);
        const T *row = qi[u] < s.nq ? qp + (long long)qi[u] * a.q_token : nullptr;
#pragma unroll
        for (int c = 0; c < C; ++c) fq[u][c] = read_fragment<T, VEC>(row, 32 * c + 8 * g, a.dim);
        top[u] = minus_infinity();
        ref[u] = sum[u] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int w_first = w.first + wave * QT * 16;   // this wavefront's queries

    auto fetch = [&](int t, auto which) {
        char *lds = decltype(which)::value ? lds1 : lds0;
        const int j0 = t * BK;
        TileReader<T, DP, BK, VEC, 256>::read(kp + (long long)j0 * a.k_token, a.k_token, s.nk - j0, a.dim, lds, tid);
        TileReader<T, DP, BK, VEC, 256>::read(vp + (long long)j0 * a.v_token, a.v_token, s.nk - j0, a.dim, lds + BK * L::PITCH, tid);
    };
    auto work = [&](int t, auto which) {
        const char *lds_k = decltype(which)::value ? lds1 : lds0, *lds_v = lds_k + BK * L::PITCH;
        const int j0 = t * BK;
        // sets of a tile or less: what lies behind their ends is left out, 16 queries and 16 keys at a time
        const int tiles = QT == 1 ? (w.last - j0 + 15) / 16 : 4;
        if (QT == 1 && w_first >= s.nq) return;
        f32x4 z[4][QT];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
            for (int u = 0; u < QT; ++u) z[kt][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            if (QT == 1 && kt >= tiles) break;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const typename Frag<T>::type fk = L::rows(lds_k, kt * 16, c, lane);
#pragma unroll
                for (int u = 0; u < QT; ++u) mma(z[kt][u], fk, fq[u][c]);
            }
        }
        settle(z);
        const bool whole = j0 + BK <= s.nk && (!a.causal || j0 + BK - 1 <= w_first + w.shift || j0 + BK <= w.prefix);
        auto seen = [&](int j, int at) { return j < s.nk && (!a.causal || j <= at || j < w.prefix); };
        typename Frag<T>::type fp[2][QT];
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            const int at = qi[u] + w.shift;
            float add = 0.f;
            if constexpr (SHAPE == CAPPED) {
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[kt][u][e] = exp2_fast(__builtin_fmaf(score.under(z[kt][u][e]), -2.f * score.cap, score.cap));
                if (!whole) {
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!seen(j0 + kt * 16 + 4 * g + e, at)) z[kt][u][e] = 0.f;
                }
            } else {
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) score.template shape<-1>(z[kt][u], at - (j0 + kt * 16 + 4 * g), nullptr);
                if (!whole) {
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!seen(j0 + kt * 16 + 4 * g + e, at)) z[kt][u][e] = minus_infinity();
                }
                float most = top[u];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = fmaxf(most, z[kt][u][e]);
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                if (__any(most != top[u])) {   // else nothing is scaled down
                    float now = most == minus_infinity() ? 0.f : most * score.unit;
                    asm volatile("" : "+v"(now));   // rounded here, not fused into the difference
                    const float keep = top[u] == minus_infinity() ? 0.f : exp2_fast(ref[u] - now);
                    top[u] = most;
                    ref[u] = now;
                    sum[u] *= keep;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[d][u] *= keep;
                }
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[kt][u][e] = exp2_fast(z[kt][u][e] * score.unit - ref[u]);
            }
#pragma unroll
            for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    add += z[kt][u][e];
                    fp[kt >> 1][u][(kt & 1) * 4 + e] = (T)z[kt][u][e];
                }
            sum[u] += add;
        }
        if constexpr (sizeof(T) == 4) {
            // float: the step's sum by itself, so that long sums are rounded once a step
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                f32x4 t4[QT];
#pragma unroll
                for (int u = 0; u < QT; ++u) t4[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (QT == 1 && 2 * c >= tiles) break;
                    const typename Frag<T>::type fv = L::columns(lds_v, c * 32, d * 16, lane);
#pragma unroll
                    for (int u = 0; u < QT; ++u) mma(t4[u], fv, fp[c][u]);
                }
                settle(t4);
#pragma unroll
                for (int u = 0; u < QT; ++u) o[d][u] += t4[u];
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (QT == 1 && 2 * c >= tiles) break;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const typename Frag<T>::type fv = L::columns(lds_v, c * 32, d * 16, lane);
#pragma unroll
                    for (int u = 0; u < QT; ++u) mma(o[d][u], fv, fp[c][u]);
                }
            }
        }
    };
    two_buffers(w.step<BK>(a, w.split), w.step<BK>(a, w.split + 1), fetch, [](int, auto) {}, work);
    settle_loop();
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        float total = sum[u];
        total += __shfl_xor(total, 16);
        total += __shfl_xor(total, 32);
        if (qi[u] >= s.nq) continue;
        const long long n = s.q0 + qi[u];
        const float reference = SHAPE == CAPPED ? 0.f : top[u] == minus_infinity() ? top[u] : ref[u];
        if (a.key_splits > 1) {
            const long long row = (w.split * a.total_q + n) * a.heads + w.head;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int d0 = d * 16 + 4 * g;
                if (d0 < a.dim) store_four(a.part + row * a.dim + d0, o[d][u], a.dim - d0, VEC);
            }
            // (capped: without keys there is no maximum either)
            if (g == 0) a.part_top[row] = make_float2(total == 0.f ? minus_infinity() : reference, total);
            continue;
        }
        const float inv = total > 0.f || total != total ? 1.f / total : 0.f;   // no key: zero
        T *out = (T *)a.o + (n * a.heads + w.head) * a.dim;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int d0 = d * 16 + 4 * g;
            if (d0 < a.dim) store_four(out + d0, o[d][u] * inv, a.dim - d0, VEC);
        }
        if (g == 0) a.lse[w.head * a.total_q + n] = natural_log(reference, total);
    }
}

// The row of a query and head that is not computed, by a wavefront: it gets `value`, and this lse.
template <class T>
__device__ __forceinline__ void clear_row(const AttentionArgs &a, long long row, int lane, float value, float lse)
{
    T *out = (T *)a.o + row * a.dim;
    if (lane < a.dim) out[lane] = (T)value;
    if (lane + 64 < a.dim) out[lane + 64] = (T)value;
    if (lane == 0) a.lse[row % a.heads * a.total_q + row / a.heads] = lse;
}

// Joins the splits of a query and head, a wavefront each, in their order.  Bound by memory, and small where splits are chosen.
template <class T>
__global__ __launch_bounds__(256) void attention_join_splits_kernel(AttentionArgs a)
{
    const long long row = (long long)group_number() * 4 + (threadIdx.x >> 6), n = row / a.heads, all = a.total_q * a.heads;
    const int head = (int)(row % a.heads), lane = threadIdx.x & 63;
    if (n >= a.total_q) return;
    if (n < a.q_off[0] || n >= a.q_off[a.sets]) {
        if (a.clear) clear_row<T>(a, row, lane, 0.f, minus_infinity());
        return;
    }
    float most = minus_infinity();
    for (int s = 0; s < a.key_splits; ++s) most = fmaxf(most, a.part_top[s * all + row].x);
    float total = 0.f, v0 = 0.f, v1 = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.key_splits; ++s) {
        const float2 ml = a.part_top[s * all + row];
        const float keep = ml.x == minus_infinity() ? (ml.y == ml.y ? 0.f : ml.y) : exp2_fast(ml.x - most);
        const float *o = a.part + (s * all + row) * a.dim;
        total += ml.y * keep;
        if (lane < a.dim) v0 += o[lane] * keep;
        if (lane + 64 < a.dim) v1 += o[lane + 64] * keep;
    }
    const float inv = total > 0.f || total != total ? 1.f / total : 0.f;   // no key: zero
    T *out = (T *)a.o + row * a.dim;
    if (lane < a.dim) out[lane] = (T)(v0 * inv);
    if (lane + 64 < a.dim) out[lane + 64] = (T)(v1 * inv);
    if (lane == 0) a.lse[head * a.total_q + n] = natural_log(most, total);
}

// Few queries per set (new tokens): the keys of a set are cut into chunks, a workgroup per chunk and key head, so that every
// key is read once for all query heads that share it.  Bound by reading the keys: each wavefront goes over its own 32 keys at
// a time, through its own two buffers of LDS without waiting for the others.  A row is a query and one of the heads of
// the group: row = query * group + head of the group.  32 sets of 100 to 16 000 keys, bf16, 32 heads of 128 on 8: 197 us, 4.9 TB/s.
template <class T, int DP, int QT, int WAVES, bool VEC, int SHAPE>
__global__ __launch_bounds__(WAVES * 64) void attention_chunk_kernel(AttentionArgs a)
{
    constexpr int C = DP / 32, DT = DP / 16, BK = 32;
    typedef Tile<T, DP> L;
    constexpr int BYTES = 2 * BK * L::PITCH;   // keys and values of one wavefront
    __shared__ __align__(1024) char lds0[WAVES * BYTES];
    __shared__ __align__(1024) char lds1[WAVES * BYTES];
    __shared__ float2 lds_ml[WAVES][QT * 16];
    static_assert(WAVES * BYTES >= WAVES * QT * DP * 16 * 4, "the wavefronts' sums fit");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
    const int group = a.heads / a.kv_heads;
    if (group_number() >= a.groups) return;
    const long long t = die_run(group_number(), a.groups);
    const int kv = (int)(t / a.tiles);
    const long long tile = t % a.tiles;
    const int p = set_of_tile(a.k_off, a.sets, a.chunk, tile);
    SetRange s = range_of(a, p);
    const long long b0 = (tile - (s.k0 / a.chunk + p)) * a.chunk;
    if (b0 < 0 || b0 >= s.nk || s.nq <= 0) return;
    const int shift = s.nk - s.nq, rows = s.nq * group < a.rows ? s.nq * group : a.rows;
    const int prefix = a.causal && a.prefix ? a.prefix[p] : 0;
    const int k_first = (int)b0, k_end = k_first + a.chunk < s.nk ? k_first + a.chunk : s.nk;
    const T *kp = (const T *)a.k + s.k0 * a.k_token + kv * a.k_head;
    const T *vp = (const T *)a.v + s.k0 * a.v_token + kv * a.v_head;

    typename Frag<T>::type fq[QT][C];
    Scores<T, SHAPE> score[QT];
    int qi[QT];
    f32x4 o[DT][QT];
    float top[QT], sum[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int r = u * 16 + (lane & 15), head = kv * group + r % group;
        qi[u] = r / group;
        const T *row = r < rows ? (const T *)a.q + (s.q0 + qi[u]) * a.q_token + head * a.q_head : nullptr;
#pragma unroll
        for (int c = 0; c < C; ++c) fq[u][c] = read_fragment<T, VEC>(row, 32 * c + 8 * g, a.dim);
        score[u].init(a, head);
        top[u] = minus_infinity();
        sum[u] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int LOADS = BYTES / 1024;   // of a wavefront for one step
    auto fetch = [&](int j0, char *lds) {
        char *own = lds + wave * BYTES;
        TileReader<T, DP, BK, VEC, 64, true>::read(kp + (long long)j0 * a.k_token, a.k_token, k_end - j0, a.dim, own, lane);
        TileReader<T, DP, BK, VEC, 64, true>::read(vp + (long long)j0 * a.v_token, a.v_token, k_end - j0, a.dim,
                                                   own + BK * L::PITCH, lane);
    };
    auto work = [&](int j0, const char *lds) {
        const char *lds_k = lds + wave * BYTES, *lds_v = lds_k + BK * L::PITCH;
        f32x4 z[2][QT];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int u = 0; u < QT; ++u) z[kt][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const typename Frag<T>::type fk = L::rows(lds_k, kt * 16, c, lane);
#pragma unroll
                for (int u = 0; u < QT; ++u) mma(z[kt][u], fk, fq[u][c]);
            }
        settle(z);
        const bool whole = j0 + BK <= k_end && (!a.causal || j0 + BK - 1 <= shift || j0 + BK <= prefix);
        typename Frag<T>::type fp[QT];
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            const int at = qi[u] + shift;
            float most = top[u];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                score[u].template shape<-1>(z[kt][u], at - (j0 + kt * 16 + 4 * g), nullptr);
                z[kt][u] *= score[u].unit;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + kt * 16 + 4 * g + e;
                    if (!whole && (j >= k_end || (a.causal && j > at && j >= prefix))) z[kt][u][e] = minus_infinity();
                    most = fmaxf(most, z[kt][u][e]);
                }
            }
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const float ref = most == minus_infinity() ? 0.f : most, keep = exp2_fast(top[u] - ref);
            top[u] = most;
            float add = 0.f;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = exp2_fast(z[kt][u][e] - ref);
                    add += v;
                    fp[u][kt * 4 + e] = (T)v;
                }
            sum[u] = sum[u] * keep + add;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d][u] *= keep;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const typename Frag<T>::type fv = L::columns(lds_v, 0, d * 16, lane);
#pragma unroll
            for (int u = 0; u < QT; ++u) mma(o[d][u], fv, fp[u]);
        }
    };
    // A step's loads are in LDS when no more than those of the step after, if there is one, are under way.
    auto arrived = [&](bool more) {
        if (VEC && more)
            __builtin_amdgcn_s_waitcnt((LOADS & 15) | (LOADS >> 4) << 14 | 0x0f70);
        else
            __builtin_amdgcn_s_waitcnt(0x0f70);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // The buffer has been read: the next loads into it come behind the last read, by a wait and not by the order in which the
    // instructions that use what was read happen to stand.
    auto read = [&]() {
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    constexpr int STEP = WAVES * BK;
    int j0 = k_first + wave * BK;
    if (j0 < k_end) fetch(j0, lds0);
    for (; j0 < k_end; j0 += 2 * STEP) {
        const bool second = j0 + STEP < k_end, third = j0 + 2 * STEP < k_end;
        if (second) fetch(j0 + STEP, lds1);
        arrived(second);
        work(j0, lds0);
        read();
        if (!second) break;
        if (third) fetch(j0 + 2 * STEP, lds0);
        arrived(third);
        work(j0 + STEP, lds1);
        read();
    }
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        sum[u] += __shfl_xor(sum[u], 16);
        sum[u] += __shfl_xor(sum[u], 32);
        if (g == 0) lds_ml[wave][u * 16 + lane] = make_float2(top[u], sum[u]);
    }
    __syncthreads();
    float *all = (float *)lds0;   // [wave][row][dim]
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        float most = minus_infinity();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, lds_ml[w][u * 16 + (lane & 15)].x);
        const float keep = most == minus_infinity() ? 0.f : exp2_fast(top[u] - most);
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *(f32x4 *)(all + ((long long)wave * QT * 16 + u * 16 + (lane & 15)) * DP + d * 16 + 4 * g) = o[d][u] * keep;
    }
    __syncthreads();
    const long long first = (tile * a.kv_heads + kv) * a.rows;
    for (int r = wave; r < rows; r += WAVES) {
        float most = minus_infinity(), total = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, lds_ml[w][r].x);
        // a row whose scores here are not numbers has no maximum, but a sum that is not a number
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 ml = lds_ml[w][r];
            total += ml.x == minus_infinity() ? ml.y : ml.y * exp2_fast(ml.x - most);
        }
        for (int d = lane; d < a.dim; d += 64) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v += all[((long long)w * QT * 16 + r) * DP + d];
            a.part[(first + r) * a.dim + d] = v;
        }
        if (lane == 0) a.part_top[first + r] = make_float2(most, total);
    }
}

// Joins the chunks of a query and head: a wavefront each, in the order of the chunks.  The same sets: 18 us, a chain of a launch and
// two trips to memory for the longest set's chunks.
template <class T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a)
{
    const long long row = (long long)group_number() * 4 + (threadIdx.x >> 6), n = row / a.heads;
    const int head = (int)(row % a.heads), lane = threadIdx.x & 63, group = a.heads / a.kv_heads, kv = head / group;
    if (n >= a.total_q) return;
    const int p = last_set(a.sets, [&](int q) { return a.q_off[q] <= n; });
    const SetRange s = range_of(a, p);
    const long long i = n - s.q0, r = i * group + head % group;
    if (a.clear && (n < a.q_off[0] || n >= a.q_off[a.sets])) return clear_row<T>(a, row, lane, 0.f, minus_infinity());
    if (i < 0 || i >= s.nq) return;
    if (r >= a.rows) {   // the set has more than max_q queries
        if (a.clear) clear_row<T>(a, row, lane, __builtin_nanf(""), __builtin_nanf(""));
        return;
    }
    const long long first = s.k0 / a.chunk + p;
    const int chunks = (s.nk + a.chunk - 1) / a.chunk;
    const long long stride = (long long)a.kv_heads * a.rows, at = (first * a.kv_heads + kv) * a.rows + r;
    float most = minus_infinity();
    for (int c = lane; c < chunks; c += 64) most = fmaxf(most, a.part_top[at + c * stride].x);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) most = fmaxf(most, __shfl_xor(most, x));
    float total = 0.f, v0 = 0.f, v1 = 0.f;
    for (int c0 = 0; c0 < chunks; c0 += 64) {   // a lane has the weight of a chunk
        float keep = 0.f, sum = 0.f;
        if (c0 + lane < chunks) {
            const float2 ml = a.part_top[at + (c0 + lane) * stride];
            keep = ml.x == minus_infinity() ? (ml.y == ml.y ? 0.f : ml.y) : exp2_fast(ml.x - most);
            sum = ml.y * keep;
        }
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
        total += sum;
        const int count = chunks - c0 < 64 ? chunks - c0 : 64;
#pragma unroll 8
        for (int c = 0; c < count; ++c) {
            const float k = __shfl(keep, c);
            const float *o = a.part + (at + (c0 + c) * stride) * a.dim;
            if (lane < a.dim) v0 += o[lane] * k;
            if (lane + 64 < a.dim) v1 += o[lane + 64] * k;
        }
    }
    const float inv = total > 0.f || total != total ? 1.f / total : 0.f;   // no key: zero
    T *out = (T *)a.o + row * a.dim;
    if (lane < a.dim) out[lane] = (T)(v0 * inv);
    if (lane + 64 < a.dim) out[lane + 64] = (T)(v1 * inv);
    if (lane == 0) a.lse[head * a.total_q + n] = natural_log(most, total);
}

// ---- backward -------------------------------------------------------------------
// sum[u] += a b[u]; float: the product by itself, so that a long sum is rounded once for 32 of its terms
template <class T, int N>
__device__ __forceinline__ void add_product(f32x4 (&sum)[N], typename Frag<T>::type a, const typename Frag<T>::type (&b)[N])
{
    if constexpr (sizeof(T) == 4) {
        f32x4 t[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            t[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            mma(t[u], a, b[u]);
        }
        settle(t);
#pragma unroll
        for (int u = 0; u < N; ++u) sum[u] += t[u];
    } else {
#pragma unroll
        for (int u = 0; u < N; ++u) mma(sum[u], a, b[u]);
    }
}

// dq: like the forward pass; dS = P (dP - delta) cut, dq = scale sum_j dS_ij k_j.
// delta_i = do_i . o_i = sum_j P_ij dP_ij.  Where a tile sees up to EXACT_KEYS keys it is formed as the second sum, in a pass of
// its own: o is large there, and its rounding to bf16 would count in dS as much as that of dS itself.  With more keys do . o is
// taken: o is an average of many v then, and small, unless a row's weight lies on few keys (steep slopes, large scores), whose dS
// is off by a rounding of o as well; the first sum costs a pass over all keys.  The delta that is used goes to a.delta for dk and dv; where dq is not asked for that is all
// that the kernel does, so that dk does not depend on it.
// Bound as the forward pass is: the documents 425 us (0.63 PFLOP/s), the small float sets 57.
constexpr int EXACT_KEYS = 256;
template <class T, int DP, int QT, bool VEC, int SHAPE>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void attention_dq_kernel(AttentionArgs a)
{
    constexpr int BQ = 64 * QT, BK = 64, C = DP / 32, DT = DP / 16;
    typedef Tile<T, DP> L;
    __shared__ __align__(1024) char lds0[2 * BK * L::PITCH];
    __shared__ __align__(1024) char lds1[2 * BK * L::PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
    const QueryTile w = query_tile<BQ>(a);
    if (!w.any) return clear_others<T, VEC>(a, a.q_off, a.total_q, (long long)a.heads * a.dim, (T *)a.dq, nullptr, nullptr);
    const SetRange s = w.s;
    Scores<T, SHAPE> score;
    score.init(a, w.head);
    const T *kp = (const T *)a.k + s.k0 * a.k_token + w.kv * a.k_head;
    const T *vp = (const T *)a.v + s.k0 * a.v_token + w.kv * a.v_head;
    typename Frag<T>::type fq[QT][C], fo[QT][C];
    int qi[QT];
    float lse[QT], delta[QT];
    f32x4 dq[DT][QT];
    const bool exact = sizeof(T) == 2 && w.last <= EXACT_KEYS;   // float: o is not rounded
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        qi[u] = w.first + (wave * QT + u) * 16 + (lane & 15);
        const bool in = qi[u] < s.nq;
        const long long n = s.q0 + (in ? qi[u] : 0);
        const T *row = in ? (const T *)a.q + n * a.q_token + w.head * a.q_head : nullptr;
        const T *dorow = in ? (const T *)a.d_o + (n * a.heads + w.head) * a.dim : nullptr;
        const T *orow = in ? (const T *)a.o + (n * a.heads + w.head) * a.dim : nullptr;
        delta[u] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            fq[u][c] = read_fragment<T, VEC>(row, 32 * c + 8 * g, a.dim);
            fo[u][c] = read_fragment<T, VEC>(dorow, 32 * c + 8 * g, a.dim);
            if (!exact) {
                const typename Frag<T>::type f = read_fragment<T, VEC>(orow, 32 * c + 8 * g, a.dim);
#pragma unroll
                for (int e = 0; e < 8; ++e) delta[u] += (float)f[e] * (float)fo[u][c][e];
            }
        }
        lse[u] = in ? Scores<T, SHAPE>::lse_in(a.lse_in[w.head * a.total_q + n]) : 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) dq[d][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int w_first = w.first + wave * QT * 16;
    auto fetch = [&](int t, auto which) {
        char *lds = decltype(which)::value ? lds1 : lds0;
        const int j0 = t * BK;
        TileReader<T, DP, BK, VEC, 256>::read(kp + (long long)j0 * a.k_token, a.k_token, s.nk - j0, a.dim, lds, tid);
        TileReader<T, DP, BK, VEC, 256>::read(vp + (long long)j0 * a.v_token, a.v_token, s.nk - j0, a.dim, lds + BK * L::PITCH, tid);
    };
    // P and dP of 32 keys from j0 on, the first of them in row r of the tiles; P is zero where the key is not seen
    auto scores = [&](const char *lds_k, const char *lds_v, int j0, int r, f32x4 (&z)[2][QT], f32x4 (&dp)[2][QT],
                      f32x4 (&cut)[2][QT]) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int u = 0; u < QT; ++u) z[kt][u] = dp[kt][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const typename Frag<T>::type fk = L::rows(lds_k, r + kt * 16, c, lane);
                const typename Frag<T>::type fv = L::rows(lds_v, r + kt * 16, c, lane);
#pragma unroll
                for (int u = 0; u < QT; ++u) {
                    mma(z[kt][u], fk, fq[u][c]);
                    mma(dp[kt][u], fv, fo[u][c]);
                }
            }
        settle(z);
        settle(dp);
        const bool whole = j0 + 32 <= s.nk && (!a.causal || j0 + 31 <= w_first + w.shift || j0 + 32 <= w.prefix);
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const int at = qi[u] + w.shift, j = j0 + kt * 16 + 4 * g;
                score.template weigh<-1>(z[kt][u], at - j, f32x4{lse[u], lse[u], lse[u], lse[u]}, cut[kt][u]);
                if (!whole) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (j + e >= s.nk || (a.causal && j + e > at && j + e >= w.prefix)) {
                            z[kt][u][e] = 0.f;
                            dp[kt][u][e] = 0.f;
                        }
                }
            }
    };
    if (exact) {
        two_buffers(0, (w.last + BK - 1) / BK, fetch, [](int, auto) {}, [&](int t, auto which) {
            const char *lds_k = decltype(which)::value ? lds1 : lds0, *lds_v = lds_k + BK * L::PITCH;
            if (QT == 1 && w_first >= s.nq) return;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (QT == 1 && t * BK + h * 32 >= w.last) break;
                f32x4 z[2][QT], dp[2][QT], cut[2][QT];
                scores(lds_k, lds_v, t * BK + h * 32, h * 32, z, dp, cut);
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) delta[u] += z[kt][u][e] * dp[kt][u][e];
            }
        });
        __syncthreads();   // the first buffer is filled again
    }
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        delta[u] += __shfl_xor(delta[u], 16);
        delta[u] += __shfl_xor(delta[u], 32);
        if (g == 0 && qi[u] < s.nq && w.split == 0) a.delta[w.head * a.total_q + s.q0 + qi[u]] = delta[u];
    }
    if (!a.dq) return;
    two_buffers(w.step<BK>(a, w.split), w.step<BK>(a, w.split + 1), fetch, [](int, auto) {}, [&](int t, auto which) {
        const char *lds_k = decltype(which)::value ? lds1 : lds0, *lds_v = lds_k + BK * L::PITCH;
        if (QT == 1 && w_first >= s.nq) return;   // short sets: see the forward kernel
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // 32 keys at a time
            if (QT == 1 && t * BK + h * 32 >= w.last) break;
            f32x4 z[2][QT], dp[2][QT], cut[2][QT];
            scores(lds_k, lds_v, t * BK + h * 32, h * 32, z, dp, cut);
            typename Frag<T>::type fs[QT];
#pragma unroll
            for (int u = 0; u < QT; ++u)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    f32x4 ds = z[kt][u] * (dp[kt][u] - delta[u]);
                    if (SHAPE != PLAIN) ds *= cut[kt][u];
#pragma unroll
                    for (int e = 0; e < 4; ++e) fs[u][kt * 4 + e] = (T)ds[e];
                }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const typename Frag<T>::type fk = L::columns(lds_k, h * 32, d * 16, lane);
                add_product<T>(dq[d], fk, fs);
            }
        }
    });
    settle_loop();
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        if (qi[u] >= s.nq) continue;
        const long long at = ((s.q0 + qi[u]) * a.heads + w.head) * a.dim;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int d0 = d * 16 + 4 * g;
            if (d0 >= a.dim) continue;
            const f32x4 v = dq[d][u] * score.rest(a);
            if (a.key_splits > 1)
                store_four(a.part + w.split * a.total_q * a.heads * a.dim + at + d0, v, a.dim - d0, VEC);
            else
                store_four((T *)a.dq + at + d0, v, a.dim - d0, VEC);
        }
    }
}

// dk, dv: four wavefronts of 16 KT keys each go over the queries of all heads that share the key head, BQ at a
// time; dv = P^T do, dk = scale dS^T q.  With few tiles the steps are dealt to a.splits workgroups, whose sums a second launch adds.
// Two products more per score than forward, and both operands are read from LDS twice: the documents 703 us (0.51 PFLOP/s) and 24 for
// the sums, the small float sets 74.
template <class T, int DP, int KT, bool VEC, int SHAPE>
__global__ __launch_bounds__(256) void attention_dkv_kernel(AttentionArgs a)
{
    constexpr int BK = 64 * KT, BQ = DP * sizeof(T) > 256 ? 32 : 64, C = DP / 32, DT = DP / 16;
    typedef Tile<T, DP> L;
    __shared__ __align__(1024) char lds0[2 * BQ * L::PITCH];
    __shared__ __align__(1024) char lds1[2 * BQ * L::PITCH];
    __shared__ __align__(16) float lds_lse[2][BQ], lds_delta[2][BQ];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4;
    const int group = a.heads / a.kv_heads;
    const unsigned id = group_number();
    if (id >= a.groups)
        return clear_others<T, VEC>(a, a.k_off, a.total_k, (long long)a.kv_heads * a.dim, (T *)a.dk, (T *)a.dv, nullptr);
    const int share = (int)(id % a.splits), kv = (int)(id / a.splits % a.kv_heads);
    const long long tile = id / (a.splits * a.kv_heads);
    const int p = set_of_tile(a.k_off, a.sets, BK, tile);
    const SetRange s = range_of(a, p);
    const long long b0 = (tile - (s.k0 / BK + p)) * BK;
    if (b0 < 0 || b0 >= s.nk) return;
    const int k_first = (int)b0, shift = s.nk - s.nq;
    const int prefix = a.causal && a.prefix ? a.prefix[p] : 0;
    // queries before `begin` see none of these keys
    int begin = 0;
    if (a.causal && k_first >= prefix) {
        begin = k_first - shift;
        begin = begin > 0 ? begin & ~(BQ - 1) : 0;
    }
    typename Frag<T>::type fk[KT][C], fv[KT][C];
    int kj[KT];
    f32x4 dk[DT][KT], dv[DT][KT];
#pragma unroll
    for (int u = 0; u < KT; ++u) {
        kj[u] = k_first + (wave * KT + u) * 16 + (lane & 15);
        const bool in = kj[u] < s.nk;
        const long long n = s.k0 + (in ? kj[u] : 0);
        const T *krow = in ? (const T *)a.k + n * a.k_token + kv * a.k_head : nullptr;
        const T *vrow = in ? (const T *)a.v + n * a.v_token + kv * a.v_head : nullptr;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            fk[u][c] = read_fragment<T, VEC>(krow, 32 * c + 8 * g, a.dim);
            fv[u][c] = read_fragment<T, VEC>(vrow, 32 * c + 8 * g, a.dim);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) dk[d][u] = dv[d][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int w_last = k_first + (wave + 1) * KT * 16 - 1;   // this wavefront's last key
    // a step: BQ queries of one head of the group
    const int each = s.nq > begin ? (s.nq - begin + BQ - 1) / BQ : 0;
    float next_lse = 0.f, next_delta = 0.f;
    auto fetch = [&](int t, auto which) {
        char *lds = decltype(which)::value ? lds1 : lds0;
        const int head = kv * group + t / each, i0 = begin + t % each * BQ;
        const T *qp = (const T *)a.q + (s.q0 + i0) * a.q_token + head * a.q_head;
        const T *op = (const T *)a.d_o + ((s.q0 + i0) * a.heads + head) * a.dim;
        if (tid < BQ) {
            const bool in = i0 + tid < s.nq;
            const long long n = head * a.total_q + s.q0 + (in ? i0 + tid : 0);
            next_lse = a.lse_in[n];
            next_delta = a.delta[n];
        }
        TileReader<T, DP, BQ, VEC, 256>::read(qp, a.q_token, s.nq - i0, a.dim, lds, tid);
        TileReader<T, DP, BQ, VEC, 256>::read(op, (long long)a.heads * a.dim, s.nq - i0, a.dim, lds + BQ * L::PITCH, tid);
    };
    auto landed = [&](int, auto which) {
        if (tid < BQ) {
            lds_lse[decltype(which)::value][tid] = Scores<T, SHAPE>::lse_in(next_lse);
            lds_delta[decltype(which)::value][tid] = next_delta;
        }
    };
    auto work = [&](int t, auto which) {
        const char *lds_q = decltype(which)::value ? lds1 : lds0, *lds_o = lds_q + BQ * L::PITCH;
        const int head = kv * group + t / each;
        Scores<T, SHAPE> score;
        score.init(a, head);
        if (KT == 1 && w_last - 15 >= s.nk) return;   // short sets: no key of this wavefront, no query of the 32
#pragma unroll
        for (int h = 0; h < BQ / 32; ++h) {   // 32 queries at a time
            const int i0 = begin + t % each * BQ + h * 32;
            if (KT == 1 && i0 >= s.nq) break;
            f32x4 z[2][KT], dp[2][KT];
#pragma unroll
            for (int qt = 0; qt < 2; ++qt)
#pragma unroll
                for (int u = 0; u < KT; ++u) z[qt][u] = dp[qt][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) {
                    const typename Frag<T>::type fq = L::rows(lds_q, h * 32 + qt * 16, c, lane);
                    const typename Frag<T>::type fo = L::rows(lds_o, h * 32 + qt * 16, c, lane);
#pragma unroll
                    for (int u = 0; u < KT; ++u) {
                        mma(z[qt][u], fq, fk[u][c]);
                        mma(dp[qt][u], fo, fv[u][c]);
                    }
                }
            settle(z);
            settle(dp);
            const bool whole = i0 + 32 <= s.nq && w_last < s.nk && (!a.causal || w_last <= i0 + shift || w_last < prefix);
            typename Frag<T>::type fp[KT], fs[KT];
#pragma unroll
            for (int qt = 0; qt < 2; ++qt) {
                const f32x4 lse = *(const f32x4 *)(lds_lse[decltype(which)::value] + h * 32 + qt * 16 + 4 * g);
                const f32x4 delta = *(const f32x4 *)(lds_delta[decltype(which)::value] + h * 32 + qt * 16 + 4 * g);
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    const int i = i0 + qt * 16 + 4 * g, j = kj[u];
                    f32x4 cut;
                    score.template weigh<1>(z[qt][u], i + shift - j, lse, cut);
                    f32x4 pr = z[qt][u], ds = pr * (dp[qt][u] - delta);
                    if (SHAPE != PLAIN) ds *= cut;
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (i + e >= s.nq || j >= s.nk || (a.causal && j > i + e + shift && j >= prefix)) pr[e] = ds[e] = 0.f;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        fp[u][qt * 4 + e] = (T)pr[e];
                        fs[u][qt * 4 + e] = (T)ds[e];
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const typename Frag<T>::type fo = L::columns(lds_o, h * 32, d * 16, lane);
                const typename Frag<T>::type fq = L::columns(lds_q, h * 32, d * 16, lane);
                add_product<T>(dv[d], fo, fp);
                add_product<T>(dk[d], fq, fs);
            }
        }
    };
    // this workgroup's share of the steps
    const long long steps = (long long)group * each;
    two_buffers((int)(steps * share / a.splits), (int)(steps * (share + 1) / a.splits), fetch, landed, work);
    settle_loop();
    const float rest = Scores<T, SHAPE>().rest(a);
#pragma unroll
    for (int u = 0; u < KT; ++u) {
        if (kj[u] >= s.nk) continue;
        const long long at = ((s.k0 + kj[u]) * a.kv_heads + kv) * a.dim;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int d0 = d * 16 + 4 * g;
            if (d0 >= a.dim) continue;
            if (a.splits > 1) {
                const long long all = a.total_k * a.kv_heads * a.dim;
                store_four(a.part + 2 * share * all + at + d0, dk[d][u] * rest, a.dim - d0, VEC);
                store_four(a.part + (2 * share + 1) * all + at + d0, dv[d][u], a.dim - d0, VEC);
            } else {
                store_four((T *)a.dk + at + d0, dk[d][u] * rest, a.dim - d0, VEC);
                store_four((T *)a.dv + at + d0, dv[d][u], a.dim - d0, VEC);
            }
        }
    }
}

// A gradient (blockIdx.y = 0, 1: of two) from the sums of `splits` workgroups, in their order: a thread adds four values of the
// `width` of a token.  Tokens in no set are not written, or become zero (clear).
template <class T>
__global__ __launch_bounds__(256) void attention_add_kernel(const float *part, int splits, long long tokens, long long width,
                                                            const int64_t *off, int sets, T *out0, T *out1, int whole,
                                                            int clear)
{
    const long long all = tokens * width, stride = all * gridDim.y, fours = (all + 3) / 4;
    const long long begin = off[0] < 0 ? 0 : off[0] * width, end = (off[sets] < tokens ? off[sets] : tokens) * width;
    T *out = blockIdx.y ? out1 : out0;
    part += blockIdx.y * all;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < fours; t += (long long)gridDim.x * 256) {
        const long long i = t * 4;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) v += load_four(part + s * stride + i, all - i < 4 ? (int)(all - i) : 4, whole);
        if (i >= begin && i + 4 <= end) {
            store_four(out + i, v, 4, whole);
        } else {
            for (int e = 0; e < 4; ++e) {
                const bool in = i + e >= begin && i + e < end;
                if (in || (clear && i + e < all)) out[i + e] = in ? (T)v[e] : (T)0.f;
            }
        }
    }
}

// one translation unit per type (kernels_attention_*.hip)
template <class T>
hipError_t attention_forward(AttentionArgs a, bool vec, int shape, hipStream_t s);
template <class T>
hipError_t attention_by_chunks(AttentionArgs a, bool vec, int shape, hipStream_t s);
template <class T>
hipError_t attention_backward(AttentionArgs a, bool vec, int shape, hipStream_t s);

}  // namespace lcn
