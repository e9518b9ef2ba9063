// Instantiates the attention kernels of one type and chooses among them.
#pragma once

#include "attention.h"

namespace lcn {

// Tiles of B tokens that sets with `total` tokens can have (see set_of_tile).
inline long long tiles_of(long long total, int sets, int B) { return total / B + sets; }

// Sets of up to 64 tokens on average: wavefronts of 16 instead of 32 queries (or keys) each, so that a set fills a workgroup.
inline bool short_sets(long long total, int sets) { return total <= 64LL * sets; }

template <class T, int DP, int QT, bool VEC, int SHAPE>
static hipError_t forward_one(AttentionArgs a, hipStream_t s)
{
    const long long tiles = tiles_of(a.total_q, a.sets, 64 * QT);
    a.tiles = (int)tiles;
    hipLaunchKernelGGL((attention_forward_kernel<T, DP, QT, VEC, SHAPE>), dim3((unsigned)(tiles * a.heads * a.key_splits)), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <class T, int DP, int QT, bool DQ, bool VEC, int SHAPE>
static hipError_t backward_one(AttentionArgs a, hipStream_t s)
{
    if constexpr (DQ) {
        const long long tiles = tiles_of(a.total_q, a.sets, 64 * QT);
        a.tiles = (int)tiles;
        hipLaunchKernelGGL((attention_dq_kernel<T, DP, QT, VEC, SHAPE>), dim3((unsigned)(tiles * a.heads * a.key_splits)), dim3(256), 0, s, a);
    } else {
        const long long tiles = tiles_of(a.total_k, a.sets, 64 * QT);
        a.tiles = (int)tiles;
        hipLaunchKernelGGL((attention_dkv_kernel<T, DP, QT, VEC, SHAPE>), dim3((unsigned)(tiles * a.kv_heads * a.splits)), dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

enum { FORWARD = 0, GRAD_Q = 1, GRAD_KV = 2 };

template <class T, int DP, int QT, int WHAT, bool VEC, int SHAPE>
static hipError_t one(const AttentionArgs &a, hipStream_t s)
{
    if constexpr (WHAT == FORWARD)
        return forward_one<T, DP, QT, VEC, SHAPE>(a, s);
    else
        return backward_one<T, DP, QT, WHAT == GRAD_Q, VEC, SHAPE>(a, s);
}
template <class T, int DP, int QT, int WHAT>
static hipError_t by_form(const AttentionArgs &a, bool vec, int shape, hipStream_t s)
{
    if (!vec) return one<T, DP, QT, WHAT, false, SHAPED>(a, s);
    if (shape == PLAIN) return one<T, DP, QT, WHAT, true, PLAIN>(a, s);
    if constexpr (sizeof(T) == 2) {
        if (shape == CAPPED) return one<T, DP, QT, WHAT, true, CAPPED>(a, s);
    }
    return one<T, DP, QT, WHAT, true, SHAPED>(a, s);
}
template <class T, int WHAT>
static hipError_t by_size(const AttentionArgs &a, bool vec, int shape, hipStream_t s)
{
    const bool few = WHAT == GRAD_KV ? short_sets(a.total_k, a.sets) : short_sets(a.total_q, a.sets);
    // wide bf16 heads: with 16 keys a wavefront two share a SIMD (249 registers instead of 424), which is worth more than
    // the fewer reads of LDS (packed documents of 16 heads of 128: dk and dv in 745 instead of 827 us)
    constexpr bool narrow_keys = WHAT == GRAD_KV && sizeof(T) == 2;
    if (a.dim <= 32) return few ? by_form<T, 32, 1, WHAT>(a, vec, shape, s) : by_form<T, 32, 2, WHAT>(a, vec, shape, s);
    if (a.dim <= 64) return few ? by_form<T, 64, 1, WHAT>(a, vec, shape, s) : by_form<T, 64, 2, WHAT>(a, vec, shape, s);
    if constexpr (narrow_keys)
        return by_form<T, 128, 1, WHAT>(a, vec, shape, s);
    else
        return few ? by_form<T, 128, 1, WHAT>(a, vec, shape, s) : by_form<T, 128, 2, WHAT>(a, vec, shape, s);
}

template <class T>
hipError_t attention_forward(AttentionArgs a, bool vec, int shape, hipStream_t s)
{
    const hipError_t e = by_size<T, FORWARD>(a, vec, shape, s);
    if (e != hipSuccess || a.key_splits == 1) return e;
    hipLaunchKernelGGL(attention_join_splits_kernel<T>, dim3((unsigned)((a.total_q * a.heads + 3) / 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <class T, int DP, int QT>
static hipError_t chunks_one(const AttentionArgs &a, bool vec, int shape, hipStream_t s)
{
    constexpr int WAVES = DP * sizeof(T) > 256 ? 2 : 4;   // two buffers of each wavefront fit into LDS
    const dim3 grid((unsigned)((long long)a.tiles * a.kv_heads)), block(WAVES * 64);
    if (vec && shape == PLAIN)   // bound by memory: a cap needs no kernel of its own
        hipLaunchKernelGGL((attention_chunk_kernel<T, DP, QT, WAVES, true, PLAIN>), grid, block, 0, s, a);
    else if (vec)
        hipLaunchKernelGGL((attention_chunk_kernel<T, DP, QT, WAVES, true, SHAPED>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((attention_chunk_kernel<T, DP, QT, WAVES, false, SHAPED>), grid, block, 0, s, a);
    return hipGetLastError();
}
template <class T, int QT>
static hipError_t chunks_by_dim(const AttentionArgs &a, bool vec, int shape, hipStream_t s)
{
    if (a.dim <= 32) return chunks_one<T, 32, QT>(a, vec, shape, s);
    if (a.dim <= 64) return chunks_one<T, 64, QT>(a, vec, shape, s);
    return chunks_one<T, 128, QT>(a, vec, shape, s);
}
template <class T>
hipError_t attention_by_chunks(AttentionArgs a, bool vec, int shape, hipStream_t s)
{
    a.tiles = (int)tiles_of(a.total_k, a.sets, a.chunk);
    hipError_t e = a.rows <= 16 ? chunks_by_dim<T, 1>(a, vec, shape, s) : chunks_by_dim<T, 2>(a, vec, shape, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(attention_join_kernel<T>, dim3((unsigned)((a.total_q * a.heads + 3) / 4)), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <class T>
static hipError_t add_sums(const AttentionArgs &a, int splits, long long tokens, long long width, const int64_t *off, void *out0,
                           void *out1, bool whole, hipStream_t s)
{
    const long long groups = (tokens * width / 4 + 255) / 256 + 1;
    hipLaunchKernelGGL(attention_add_kernel<T>, dim3((unsigned)(groups < 4096 ? groups : 4096), out1 ? 2 : 1), dim3(256), 0, s,
                       a.part, splits, tokens, width, off, a.sets, (T *)out0, (T *)out1, whole ? 1 : 0);
    return hipGetLastError();
}
template <class T>
hipError_t attention_backward(AttentionArgs a, bool vec, int shape, hipStream_t s)
{
    hipError_t e = hipSuccess;
    if (a.total_q > 0 && a.dq) {
        e = by_size<T, GRAD_Q>(a, vec, shape, s);
        if (e == hipSuccess && a.key_splits > 1)
            e = add_sums<T>(a, a.key_splits, a.total_q, (long long)a.heads * a.dim, a.q_off, a.dq, nullptr, vec, s);
    } else if (a.total_q > 0) {
        const long long rows = a.total_q * a.heads;
        hipLaunchKernelGGL(attention_delta_kernel<T>, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, s, (const T *)a.o,
                           (const T *)a.d_o, a.total_q, a.heads, a.dim, a.delta);
        e = hipGetLastError();
    }
    if (e != hipSuccess || !a.dk || a.total_k == 0) return e;
    e = by_size<T, GRAD_KV>(a, vec, shape, s);
    if (e != hipSuccess || a.splits == 1) return e;
    return add_sums<T>(a, a.splits, a.total_k, (long long)a.kv_heads * a.dim, a.k_off, a.dk, a.dv, vec, s);
}

}  // namespace lcn
