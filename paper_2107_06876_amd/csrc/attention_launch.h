// Instantiates the attention kernels of one type and chooses among them.
#pragma once

#include "attention.h"

namespace lcn {

// The grid of a.groups workgroups and, where they write their outputs themselves, of those that clear the others' (see clear_others).
static dim3 grid_with_clearers(const AttentionArgs &a, bool own) { return grid_of((long long)a.groups + (a.clear && own ? CLEARERS : 0)); }

// Tiles of B tokens that sets with `total` tokens can have (see set_of_tile).
inline long long tiles_of(long long total, int sets, int B) { return total / B + sets; }

template <class T, int DP, int QT, bool VEC, int SHAPE>
static hipError_t forward_one(AttentionArgs a, hipStream_t s)
{
    const long long tiles = tiles_of(a.total_q, a.sets, 64 * QT);
    a.tiles = (int)tiles;
    a.groups = (unsigned)(tiles * a.heads * a.key_splits);
    hipLaunchKernelGGL((attention_forward_kernel<T, DP, QT, VEC, SHAPE>), grid_with_clearers(a, a.key_splits == 1), dim3(256), 0, s,
                       a);
    return hipGetLastError();
}
template <class T, int DP, int QT, bool DQ, bool VEC, int SHAPE>
static hipError_t backward_one(AttentionArgs a, hipStream_t s)
{
    if constexpr (DQ) {
        const long long tiles = tiles_of(a.total_q, a.sets, 64 * QT);
        a.tiles = (int)tiles;
        a.groups = (unsigned)(tiles * a.heads * a.key_splits);
        hipLaunchKernelGGL((attention_dq_kernel<T, DP, QT, VEC, SHAPE>), grid_with_clearers(a, a.dq && a.key_splits == 1), dim3(256),
                           0, s, a);
    } else {
        const long long tiles = tiles_of(a.total_k, a.sets, 64 * QT);
        a.tiles = (int)tiles;
        a.groups = (unsigned)(tiles * a.kv_heads * a.splits);
        hipLaunchKernelGGL((attention_dkv_kernel<T, DP, QT, VEC, SHAPE>), grid_with_clearers(a, a.splits == 1), dim3(256), 0, s, a);
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
// A wavefront has 16 or 32 queries (dk and dv: keys).  32 halve the reads of LDS, 16 take half of the registers, so that two
// wavefronts share a SIMD, fill a tile of half the size and leave out what lies behind a short set's end.  Measured, 16 / 32,
// four heads of 32, 64, 128 on sets of 500 tokens and of 2000 (some 32 000 in all), us:
//   dk, dv bf16   saves 12, 53, 0 / 76, 166, 0 of the whole backward pass    -> always 16
//   dk, dv float  saves 67, 112, 122 / 189, 195, -205                         -> 32 for wide heads in long sets alone
//   dq bf16       saves 8, 13, -7 / 8, 0, -79; float 41, 86, 122 / 20, 39, -131   -> wide heads: 32 in long sets
//   (dq, dk and dv of float with 32 rows of 65 to 128 values do not fit: 99 to 121 registers per lane are spilled, 239 where rows are
//   not whole pieces; bf16 with 32 queries spills 8 to 34 in the forward and dq kernels of that width)
//   forward bf16  33, 46, 84 / 32, 49, 74 and 95, 138, 262 / 76, 115, 178; float 98, 190, 462 / 118, 247, 452 and
//                 346, 712, 1706 / 339, 725, 1357                              -> 32 in long sets, bf16 wide heads from 65 on
template <class T, int WHAT>
static hipError_t by_size(const AttentionArgs &a, bool vec, int shape, hipStream_t s)
{
    constexpr bool wide_type = sizeof(T) == 4;
    const long long total = WHAT == GRAD_KV ? a.total_k : a.total_q;
    const bool up_to_512 = total <= 512LL * a.sets, up_to_64 = total <= 64LL * a.sets;
    if constexpr (WHAT != FORWARD) {
        if (a.dim <= 32) return by_form<T, 32, 1, WHAT>(a, vec, shape, s);
        if (a.dim <= 64) return by_form<T, 64, 1, WHAT>(a, vec, shape, s);
    } else {
        if (a.dim <= 32) return up_to_512 ? by_form<T, 32, 1, WHAT>(a, vec, shape, s) : by_form<T, 32, 2, WHAT>(a, vec, shape, s);
        if (a.dim <= 64) return up_to_512 ? by_form<T, 64, 1, WHAT>(a, vec, shape, s) : by_form<T, 64, 2, WHAT>(a, vec, shape, s);
    }
    if constexpr (WHAT == GRAD_KV && !wide_type)
        return by_form<T, 128, 1, WHAT>(a, vec, shape, s);
    else
        return (wide_type ? up_to_512 : up_to_64) ? by_form<T, 128, 1, WHAT>(a, vec, shape, s) : by_form<T, 128, 2, WHAT>(a, vec, shape, s);
}

template <class T>
hipError_t attention_forward(AttentionArgs a, bool vec, int shape, hipStream_t s)
{
    const hipError_t e = by_size<T, FORWARD>(a, vec, shape, s);
    if (e != hipSuccess || a.key_splits == 1) return e;
    hipLaunchKernelGGL(attention_join_splits_kernel<T>, grid_of((a.total_q * a.heads + 3) / 4), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <class T, int DP, int QT>
static hipError_t chunks_one(const AttentionArgs &a, bool vec, int shape, hipStream_t s)
{
    constexpr int WAVES = DP * sizeof(T) > 256 ? 2 : 4;   // two buffers of each wavefront fit into LDS
    const dim3 grid = grid_of(a.groups), block(WAVES * 64);
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
    a.groups = (unsigned)((long long)a.tiles * a.kv_heads);
    hipError_t e = a.rows <= 16 ? chunks_by_dim<T, 1>(a, vec, shape, s) : chunks_by_dim<T, 2>(a, vec, shape, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(attention_join_kernel<T>, grid_of((a.total_q * a.heads + 3) / 4), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <class T>
static hipError_t add_sums(const AttentionArgs &a, int splits, long long tokens, long long width, const int64_t *off, void *out0,
                           void *out1, hipStream_t s)
{
    const long long groups = (tokens * width / 4 + 255) / 256 + 1;
    hipLaunchKernelGGL(attention_add_kernel<T>, dim3((unsigned)(groups < 4096 ? groups : 4096), out1 ? 2 : 1), dim3(256), 0, s,
                       a.part, splits, tokens, width, off, a.sets, (T *)out0, (T *)out1, a.clear);
    return hipGetLastError();
}
template <class T>
hipError_t attention_backward(AttentionArgs a, bool vec, int shape, hipStream_t s)
{
    hipError_t e = hipSuccess;
    if (a.total_q > 0) {
        if (!a.dq) a.key_splits = 1;   // delta alone: formed by one workgroup of a tile
        e = by_size<T, GRAD_Q>(a, vec, shape, s);
        if (e == hipSuccess && a.key_splits > 1)
            e = add_sums<T>(a, a.key_splits, a.total_q, (long long)a.heads * a.dim, a.q_off, a.dq, nullptr, s);
    }
    if (e != hipSuccess || !a.dk || a.total_k == 0) return e;
    e = by_size<T, GRAD_KV>(a, vec, shape, s);
    if (e != hipSuccess || a.splits == 1) return e;
    return add_sums<T>(a, a.splits, a.total_k, (long long)a.kv_heads * a.dim, a.k_off, a.dk, a.dv, s);
}

}  // namespace lcn
