// Operands of the 16x16 matrix instructions with 32 values of k, for bf16 and float alike: lane l holds index l % 16 and
// eight values of k, 8 (l / 16) + 0 .. 7 or, where two accumulators become an operand, 4 (l / 16) + 0 .. 3 and
// 16 + 4 (l / 16) + 0 .. 3.  bf16 takes the 16x16x32 instruction, float eight 16x16x4 ones on the same registers (each
// adds one of a lane's eight values; which k they stand for does not matter as long as both operands agree).
#pragma once

#include "operators.h"

namespace lcn {

template <class T>
struct Frag;
template <>
struct Frag<__bf16> {
    typedef bf16x8 type;
};
template <>
struct Frag<float> {
    typedef float type __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ void mma(f32x4 &c, bf16x8 a, bf16x8 b) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mma(f32x4 &c, Frag<float>::type a, Frag<float>::type b)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
}

// A tile in LDS: ROWS rows of DP values, in pieces of 16 bytes permuted so that neither 16 rows' pieces of one place nor
// the transposing reads of eight rows meet in a bank.
template <class T, int DP>
struct Tile {
    static constexpr int PITCH = DP * (int)sizeof(T), PIECES = PITCH / 16, EACH = 16 / (int)sizeof(T);
    static __device__ __forceinline__ int swizzle(int r)
    {
        if (PIECES >= 16) return ((r & 7) << 1) | ((r >> 3) & 1);
        if (PIECES == 8) return (((r >> 1) & 3) << 1) | ((r >> 3) & 1);
        return (((r >> 2) & 1) << 1) | ((r >> 3) & 1);
    }
    static __device__ __forceinline__ int place(int r, int piece) { return r * PITCH + ((piece ^ swizzle(r)) << 4); }

    // rows r0 .. r0 + 15 (lane % 16), values 32 c + 8 (lane / 16) + 0 .. 7
    static __device__ __forceinline__ typename Frag<T>::type rows(const char *lds, int r0, int c, int lane)
    {
        const int r = r0 + (lane & 15), g = lane >> 4;
        if constexpr (sizeof(T) == 2) {
            return *(const bf16x8 *)(lds + place(r, 4 * c + g));
        } else {
            union {
                f32x4 h[2];
                Frag<float>::type v;
            } f;
            f.h[0] = *(const f32x4 *)(lds + place(r, 8 * c + 2 * g));
            f.h[1] = *(const f32x4 *)(lds + place(r, 8 * c + 2 * g + 1));
            return f.v;
        }
    }
    // values d0 .. d0 + 15 (lane % 16) of rows r0 + 4 g + 0 .. 3 and r0 + 16 + 4 g + 0 .. 3, g = lane / 16
    static __device__ __forceinline__ typename Frag<T>::type columns(const char *lds, int r0, int d0, int lane)
    {
        const int g = lane >> 4;
        if constexpr (sizeof(T) == 2) {
            const int r = r0 + 4 * g + ((lane & 15) >> 2), piece = (d0 >> 3) + ((lane & 3) >> 1), part = (lane & 1) * 8;
            union {
                s16x4 h[2];
                bf16x8 v;
            } f;
            f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + place(r, piece) + part));
            f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + place(r + 16, piece) + part));
            return f.v;
        } else {
            Frag<float>::type f;
            const int d = d0 + (lane & 15), piece = d >> 2, part = (d & 3) * 4;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int r = r0 + 4 * g + (e & 3) + (e >> 2) * 16;
                f[e] = *(const float *)(lds + place(r, piece) + part);
            }
            return f;
        }
    }
};

// Brings rows of a tensor into a tile.  VEC: 16-byte pieces of rows are aligned and whole; they go straight into LDS.
// Otherwise values are read one by one.  What is outside (rows from `left` on, values from dim on) becomes zero.
// REPEAT: rows from `left` on repeat the last one instead (left > 0), so that every load reads something.
template <class T, int DP, int ROWS, bool VEC, int THREADS, bool REPEAT = false>
struct TileReader {
    typedef Tile<T, DP> L;
    static constexpr int ALL = ROWS * L::PIECES, LOADS = (ALL + THREADS - 1) / THREADS;
    static_assert(ALL % 64 == 0, "whole wavefronts of pieces");
    static __device__ __forceinline__ void read(const T *first, long long token, int left, int dim, char *lds, int tid)
    {
        const int lane = tid & 63, wave = THREADS > 64 ? __builtin_amdgcn_readfirstlane(tid >> 6) : 0;
        if constexpr (VEC) {
            const int rows = left < ROWS ? left : ROWS;
            const unsigned pitch = (unsigned)token * (unsigned)sizeof(T);
            __amdgpu_buffer_rsrc_t res = __builtin_amdgcn_make_buffer_rsrc(
                (void *)first, 0, rows > 0 ? (unsigned)(rows - 1) * pitch + (unsigned)(dim * sizeof(T)) : 0, 0x00020000);
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int at = (u * (THREADS / 64) + wave) * 64, c = at + lane;
                if (at >= ALL) break;
                const int r = c / L::PIECES, piece = (c % L::PIECES) ^ L::swizzle(r), from = REPEAT && r >= rows ? rows - 1 : r;
                unsigned off = (unsigned)from * pitch + (unsigned)piece * 16;
                off = from < rows && piece * L::EACH < dim ? off : 0x80000000u;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(res, (lds_void *)(lds + at * 16), 16, (int)off, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                if (u * THREADS + tid >= ALL) break;
                const int c = u * THREADS + tid, r = c / L::PIECES, piece = (c % L::PIECES) ^ L::swizzle(r);
                typedef T pieces __attribute__((ext_vector_type(L::EACH)));
                pieces p;
#pragma unroll
                for (int e = 0; e < L::EACH; ++e) {
                    const int d = piece * L::EACH + e;
                    p[e] = r < left && d < dim ? first[(long long)r * token + d] : (T)0.f;
                }
                *(pieces *)(lds + c * 16) = p;
            }
        }
    }
};

// A fragment straight from memory: row `row` (nullptr: zeros), values 32 c + 8 g + 0 .. 7.
template <class T, bool VEC>
__device__ __forceinline__ typename Frag<T>::type read_fragment(const T *row, int d0, int dim)
{
    typename Frag<T>::type f;
    if constexpr (VEC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (T)0.f;
        if (row && d0 < dim) {
            constexpr int EACH = 16 / (int)sizeof(T);
            typedef T pieces __attribute__((ext_vector_type(EACH)));
#pragma unroll
            for (int h = 0; h < 8 / EACH; ++h)
                if (d0 + h * EACH < dim) {
                    const pieces p = *(const pieces *)(row + d0 + h * EACH);
#pragma unroll
                    for (int e = 0; e < EACH; ++e) f[h * EACH + e] = p[e];
                }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = row && d0 + e < dim ? row[d0 + e] : (T)0.f;
    }
    return f;
}

}  // namespace lcn
