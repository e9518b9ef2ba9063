// Shared by the kernels of the gated layer: what its forward pass keeps, its gates and their slopes.
#pragma once

#include "fragments.h"

namespace lcn {

// ---- what is kept of g and u: rows x 2 (g, u) x padded(d_out), in pieces of eight values ----
// Float: as they are.  bf16 tensors: eight 16-bit words, of which the upper 15 bits are a value's multiple of a power of two and the
// lowest is a bit of the piece's exponent code, so that a piece is 16 bytes.  The code is the largest value's exponent field (15 at
// least): multiples are rounded to half of 2^-14 of the power of two above the largest value, 1.8e-5 of it in the root mean square where
// bf16 leaves 1.6e-3 of each value.  Code 255, with a value that is not finite: the words are bf16, but for their lowest bits.
template <class T>
struct Keep;
template <>
struct Keep<float> {
    typedef float type;
    static __device__ __forceinline__ void store(float *p, const f32x4 (&v)[2])
    {
        ((f32x4 *)p)[0] = v[0];
        ((f32x4 *)p)[1] = v[1];
    }
    static __device__ __forceinline__ void load(const float *p, f32x4 (&v)[2])
    {
        v[0] = ((const f32x4 *)p)[0];
        v[1] = ((const f32x4 *)p)[1];
    }
};
template <>
struct Keep<__bf16> {
    typedef unsigned short type;
    typedef unsigned words __attribute__((ext_vector_type(4)));   // values 2 i and 2 i + 1 of the piece
    static __device__ __forceinline__ void store(unsigned short *p, const f32x4 (&v)[2])
    {
        unsigned top = 15u << 23;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = v[e >> 2][e & 3];
            const unsigned b = __builtin_bit_cast(unsigned, x) & 0x7fffffffu;
            top = b > top ? b : top;
        }
        const unsigned code = top >> 23;
        words w;
        if (code < 255) {
            // multiples of up to 16383: 2^(140 - code) 16383 / 16384; adding 3 * 2^22 leaves them in the lowest bits, rounded
            const float scale = __builtin_bit_cast(float, (267u - code) << 23) * (16383.f / 16384.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = __builtin_fmaf(v[i >> 1][(i & 1) * 2], scale, 12582912.f);
                const float b = __builtin_fmaf(v[i >> 1][(i & 1) * 2 + 1], scale, 12582912.f);
                w[i] = (__builtin_bit_cast(unsigned, a) << 1 & 0xfffeu) | __builtin_bit_cast(unsigned, b) << 17;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned short a = __builtin_bit_cast(unsigned short, (__bf16)v[i >> 1][(i & 1) * 2]);
                const unsigned short b = __builtin_bit_cast(unsigned short, (__bf16)v[i >> 1][(i & 1) * 2 + 1]);
                w[i] = (a & 0xfffeu) | (b & 0xfffeu) << 16;
            }
        }
        const unsigned bits = (code & 15u) | (code & 0xf0u) << 12;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] |= bits >> i & 0x10001u;
        *(words *)p = w;
    }
    static __device__ __forceinline__ void load(const unsigned short *p, f32x4 (&v)[2])
    {
        const words w = *(const words *)p;
        unsigned bits = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) bits |= (w[i] & 0x10001u) << i;
        const unsigned code = (bits & 15u) | (bits >> 12 & 0xf0u);
        // 2^(code - 141), the words being twice the multiples
        const float scale = __builtin_bit_cast(float, (code - 14u) << 23) * (16384.f / 16383.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned one = w[i] & 0xfffeu, two = w[i] & 0xfffe0000u;
            v[i >> 1][(i & 1) * 2] = (float)(short)one * scale;
            v[i >> 1][(i & 1) * 2 + 1] = (float)((int)two >> 16) * scale;
        }
        if (code == 255)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i >> 1][(i & 1) * 2] = __builtin_bit_cast(float, (w[i] & 0xfffeu) << 16);
                v[i >> 1][(i & 1) * 2 + 1] = __builtin_bit_cast(float, w[i] & 0xfffe0000u);
            }
    }
};

// act(g), and its slope.  With bf16 tensors the sigmoid is the exponential and reciprocal instructions alone, each within 2^-22: the
// kernels here are bound by such operations otherwise (gated_slope_kernel 192 us instead of 138 for 16391 x 4096).
template <class T>
__device__ __forceinline__ float sigmoid(float z)
{
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.f + exp2_fast(z * -1.44269504088896341f));
    return 1.f / (1.f + expf(-z));
}
template <class T, int ACT>
__device__ __forceinline__ float gate(float g)
{
    if constexpr (ACT == LCN_ACT_SILU) return g * sigmoid<T>(g);
    return activate<ACT>(g);
}
template <class T, int ACT>
__device__ __forceinline__ void gate_and_slope(float g, float &a, float &slope)
{
    if constexpr (ACT == LCN_ACT_SILU) {
        const float f = sigmoid<T>(g);
        a = g * f;
        slope = __builtin_fmaf(a, 1.f - f, f);
    } else if constexpr (ACT == LCN_ACT_TANH) {
        a = tanhf(g);
        slope = 1.f - a * a;
    } else if constexpr (ACT == LCN_ACT_GELU) {
        const float f = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        a = g * f;
        slope = f + g * expf(-0.5f * g * g) * 0.39894228040143268f;
    } else {
        a = activate<ACT>(g);
        slope = activate_slope<ACT>(g);
    }
}

template <class T>
struct GatedArgs {
    const T *bias;   // 2 width
    T *y;
    typename Keep<T>::type *kept;   // nullable
    int act;
};

// Narrow layers (kernels_gated_narrow.hip): up to 64 inputs and outputs, on many rows.
bool gated_narrow(int64_t rows, int32_t d_in, int32_t d_out);
// Some rows of floats (the same file), more than FEW_ROWS.
bool gated_some(int64_t rows, int32_t d_in, int32_t dtype);
hipError_t launch_gated_some(const GatedArgs<float> &e, const float *x, const float *w, int rows, int d_in, int d_out, hipStream_t s);
// workgroups of the backward pass of narrow layers, each of which leaves partial sums of dW and db, 2 d_out (d_in + 1) floats
int gated_narrow_groups(int64_t rows);
template <class T>
hipError_t launch_gated_narrow(const GatedArgs<T> &e, const T *x, const T *w, int64_t rows, int32_t d_in, int32_t d_out, hipStream_t s);
template <class T>
hipError_t launch_gated_narrow_backward(const T *x, const T *w, const typename Keep<T>::type *kept, const T *dy, int64_t rows, int32_t d_in,
                                        int32_t d_out, int32_t act, T *dx, T *dw, T *db, float *part, hipStream_t s);

}  // namespace lcn
