// Shared by the kernels of the gated layer: what its forward pass keeps, its gates and their slopes.
#pragma once

#include "fragments.h"

namespace lcn {

// ---- what is kept of g and u: rows x 2 (g, u) x padded(d_out), in pieces of eight values ----
// Float: as they are.  bf16 tensors: eight 16-bit words, 16 bytes, of which the upper 15 bits are a value and the lowest is a bit of the
// piece's code: E, the exponent field of its largest value, rounded up to an even number, and whether its values are far apart.
//   Near, all from 2^-13 of the largest on: sign, 4 bits of exponent below E's and 10 of significand: within 2^-11 of each value, 2.1e-4
//   of it in the root mean square, where bf16 leaves 1.6e-3.  Eight normally distributed values are 999 times in 1000.
//   Far, all but zeros from 2^-27 of the largest on: 5 bits of exponent and 9 of significand, within 2^-10 of each value.
//   Farther, or with a value that is not finite (code 0): bf16 with 6 bits of significand, within 2^-7.
// So a value is as exact beside a large one as elsewhere; one exponent and 15-bit multiples for all eight are 1 % off beside one 2^8 times
// as large (16 391 rows, 1024 -> 4096, a training step 980 us with those, 990 so).  Zeros stay zeros.
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
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ unsigned as_fp16(float a, float b) { return __builtin_bit_cast(unsigned, pair{(_Float16)a, (_Float16)b}); }
    static __device__ __forceinline__ unsigned bits_of(float x) { return __builtin_bit_cast(unsigned, x); }
    static __device__ __forceinline__ float value_of(unsigned b) { return __builtin_bit_cast(float, b); }
    static __device__ __forceinline__ float value(const f32x4 (&v)[2], int e) { return v[e >> 2][e & 3]; }
    // sign and 14 bits, rounded; finite values stay finite
    static __device__ __forceinline__ unsigned short_bf16(float x)
    {
        constexpr unsigned INFINITE = 0x7f800000u;
        const unsigned b = bits_of(x) & 0x7fffffffu, up = b + 0x10000u;
        const unsigned r = b > INFINITE ? 0x7fc00000u : b == INFINITE ? b : up < INFINITE ? up : INFINITE - 1;
        return ((bits_of(x) & 0x80000000u) | r) >> 16 & 0xfffeu;
    }
    // what is not near (zeros beside other values among it): the words, and the code
    static __device__ __forceinline__ unsigned store_far(words &w, const f32x4 (&v)[2], unsigned top, int E)
    {
        unsigned least = ~0u;   // of those that are not zero, less 1
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned b = (bits_of(value(v, e)) & 0x7fffffffu) - 1;
            least = b < least ? b : least;
        }
        if (top < 0x7f800000u && (int)((least + 1) >> 23) >= E - 28) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) x[u] = __builtin_ldexpf(value_of((bits_of(value(v, 2 * i + u)) + 0x2000u) & 0xffffc000u), 141 - E);
                w[i] = as_fp16(x[0], x[1]);   // below 2^15
            }
            return (unsigned)E | 1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = short_bf16(value(v, 2 * i)) | short_bf16(value(v, 2 * i + 1)) << 16;
        return 0;
    }
    static __device__ __forceinline__ void store(unsigned short *p, const f32x4 (&v)[2])
    {
        unsigned top = 0;
        float least = __builtin_fabsf(v[0][0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned b = bits_of(value(v, e)) & 0x7fffffffu;
            top = b > top ? b : top;
            if (e) least = __builtin_fminf(least, __builtin_fabsf(value(v, e)));
        }
        int E = (int)((top >> 23) + 1) & ~1;
        E = E < 2 ? 2 : E;
        unsigned code = (unsigned)E;
        words w;
        if (E <= 252 && (int)(bits_of(least) >> 23) >= E - 14) {
            // values below 2, and a little less, so that none is rounded to 2: the exponent's highest bit stays zero
            const float scale = value_of((unsigned)(254 - E) << 23) * (4095.f / 4096.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned h = as_fp16(value(v, 2 * i) * scale, value(v, 2 * i + 1) * scale);
                w[i] = (h & 0x80008000u) | (h << 1 & 0x7ffe7ffeu);
            }
        } else {
            code = store_far(w, v, top, E);
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
        const float scale = value_of(code << 23) * (4096.f / 4095.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const pair h = __builtin_bit_cast(pair, (w[i] & 0x80008000u) | (w[i] >> 1 & 0x3fff3fffu));
            v[i >> 1][(i & 1) * 2] = (float)h[0] * scale;
            v[i >> 1][(i & 1) * 2 + 1] = (float)h[1] * scale;
        }
        if (code & 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const pair h = __builtin_bit_cast(pair, w[i] & 0xfffefffeu);
                v[i >> 1][(i & 1) * 2] = __builtin_ldexpf((float)h[0], (int)code - 142);
                v[i >> 1][(i & 1) * 2 + 1] = __builtin_ldexpf((float)h[1], (int)code - 142);
            }
        if (code == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i >> 1][(i & 1) * 2] = value_of((w[i] & 0xfffeu) << 16);
                v[i >> 1][(i & 1) * 2 + 1] = value_of(w[i] & 0xfffe0000u);
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
