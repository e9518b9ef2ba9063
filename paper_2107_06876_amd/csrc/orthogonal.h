// Products of the orthogonalisation: matrices in two planes of fp16, a batch of them in one launch.
//
// x1 = fp16(x), x2 = fp16(x - x1) leave 2^-24 |x| where x2 is no subnormal, and the three products but x2 y2 are as exact as a
// single-precision one, at half the cost of the six of three bf16 planes.  That takes values whose range is known.
#pragma once

#include "fragments.h"

namespace lcn {

typedef _Float16 f16;
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));

// the same for a register's bits as fp16
__device__ __forceinline__ f32x4 mfma_f16(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}


// The largest singular value of X that a step may leave, the largest of a + b t + c t^2 in its way, and what X, A and B are
// multiplied with: values up to 32 768 of fp16's 65 504.
constexpr double MOST_X = 4.0, MOST_POLY = 64.0;
constexpr float SCALE_X = 8192.f, SCALE_A = 2048.f, SCALE_B = 512.f;
constexpr int MOST_STEPS = 64, NORM_GROUPS = 64;
struct SmallSteps {
    float c[MOST_STEPS][3];
};

// Matrices in two planes, one behind the other: rows of `ld` values, ld a multiple of 8, zeros behind a row's values
struct Planes {
    f16 *p;
    long long plane, ld;   // values from a plane to the next, from a row to the next
};

__device__ __forceinline__ void store_planes(const Planes &o, long long at, const f32x4 (&v)[2])
{
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[e >> 2][e & 3];
        hi[e] = (f16)x;
        lo[e] = (f16)(x - (float)hi[e]);
    }
    *(f16x8 *)(o.p + at) = hi;
    *(f16x8 *)(o.p + o.plane + at) = lo;
}

struct PairArgs {
    Operand a, b;
    long long a_batch, b_batch;   // bytes from a matrix to the next
    float *part;                  // with splits: sums of [split][tile], in the order of the accumulators
    int m, n, k, splits, batches, tiles_m, tiles_n;
};

// Planes of both operands, and whether the small products are added up by themselves: sums of a float's precision, at the cost of
// registers, so not for the largest tile.
enum { PAIR_ONE = 0, PAIR_TWO = 1, PAIR_FLOAT = 2 };

// tile shapes
enum { PAIR_256 = 0, PAIR_128 = 1, PAIR_64 = 2, PAIR_32 = 3, PAIR_SHAPES = 4 };
inline int pair_tile_of(int shape) { return shape == PAIR_256 ? 256 : shape == PAIR_128 ? 128 : shape == PAIR_64 ? 64 : 32; }
struct PairPlan {
    int shape, splits;   // workgroups that share a tile's k
};
PairPlan plan_pair(long long m, long long n, long long k, long long batches, bool symmetric, bool bf16);
// bytes of the partial sums of a symmetric product of n x n
inline size_t pair_part_bytes(const PairPlan &p, long long n, long long batches)
{
    const long long w = pair_tile_of(p.shape), t = (n + w - 1) / w;
    return p.splits > 1 ? (size_t)(p.splits * batches * (t * (t + 1) / 2)) * w * w * 4 : 0;
}

// A symmetric result in planes: factor * ratio^2 * product + linear * gram + constant on the diagonal
struct GramArgs {
    Planes out;
    long long batch;      // values from a matrix to the next, of out and gram
    Planes gram;          // p: nullable
    float factor, linear, constant;
    const float *ratio;   // of every matrix, nullable (1)
};
// X in planes: factor * ratio * product
struct ApplyArgs {
    Planes out;
    long long batch;
    float factor;
    const float *ratio;
};
// the same, rounded to the caller's type: float with PAIR_FLOAT, else bf16
struct LastArgs {
    void *out;
    long long batch, ld;
    float factor;
    const float *ratio;
};
// wide: both operands lie with k contiguous, else with their own index
hipError_t launch_gram(const PairPlan &plan, const PairArgs &p, const GramArgs &e, bool wide, int planes, hipStream_t s);
// wide: a = X with its own index contiguous, b = B;  else a = B, b = X, both with k contiguous.  PAIR_ONE: X is one plane.
hipError_t launch_apply(const PairPlan &plan, const PairArgs &p, const ApplyArgs &e, bool wide, int planes, hipStream_t s);
hipError_t launch_apply_last(const PairPlan &plan, const PairArgs &p, const LastArgs &e, bool wide, int planes, hipStream_t s);

}  // namespace lcn
