// Host-callable launchers of the dense companions of the layer (lmkan_ortho.hip, lmkan_linear.hip).
// Every launcher enqueues on the given stream and returns; arguments have been validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lmkan.h"

namespace lmkan {

// A batch of matrices seen with the shorter side first: m x n, the transpose of what is stored when `flip`.
struct MatrixShape {
    int64_t batch;
    int rows, cols;
    int dtype;
    float eps;
    __host__ __device__ bool flip() const { return rows > cols; }
    __host__ __device__ int m() const { return rows > cols ? cols : rows; }
    __host__ __device__ int n() const { return rows > cols ? rows : cols; }
    __host__ __device__ int64_t elems() const { return (int64_t)rows * cols; }
};

// What a step does around the products: the update's direction from gradient and momentum, and the weights.
// Plain orthogonalisation is the case without momentum (null) that writes `out`.
struct UpdateArgs {
    const void *grad;   // or x; in the shape's dtype
    float *momentum;    // null: the direction is `grad` itself
    float *weight;      // null: the result goes to `out`
    void *out;          // in the shape's dtype
    float beta;
    bool nesterov;
    float keep;         // W <- keep W + add O
    float add;
};

// What the steps of a schedule can make of singular values in [0, 1]; false when a coefficient is not finite or
// a step exceeds the limits below.
constexpr double kMaxSingular = 4.0, kMaxFactor = 64.0;
struct ScheduleBounds {
    float singular[LMKAN_MAX_ORTHO_STEPS + 1];  // largest singular value before step k (and after the last)
    float factor[LMKAN_MAX_ORTHO_STEPS];        // largest |a + b s^2 + c s^4| of step k
};
bool schedule_bounds(int steps, const float *schedule, ScheduleBounds *bounds);

// Steps that are taken on one Gram matrix before the polynomial is applied and a new one is formed: the step after the
// last of those that begin with step k (lmkan_ortho.hip)
int steps_until(const MatrixShape &s, const ScheduleBounds &bounds, int steps, int k);

// The power of two that brings values up to `bound` to the upper end of float16's range (65504), with room for rounding.
// Bounds end at 2^-113, so that every scale and every inverse of one is a float32 value: what a schedule takes below
// that has fewer bits, and none from 2^-152 on.
float pair_scale(double bound);

// A step on a Gram matrix A held in pairs: what takes products of pairs to pairs of their results.  (Worked out in
// float64: of scales that are far apart no two may be multiplied in float32 first.)
struct ChainStep {
    float a, b, c;                   // B = a I + b A + c A^2, from pairs of A and their products
    float to_w, to_gram, to_p;       // B A, (B A) B and B P
    float step_inverse, p_inverse;   // of the scales of B, and of P before the step
};
// `factor`: the product of the factors of the steps before on the same Gram matrix, and of this one afterwards
ChainStep chain_step(const ScheduleBounds &bounds, const float *schedule, int k, double *factor);

// Workgroups of a launch at most, of up to 1024 threads: the runtime takes fewer than 2^32 threads along a dimension
constexpr int64_t kMostGroups = 1 << 21;

size_t ortho_workspace_bytes(const MatrixShape &s);
void launch_ortho(const MatrixShape &s, int steps, const float *schedule, const UpdateArgs &u, void *workspace,
                  hipStream_t stream);

// Matrices whose shorter side is at most 64 (lmkan_ortho_small.hip); reached through launch_ortho
bool ortho_small_applicable(const MatrixShape &s, int steps);
size_t ortho_small_workspace_bytes(const MatrixShape &s);
void launch_ortho_small(const MatrixShape &s, int steps, const float *schedule, const UpdateArgs &u, void *workspace,
                        hipStream_t stream);

struct LinearShape {
    int64_t batch;
    int n_in, n_out;
    int x_dtype, y_dtype;
    bool relu;
};

void launch_quantize_rows(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, float *scale,
                          hipStream_t stream);
size_t linear_i8_workspace_bytes(const LinearShape &s);
void launch_linear_i8(const LinearShape &s, const void *x, const int8_t *w, const float *w_scale, const float *bias,
                      float beta, void *y, void *workspace, hipStream_t stream);

// Element types by their lmkan_dtype
__device__ __forceinline__ float load_as_float(const void *p, int64_t i, int dtype)
{
    if (dtype == LMKAN_F32) return static_cast<const float *>(p)[i];
    const uint16_t b = static_cast<const uint16_t *>(p)[i];
    if (dtype == LMKAN_F16) return (float)__builtin_bit_cast(_Float16, b);
    return __builtin_bit_cast(float, (uint32_t)b << 16);
}

// float32 -> bfloat16, to nearest, ties to even; NaN stays NaN
__device__ __forceinline__ uint16_t bf16_bits(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);
    return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1)) >> 16);
}

__device__ __forceinline__ void store_from_float(void *p, int64_t i, int dtype, float v)
{
    if (dtype == LMKAN_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == LMKAN_F16) static_cast<uint16_t *>(p)[i] = __builtin_bit_cast(uint16_t, (_Float16)v);
    else static_cast<uint16_t *>(p)[i] = bf16_bits(v);
}

// The direction's element `at` in two halves, so that many loads can be under way: what it is made of, and the element.
// `move`: the momentum moves.
struct Raw {
    float g, m;
};
__device__ __forceinline__ Raw fetch(const UpdateArgs &u, int dtype, int64_t at, bool move)
{
    Raw r;
    r.g = !u.momentum || u.nesterov || move ? load_as_float(u.grad, at, dtype) : 0.0f;
    r.m = u.momentum ? u.momentum[at] : 0.0f;
    return r;
}
__device__ __forceinline__ float direction(const UpdateArgs &u, Raw r, int64_t at, bool move)
{
    if (!u.momentum) return r.g;
    if (move) u.momentum[at] = r.m = u.beta * r.m + (1.0f - u.beta) * r.g;
    return u.nesterov ? u.beta * r.m + (1.0f - u.beta) * r.g : r.m;
}

// two adjacent 16-bit elements, the first in the lower half
__device__ __forceinline__ uint32_t two_from_float(int dtype, float a, float b)
{
    if (dtype == LMKAN_F16)
        return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
    return (uint32_t)bf16_bits(a) | (uint32_t)bf16_bits(b) << 16;
}

}  // namespace lmkan
