// What the operators on rows share (lmkan_norm.hip, lmkan_checkpoint.hip, lmkan_linear_grad.hip, lmkan_adapters.hip):
// their launchers, the blocks of a checkpoint.
// Every launcher enqueues on the given stream and returns; arguments have been validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lmkan_dense.h"

namespace lmkan {

constexpr int kBlock = LMKAN_CHECKPOINT_BLOCK;
constexpr int kExpBias = 133, kMostExp = 121;   // a block's byte is its exponent + 133
constexpr int kExpNan = 255;

__host__ __device__ __forceinline__ int exp_blocks(int cols) { return (cols + kBlock - 1) / kBlock; }

// The byte of a block whose largest magnitude has the bits `top` (ordered like the values; NaN above infinity)
__device__ __forceinline__ int block_byte(uint32_t top)
{
    if (top >= 0x7f800000u) return kExpNan;
    if (top == 0) return 0;
    const float t = __builtin_bit_cast(float, top);
    int e = __builtin_amdgcn_frexp_expf(t) - 7;                        // t / 2^e in [64, 128)
    e += rintf(__builtin_amdgcn_ldexpf(t, -e)) > 127.0f;
    e = e < -kExpBias ? -kExpBias : e > kMostExp ? kMostExp : e;
    return e + kExpBias;
}

// Code of an element of a block (top finite), and the value that a code stands for.  Both scalings are exact, so that
// rounding to a whole number is the only one.
__device__ __forceinline__ int code_of(float v, int byte)
{
    if (byte == kExpNan) return 0;
    const float c = rintf(__builtin_amdgcn_ldexpf(v, kExpBias - byte));
    return (int)(c > 127.0f ? 127.0f : c < -127.0f ? -127.0f : c);
}
__device__ __forceinline__ float value_of(int code, int byte)
{
    return byte == kExpNan ? __builtin_nanf("") : __builtin_amdgcn_ldexpf((float)code, byte - kExpBias);
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
// max(v, 0); a NaN stays one
__device__ __forceinline__ float rectify(float v, bool relu) { return relu && v < 0.0f ? 0.0f : v; }

struct NormShape {
    int64_t rows;
    int cols;
    int x_dtype, y_dtype;
    float eps;
    bool accumulate;
};

struct NormBackwardArgs {
    const void *x;          // or null, and the checkpoint
    const int8_t *codes;
    const uint8_t *exps;
    const float *stats, *weight;
    const void *grad_y;
    void *grad_x;
    float *grad_weight, *grad_bias;
};

void launch_checkpoint(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, uint8_t *exps, hipStream_t stream);
void launch_restore(int64_t rows, int cols, int dtype, bool relu, const int8_t *codes, const uint8_t *exps, const float *weight,
                    const float *bias, void *y, hipStream_t stream);

void launch_layer_norm(const NormShape &s, const void *x, const float *weight, const float *bias, void *y, float *stats, int8_t *codes,
                       uint8_t *exps, hipStream_t stream);
size_t layer_norm_backward_workspace_bytes(const NormShape &s);
void launch_layer_norm_backward(const NormShape &s, const NormBackwardArgs &a, void *workspace, hipStream_t stream);

// y_dtype: of grad_y
size_t linear_grad_workspace_bytes(const LinearShape &s);
void launch_linear_grad(const LinearShape &s, bool accumulate, const int8_t *codes, const uint8_t *exps, const void *grad_y,
                        float *grad_weight, float *grad_bias, void *workspace, hipStream_t stream);

struct AdapterShape {
    int64_t batch;
    int count, rank, n_in, n_out;
    int dtype, x_dtype, y_dtype;
    bool relu;
};
size_t adapters_workspace_bytes(const AdapterShape &s);
void launch_adapters(const AdapterShape &s, const void *x, const int32_t *index, const void *a, const void *b, const float *scale, void *y,
                     void *workspace, hipStream_t stream);

}  // namespace lmkan
