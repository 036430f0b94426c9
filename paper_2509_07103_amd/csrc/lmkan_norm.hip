// Layer norm over the columns of rows, and its gradients.
#include "lmkan_rows.h"

namespace lmkan {

namespace {

constexpr int kThreads = 256;

template <class V>
__device__ __forceinline__ V wave_sum(V v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Sum over a workgroup, the same in every thread
template <class V>
__device__ __forceinline__ V group_sum(V v, V *shared)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < kThreads / 64; ++w) v += shared[w];
    return v;
}

struct NormArgs {
    int64_t rows;
    int cols, x_dtype, y_dtype;
    float eps;
    const void *x;
    const float *weight, *bias;
    void *y;
    float *stats;
    int8_t *codes;
    uint8_t *exps;
};

__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a)
{
    __shared__ double sums[kThreads / 64];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = row * a.cols;
        double sum = 0.0;
        for (int c = threadIdx.x; c < a.cols; c += kThreads) sum += (double)load_as_float(a.x, at + c, a.x_dtype);
        const double centre = group_sum(sum, sums) / a.cols;
        sum = 0.0;
        for (int c = threadIdx.x; c < a.cols; c += kThreads) {
            const double d = (double)load_as_float(a.x, at + c, a.x_dtype) - centre;
            sum += d * d;
        }
        const float mean = (float)centre, rstd = (float)(1.0 / sqrt(group_sum(sum, sums) / a.cols + (double)a.eps));
        if (a.stats && threadIdx.x == 0) a.stats[2 * row] = mean, a.stats[2 * row + 1] = rstd;
        for (int c0 = 0; c0 < a.cols; c0 += kThreads) {
            const int c = c0 + threadIdx.x;
            const float hat = c < a.cols ? __fmul_rn(__fsub_rn(load_as_float(a.x, at + c, a.x_dtype), mean), rstd) : 0.0f;
            if (a.codes) {
                uint32_t top = magnitude_bits(hat);
                for (int d = 16; d > 0; d >>= 1) {
                    const uint32_t other = (uint32_t)__shfl_xor((int)top, d, 64);
                    top = top > other ? top : other;
                }
                const int byte = block_byte(top);
                if (c < a.cols) a.codes[at + c] = (int8_t)code_of(hat, byte);
                if ((threadIdx.x & 31) == 0 && c < a.cols) a.exps[row * exp_blocks(a.cols) + c / kBlock] = (uint8_t)byte;
            }
            if (c < a.cols) store_from_float(a.y, at + c, a.y_dtype, fmaf(a.weight ? a.weight[c] : 1.0f, hat, a.bias ? a.bias[c] : 0.0f));
        }
    }
}

__device__ __forceinline__ float hat_of(const NormShape &s, const NormBackwardArgs &a, int64_t row, int c)
{
    const int64_t at = row * s.cols + c;
    if (!a.x) return value_of(a.codes[at], a.exps[row * exp_blocks(s.cols) + c / kBlock]);
    return (load_as_float(a.x, at, s.x_dtype) - a.stats[2 * row]) * a.stats[2 * row + 1];
}

__global__ __launch_bounds__(kThreads) void norm_grad_x_kernel(NormShape s, NormBackwardArgs a)
{
    __shared__ float sums[kThreads / 64];
    for (int64_t row = blockIdx.x; row < s.rows; row += gridDim.x) {
        const float rstd = a.stats[2 * row + 1];
        float d = 0.0f, dh = 0.0f;
        for (int c = threadIdx.x; c < s.cols; c += kThreads) {
            const float g = load_as_float(a.grad_y, row * s.cols + c, s.y_dtype) * (a.weight ? a.weight[c] : 1.0f);
            d += g, dh += g * hat_of(s, a, row, c);
        }
        d = group_sum(d, sums) / s.cols;
        dh = group_sum(dh, sums) / s.cols;
        for (int c = threadIdx.x; c < s.cols; c += kThreads) {
            const float g = load_as_float(a.grad_y, row * s.cols + c, s.y_dtype) * (a.weight ? a.weight[c] : 1.0f);
            store_from_float(a.grad_x, row * s.cols + c, s.x_dtype, rstd * (g - d - hat_of(s, a, row, c) * dh));
        }
    }
}

constexpr int kParts = 256;

// A column a thread, every kParts-th row; parts [2][kParts][cols]
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(NormShape s, NormBackwardArgs a, float *parts)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= s.cols) return;
    float w = 0.0f, b = 0.0f;
    for (int64_t row = blockIdx.y; row < s.rows; row += kParts) {
        const float g = load_as_float(a.grad_y, row * s.cols + c, s.y_dtype);
        b += g, w += g * hat_of(s, a, row, c);
    }
    parts[(int64_t)blockIdx.y * s.cols + c] = w;
    parts[(int64_t)(kParts + blockIdx.y) * s.cols + c] = b;
}

__global__ __launch_bounds__(kThreads) void norm_join_kernel(NormShape s, NormBackwardArgs a, const float *parts)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    float *to = blockIdx.y ? a.grad_bias : a.grad_weight;
    if (c >= s.cols || !to) return;
    float sum = 0.0f;
    if (s.rows > 0)
        for (int p = 0; p < kParts; ++p) sum += parts[((int64_t)blockIdx.y * kParts + p) * s.cols + c];
    to[c] = s.accumulate ? to[c] + sum : sum;
}

}  // namespace

void launch_layer_norm(const NormShape &s, const void *x, const float *weight, const float *bias, void *y, float *stats, int8_t *codes,
                       uint8_t *exps, hipStream_t stream)
{
    const NormArgs a{s.rows, s.cols, s.x_dtype, s.y_dtype, s.eps, x, weight, bias, y, stats, codes, exps};
    norm_kernel<<<(unsigned)(s.rows < 65536 ? s.rows : 65536), kThreads, 0, stream>>>(a);
}

size_t layer_norm_backward_workspace_bytes(const NormShape &s) { return s.rows ? (size_t)2 * kParts * s.cols * sizeof(float) : 0; }

void launch_layer_norm_backward(const NormShape &s, const NormBackwardArgs &a, void *workspace, hipStream_t stream)
{
    if (a.grad_x && s.rows > 0) norm_grad_x_kernel<<<(unsigned)(s.rows < 65536 ? s.rows : 65536), kThreads, 0, stream>>>(s, a);
    if (!a.grad_weight && !a.grad_bias) return;
    float *parts = static_cast<float *>(workspace);
    const unsigned across = (s.cols + kThreads - 1) / kThreads;
    if (s.rows > 0) norm_columns_kernel<<<dim3(across, kParts), kThreads, 0, stream>>>(s, a, parts);
    norm_join_kernel<<<dim3(across, 2), kThreads, 0, stream>>>(s, a, parts);
}

}  // namespace lmkan
