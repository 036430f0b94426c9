// Gradients of the linear term's weights and bias from a checkpoint of its input.
#include "lmkan_rows.h"

namespace lmkan {

namespace {

struct GradArgs {
    int64_t batch;
    int n_in, n_out, dtype;
    bool relu, accumulate;
    const int8_t *codes;
    const uint8_t *exps;
    const void *grad_y;
    float *grad_weight, *grad_bias;
};

// 32 x 32 results of a workgroup, four a thread, 32 rows of the batch at a time
__global__ __launch_bounds__(256) void linear_grad_kernel(GradArgs a)
{
    __shared__ float g[32][33], v[32][33];
    const int across = (a.n_in + 31) / 32, ti = blockIdx.x / across, tj = blockIdx.x - ti * across;
    const int j0 = ti * 32, e0 = tj * 32, lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    float acc[4] = {}, bias[4] = {};
    for (int64_t n0 = 0; n0 < a.batch; n0 += 32) {
        for (int k = part; k < 32; k += 8) {
            const int64_t n = n0 + k;
            const int j = j0 + lane, e = e0 + lane;
            g[k][lane] = n < a.batch && j < a.n_out ? load_as_float(a.grad_y, n * a.n_out + j, a.dtype) : 0.0f;
            v[k][lane] = n < a.batch && e < a.n_in
                             ? rectify(value_of(a.codes[n * a.n_in + e], a.exps[n * exp_blocks(a.n_in) + e / kBlock]), a.relu)
                             : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < 32; ++k)
            for (int i = 0; i < 4; ++i) {
                acc[i] = fmaf(g[k][part * 4 + i], v[k][lane], acc[i]);
                bias[i] += g[k][part * 4 + i];
            }
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int j = j0 + part * 4 + i, e = e0 + lane;
        if (j >= a.n_out) continue;
        if (e < a.n_in) {
            float *to = a.grad_weight + (int64_t)j * a.n_in + e;
            *to = a.accumulate ? *to + acc[i] : acc[i];
        }
        if (a.grad_bias && e == 0) a.grad_bias[j] = a.accumulate ? a.grad_bias[j] + bias[i] : bias[i];
    }
}

}  // namespace

size_t linear_grad_workspace_bytes(const LinearShape &) { return 0; }

void launch_linear_grad(const LinearShape &s, bool accumulate, const int8_t *codes, const uint8_t *exps, const void *grad_y,
                        float *grad_weight, float *grad_bias, void *, hipStream_t stream)
{
    const GradArgs a{s.batch, s.n_in, s.n_out, s.y_dtype, s.relu, accumulate, codes, exps, grad_y, grad_weight, grad_bias};
    const int64_t tiles = (int64_t)((s.n_in + 31) / 32) * ((s.n_out + 31) / 32);
    linear_grad_kernel<<<(unsigned)tiles, 256, 0, stream>>>(a);
}

}  // namespace lmkan
