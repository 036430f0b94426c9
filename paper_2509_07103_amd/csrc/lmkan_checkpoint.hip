// Activations to 8-bit checkpoints and back.  A block of 32 columns shares a power of two, so that both directions are
// exact but for the one rounding to a whole number, and a value (7 bits and a sign) is exact in 16-bit types too.
#include "lmkan_rows.h"

namespace lmkan {

namespace {

// 32 lanes a block of a row
__global__ __launch_bounds__(256) void checkpoint_kernel(int64_t blocks, int cols, int dtype, bool relu, const void *x, int8_t *codes, uint8_t *exps)
{
    const int per_row = exp_blocks(cols);
    for (int64_t b = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); b < blocks; b += (int64_t)gridDim.x * 8) {
        const int64_t row = b / per_row;
        const int col = (int)(b - row * per_row) * kBlock + (threadIdx.x & 31);
        const float v = col < cols ? rectify(load_as_float(x, row * cols + col, dtype), relu) : 0.0f;
        uint32_t top = magnitude_bits(v);
        for (int d = 16; d > 0; d >>= 1) {
            const uint32_t other = (uint32_t)__shfl_xor((int)top, d, 64);
            top = top > other ? top : other;
        }
        const int byte = block_byte(top);
        if (col < cols) codes[row * cols + col] = (int8_t)code_of(v, byte);
        if ((threadIdx.x & 31) == 0) exps[b] = (uint8_t)byte;
    }
}

__global__ __launch_bounds__(256) void restore_kernel(int64_t elems, int cols, int dtype, bool relu, const int8_t *codes, const uint8_t *exps,
                                                      const float *weight, const float *bias, void *y)
{
    const int per_row = exp_blocks(cols);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < elems; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / cols;
        const int col = (int)(i - row * cols);
        float v = value_of(codes[i], exps[row * per_row + col / kBlock]);
        v = fmaf(weight ? weight[col] : 1.0f, v, bias ? bias[col] : 0.0f);
        store_from_float(y, i, dtype, rectify(v, relu));
    }
}

int64_t at_most(int64_t n, int64_t most) { return n < most ? n : most; }

}  // namespace

void launch_checkpoint(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, uint8_t *exps, hipStream_t stream)
{
    const int64_t blocks = rows * exp_blocks(cols);
    checkpoint_kernel<<<(unsigned)at_most((blocks + 7) / 8, 8192), 256, 0, stream>>>(blocks, cols, dtype, relu, x, codes, exps);
}

void launch_restore(int64_t rows, int cols, int dtype, bool relu, const int8_t *codes, const uint8_t *exps, const float *weight,
                    const float *bias, void *y, hipStream_t stream)
{
    const int64_t elems = rows * cols;
    restore_kernel<<<(unsigned)at_most((elems + 255) / 256, 8192), 256, 0, stream>>>(elems, cols, dtype, relu, codes, exps, weight, bias, y);
}

}  // namespace lmkan
