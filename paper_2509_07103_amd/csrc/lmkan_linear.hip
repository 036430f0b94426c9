// The linear term in 8-bit whole numbers: rows scaled to codes one by one, products of codes summed exactly,
//   y = beta y + xscale wscale sum(xcode wcode) + bias.
#include "lmkan_dense.h"

namespace lmkan {

namespace {

// A wave per row.  The largest magnitude is found on the bits (ordered like the values for non-negative
// floats, NaN above infinity), so that a row with a NaN or an infinity ends with a scale that is not finite.
__global__ __launch_bounds__(256) void quantize_kernel(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, float *scale)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int lane = threadIdx.x & 63;
    const auto value = [&](int e) {
        const float v = load_as_float(x, row * cols + e, dtype);
        return relu && v < 0.0f ? 0.0f : v;
    };
    uint32_t top = 0;
    for (int e = lane; e < cols; e += 64) {
        const uint32_t b = __builtin_bit_cast(uint32_t, value(e)) & 0x7fffffffu;
        top = b > top ? b : top;
    }
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)top, d, 64);
        top = o > top ? o : top;
    }
    const float r = __builtin_bit_cast(float, top);
    const bool finite = top < 0x7f800000u;
    const float f = finite && 127.0f / r < INFINITY ? 127.0f / r : 0.0f;
    for (int e = lane; e < cols; e += 64) codes[row * cols + e] = finite ? (int8_t)(int)rintf(value(e) * f) : (int8_t)0;
    if (lane == 0) scale[row] = r / 127.0f;
}

constexpr int kTile = 32, kDepth = 64;

struct Args {
    const int8_t *x;
    const float *x_scale;
    const int8_t *w;
    const float *w_scale, *bias;
    float beta;
    void *y;
    int64_t batch;
    int n_in, n_out, y_dtype;
};

__global__ __launch_bounds__(256) void linear_kernel(Args a)
{
    __shared__ int8_t l[kTile][kDepth + 4], r[kTile][kDepth + 4];
    const unsigned across = (unsigned)((a.n_out + kTile - 1) / kTile);
    const int64_t i0 = (int64_t)(blockIdx.x / across) * kTile;
    const int j0 = (int)(blockIdx.x % across) * kTile, tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    int acc[4] = {};
    for (int k0 = 0; k0 < a.n_in; k0 += kDepth) {
        for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
            const int k = e & (kDepth - 1), i = e / kDepth;
            l[i][k] = i0 + i < a.batch && k0 + k < a.n_in ? a.x[(i0 + i) * a.n_in + k0 + k] : (int8_t)0;
            r[i][k] = j0 + i < a.n_out && k0 + k < a.n_in ? a.w[(int64_t)(j0 + i) * a.n_in + k0 + k] : (int8_t)0;
        }
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
            for (int p = 0; p < 4; ++p) acc[p] += (int)l[ty * 4 + p][k] * (int)r[tx][k];
        __syncthreads();
    }
    for (int p = 0; p < 4; ++p) {
        const int64_t i = i0 + ty * 4 + p;
        const int j = j0 + tx;
        if (i >= a.batch || j >= a.n_out) continue;
        float v = (float)acc[p] * (a.x_scale[i] * a.w_scale[j]) + (a.bias ? a.bias[j] : 0.0f);
        if (a.beta != 0.0f) v += a.beta * load_as_float(a.y, i * a.n_out + j, a.y_dtype);
        store_from_float(a.y, i * a.n_out + j, a.y_dtype, v);
    }
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

void launch_quantize_rows(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, float *scale, hipStream_t stream)
{
    quantize_kernel<<<(unsigned)((rows + 3) / 4), 256, 0, stream>>>(rows, cols, dtype, relu, x, codes, scale);
}

size_t linear_i8_workspace_bytes(const LinearShape &s)
{
    return align256((size_t)s.batch * s.n_in) + align256((size_t)s.batch * sizeof(float));
}

void launch_linear_i8(const LinearShape &s, const void *x, const int8_t *w, const float *w_scale, const float *bias,
                      float beta, void *y, void *workspace, hipStream_t stream)
{
    int8_t *codes = static_cast<int8_t *>(workspace);
    float *scale = reinterpret_cast<float *>(codes + align256((size_t)s.batch * s.n_in));
    launch_quantize_rows(s.batch, s.n_in, s.x_dtype, s.relu, x, codes, scale, stream);
    const Args a{codes, scale, w, w_scale, bias, beta, y, s.batch, s.n_in, s.n_out, s.y_dtype};
    const int64_t tiles = ((s.batch + kTile - 1) / kTile) * ((s.n_out + kTile - 1) / kTile);
    linear_kernel<<<(unsigned)tiles, 256, 0, stream>>>(a);
}

}  // namespace lmkan
