// Low-rank adapters of many requests beside a shared linear term: y[n] += scale[r] B_r (A_r f(x[n])), r = index[n].
#include "lmkan_rows.h"

namespace lmkan {

namespace {

struct AdapterArgs {
    AdapterShape s;
    const void *x;
    const int32_t *index;
    const void *a, *b;
    const float *scale;
    void *y;
    float *low;   // [batch][rank]: A f(x)
};

// A wave a value of A f(x)
__global__ __launch_bounds__(256) void adapters_down_kernel(AdapterArgs a)
{
    const AdapterShape &s = a.s;
    const int lane = threadIdx.x & 63;
    for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < s.batch * s.rank; i += (int64_t)gridDim.x * 4) {
        const int64_t n = i / s.rank;
        const int k = (int)(i - n * s.rank), r = a.index[n];
        if (r < 0 || r >= s.count) continue;
        float sum = 0.0f;
        for (int e = lane; e < s.n_in; e += 64)
            sum = fmaf(load_as_float(a.a, ((int64_t)r * s.rank + k) * s.n_in + e, s.dtype), rectify(load_as_float(a.x, n * s.n_in + e, s.x_dtype), s.relu), sum);
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
        if (lane == 0) a.low[i] = sum;
    }
}

// A thread an output
__global__ __launch_bounds__(256) void adapters_up_kernel(AdapterArgs a)
{
    const AdapterShape &s = a.s;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < s.batch * s.n_out; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / s.n_out;
        const int j = (int)(i - n * s.n_out), r = a.index[n];
        if (r < 0 || r >= s.count) continue;
        float sum = 0.0f;
        for (int k = 0; k < s.rank; ++k) sum = fmaf(load_as_float(a.b, ((int64_t)r * s.n_out + j) * s.rank + k, s.dtype), a.low[n * s.rank + k], sum);
        store_from_float(a.y, i, s.y_dtype, fmaf(a.scale ? a.scale[r] : 1.0f, sum, load_as_float(a.y, i, s.y_dtype)));
    }
}

}  // namespace

size_t adapters_workspace_bytes(const AdapterShape &s) { return (size_t)s.batch * s.rank * sizeof(float); }

void launch_adapters(const AdapterShape &s, const void *x, const int32_t *index, const void *a, const void *b, const float *scale, void *y,
                     void *workspace, hipStream_t stream)
{
    const AdapterArgs args{s, x, index, a, b, scale, y, static_cast<float *>(workspace)};
    const int64_t down = (s.batch * s.rank + 3) / 4, up = (s.batch * s.n_out + 255) / 256;
    adapters_down_kernel<<<(unsigned)(down < 65536 ? down : 65536), 256, 0, stream>>>(args);
    adapters_up_kernel<<<(unsigned)(up < 65536 ? up : 65536), 256, 0, stream>>>(args);
}

}  // namespace lmkan
