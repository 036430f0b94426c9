// Orthogonalisation of matrices by Newton-Schulz products, and the optimiser's step round it.
//
//   X_0 = U / (|U|_F + eps),  A = X X^T,  X <- a X + (b A + c A^2) X
//
// in float32 on the vector pipe, one product after the other: 64 x 64 tiles of a product staged through LDS.
#include "lmkan_dense.h"

#include <math.h>

namespace lmkan {

namespace {

constexpr int kTile = 64, kDepth = 16;

// the direction's element i of one matrix (momentum already moved when `moved`)
__device__ __forceinline__ float direction(const UpdateArgs &u, int dtype, int64_t i)
{
    if (!u.momentum) return load_as_float(u.grad, i, dtype);
    const float m = u.momentum[i];
    return u.nesterov ? u.beta * m + (1.0f - u.beta) * load_as_float(u.grad, i, dtype) : m;
}

// a workgroup per matrix: the momentum moves, the norm of the direction is summed in float64
__global__ __launch_bounds__(256) void norm_kernel(MatrixShape s, UpdateArgs u, int64_t first, float *inverse)
{
    __shared__ double part[256];
    const int64_t base = (first + blockIdx.x) * s.elems();
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < s.elems(); i += 256) {
        if (u.momentum) u.momentum[base + i] = u.beta * u.momentum[base + i] + (1.0f - u.beta) * load_as_float(u.grad, base + i, s.dtype);
        const double v = direction(u, s.dtype, base + i);
        sum += v * v;
    }
    part[threadIdx.x] = sum;
    for (int half = 128; half > 0; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < half) part[threadIdx.x] += part[threadIdx.x + half];
    }
    if (threadIdx.x == 0) inverse[blockIdx.x] = (float)(1.0 / (sqrt(part[0]) + (double)s.eps));
}

// X [m][n] of one matrix after the other
__global__ __launch_bounds__(256) void scale_kernel(MatrixShape s, UpdateArgs u, int64_t first, int64_t count, const float *inverse, float *x)
{
    const int64_t per = s.elems();
    const int n = s.n();
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < count * per; at += (int64_t)gridDim.x * 256) {
        const int64_t b = at / per, i = at - b * per, r = i / n, c = i - r * n;
        const int64_t from = s.flip() ? c * s.cols + r : i;
        x[at] = inverse[b] * direction(u, s.dtype, (first + b) * per + from);
    }
}

// D = alpha C + beta L R for each matrix: L [rows][depth], R either [cols][depth] (its rows are summed over
// with L's) or [depth][cols]
struct ProductArgs {
    const float *L, *R, *C;
    float *D;
    int64_t sl, sr, sd;  // from one matrix to the next
    int rows, cols, depth;
    bool transposed;     // R is [cols][depth]
    float alpha, beta;
};

__global__ __launch_bounds__(256) void product_kernel(ProductArgs a)
{
    __shared__ float l[kDepth][kTile + 4], r[kDepth][kTile + 4];
    const float *L = a.L + blockIdx.z * a.sl, *R = a.R + blockIdx.z * a.sr;
    const int i0 = blockIdx.y * kTile, j0 = blockIdx.x * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < a.depth; k0 += kDepth) {
        for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
            const int k = e & (kDepth - 1), i = e / kDepth;
            l[k][i] = i0 + i < a.rows && k0 + k < a.depth ? L[(int64_t)(i0 + i) * a.depth + k0 + k] : 0.0f;
            if (a.transposed) r[k][i] = j0 + i < a.cols && k0 + k < a.depth ? R[(int64_t)(j0 + i) * a.depth + k0 + k] : 0.0f;
        }
        if (!a.transposed)
            for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
                const int j = e & (kTile - 1), k = e / kTile;
                r[k][j] = j0 + j < a.cols && k0 + k < a.depth ? R[(int64_t)(k0 + k) * a.cols + j0 + j] : 0.0f;
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[p][q] += l[k][ty * 4 + p] * r[k][tx * 4 + q];
        __syncthreads();
    }
    for (int p = 0; p < 4; ++p)
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + ty * 4 + p, j = j0 + tx * 4 + q;
            if (i >= a.rows || j >= a.cols) continue;
            const int64_t at = blockIdx.z * a.sd + (int64_t)i * a.cols + j;
            a.D[at] = (a.C ? a.alpha * a.C[at] : 0.0f) + a.beta * acc[p][q];
        }
}

__global__ __launch_bounds__(256) void finish_kernel(MatrixShape s, UpdateArgs u, int64_t first, int64_t count, const float *x)
{
    const int64_t per = s.elems();
    const int n = s.n();
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < count * per; at += (int64_t)gridDim.x * 256) {
        const int64_t b = at / per, i = at - b * per, r = i / s.cols, c = i - r * s.cols;
        const float v = x[b * per + (s.flip() ? c * n + r : i)];
        const int64_t to = (first + b) * per + i;
        if (u.weight) u.weight[to] = u.keep * u.weight[to] + u.add * v;
        else store_from_float(u.out, to, s.dtype, v);
    }
}

// matrices that share the workspace at a time
int64_t matrices_at_once(const MatrixShape &s)
{
    const int64_t some = ((int64_t)64 << 20) / s.elems();
    return some < 1 ? 1 : some > s.batch ? s.batch : some > 1024 ? 1024 : some;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

unsigned blocks(int64_t n) { return (unsigned)((n + 255) / 256 > 65536 ? 65536 : (n + 255) / 256); }

}  // namespace

bool schedule_bounds(int steps, const float *schedule, ScheduleBounds *bounds)
{
    // extremes of a polynomial of u = s^2 on [0, r^2]: the ends, and where a derivative vanishes
    double r = 1.0;
    bounds->singular[0] = 1.0f;
    for (int k = 0; k < steps; ++k) {
        const double a = schedule[3 * k], b = schedule[3 * k + 1], c = schedule[3 * k + 2], end = r * r;
        if (!isfinite(a) || !isfinite(b) || !isfinite(c)) return false;
        double factor = 0.0, singular = 0.0;
        const auto visit = [&](double u) {
            if (!(u >= 0.0)) return;
            u = u < end ? u : end;
            const double f = fabs(a + u * (b + u * c));
            factor = f > factor ? f : factor;
            singular = f * sqrt(u) > singular ? f * sqrt(u) : singular;
        };
        visit(0.0);
        visit(end);
        if (c != 0.0) visit(-b / (2.0 * c));
        const double root = sqrt(9.0 * b * b - 20.0 * a * c);  // of a + 3 b u + 5 c u^2 (NaN: none)
        if (c != 0.0) {
            visit((-3.0 * b + root) / (10.0 * c));
            visit((-3.0 * b - root) / (10.0 * c));
        } else if (b != 0.0) {
            visit(-a / (3.0 * b));
        }
        if (!(singular <= kMaxSingular) || !(factor <= kMaxFactor)) return false;
        r = singular;
        bounds->factor[k] = (float)factor;
        bounds->singular[k + 1] = (float)singular;
    }
    return true;
}

size_t ortho_workspace_bytes(const MatrixShape &s)
{
    const int64_t c = matrices_at_once(s);
    const size_t gram = (size_t)s.m() * s.m();
    return align256(c * sizeof(float)) + 2 * align256(c * s.elems() * sizeof(float)) + 2 * align256(c * gram * sizeof(float));
}

void launch_ortho(const MatrixShape &s, int steps, const float *schedule, const UpdateArgs &u, void *workspace, hipStream_t stream)
{
    const int64_t most = matrices_at_once(s), gram = (int64_t)s.m() * s.m();
    char *at = static_cast<char *>(workspace);
    const auto take = [&](size_t bytes) { char *p = at; at += align256(bytes); return reinterpret_cast<float *>(p); };
    float *inverse = take(most * sizeof(float));
    float *x = take(most * s.elems() * sizeof(float)), *y = take(most * s.elems() * sizeof(float));
    float *a = take(most * gram * sizeof(float)), *p = take(most * gram * sizeof(float));
    const int m = s.m(), n = s.n(), tm = (m + kTile - 1) / kTile, tn = (n + kTile - 1) / kTile;
    for (int64_t first = 0; first < s.batch; first += most) {
        const int64_t count = s.batch - first < most ? s.batch - first : most;
        norm_kernel<<<(unsigned)count, 256, 0, stream>>>(s, u, first, inverse);
        scale_kernel<<<blocks(count * s.elems()), 256, 0, stream>>>(s, u, first, count, inverse, x);
        for (int k = 0; k < steps; ++k) {
            const float *abc = schedule + 3 * k;
            const ProductArgs gram_of{x, x, nullptr, a, s.elems(), s.elems(), gram, m, m, n, true, 0.0f, 1.0f};
            product_kernel<<<dim3(tm, tm, (unsigned)count), 256, 0, stream>>>(gram_of);
            const ProductArgs poly{a, a, a, p, gram, gram, gram, m, m, m, false, abc[1], abc[2]};
            product_kernel<<<dim3(tm, tm, (unsigned)count), 256, 0, stream>>>(poly);
            const ProductArgs apply{p, x, x, y, gram, s.elems(), s.elems(), m, n, m, false, abc[0], 1.0f};
            product_kernel<<<dim3(tn, tm, (unsigned)count), 256, 0, stream>>>(apply);
            float *t = x;
            x = y, y = t;
        }
        finish_kernel<<<blocks(count * s.elems()), 256, 0, stream>>>(s, u, first, count, x);
    }
}

}  // namespace lmkan
