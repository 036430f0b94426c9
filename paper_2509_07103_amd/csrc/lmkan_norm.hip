// Layer norm over the columns of rows, and its gradients.
//
// Both are bound by memory: a row is read once and stays in registers, H pieces of E adjacent elements a lane, while its
// sums are taken across the lanes it is spread over (8 to 64 of a wave, or all waves of a workgroup).  Workgroups take
// row after row, with the columns' weights in registers; the backward pass keeps its sums over rows there too, writes one
// part a workgroup, and a second launch adds the parts.
#include "lmkan_rows.h"

namespace lmkan {

namespace {

template <class V>
struct Plus {
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

// How a row lies over lanes: `lanes` of them (a power of two), or a workgroup of THREADS when GROUP
template <int E, int H, int THREADS, bool GROUP>
struct Spread {
    static constexpr int kWaves = THREADS / 64;
    int lanes, lane, row, rows;   // rows: of the workgroup at a time
    __device__ __forceinline__ explicit Spread(int lanes_log)
    {
        lanes = GROUP ? THREADS : 1 << lanes_log;
        lane = GROUP ? (int)threadIdx.x : (int)(threadIdx.x & (lanes - 1));
        row = GROUP ? 0 : (int)threadIdx.x >> lanes_log;
        rows = GROUP ? 1 : THREADS >> lanes_log;
    }
    __device__ __forceinline__ int column(int h) const { return (h * lanes + lane) * E; }
    // sum over the row, in all of its lanes; `shared`: kWaves values
    template <class V>
    __device__ __forceinline__ V sum(V v, V *shared) const
    {
        v = over_lanes(v, GROUP ? 64 : lanes, Plus<V>());
        if constexpr (GROUP) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
            __syncthreads();
            v = shared[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v += shared[w];
        }
        return v;
    }
    template <class V>
    __device__ __forceinline__ void two_sums(V &a, V &b, V *shared) const
    {
        a = over_lanes(a, GROUP ? 64 : lanes, Plus<V>());
        b = over_lanes(b, GROUP ? 64 : lanes, Plus<V>());
        if constexpr (GROUP) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) shared[2 * (threadIdx.x >> 6)] = a, shared[2 * (threadIdx.x >> 6) + 1] = b;
            __syncthreads();
            a = shared[0], b = shared[1];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) a += shared[2 * w], b += shared[2 * w + 1];
        }
    }
};

template <int E, int H, int DTYPE>
__device__ __forceinline__ void load_row_as(const void *p, int64_t first, int lanes, int lane, int cols, float (&v)[H][E])
{
    p = row_at(p, first, DTYPE);
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int c = (h * lanes + lane) * E;
        load_piece<E, DTYPE>(p, c < cols ? c : 0, v[h]);
    }
}
// A lane's pieces of a row that begins at `first`; what lies beyond the end is anything that the row holds
template <int E, int H>
__device__ __forceinline__ void load_row(const void *p, int64_t first, int dtype, int lanes, int lane, int cols, float (&v)[H][E])
{
    if (dtype == LMKAN_F32) load_row_as<E, H, LMKAN_F32>(p, first, lanes, lane, cols, v);
    else if (dtype == LMKAN_F16) load_row_as<E, H, LMKAN_F16>(p, first, lanes, lane, cols, v);
    else load_row_as<E, H, LMKAN_BF16>(p, first, lanes, lane, cols, v);
}
// columns' weights or the like: `other` where there are none, zero beyond the end
template <int E, int H>
__device__ __forceinline__ void load_columns(const float *p, float other, int lanes, int lane, int cols, float (&v)[H][E])
{
    if (p) load_row_as<E, H, LMKAN_F32>(p, 0, lanes, lane, cols, v);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < E; ++i) v[h][i] = (h * lanes + lane) * E < cols ? (p ? v[h][i] : other) : 0.0f;
}

struct NormArgs {
    int64_t rows;
    int cols, x_dtype, y_dtype, lanes_log;
    float eps;
    const void *x;
    const float *weight, *bias;
    void *y;
    float *stats;
    int8_t *codes;
    uint8_t *exps;
};

// (x - mean) rstd: two roundings, as the checkpoint's definition has it
__device__ __forceinline__ float normal(float x, float mean, float rstd) { return __fmul_rn(__fsub_rn(x, mean), rstd); }

template <int E, int H, int THREADS, bool GROUP>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a)
{
    __shared__ double sums[THREADS / 64];
    const Spread<E, H, THREADS, GROUP> s(a.lanes_log);
    float w[H][E], b[H][E];
    load_columns(a.weight, 1.0f, s.lanes, s.lane, a.cols, w);
    load_columns(a.bias, 0.0f, s.lanes, s.lane, a.cols, b);
    for (int64_t row = (int64_t)blockIdx.x * s.rows + s.row; row < a.rows; row += (int64_t)gridDim.x * s.rows) {
        const int64_t first = row * a.cols;
        float x[H][E];
        load_row(a.x, first, a.x_dtype, s.lanes, s.lane, a.cols, x);
        double sum = 0.0;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            double part = 0.0;
#pragma unroll
            for (int i = 0; i < E; ++i) part += (double)x[h][i];
            sum += s.column(h) < a.cols ? part : 0.0;
        }
        const double centre = s.sum(sum, sums) / a.cols;
        sum = 0.0;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            double part = 0.0;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const double d = (double)x[h][i] - centre;
                part = fma(d, d, part);
            }
            sum += s.column(h) < a.cols ? part : 0.0;
        }
        const float mean = (float)centre, rstd = (float)(1.0 / sqrt(s.sum(sum, sums) / a.cols + (double)a.eps));
        if (a.stats && s.lane == 0) a.stats[2 * row] = mean, a.stats[2 * row + 1] = rstd;
        void *const y = row_at(a.y, first, a.y_dtype);
        int8_t *const codes = a.codes + first;
        uint8_t *const exps = a.exps + row * exp_blocks(a.cols);
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const int c = s.column(h);
            float hat[E];
#pragma unroll
            for (int i = 0; i < E; ++i) hat[i] = c < a.cols ? normal(x[h][i], mean, rstd) : 0.0f;
            if (a.codes) {
                uint32_t coded[(E + 3) / 4];
                const int byte = encode_piece(hat, coded);
                if (c < a.cols) {
                    store_codes_piece<E>(codes + c, coded);
                    if (c % kBlock == 0) exps[c / kBlock] = (uint8_t)byte;
                }
            }
            if (c < a.cols) {
#pragma unroll
                for (int i = 0; i < E; ++i) hat[i] = fmaf(w[h][i], hat[i], b[h][i]);
                store_piece(y, c, a.y_dtype, hat);
            }
        }
    }
}

// Rows that registers do not hold are read three times (from the L2 or the last cache after the first)
template <int E>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a)
{
    __shared__ double sums[16];
    const Spread<E, 1, 1024, true> s(0);
    const int lane = threadIdx.x * E;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const void *const x = row_at(a.x, row * a.cols, a.x_dtype);
        void *const y = row_at(a.y, row * a.cols, a.y_dtype);
        double sum = 0.0;
#pragma unroll 4
        for (int c = lane; c < a.cols; c += 1024 * E) {
            float v[E];
            load_piece(x, c, a.x_dtype, v);
#pragma unroll
            for (int i = 0; i < E; ++i) sum += (double)v[i];
        }
        const double centre = s.sum(sum, sums) / a.cols;
        sum = 0.0;
#pragma unroll 4
        for (int c = lane; c < a.cols; c += 1024 * E) {
            float v[E];
            load_piece(x, c, a.x_dtype, v);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const double d = (double)v[i] - centre;
                sum = fma(d, d, sum);
            }
        }
        const float mean = (float)centre, rstd = (float)(1.0 / sqrt(s.sum(sum, sums) / a.cols + (double)a.eps));
        if (a.stats && threadIdx.x == 0) a.stats[2 * row] = mean, a.stats[2 * row + 1] = rstd;
        for (int c0 = 0; c0 < a.cols; c0 += 1024 * E) {
            const int c = c0 + lane;
            float hat[E];
            load_piece(x, c < a.cols ? c : 0, a.x_dtype, hat);
#pragma unroll
            for (int i = 0; i < E; ++i) hat[i] = c < a.cols ? normal(hat[i], mean, rstd) : 0.0f;
            if (a.codes) {
                uint32_t coded[(E + 3) / 4];
                const int byte = encode_piece(hat, coded);
                if (c < a.cols) {
                    store_codes_piece<E>(a.codes + row * a.cols + c, coded);
                    if (c % kBlock == 0) a.exps[row * exp_blocks(a.cols) + c / kBlock] = (uint8_t)byte;
                }
            }
            if (c < a.cols) {
#pragma unroll
                for (int i = 0; i < E; ++i) hat[i] = fmaf(a.weight ? a.weight[c + i] : 1.0f, hat[i], a.bias ? a.bias[c + i] : 0.0f);
                store_piece(y, c, a.y_dtype, hat);
            }
        }
    }
}

// ---- gradients -------------------------------------------------------------------------------------------------------

struct GradArgs {
    NormShape s;
    NormBackwardArgs a;
    int lanes_log;
    float *parts;   // [workgroups][2][cols], or null: no gradients of weight and bias
};

template <int E, int H, int THREADS, bool GROUP>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(GradArgs g)
{
    const NormBackwardArgs &a = g.a;
    const int cols = g.s.cols;
    __shared__ float sums[2 * (THREADS / 64)];
    __shared__ float joined[GROUP ? 1 : THREADS * E];
    const Spread<E, H, THREADS, GROUP> s(g.lanes_log);
    float w[H][E], gw[H][E], gb[H][E];
    load_columns(a.weight, 1.0f, s.lanes, s.lane, cols, w);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < E; ++i) gw[h][i] = gb[h][i] = 0.0f;
    for (int64_t row = (int64_t)blockIdx.x * s.rows + s.row; row < g.s.rows; row += (int64_t)gridDim.x * s.rows) {
        const int64_t first = row * cols;
        float d[H][E], hat[H][E];
        load_row(a.grad_y, first, g.s.y_dtype, s.lanes, s.lane, cols, d);
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        if (a.x) {
            load_row(a.x, first, g.s.x_dtype, s.lanes, s.lane, cols, hat);
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int i = 0; i < E; ++i) hat[h][i] = (hat[h][i] - mean) * rstd;
        } else {
            const int8_t *codes = a.codes + first;
            const uint8_t *exps = a.exps + row * exp_blocks(cols);
            uint32_t coded[H][(E + 3) / 4];
            int byte[H];
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const int c = s.column(h) < cols ? s.column(h) : 0;
                load_codes_piece<E>(codes + c, coded[h]);
                byte[h] = exps[c / kBlock];
            }
#pragma unroll
            for (int h = 0; h < H; ++h) values_of<E>(coded[h], byte[h], hat[h]);
        }
        float of_d = 0.0f, of_dh = 0.0f;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            if (s.column(h) < cols) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    gb[h][i] += d[h][i];
                    gw[h][i] = fmaf(d[h][i], hat[h][i], gw[h][i]);
                    d[h][i] *= w[h][i];
                    of_d += d[h][i];
                    of_dh = fmaf(d[h][i], hat[h][i], of_dh);
                }
            }
        }
        if (a.grad_x) {
            s.two_sums(of_d, of_dh, sums);
            of_d /= cols, of_dh /= cols;
            void *const grad_x = row_at(a.grad_x, first, g.s.x_dtype);
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const int c = s.column(h);
                if (c < cols) {
#pragma unroll
                    for (int i = 0; i < E; ++i) d[h][i] = rstd * (d[h][i] - of_d - hat[h][i] * of_dh);
                    store_piece(grad_x, c, g.s.x_dtype, d[h]);
                }
            }
        }
    }
    if (!g.parts) return;
    // the workgroup's rows of lanes, joined in LDS
    float *to = g.parts + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int c = s.column(h);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float(&v)[E] = which ? gb[h] : gw[h];
            if constexpr (!GROUP) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < E; ++i) joined[i * THREADS + threadIdx.x] = v[i];
                __syncthreads();
                if (s.row == 0)
                    for (int r = 1; r < s.rows; ++r)
#pragma unroll
                        for (int i = 0; i < E; ++i) v[i] += joined[i * THREADS + r * s.lanes + s.lane];
            }
            if (s.row == 0 && c < cols)
#pragma unroll
                for (int i = 0; i < E; ++i) to[which * cols + c + i] = v[i];
        }
    }
}

template <int E>
__device__ __forceinline__ void load_hat(const NormShape &s, const NormBackwardArgs &a, int64_t row, int c, float (&hat)[E])
{
    if (a.x) {
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        load_piece(row_at(a.x, row * s.cols, s.x_dtype), c, s.x_dtype, hat);
#pragma unroll
        for (int i = 0; i < E; ++i) hat[i] = (hat[i] - mean) * rstd;
    } else {
        uint32_t coded[(E + 3) / 4];
        load_codes_piece<E>(a.codes + row * s.cols + c, coded);
        values_of<E>(coded, a.exps[row * exp_blocks(s.cols) + c / kBlock], hat);
    }
}

// Rows that registers do not hold: the rows' gradients, read twice ..
template <int E>
__global__ __launch_bounds__(1024) void norm_long_grad_x_kernel(NormShape s, NormBackwardArgs a)
{
    __shared__ float sums[32];
    const Spread<E, 1, 1024, true> spread(0);
    for (int64_t row = blockIdx.x; row < s.rows; row += gridDim.x) {
        const float rstd = a.stats[2 * row + 1];
        const void *const gy = row_at(a.grad_y, row * s.cols, s.y_dtype);
        void *const gx = row_at(a.grad_x, row * s.cols, s.x_dtype);
        const auto load = [&](int c, float (&d)[E], float (&hat)[E]) {
            load_piece(gy, c, s.y_dtype, d);
            load_hat(s, a, row, c, hat);
            if (a.weight)
#pragma unroll
                for (int i = 0; i < E; ++i) d[i] *= a.weight[c + i];
        };
        float of_d = 0.0f, of_dh = 0.0f;
        for (int c = threadIdx.x * E; c < s.cols; c += 1024 * E) {
            float d[E], hat[E];
            load(c, d, hat);
#pragma unroll
            for (int i = 0; i < E; ++i) of_d += d[i], of_dh = fmaf(d[i], hat[i], of_dh);
        }
        spread.two_sums(of_d, of_dh, sums);
        of_d /= s.cols, of_dh /= s.cols;
        for (int c = threadIdx.x * E; c < s.cols; c += 1024 * E) {
            float d[E], hat[E];
            load(c, d, hat);
#pragma unroll
            for (int i = 0; i < E; ++i) d[i] = rstd * (d[i] - of_d - hat[i] * of_dh);
            store_piece(gx, c, s.x_dtype, d);
        }
    }
}

// .. and the columns' sums, a piece of columns a thread
template <int E>
__global__ __launch_bounds__(256) void norm_long_columns_kernel(NormShape s, NormBackwardArgs a, float *parts)
{
    const int c = (blockIdx.x * 256 + threadIdx.x) * E;
    if (c >= s.cols) return;
    float w[E] = {}, b[E] = {};
    for (int64_t row = blockIdx.y; row < s.rows; row += gridDim.y) {
        float g[E], hat[E];
        load_piece(row_at(a.grad_y, row * s.cols, s.y_dtype), c, s.y_dtype, g);
        load_hat(s, a, row, c, hat);
#pragma unroll
        for (int i = 0; i < E; ++i) b[i] += g[i], w[i] = fmaf(g[i], hat[i], w[i]);
    }
    float *const to = parts + (int64_t)blockIdx.y * 2 * s.cols;
#pragma unroll
    for (int i = 0; i < E; ++i) to[c + i] = w[i], to[s.cols + c + i] = b[i];
}

// The parts' sums: 32 columns a workgroup, every 32nd part a thread
__global__ __launch_bounds__(1024) void norm_join_kernel(NormShape s, NormBackwardArgs a, int parts, const float *from)
{
    __shared__ double sums[32][33];
    const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + col;
    float *const to = blockIdx.y ? a.grad_bias : a.grad_weight;
    if (!to) return;
    double sum = 0.0;
    if (c < s.cols)
#pragma unroll 8
        for (int p = slice; p < parts; p += 32) sum += (double)from[((int64_t)p * 2 + blockIdx.y) * s.cols + c];
    sums[slice][col] = sum;
    __syncthreads();
    if (slice > 0 || c >= s.cols) return;
    for (int k = 1; k < 32; ++k) sum += sums[k][col];
    to[c] = s.accumulate ? to[c] + (float)sum : (float)sum;
}

// ---- host ------------------------------------------------------------------------------------------------------------

// Elements of a row that a lane holds (8 where they lie one by one), and a workgroup of 512; workgroups of 1024 would leave
// 128 registers a lane, which spill.
constexpr int lane_holds(int e) { return e == 1 ? 8 : 16; }
constexpr int most_held(int e) { return 512 * lane_holds(e); }
constexpr int kUnits = 256;                       // compute units

// How a row of `cols` columns is spread: pieces of e elements; its lanes, or the threads of a workgroup
struct Plan {
    int e, held, lanes_log, threads;   // threads: 0, lanes of a wave
};

Plan plan_of(int cols, int e)
{
    Plan p = {e, 1, e == 1 ? 5 : e == 4 ? 3 : 2, 0};
    while (p.lanes_log < 6 && cols > lane_holds(e) << p.lanes_log) ++p.lanes_log;
    int lanes = 1 << p.lanes_log;
    if (cols > lane_holds(e) * 64) {
        p.threads = 256;
        while (cols > lane_holds(e) * p.threads) p.threads *= 2;
        lanes = p.threads;
    }
    while (p.held * e * lanes < cols) p.held *= 2;
    return p;
}

// calls f with E, H, THREADS and GROUP as constants
template <int E, int H, int THREADS, bool GROUP>
struct Sizes {
    static constexpr int e = E, h = H, threads = THREADS;
    static constexpr bool group = GROUP;
};
template <int E, class F>
void with_held(const Plan &p, F &&f)
{
    constexpr int kMost = lane_holds(E) / E;
    if (p.threads == 512) f(Sizes<E, kMost, 512, true>());
    else if (p.threads == 256 && p.held == kMost) f(Sizes<E, kMost, 256, true>());
    else if (p.threads == 256) f(Sizes<E, kMost / 2, 256, true>());
    else if (p.held == kMost) f(Sizes<E, kMost, 256, false>());
    else if (p.held == kMost / 2) f(Sizes<E, kMost / 2, 256, false>());
    else if constexpr (E == 4) f(Sizes<E, 1, 256, false>());
    else if constexpr (E == 1) f(Sizes<E, 2, 256, false>());
}
template <class F>
void with_sizes(const Plan &p, F &&f)
{
    if (p.e == 8) with_held<8>(p, f);
    else if (p.e == 4) with_held<4>(p, f);
    else with_held<1>(p, f);
}

unsigned groups_of(const Plan &p, int64_t rows, int most)
{
    const int64_t at_once = p.threads ? 1 : 256 >> p.lanes_log, n = (rows + at_once - 1) / at_once;
    return (unsigned)(n < most ? n : most);
}

int piece_of(int cols, const void *const (&p)[4], const int (&dtypes)[4], const float *w, const float *b, const int8_t *codes, bool narrow)
{
    const auto fits = [&](int e) {
        for (int i = 0; i < 4; ++i)
            if (p[i] && !pieces_ok(e, cols, p[i], dtypes[i])) return false;
        return cols % e == 0 && reinterpret_cast<uintptr_t>(codes) % e == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0 && reinterpret_cast<uintptr_t>(b) % 16 == 0;
    };
    return narrow && fits(8) ? 8 : fits(4) ? 4 : 1;
}

constexpr int kGradGroups = 2 * kUnits;   // workgroups of the backward pass, and parts

}  // namespace

void launch_layer_norm(const NormShape &s, const void *x, const float *weight, const float *bias, void *y, float *stats, int8_t *codes,
                       uint8_t *exps, hipStream_t stream)
{
    NormArgs a{s.rows, s.cols, s.x_dtype, s.y_dtype, 0, s.eps, x, weight, bias, y, stats, codes, exps};
    const int e = piece_of(s.cols, {x, y, nullptr, nullptr}, {s.x_dtype, s.y_dtype}, weight, bias, codes, s.x_dtype != LMKAN_F32);
    if (s.cols > most_held(e)) {
        const unsigned groups = (unsigned)(s.rows < kMostGroups ? s.rows : kMostGroups);
        if (e > 1) norm_long_kernel<4><<<groups, 1024, 0, stream>>>(a);
        else norm_long_kernel<1><<<groups, 1024, 0, stream>>>(a);
        return;
    }
    const Plan p = plan_of(s.cols, e);
    a.lanes_log = p.lanes_log;
    with_sizes(p, [&](auto sizes) {
        typedef decltype(sizes) S;
        const int most = 8 * kUnits * 256 / S::threads;
        norm_kernel<S::e, S::h, S::threads, S::group><<<groups_of(p, s.rows, most), S::threads, 0, stream>>>(a);
    });
}

size_t layer_norm_backward_workspace_bytes(const NormShape &s)
{
    const int64_t parts = s.rows < kGradGroups ? s.rows : kGradGroups;
    return (size_t)parts * 2 * s.cols * sizeof(float);
}

void launch_layer_norm_backward(const NormShape &s, const NormBackwardArgs &a, void *workspace, hipStream_t stream)
{
    const bool columns = a.grad_weight || a.grad_bias;
    float *const parts = static_cast<float *>(workspace);
    unsigned groups = 0;
    const bool narrow = s.y_dtype != LMKAN_F32 && (!a.x || s.x_dtype != LMKAN_F32);
    const int e = piece_of(s.cols, {a.x, a.grad_y, a.grad_x, nullptr}, {s.x_dtype, s.y_dtype, s.x_dtype}, a.weight, nullptr, a.codes, narrow);
    if (s.rows > 0 && s.cols > most_held(e)) {
        const unsigned rows = (unsigned)(s.rows < kMostGroups ? s.rows : kMostGroups);
        if (a.grad_x) {
            if (e > 1) norm_long_grad_x_kernel<4><<<rows, 1024, 0, stream>>>(s, a);
            else norm_long_grad_x_kernel<1><<<rows, 1024, 0, stream>>>(s, a);
        }
        groups = rows < 64 ? rows : 64;
        if (columns) {
            if (e > 1) norm_long_columns_kernel<4><<<dim3((s.cols / 4 + 255) / 256, groups), 256, 0, stream>>>(s, a, parts);
            else norm_long_columns_kernel<1><<<dim3((s.cols + 255) / 256, groups), 256, 0, stream>>>(s, a, parts);
        }
    } else if (s.rows > 0) {
        GradArgs g{s, a, 0, columns ? parts : nullptr};
        const Plan p = plan_of(s.cols, e);
        g.lanes_log = p.lanes_log;
        groups = groups_of(p, s.rows, kGradGroups);
        with_sizes(p, [&](auto sizes) {
            typedef decltype(sizes) S;
            norm_grad_kernel<S::e, S::h, S::threads, S::group><<<groups, S::threads, 0, stream>>>(g);
        });
    }
    if (columns) norm_join_kernel<<<dim3((s.cols + 31) / 32, 2), 1024, 0, stream>>>(s, a, (int)groups, parts);
}

}  // namespace lmkan
