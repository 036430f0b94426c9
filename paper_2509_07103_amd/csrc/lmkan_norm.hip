// Layer norm over the columns of rows, and its gradients:
//   hat = (x - mean) rstd,  y = weight hat + bias
//   grad_x = rstd (d - <d> - hat <d hat>),  d = weight grad_y;  grad_weight = sum_n grad_y hat,  grad_bias = sum_n grad_y
//
// Both are bound by memory: a row is read once and stays in registers, H pieces of E adjacent elements a lane, while its
// sums are taken across the lanes it is spread over (8 to 64 of a wave, or all waves of a workgroup).  Workgroups take
// row after row, with the columns' weights in registers; the backward pass keeps its sums over rows there too, writes one
// part a workgroup, and a second launch adds the parts.  Statistics in float64 take no time beside the memory.
//
// Measured (us; TB/s of what has to be read and written, of which a copy reaches 5.2 to 5.4): 65536 x 1024 float32 forward 100
// (5.4), with a checkpoint 116 (5.2), backward 151 (5.3), from the checkpoint 113 (5.4); 8192 x 1024 backward 23 (4.4), of which
// 3.9 are the second launch; 262144 x 128 bfloat16 from the checkpoint 39 (4.3); 100000 x 333 from bfloat16 to float32, rows at any
// address, forward 48 (4.1), backward 63 (4.2); 4096 x 16384 float32 forward 130 (4.1), backward 185 (4.4); 2000 x 40000, which
// registers do not hold, 266 (2.4) and 419 (2.3).
#include "lmkan_rows.h"

namespace lmkan {

namespace {

template <class V>
struct Plus {
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

// How a row lies over lanes: `lanes` of them (a power of two), or a workgroup of THREADS when GROUP; H pieces of kind K a lane
template <int K, int H, int THREADS, bool GROUP>
struct Spread {
    static constexpr int kWaves = THREADS / 64, E = elements_of(K);
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
    // A lane's pieces of a row, as they lie in memory
    __device__ __forceinline__ void load(const void *p, int64_t first, int dtype, int cols, uint32_t (&w)[H][E]) const
    {
        p = row_at(p, first, dtype);
        if (dtype == LMKAN_F32) {
#pragma unroll
            for (int h = 0; h < H; ++h) load_raw<K, true>(p, column(h), cols, w[h]);
        } else {
#pragma unroll
            for (int h = 0; h < H; ++h) load_raw<K, false>(p, column(h), cols, w[h]);
        }
    }
    // ... and as float32, in place
    __device__ __forceinline__ void take(const uint32_t (&w)[H][E], int dtype, int cols, float (&v)[H][E]) const
    {
        if (dtype == LMKAN_F32) {
#pragma unroll
            for (int h = 0; h < H; ++h) convert<LMKAN_F32>(w[h], v[h]);
        } else if (dtype == LMKAN_F16) {
#pragma unroll
            for (int h = 0; h < H; ++h) convert<LMKAN_F16>(w[h], v[h]);
        } else {
#pragma unroll
            for (int h = 0; h < H; ++h) convert<LMKAN_BF16>(w[h], v[h]);
        }
        place(v, cols);
    }
    // (pieces that are aligned exist or do not: who takes them asks)
    __device__ __forceinline__ void place(float (&v)[H][E], int cols) const
    {
        if constexpr (K < 0)
#pragma unroll
            for (int h = 0; h < H; ++h) settle<K>(v[h], column(h), cols);
    }
    // columns' weights or the like: `other` where there are none, zero beyond the end
    __device__ __forceinline__ void load_columns(const float *p, float other, int h, int cols, float (&v)[E]) const
    {
        if (p) load_piece_as<K, LMKAN_F32>(p, column(h), cols, v);
        if (K < 0) settle<K>(v, column(h), cols);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = exists<K>(column(h), i, cols) ? (p ? v[i] : other) : 0.0f;
    }
    __device__ __forceinline__ void load_columns(const float *p, float other, int cols, float (&v)[H][E]) const
    {
#pragma unroll
        for (int h = 0; h < H; ++h) load_columns(p, other, h, cols, v[h]);
    }
};

// Elements of a row that a lane holds, and of the longest rows that registers hold
constexpr int kLaneHolds = 16, kLaneHoldsMost = 32, kMostHeld = 512 * kLaneHoldsMost;
// Weights stay in registers beside 16 elements of the row; beside 32 they are read for every row
constexpr bool weights_held(int held) { return held <= kLaneHolds; }

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

template <int K, int H, int THREADS, bool GROUP>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a)
{
    constexpr int E = elements_of(K);
    __shared__ double sums[THREADS / 64];
    const Spread<K, H, THREADS, GROUP> s(a.lanes_log);
    constexpr bool kHeld = weights_held(H * E);
    float w[H][E], b[H][E];
    if (kHeld) {
        s.load_columns(a.weight, 1.0f, a.cols, w);
        s.load_columns(a.bias, 0.0f, a.cols, b);
    }
    for (int64_t row = (int64_t)blockIdx.x * s.rows + s.row; row < a.rows; row += (int64_t)gridDim.x * s.rows) {
        const int64_t first = row * a.cols;
        uint32_t raw[H][E];
        s.load(a.x, first, a.x_dtype, a.cols, raw);
        float x[H][E];
        s.take(raw, a.x_dtype, a.cols, x);
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
                double d = (double)x[h][i] - centre;
                if (K < 0 && i > 0) d = exists<K>(s.column(h), i, a.cols) ? d : 0.0;
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
            for (int i = 0; i < E; ++i) hat[i] = exists<K>(c, i, a.cols) ? normal(x[h][i], mean, rstd) : 0.0f;
            if (a.codes) {
                uint32_t coded[(E + 3) / 4];
                const int byte = encode_piece(hat, coded);
                if (c < a.cols) {
                    store_codes_piece<K>(codes, c, a.cols, coded);
                    if (c % kBlock == 0) exps[c / kBlock] = (uint8_t)byte;
                }
            }
            if (c < a.cols) {
                float wh[E], bh[E];
                if constexpr (kHeld) {
#pragma unroll
                    for (int i = 0; i < E; ++i) wh[i] = w[h][i], bh[i] = b[h][i];
                } else {
                    s.load_columns(a.weight, 1.0f, h, a.cols, wh);
                    s.load_columns(a.bias, 0.0f, h, a.cols, bh);
                }
#pragma unroll
                for (int i = 0; i < E; ++i) hat[i] = fmaf(wh[i], hat[i], bh[i]);
                store_piece<K>(y, c, a.cols, a.y_dtype, hat);
            }
        }
    }
}

// Rows that registers do not hold are read three times (from the L2 or the last cache after the first).  4096 x 16384 float32
// would take 216 us this way where rows in registers take 130, and 330 instead of 185 in the backward pass.
template <int K>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a)
{
    constexpr int E = elements_of(K);
    __shared__ double sums[16];
    const Spread<K, 1, 1024, true> s(0);
    const int lane = threadIdx.x * E;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const void *const x = row_at(a.x, row * a.cols, a.x_dtype);
        void *const y = row_at(a.y, row * a.cols, a.y_dtype);
        double sum = 0.0;
#pragma unroll 4
        for (int c = lane; c < a.cols; c += 1024 * E) {
            float v[E];
            load_piece<K>(x, c, a.cols, a.x_dtype, v);
            settle<K>(v, c, a.cols);
#pragma unroll
            for (int i = 0; i < E; ++i) sum += (double)v[i];
        }
        const double centre = s.sum(sum, sums) / a.cols;
        sum = 0.0;
#pragma unroll 4
        for (int c = lane; c < a.cols; c += 1024 * E) {
            float v[E];
            load_piece<K>(x, c, a.cols, a.x_dtype, v);
            settle<K>(v, c, a.cols);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const double d = exists<K>(c, i, a.cols) ? (double)v[i] - centre : 0.0;
                sum = fma(d, d, sum);
            }
        }
        const float mean = (float)centre, rstd = (float)(1.0 / sqrt(s.sum(sum, sums) / a.cols + (double)a.eps));
        if (a.stats && threadIdx.x == 0) a.stats[2 * row] = mean, a.stats[2 * row + 1] = rstd;
        for (int c0 = 0; c0 < a.cols; c0 += 1024 * E) {
            const int c = c0 + lane;
            float hat[E];
            load_piece<K>(x, c, a.cols, a.x_dtype, hat);
            settle<K>(hat, c, a.cols);
#pragma unroll
            for (int i = 0; i < E; ++i) hat[i] = exists<K>(c, i, a.cols) ? normal(hat[i], mean, rstd) : 0.0f;
            if (a.codes) {
                uint32_t coded[(E + 3) / 4];
                const int byte = encode_piece(hat, coded);
                if (c < a.cols) {
                    store_codes_piece<K>(a.codes + row * a.cols, c, a.cols, coded);
                    if (c % kBlock == 0) a.exps[row * exp_blocks(a.cols) + c / kBlock] = (uint8_t)byte;
                }
            }
            if (c < a.cols) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int at = c + i < a.cols ? c + i : c;
                    hat[i] = fmaf(a.weight ? a.weight[at] : 1.0f, hat[i], a.bias ? a.bias[at] : 0.0f);
                }
                store_piece<K>(y, c, a.cols, a.y_dtype, hat);
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

// KEPT: from the checkpoint.  One kernel for both would hold the registers of both: 142 instead of 110 for 8192 columns of
// bfloat16, 8192 x 4096 from the checkpoint 44 us instead of 38.
template <bool KEPT, int K, int H, int THREADS, bool GROUP>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(GradArgs g)
{
    constexpr int E = elements_of(K);
    const NormBackwardArgs &a = g.a;
    const int cols = g.s.cols;
    __shared__ float sums[2 * (THREADS / 64)];
    __shared__ float joined[GROUP ? 1 : THREADS * E];
    const Spread<K, H, THREADS, GROUP> s(g.lanes_log);
    const float part = 1.0f / (float)cols;
    float w[H][E], gw[H][E], gb[H][E];
    if (weights_held(H * E)) s.load_columns(a.weight, 1.0f, cols, w);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < E; ++i) gw[h][i] = gb[h][i] = 0.0f;
    for (int64_t row = (int64_t)blockIdx.x * s.rows + s.row; row < g.s.rows; row += (int64_t)gridDim.x * s.rows) {
        const int64_t first = row * cols;
        // (all loads of the row are under way before the first is used, but for the longest unaligned rows, for which registers
        // are short: 60 bytes a lane of theirs go to memory and back for every row all the same)
        constexpr bool kOneByOne = KEPT && K < 0 && !weights_held(H * E);
        uint32_t raw_d[H][E], raw_x[H][E], coded[H][(E + 3) / 4];
        int byte[H];
        float d[H][E], hat[H][E];
        s.load(a.grad_y, first, g.s.y_dtype, cols, raw_d);
        if constexpr (kOneByOne) {
            s.take(raw_d, g.s.y_dtype, cols, d);
            __builtin_amdgcn_sched_barrier(0);
        }
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        if constexpr (!KEPT) {
            s.load(a.x, first, g.s.x_dtype, cols, raw_x);
        } else {
            const int8_t *codes = a.codes + first;
            const uint8_t *exps = a.exps + row * exp_blocks(cols);
#pragma unroll
            for (int h = 0; h < H; ++h) {
                load_codes_piece<K>(codes, s.column(h), cols, coded[h]);
                byte[h] = exps[(s.column(h) < cols ? s.column(h) : 0) / kBlock];
            }
        }
        if constexpr (!kOneByOne) s.take(raw_d, g.s.y_dtype, cols, d);
        if constexpr (!KEPT) {
            s.take(raw_x, g.s.x_dtype, cols, hat);
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int i = 0; i < E; ++i) hat[h][i] = (hat[h][i] - mean) * rstd;
        } else {
#pragma unroll
            for (int h = 0; h < H; ++h) values_of<E>(coded[h], byte[h], hat[h]);
            s.place(hat, cols);
        }
        float of_d = 0.0f, of_dh = 0.0f;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            if (s.column(h) < cols) {
                float of_h[E];
                if constexpr (weights_held(H * E)) {
#pragma unroll
                    for (int i = 0; i < E; ++i) of_h[i] = w[h][i];
                } else {
                    s.load_columns(a.weight, 1.0f, h, cols, of_h);
                }
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    gb[h][i] += d[h][i];
                    gw[h][i] = fmaf(d[h][i], hat[h][i], gw[h][i]);
                    d[h][i] *= of_h[i];
                    of_d += d[h][i];
                    of_dh = fmaf(d[h][i], hat[h][i], of_dh);
                }
            }
        }
        if (a.grad_x) {
            s.two_sums(of_d, of_dh, sums);
            of_d *= part, of_dh *= part;
            void *const grad_x = row_at(a.grad_x, first, g.s.x_dtype);
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const int c = s.column(h);
                if (c < cols) {
#pragma unroll
                    for (int i = 0; i < E; ++i) d[h][i] = rstd * (d[h][i] - of_d - hat[h][i] * of_dh);
                    store_piece<K>(grad_x, c, cols, g.s.x_dtype, d[h]);
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
                for (int i = 0; i < E; ++i)
                    if (exists<K>(c, i, cols)) to[which * cols + c + i] = v[i];
        }
    }
}

template <int K, int E>
__device__ __forceinline__ void load_hat(const NormShape &s, const NormBackwardArgs &a, int64_t row, int c, float (&hat)[E])
{
    if (a.x) {
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        load_piece<K>(row_at(a.x, row * s.cols, s.x_dtype), c, s.cols, s.x_dtype, hat);
#pragma unroll
        for (int i = 0; i < E; ++i) hat[i] = (hat[i] - mean) * rstd;
    } else {
        uint32_t coded[(E + 3) / 4];
        load_codes_piece<K>(a.codes + row * s.cols, c, s.cols, coded);
        values_of<E>(coded, a.exps[row * exp_blocks(s.cols) + c / kBlock], hat);
    }
    settle<K>(hat, c, s.cols);
}

// Rows that registers do not hold: the rows' gradients, read twice ..
template <int K>
__global__ __launch_bounds__(1024) void norm_long_grad_x_kernel(NormShape s, NormBackwardArgs a)
{
    constexpr int E = elements_of(K);
    __shared__ float sums[32];
    const Spread<K, 1, 1024, true> spread(0);
    for (int64_t row = blockIdx.x; row < s.rows; row += gridDim.x) {
        const float rstd = a.stats[2 * row + 1];
        const void *const gy = row_at(a.grad_y, row * s.cols, s.y_dtype);
        void *const gx = row_at(a.grad_x, row * s.cols, s.x_dtype);
        const auto load = [&](int c, float (&d)[E], float (&hat)[E]) {
            load_piece<K>(gy, c, s.cols, s.y_dtype, d);
            settle<K>(d, c, s.cols);
            load_hat<K>(s, a, row, c, hat);
            if (a.weight)
#pragma unroll
                for (int i = 0; i < E; ++i) d[i] *= a.weight[c + i < s.cols ? c + i : c];
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
            store_piece<K>(gx, c, s.cols, s.x_dtype, d);
        }
    }
}

// .. and the columns' sums, a piece of columns a thread
template <int K>
__global__ __launch_bounds__(256) void norm_long_columns_kernel(NormShape s, NormBackwardArgs a, float *parts)
{
    constexpr int E = elements_of(K);
    const int c = (blockIdx.x * 256 + threadIdx.x) * E;
    if (c >= s.cols) return;
    float w[E] = {}, b[E] = {};
    for (int64_t row = blockIdx.y; row < s.rows; row += gridDim.y) {
        float g[E], hat[E];
        load_piece<K>(row_at(a.grad_y, row * s.cols, s.y_dtype), c, s.cols, s.y_dtype, g);
        settle<K>(g, c, s.cols);
        load_hat<K>(s, a, row, c, hat);
#pragma unroll
        for (int i = 0; i < E; ++i) b[i] += g[i], w[i] = fmaf(g[i], hat[i], w[i]);
    }
    float *const to = parts + (int64_t)blockIdx.y * 2 * s.cols;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (c + i < s.cols) to[c + i] = w[i], to[s.cols + c + i] = b[i];
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
#pragma unroll 16
        for (int p = slice; p < parts; p += 32) sum += (double)from[((int64_t)p * 2 + blockIdx.y) * s.cols + c];
    sums[slice][col] = sum;
    __syncthreads();
    if (slice > 0 || c >= s.cols) return;
    for (int k = 1; k < 32; ++k) sum += sums[k][col];
    to[c] = s.accumulate ? to[c] + (float)sum : (float)sum;
}

// ---- host ------------------------------------------------------------------------------------------------------------

constexpr int kUnits = 256;                       // compute units

// How a row of `cols` columns is spread: pieces of a kind; its lanes, or the threads of a workgroup
struct Plan {
    int kind, held, lanes_log, threads;   // threads: 0, lanes of a wave
};

Plan plan_of(int cols, int kind)
{
    const int e = elements_of(kind);
    Plan p = {kind, 1, e == 1 ? 5 : e == 4 ? 3 : 2, 0};
    while (p.lanes_log < 6 && cols > kLaneHolds << p.lanes_log) ++p.lanes_log;
    int lanes = 1 << p.lanes_log;
    if (cols > kLaneHolds * 64) {
        p.threads = cols > kLaneHolds * 256 ? 512 : 256;
        lanes = p.threads;
    }
    while (p.held * e * lanes < cols) p.held *= 2;
    return p;
}

// calls f with K, H, THREADS and GROUP as constants
template <int K, int H, int THREADS, bool GROUP>
struct Sizes {
    static constexpr int k = K, h = H, threads = THREADS;
    static constexpr bool group = GROUP;
};
template <int K, class F>
void with_held(const Plan &p, F &&f)
{
    constexpr int kMost = kLaneHolds / elements_of(K);
    if (p.held == 2 * kMost) f(Sizes<K, 2 * kMost, 512, true>());
    else if (p.threads == 512) f(Sizes<K, kMost, 512, true>());
    else if (p.threads == 256 && p.held == kMost) f(Sizes<K, kMost, 256, true>());
    else if (p.threads == 256) f(Sizes<K, kMost / 2, 256, true>());
    else if (p.held == kMost) f(Sizes<K, kMost, 256, false>());
    else if (p.held == kMost / 2) f(Sizes<K, kMost / 2, 256, false>());
    else if constexpr (kMost == 4) f(Sizes<K, 1, 256, false>());
}
template <class F>
void with_sizes(const Plan &p, F &&f)
{
    if (p.kind == 8) with_held<8>(p, f);
    else if (p.kind == 4) with_held<4>(p, f);
    else if (p.kind == -4) with_held<-4>(p, f);
    else f(Sizes<1, 1, 256, false>());   // (fewer than four columns)
}

unsigned groups_of(const Plan &p, int64_t rows, int most)
{
    const int64_t at_once = p.threads ? 1 : 256 >> p.lanes_log, n = (rows + at_once - 1) / at_once;
    return (unsigned)(n < most ? n : most);
}

// Pieces of eight where all rows are of 16 bits, and from those to float32 with a checkpoint.  Measured (us, eight / four):
// 262144 x 128 bfloat16 forward 26 / 30, with a checkpoint 33 / 41, backward 44 / 50, from the checkpoint 41 / 47; bfloat16 to
// float32 65536 x 1024 89 / 79, 16384 x 512 with a checkpoint 12.9 / 15.0; gradients of float32 rows from bfloat16 ones and a
// checkpoint 60000 x 1000 91 / 82
int kind_of(int cols, const void *const (&p)[4], const int (&dtypes)[4], const float *w, const float *b, const int8_t *codes, bool narrow)
{
    const auto fits = [&](int e) {
        for (int i = 0; i < 4; ++i)
            if (p[i] && !pieces_ok(e, cols, p[i], dtypes[i])) return false;
        return cols % e == 0 && reinterpret_cast<uintptr_t>(codes) % e == 0 && reinterpret_cast<uintptr_t>(w) % 16 == 0 && reinterpret_cast<uintptr_t>(b) % 16 == 0;
    };
    return narrow && fits(8) ? 8 : fits(4) ? 4 : unaligned_kind(cols);
}

// Workgroups of the backward pass at most, and parts: more of them read more weights and leave more parts, fewer are too few for
// the memory.  Measured (us, 256 / 512 / 1024): 65536 x 1024 float32 175 / 153 / 163, 8192 x 1024 26.7 / 23.1 / 25.6, 262144 x 128
// bfloat16 64 / 44 / 45, 100000 x 333 105 / 63 / 72.  Rows of which a lane holds 32 elements: one workgroup fills a unit
constexpr int kGradGroups = 2 * kUnits;

}  // namespace

void launch_layer_norm(const NormShape &s, const void *x, const float *weight, const float *bias, void *y, float *stats, int8_t *codes,
                       uint8_t *exps, hipStream_t stream)
{
    NormArgs a{s.rows, s.cols, s.x_dtype, s.y_dtype, 0, s.eps, x, weight, bias, y, stats, codes, exps};
    const bool narrow = s.x_dtype != LMKAN_F32 && (s.y_dtype != LMKAN_F32 || codes);
    const int kind = kind_of(s.cols, {x, y, nullptr, nullptr}, {s.x_dtype, s.y_dtype}, weight, bias, codes, narrow);
    if (s.cols > kMostHeld) {
        const unsigned groups = (unsigned)(s.rows < kMostGroups ? s.rows : kMostGroups);
        if (kind > 0) norm_long_kernel<4><<<groups, 1024, 0, stream>>>(a);
        else norm_long_kernel<-4><<<groups, 1024, 0, stream>>>(a);
        return;
    }
    const Plan p = plan_of(s.cols, kind);
    a.lanes_log = p.lanes_log;
    with_sizes(p, [&](auto sizes) {
        typedef decltype(sizes) S;
        const int most = 8 * kUnits * 256 / S::threads;
        norm_kernel<S::k, S::h, S::threads, S::group><<<groups_of(p, s.rows, most), S::threads, 0, stream>>>(a);
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
    const bool narrow = s.y_dtype != LMKAN_F32 && s.x_dtype != LMKAN_F32;
    const int kind = kind_of(s.cols, {a.x, a.grad_y, a.grad_x, nullptr}, {s.x_dtype, s.y_dtype, s.x_dtype}, a.weight, nullptr, a.codes, narrow);
    if (s.rows > 0 && s.cols > kMostHeld) {
        const unsigned rows = (unsigned)(s.rows < kMostGroups ? s.rows : kMostGroups);
        if (a.grad_x) {
            if (kind > 0) norm_long_grad_x_kernel<4><<<rows, 1024, 0, stream>>>(s, a);
            else norm_long_grad_x_kernel<-4><<<rows, 1024, 0, stream>>>(s, a);
        }
        groups = rows < 64 ? rows : 64;
        if (columns) {
            const dim3 across((s.cols + 1023) / 1024, groups);
            if (kind > 0) norm_long_columns_kernel<4><<<across, 256, 0, stream>>>(s, a, parts);
            else norm_long_columns_kernel<-4><<<across, 256, 0, stream>>>(s, a, parts);
        }
    } else if (s.rows > 0) {
        GradArgs g{s, a, 0, columns ? parts : nullptr};
        const Plan p = plan_of(s.cols, kind);
        g.lanes_log = p.lanes_log;
        groups = groups_of(p, s.rows, s.cols > kLaneHolds * 512 ? kUnits : kGradGroups);
        with_sizes(p, [&](auto sizes) {
            typedef decltype(sizes) S;
            if (a.x) norm_grad_kernel<false, S::k, S::h, S::threads, S::group><<<groups, S::threads, 0, stream>>>(g);
            else norm_grad_kernel<true, S::k, S::h, S::threads, S::group><<<groups, S::threads, 0, stream>>>(g);
        });
    }
    if (columns) norm_join_kernel<<<dim3((s.cols + 31) / 32, 2), 1024, 0, stream>>>(s, a, (int)groups, parts);
}

}  // namespace lmkan
