// Orthogonalisation of matrices by Newton-Schulz products, and the optimiser's step round it.
//
//   X_0 = U / (|U|_F + eps),  A_k = X_k X_k^T,  X_{k+1} = B_k X_k,  B_k = a_k I + b_k A_k + c_k A_k^2
//
// with X of m x n, m <= n (the transpose of what is stored where that has more rows than columns).  Everything
// between X_0 and the result is a polynomial of A_0, and polynomials of one symmetric matrix commute, so that
// several steps can be taken on m x m matrices alone,
//   A_{k+1} = B_k A_k B_k,   P_{k+1} = B_k P_k,
// and then X_{k+s} = P X_k.  All products but that one are symmetric: half their tiles are computed and mirrored.
// Five steps take 15 m^2 n + 5 m^3 operations as written, 9 m^2 n + 11 m^3 two at a time and 6 m^2 n + 14 m^3 three
// at a time, and X is read and written five, three or two times.  An error of A is relative to its largest eigenvalue
// and grows by up to a^2 (11.9) a step where the eigenvalue is small, which is why not all are taken at once, and
// steps_until() chooses.
//
// Factors are pairs of float16 (lmkan_tile.h): three instructions at the rate of float16 keep 22 bits, which float32
// instructions do at a seventh of that rate (library products: 154 against 1130 to 1240 TFLOP/s).  The power of two that
// a matrix is scaled by follows from the bound of its singular values (schedule_bounds); for X, which is smaller where
// |U| is not large beside eps, also from |X_0| and the factors of the steps behind it (extra_bits).
#include "lmkan_dense.h"

#include <math.h>

#include "lmkan_kernels.h"
#include "lmkan_tile.h"

namespace lmkan {

namespace {

constexpr int kStepsAtOnce = 3;   // steps on one Gram matrix, at most
constexpr int kAtOnce = 8;        // elements that a thread loads before it uses them
constexpr int kNormParts = 1024;  // workgroups that sum the norm of one matrix, at most

// A batch of matrices of pairs (lmkan_tile.h); element values are held times `scale`
struct PairMatrix {
    char *base;
    int64_t stride;  // bytes from one matrix to the next
    int rows, depth;
    float scale, inverse;   // a power of two, and one over it
};

// X is held times a power of two of its own besides: its norm is at most |X_0| times `grow`, and `bound`
struct Extra {
    float grow, bound;
    int most;          // bits
};
// How many bits a matrix X with |X_0| = size stays below its bound
__device__ __forceinline__ int extra_bits(const Extra &x, float size)
{
    const float now = size * x.grow;
    if (!(now > 0.0f && now < x.bound)) return 0;
    const int bits = (int)(__builtin_bit_cast(uint32_t, x.bound) >> 23) - (int)(__builtin_bit_cast(uint32_t, now) >> 23) - 1;
    return min(max(bits, 0), x.most);
}

// Sum over the 256 threads in a fixed order, for all of them
__device__ __forceinline__ double sum_of_threads(double v, double *shared)
{
    shared[threadIdx.x] = v;
    for (int half = 128; half > 0; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < half) shared[threadIdx.x] += shared[threadIdx.x + half];
    }
    __syncthreads();
    return shared[0];
}

// Moves the momentum and sums the squares of the direction in float64: grid (parts, matrices)
__global__ __launch_bounds__(256) void norm_kernel(MatrixShape s, UpdateArgs u, int64_t first, double *part)
{
    __shared__ double sums[256];
    const int64_t per = s.elems(), base = (first + blockIdx.y) * per;
    const int64_t each = (per + gridDim.x - 1) / gridDim.x, begin = blockIdx.x * each;
    const int64_t end = begin + each < per ? begin + each : per;
    double sum = 0.0;
    for (int64_t i0 = begin + threadIdx.x; i0 < end; i0 += 256 * kAtOnce) {
        Raw raw[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (i0 + 256 * k < end) raw[k] = fetch(u, s.dtype, base + i0 + 256 * k, true);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (i0 + 256 * k < end) {
                const double v = direction(u, raw[k], base + i0 + 256 * k, true);
                sum += v * v;
            }
    }
    sum = sum_of_threads(sum, sums);
    if (threadIdx.x == 0) part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// What takes elements to X_0 (a matrix of pairs: to what they are held as), in two factors, as it may be beyond float32
// either way: a power of two that brings elements near one without a rounding, and the rest.  (In scalar registers: two
// vector registers more and split_kernel has six waves a SIMD instead of seven, 132 us instead of 124 for 441 of 250 x 333.)
struct Inverse {
    float power, rest, size;   // size: |X_0|
    __device__ __forceinline__ float of(float v) const { return v * power * rest; }
};
__device__ __forceinline__ Inverse inverse_norm(const MatrixShape &s, const double *part, int parts, int64_t matrix, float scale, const Extra &extra, double *shared)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) sum += part[matrix * parts + i];
    const double norm = sqrt(sum_of_threads(sum, shared)), inverse = 1.0 / (norm + (double)s.eps);
    const int exponent = (int)(__builtin_bit_cast(uint64_t, norm) >> 52) - 1023;   // (not below zero)
    const int power = min(max(exponent, -127), 126);                               // elements times 2^-power
    const float size = uniform((float)(norm * inverse));
    const int up = power + extra_bits(extra, size);
    const double rest = inverse * scale * __builtin_bit_cast(double, (uint64_t)(1023 + up) << 52);
    return {uniform(__builtin_bit_cast(float, (uint32_t)(127 - power) << 23)), uniform((float)rest), size};
}

__device__ __forceinline__ void split(float v, _Float16 *hi, _Float16 *lo)
{
    *hi = (_Float16)v;
    *lo = (_Float16)(v - (float)*hi);
}

// X_0 as pairs, both ways round: `by_rows` has the stored rows (summed over columns), `by_cols` the stored columns.
// grid: 64 x 64 tiles of the stored matrices.
struct SplitArgs {
    MatrixShape s;
    UpdateArgs u;
    int64_t first;
    const double *part;
    int parts;
    PairMatrix by_rows, by_cols;
    Extra extra;
    float *size;
};
__global__ __launch_bounds__(256) void split_kernel(SplitArgs a)
{
    __shared__ float tile[64][65];
    __shared__ double sums[256];
    const int64_t matrix = blockIdx.z, per = a.s.elems();
    const int across = (a.s.cols + 63) / 64;
    const int r0 = (int)(blockIdx.x / across) * 64, c0 = (int)(blockIdx.x % across) * 64;
    const Inverse f = inverse_norm(a.s, a.part, a.parts, matrix, a.by_rows.scale, a.extra, sums);
    if (blockIdx.x == 0 && threadIdx.x == 0) a.size[matrix] = f.size;
    const int c = threadIdx.x & 63;
    const int64_t from = (a.first + matrix) * per + (int64_t)r0 * a.s.cols + c0 + c;
    for (int b = threadIdx.x >> 6; b < 64; b += 4 * kAtOnce) {
        Raw raw[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int r = b + 4 * k;
            if (r0 + r < a.s.rows && c0 + c < a.s.cols) raw[k] = fetch(a.u, a.s.dtype, from + (int64_t)r * a.s.cols, false);
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int r = b + 4 * k;
            const bool in = r0 + r < a.s.rows && c0 + c < a.s.cols;
            tile[r][c] = in ? f.of(direction(a.u, raw[k], 0, false)) : 0.0f;
        }
    }
    __syncthreads();
    // a chunk of eight values at a time: 64 lines, two panels, four chunks
    for (int e = threadIdx.x; e < 64 * 2 * 4; e += 256) {
        const int r = e >> 3, panel = (e >> 2) & 1, chunk = e & 3;
        for (int way = 0; way < 2; ++way) {
            const PairMatrix &d = way ? a.by_cols : a.by_rows;
            const int row = (way ? c0 : r0) + r, p = (way ? r0 : c0) / kPanel + panel;
            if (row >= d.rows || p >= panels(d.depth)) continue;
            half8 hi, lo;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int at = panel * kPanel + chunk * 8 + k;
                _Float16 h, l;
                split(way ? tile[at][r] : tile[r][at], &h, &l);
                hi[k] = h, lo[k] = l;
            }
            char *to = d.base + matrix * d.stride;
            *reinterpret_cast<half8 *>(to + pair_at(d.rows, row, p, chunk)) = hi;
            *reinterpret_cast<half8 *>(to + pair_at(d.rows, row, p, 4 + chunk)) = lo;
        }
    }
}

constexpr int kPitch = 36;                                // floats of a row of a wave's tile in LDS
constexpr int kWaveScratch = 32 * kPitch * (int)sizeof(float);

// A wave's 32 x 32 tile at (row, col) of the output, values as in for_wave_tiles, to a matrix of pairs: by lines
// through LDS, 1 KiB adjacent at a time
__device__ __forceinline__ void store_pairs(const PairMatrix &d, char *to, int row, int col, const uint2 (&hi)[4], const uint2 (&lo)[4],
                                            char *scratch, int lane)
{
    const int r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int line = 16 * (g >> 1) + r, chunk = 2 * (g & 1) + (q >> 1);
        *reinterpret_cast<uint2 *>(scratch + line * kLine + slot_of(line, chunk) * 16 + (q & 1) * 8) = hi[g];
        *reinterpret_cast<uint2 *>(scratch + line * kLine + slot_of(line, 4 + chunk) * 16 + (q & 1) * 8) = lo[g];
    }
    char *line = to + ((int64_t)(col / kPanel) * d.rows + row) * kLine;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int at = t * 1024 + lane * 16;
        const uint4 v = *reinterpret_cast<const uint4 *>(scratch + at);
        if (row + at / kLine < d.rows) *reinterpret_cast<uint4 *>(line + at) = v;
    }
}

// the same tile turned: its columns are rows of `d`
__device__ __forceinline__ void store_turned(const PairMatrix &d, char *to, int row, int col, const uint2 (&hi)[4], const uint2 (&lo)[4], int lane)
{
    const int q = lane >> 4, k = (lane & 15) >> 2;   // the lane's four values along the depth: 4 k ..
    char *line = to + ((int64_t)(row / kPanel) * d.rows + col) * kLine + (k & 1) * 8;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int r = 16 * (g & 1) + 4 * q + (lane & 3), chunk = 2 * (g >> 1) + (k >> 1);
        const uint2 th = turn_quad(hi[g], lane), tl = turn_quad(lo[g], lane);
        if (col + r < d.rows) {
            *reinterpret_cast<uint2 *>(line + r * kLine + slot_of(r, chunk) * 16) = th;
            *reinterpret_cast<uint2 *>(line + r * kLine + slot_of(r, 4 + chunk) * 16) = tl;
        }
    }
}

// What becomes of a product
enum Finish {
    kKeep,      // pairs, both ways round
    kKeepX,     // the same, with X among the factors
    kPoly,      // a I + b A + c (product), pairs
    kResult,    // the result of the call (X is a factor)
};

struct Product {
    PairMatrix rows, cols;     // the factors: by the rows and by the columns of the output
    PairMatrix out, mirror;    // mirror: the output's transpose (the same matrix when symmetric); no base: none
    PairMatrix gram;           // kPoly: A
    bool symmetric;
    float a, b, c;             // kPoly: from products and pairs of A to pairs
    float to_out;              // kKeep: from products to pairs
};
struct ProductArgs {
    Product p[2];
    int problems;
    int matrices;
    int tiles_down, tiles_across;
    int tiles;                 // of one matrix and problem
    WorkSplit work;
    floatx4 *parts;
    const float *size;         // |X_0| of every matrix
    int x_factors;             // kKeepX, kResult: how many of the factors are X
    Extra in, out;             // of X as a factor, and as the product
    // kResult
    MatrixShape s;
    UpdateArgs u;
    int64_t first;
    bool by_four;              // rows of the result take accesses of four elements
};

// Where a tile of the launch is
struct Place {
    int matrix, problem, ti, tj;
};
__device__ __forceinline__ Place place_of(const ProductArgs &a, int t)
{
    const int which = t / a.tiles, tile = t - which * a.tiles;
    const int matrix = a.problems == 1 ? which : which >> 1;
    int ti, tj;
    if (a.p[0].symmetric) upper_tile(tile, a.tiles_across, &ti, &tj);
    else grouped_tile(tile, a.tiles_down, a.tiles_across, &ti, &tj);
    return Place{uniform(matrix), uniform(which - matrix * a.problems), uniform(ti), uniform(tj)};
}

// (two products at a time are kept ones)
template <int FINISH>
__device__ __forceinline__ const Product &product_of(const ProductArgs &a, const Place &w)
{
    return FINISH == kKeep && w.problem ? a.p[1] : a.p[0];
}

// A wave's 32 x 32 tile at (row, col), values as in for_wave_tiles, to pairs; what lies beyond n_rows x n_cols is zero
__device__ __forceinline__ void to_pairs(const floatx4 (&v)[4], float scale, int row, int col, int n_rows, int n_cols, int lane, uint2 (&hi)[4], uint2 (&lo)[4])
{
    const bool inside = row + 32 <= n_rows && col + 32 <= n_cols;
    const int r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        floatx4 f = v[g] * scale;
        if (!inside) {
            const int i = row + 16 * (g >> 1) + r, j = col + 16 * (g & 1) + 4 * q;
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = i < n_rows && j + e < n_cols ? f[e] : 0.0f;
        }
        half4 vh, vl;
#pragma unroll
        for (int e = 0; e < 4; ++e) vh[e] = (_Float16)f[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) vl[e] = (_Float16)__builtin_fmaf((float)vh[e], -1.0f, f[e]);
        hi[g] = __builtin_bit_cast(uint2, vh), lo[g] = __builtin_bit_cast(uint2, vl);
    }
}

// |X_0| of a tile's matrix, for products with X
template <int FINISH>
__device__ __forceinline__ float size_of(const ProductArgs &a, const Place &w) { return FINISH == kKeepX || FINISH == kResult ? a.size[w.matrix] : 0.0f; }

// `scratch`: kWaveScratch bytes of LDS of the wave's own
template <class T, int FINISH>
__device__ __forceinline__ void finish_tile(const ProductArgs &a, const Place &w, const floatx4 (&acc)[T::CT][T::RT], float size, char *scratch, int wave)
{
    const Product &p = product_of<FINISH>(a, w);
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // (the addresses below are worked out here, not kept in registers through the main loop)
    const int r = lane & 15, q = lane >> 4;
    const int n_rows = p.rows.rows, n_cols = p.cols.rows;
    // for what X is held times besides its scale
    const float adjust = FINISH == kKeepX || FINISH == kResult ? uniform(ldexpf(1.0f, extra_bits(a.out, size) - a.x_factors * extra_bits(a.in, size))) : 1.0f;
    // what a lane finishes of a 32 x 32 tile of the result, after the tile went through LDS: rows 8 t + lane / 8, four columns
    const int fr = lane >> 3, fc = (lane & 7) * 4;
    const int64_t start = FINISH == kResult ? (a.first + w.matrix) * a.s.elems() : 0;
    const char *gram = FINISH == kPoly ? p.gram.base + w.matrix * p.gram.stride : nullptr;
    struct Held {
        floatx4 w[4];        // kResult: weights
        half4 hi[4], lo[4];  // kPoly: elements of A
    };
    // (rows and columns beyond the end: others are loaded, and not used)
    const auto ahead = [&](int row, int col) {
        Held h;
        row += w.ti * T::ROWS, col += w.tj * T::COLS;
        if (FINISH == kResult && a.u.weight && a.by_four) {
            const int j = min(col + fc, n_cols - 4);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                h.w[t] = *reinterpret_cast<const floatx4 *>(a.u.weight + start + (int64_t)min(row + 8 * t + fr, n_rows - 1) * a.s.cols + j);
        }
        if (FINISH == kPoly) {
            const int panel = min(col, n_cols - 1) / kPanel;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int i = min(row + 16 * (g >> 1) + r, n_rows - 1), chunk = 2 * (g & 1) + (q >> 1);
                h.hi[g] = *reinterpret_cast<const half4 *>(gram + pair_at(p.gram.rows, i, panel, chunk) + (q & 1) * 8);
                h.lo[g] = *reinterpret_cast<const half4 *>(gram + pair_at(p.gram.rows, i, panel, 4 + chunk) + (q & 1) * 8);
            }
        }
        return h;
    };
    for_wave_tiles<T>(acc, wave, ahead, [&](int row, int col, const floatx4 (&v)[4], const Held &held) {
        row += w.ti * T::ROWS, col += w.tj * T::COLS;
        if (FINISH == kResult) {
            if (row >= n_rows || col >= n_cols) return;
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<floatx4 *>(scratch + ((16 * (g >> 1) + r) * kPitch + 16 * (g & 1) + 4 * q) * 4) = v[g] * p.rows.inverse * p.cols.inverse * adjust;
            if (a.by_four) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int i = row + 8 * t + fr, j = col + fc;
                    const floatx4 o = *reinterpret_cast<const floatx4 *>(scratch + ((8 * t + fr) * kPitch + fc) * 4);
                    if (i >= n_rows || j >= n_cols) continue;
                    const int64_t at = start + (int64_t)i * a.s.cols + j;
                    if (a.u.weight) *reinterpret_cast<floatx4 *>(a.u.weight + at) = a.u.keep * held.w[t] + a.u.add * o;
                    else if (a.s.dtype == LMKAN_F32) *reinterpret_cast<floatx4 *>(static_cast<float *>(a.u.out) + at) = o;
                    else
                        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.u.out) + at) =
                            make_uint2(two_from_float(a.s.dtype, o[0], o[1]), two_from_float(a.s.dtype, o[2], o[3]));
                }
            } else {
                const int j = lane & 31;
#pragma unroll 1
                for (int i = lane >> 5; i < 32; i += 2) {
                    if (row + i >= n_rows || col + j >= n_cols) continue;
                    const int64_t at = start + (int64_t)(row + i) * a.s.cols + col + j;
                    const float o = *reinterpret_cast<const float *>(scratch + (i * kPitch + j) * 4);
                    if (a.u.weight) a.u.weight[at] = a.u.keep * a.u.weight[at] + a.u.add * o;
                    else store_from_float(a.u.out, at, a.s.dtype, o);
                }
            }
            return;
        }
        const bool direct = row < n_rows && col < panels(n_cols) * kPanel;
        const bool turned = p.mirror.base && !(p.symmetric && w.ti == w.tj) && col < n_cols && row < panels(n_rows) * kPanel;
        if (!direct && !turned) return;
        uint2 hi[4], lo[4];
        if (FINISH == kPoly) {
            floatx4 f[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int i = row + 16 * (g >> 1) + r, j = col + 16 * (g & 1) + 4 * q;
#pragma unroll
                for (int e = 0; e < 4; ++e) f[g][e] = p.c * v[g][e] + p.b * ((float)held.hi[g][e] + (float)held.lo[g][e]) + (i == j + e ? p.a : 0.0f);
            }
            to_pairs(f, 1.0f, row, col, n_rows, n_cols, lane, hi, lo);
        } else {
            to_pairs(v, p.to_out * adjust, row, col, n_rows, n_cols, lane, hi, lo);
        }
        if (direct) store_pairs(p.out, p.out.base + w.matrix * p.out.stride, row, col, hi, lo, scratch, lane);
        if (turned) store_turned(p.mirror, p.mirror.base + w.matrix * p.mirror.stride, row, col, hi, lo, lane);
    });
}

template <class T, int FINISH, bool ALONE>
__global__ __launch_bounds__(T::THREADS) void product_kernel(ProductArgs a)
{
    extern __shared__ __align__(16) char lds[];
    for_work(a.work, blockIdx.x, [&](int tile, int from, int to, int slot) {
        const Place w = place_of(a, tile);
        const Product &p = product_of<FINISH>(a, w);
        const auto operand = [&](const PairMatrix &m, int first_row) {
            return Operand{uniform(m.base + w.matrix * m.stride + (int64_t)first_row * kLine), uniform((int64_t)m.rows * kLine), m.rows - 1 - first_row, true, 0, 0};
        };
        const float size = size_of<FINISH>(a, w);   // (under way through the main loop)
        floatx4 acc[T::CT][T::RT];
        // (a workgroup that finishes a tile goes before one that multiplies: 1 to 3 %)
        __builtin_amdgcn_s_setprio(0);
        if constexpr (ALONE) multiply_alone<T, PairProduct>(operand(p.rows, w.ti * T::ROWS), operand(p.cols, w.tj * T::COLS), from, to, lds, acc);
        else multiply<T, PairProduct>(operand(p.rows, w.ti * T::ROWS), operand(p.cols, w.tj * T::COLS), from, to, lds, acc);
        __builtin_amdgcn_s_setprio(2);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (slot < 0) finish_tile<T, FINISH>(a, w, acc, size, lds + wave * kWaveScratch, wave);
        else store_part<T>(a.parts, slot, acc);
        __syncthreads();
    });
}

// A wave's share of a tile that was cut, a workgroup each
template <class T, int FINISH>
__global__ __launch_bounds__(64 * joiners<T>()) void join_kernel(ProductArgs a)
{
    __shared__ __align__(16) char lds[kWaveScratch + join_lds<T>()];
    const int tile = blockIdx.x / T::WAVES, wave = blockIdx.x % T::WAVES;
    const Place w = place_of(a, a.work.whole + tile);
    const float size = size_of<FINISH>(a, w);
    floatx4 acc[T::CT][T::RT];
    if (!join_parts<T, joiners<T>()>(a.work, tile, wave, a.parts, reinterpret_cast<floatx4 *>(lds + kWaveScratch), acc)) return;
    finish_tile<T, FINISH>(a, w, acc, size, lds, wave);
}

// The steps on one Gram matrix of up to 128 x 128 in one launch: a workgroup per matrix, A and B in LDS, P in memory
// (three matrices of pairs do not fit).  A wave has one 32 x 32 tile of the upper triangle; all read, then all write,
// so that a product may take the place of a factor.  A product takes 3.7 us of 128 x 128, a launch for it 6.
constexpr int kSide = 128, kSideTiles = kSide / 32, kChainWaves = kSideTiles * (kSideTiles + 1) / 2;
constexpr int kSideBytes = kSide / kPanel * kSide * kLine;

struct ChainArgs {
    PairMatrix gram;           // of the first step
    PairMatrix p[2];           // P after every step by turns, the first in p[0]
    int steps;
    ChainStep step[kStepsAtOnce];
};

__device__ __forceinline__ void lds_store_tile(char *lds, int row, int col, const uint2 (&hi)[4], const uint2 (&lo)[4], bool turned, int lane)
{
    const int r = lane & 15, q = lane >> 4, k = r >> 2;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int line = row + 16 * (g >> 1) + r, chunk = 2 * (g & 1) + (q >> 1);
        char *to = lds + (col / kPanel * kSide + line) * kLine + (q & 1) * 8;
        *reinterpret_cast<uint2 *>(to + slot_of(line, chunk) * 16) = hi[g];
        *reinterpret_cast<uint2 *>(to + slot_of(line, 4 + chunk) * 16) = lo[g];
        if (turned) {
            const int other = col + 16 * (g & 1) + 4 * q + (lane & 3), piece = 2 * (g >> 1) + (k >> 1);
            char *back = lds + (row / kPanel * kSide + other) * kLine + (k & 1) * 8;
            *reinterpret_cast<uint2 *>(back + slot_of(other, piece) * 16) = turn_quad(hi[g], lane);
            *reinterpret_cast<uint2 *>(back + slot_of(other, 4 + piece) * 16) = turn_quad(lo[g], lane);
        }
    }
}
// the same to memory, lines of `d`
__device__ __forceinline__ void memory_store_tile(const PairMatrix &d, char *to, int row, int col, const uint2 (&hi)[4], const uint2 (&lo)[4], bool turned, int lane)
{
    const int r = lane & 15, q = lane >> 4;
    if (col < panels(d.depth) * kPanel)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int line = row + 16 * (g >> 1) + r, chunk = 2 * (g & 1) + (q >> 1);
            if (line < d.rows) {
                *reinterpret_cast<uint2 *>(to + pair_at(d.rows, line, col / kPanel, chunk) + (q & 1) * 8) = hi[g];
                *reinterpret_cast<uint2 *>(to + pair_at(d.rows, line, col / kPanel, 4 + chunk) + (q & 1) * 8) = lo[g];
            }
        }
    if (turned && row < panels(d.depth) * kPanel) store_turned(d, to, row, col, hi, lo, lane);
}

__global__ __launch_bounds__(64 * kChainWaves) void chain_kernel(ChainArgs a)
{
    extern __shared__ __align__(16) char lds[];
    char *gram = lds, *step = lds + kSideBytes;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int m = a.gram.rows, lines = panels(m);
    int ti, tj;
    upper_tile(wave, kSideTiles, &ti, &tj);
    const int row = uniform(ti) * 32, col = uniform(tj) * 32;
    const bool there = row < m && col < lines * kPanel, turned = row != col;
    const char *from = a.gram.base + (int64_t)blockIdx.x * a.gram.stride;
    for (int e = threadIdx.x; e < 2 * kSideBytes / 16; e += 64 * kChainWaves) {
        const int line = e / 8, at = line % kSide, panel = line / kSide;
        const bool in = at < m && panel < lines;
        *reinterpret_cast<uint4 *>(lds + e * 16) = in ? *reinterpret_cast<const uint4 *>(from + ((int64_t)panel * m + at) * kLine + e % 8 * 16) : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    const FragmentPlace place(lane);
    typedef Fragment<half8> Frag;
    const auto read = [&](const char *matrix, int panel, int first, Frag (&f)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) place.load(f[i], matrix + (panel * kSide + first) * kLine, i);
    };
    const auto read_memory = [&](const char *matrix, int panel, int first, Frag (&f)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = min(first + 16 * i + r, m - 1);
            f[i].half[0] = *reinterpret_cast<const half8 *>(matrix + pair_at(m, at, panel, q));
            f[i].half[1] = *reinterpret_cast<const half8 *>(matrix + pair_at(m, at, panel, 4 + q));
        }
    };
    // the wave's tile of L R, R in LDS or in memory; v[2 i + j] as in for_wave_tiles
    floatx4 v[4];
    const auto product = [&](const char *l, auto &&read_right, const char *right) {
#pragma unroll
        for (int g = 0; g < 4; ++g) v[g] = floatx4{0, 0, 0, 0};
        if (!there) return;
        for (int k = 0; k < lines; ++k) {
            Frag rows[2], cols[2];
            read(l, k, row, rows);
            read_right(right, k, col, cols);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                floatx4 sum[2];
                PairProduct::line(rows, cols[j], sum);
                v[j] += sum[0], v[2 + j] += sum[1];
            }
        }
    };
    uint2 hi[4], lo[4];
    for (int k = 0; k < a.steps; ++k) {
        const ChainStep &now = a.step[k];
        char *p_now = a.p[k & 1].base + (int64_t)blockIdx.x * a.p[k & 1].stride;
        product(gram, read, gram);
        if (there) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int i = row + 16 * (g >> 1) + r, chunk = 2 * (g & 1) + (q >> 1), j = col + 16 * (g & 1) + 4 * q;
                const char *at = gram + (col / kPanel * kSide + i) * kLine + (q & 1) * 8;
                const half4 h = *reinterpret_cast<const half4 *>(at + slot_of(i, chunk) * 16), l = *reinterpret_cast<const half4 *>(at + slot_of(i, 4 + chunk) * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[g][e] = now.c * v[g][e] + now.b * ((float)h[e] + (float)l[e]) + (i == j + e ? now.a : 0.0f);
            }
            // (B is not read by anybody at this point)
            to_pairs(v, 1.0f, row, col, m, m, lane, hi, lo);
            lds_store_tile(step, row, col, hi, lo, turned, lane);
            if (k == 0) memory_store_tile(a.p[0], p_now, row, col, hi, lo, turned, lane);
        }
        __syncthreads();
        if (k > 0) {
            // P in memory was written by this workgroup, before a barrier, to lines that it had not read
            const char *before = a.p[(k - 1) & 1].base + (int64_t)blockIdx.x * a.p[0].stride;
            product(step, read_memory, before);
            if (there) {
                to_pairs(v, now.to_p, row, col, m, m, lane, hi, lo);
                memory_store_tile(a.p[k & 1], p_now, row, col, hi, lo, turned, lane);
            }
        }
        if (k + 1 < a.steps) {
            product(step, read, gram);
            __syncthreads();
            if (there) {
                to_pairs(v, now.to_w, row, col, m, m, lane, hi, lo);
                lds_store_tile(gram, row, col, hi, lo, turned, lane);
            }
            __syncthreads();
            product(gram, read, step);
            __syncthreads();
            if (there) {
                to_pairs(v, now.to_gram, row, col, m, m, lane, hi, lo);
                lds_store_tile(gram, row, col, hi, lo, turned, lane);
            }
            __threadfence_block();
            __syncthreads();
        }
    }
}

// No steps: X_0 itself is the result
__global__ __launch_bounds__(256) void unscaled_kernel(MatrixShape s, UpdateArgs u, int64_t first, const double *part, int parts)
{
    __shared__ double sums[256];
    const int64_t per = s.elems(), base = (first + blockIdx.y) * per;
    const Inverse f = inverse_norm(s, part, parts, blockIdx.y, 1.0f, Extra{}, sums);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (int64_t)gridDim.x * 256) {
        const float v = f.of(direction(u, fetch(u, s.dtype, base + i, false), base + i, false));
        if (u.weight) u.weight[base + i] = u.keep * u.weight[base + i] + u.add * v;
        else store_from_float(u.out, base + i, s.dtype, v);
    }
}

typedef TileShape<64, 64, 2, 2, 4> Tile64;
typedef TileShape<64, 64, 2, 2, 2> Tile64Alone;
typedef TileShape<128, 128, 2, 2, 2> Tile128;
typedef TileShape<256, 256, 4, 2, 2> Tile256;

constexpr int kUnits = 256;      // compute units

// `count` products of rows x cols, summed over `depth`
struct Batch {
    int rows, cols, depth;
    bool symmetric;
    int64_t count;
    int64_t tiles(int tile) const
    {
        const int64_t down = (rows + tile - 1) / tile, across = (cols + tile - 1) / tile;
        return symmetric ? down * (down + 1) / 2 : down * across;
    }
};

// How a batch of products is launched: the tiles, and who takes which of them.
// The larger the tile, the less is read per product and the more of a tile that straddles the diagonal or the end is
// wasted.  Measured (us, tiles of 64 / 128 / 256): 441 of 250 x 333 1720 / 1640 / 1800; 289 of 512 x 1024 7000 /
// 5480 / 5800; one of 4096 x 4096 5900 / 4770 / 4380; one of 1024 x 1024 300 / 563 / 997.  Rows of 193 to 256 fill two
// tiles of 128, which pays where there are tiles for one and a half turns of the units (two workgroups each): 441 of
// 200 x 300 1289 / 1178, 300 of 193 x 386 962 / 907, but 200 of 256 x 512 858 / 964.
struct Plan {
    int tile;
    bool alone;
    WorkSplit work;
    size_t parts() const { return work.cut() ? (size_t)2 * work.cutters * tile * tile * sizeof(float) : 0; }
};
// (joining takes 6 us, a stage of the smallest tile 0.25; 20 us and 1.8 for the largest)
template <class T, bool ALONE = false>
Plan plan_with(const Batch &b)
{
    const int workers = kUnits * ((ALONE ? Alone<T>::LDS : T::LDS) <= 80 * 1024 ? 2 : 1);
    return {T::ROWS, ALONE, WorkSplit::of((int)(b.tiles(T::ROWS) * b.count), panels(b.depth), workers, T::ROWS == 64 ? 24 : T::ROWS == 128 ? 20 : 12)};
}
Plan plan_of(const MatrixShape &s, const Batch &b)
{
    const int shorter = s.m();
    if (shorter > 512 && b.tiles(256) * b.count >= kUnits / 2) return plan_with<Tile256>(b);
    if (shorter > 192 && b.tiles(128) * b.count >= (shorter > 256 ? 2 : 3) * kUnits) return plan_with<Tile128>(b);
    if (b.tiles(64) * b.count > kUnits) return plan_with<Tile64>(b);
    return plan_with<Tile64Alone, true>(b);
}

template <class T, int FINISH, bool ALONE = false>
void launch_product_with(const ProductArgs &a, hipStream_t stream)
{
    constexpr int kLds = ALONE ? Alone<T>::LDS : T::LDS;
    if (kLds > 65536) allow_large_lds(reinterpret_cast<const void *>(product_kernel<T, FINISH, ALONE>), kLds);
    product_kernel<T, FINISH, ALONE><<<a.work.workers, T::THREADS, kLds, stream>>>(a);
    if (a.work.cut()) join_kernel<T, FINISH><<<a.work.left() * T::WAVES, 64 * joiners<T>(), 0, stream>>>(a);
}

template <int FINISH>
void launch_product(ProductArgs &a, hipStream_t stream)
{
    const Product &p = a.p[0];
    const Batch b{p.rows.rows, p.cols.rows, p.rows.depth, p.symmetric, (int64_t)a.matrices * a.problems};
    const Plan plan = plan_of(a.s, b);
    a.tiles_down = (b.rows + plan.tile - 1) / plan.tile;
    a.tiles_across = (b.cols + plan.tile - 1) / plan.tile;
    a.tiles = (int)b.tiles(plan.tile);
    a.work = plan.work;
    if (plan.tile == 256) launch_product_with<Tile256, FINISH>(a, stream);
    else if (plan.tile == 128) launch_product_with<Tile128, FINISH>(a, stream);
    else if (!plan.alone) launch_product_with<Tile64, FINISH>(a, stream);
    else launch_product_with<Tile64Alone, FINISH, true>(a, stream);
}

// Matrices that share the workspace at a time: the batch in equal parts of at most 256 M elements (parts of 32 M and
// less leave compute units without work at the end of every launch: 289 of 512 x 1024 took 7.7 ms instead of 6.2)
int64_t matrices_at_once(const MatrixShape &s)
{
    int64_t most = ((int64_t)256 << 20) / s.elems();
    most = most < 1 ? 1 : most > 16384 ? 16384 : most;
    const int64_t parts = (s.batch + most - 1) / most;
    return (s.batch + parts - 1) / parts;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// the workspace of `count` matrices
struct Layout {
    size_t norm, u, v[2], a, w, b[2], p[2], parts, size, total;
};
Layout layout_of(const MatrixShape &s, int64_t count)
{
    const size_t u = align256(count * pair_bytes(s.m(), s.n())), v = align256(count * pair_bytes(s.n(), s.m()));
    const size_t g = align256(count * pair_bytes(s.m(), s.m()));
    Layout l;
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += bytes; return here; };
    l.norm = take(align256(count * kNormParts * sizeof(double)));
    l.u = take(u), l.v[0] = take(v), l.v[1] = take(v);
    l.a = take(g), l.w = take(g), l.b[0] = take(g), l.b[1] = take(g), l.p[0] = take(g), l.p[1] = take(g);
    // what the products of a call have of parts at most: Gram matrices, products of polynomials, one or two at a time, X
    const int m = s.m(), n = s.n();
    size_t parts = 0;
    for (const Batch &b : {Batch{m, m, n, true, count}, Batch{m, m, m, true, count}, Batch{m, m, m, true, 2 * count}, Batch{s.flip() ? n : m, s.flip() ? m : n, m, false, count},
                           Batch{m, n, m, false, count}}) {
        const size_t bytes = plan_of(s, b).parts();
        parts = bytes > parts ? bytes : parts;
    }
    l.parts = take(align256(parts));
    // (last: matrices of pairs that start 256 bytes off multiples of 8 KiB make products 2 % slower)
    l.size = take(align256(count * sizeof(float)));
    l.total = at;
    return l;
}

}  // namespace

// The error against float64 is to stay within 1.5 times that of the steps as written in float32, for schedules that leave
// singular values apart (one that converges ends nearer to it than pairs are held: below).  float32's error grows with m,
// as its sums get longer; that of pairs comes from their rounding (2^-23 of a factor, float32 2^-24) and hardly grows.  So
// float32 wins where m is small: from 33 rows, where the polynomials go over to pairs, to 48 a step by itself already costs
// up to 1.3 times float32's error, two of them 1.3 to 2.  The error of a Gram matrix is multiplied by the square of a step's
// factor where the singular value is small, and so is that of long rows, whose eigenvalues are small.  Measured, the error
// relative to that of float32 for gradients with a few strong directions and five steps of a factor of 3.44 (64 and fewer
// matrices a shape, geometric mean):
//   m x n       one   two   three at once  |  m x n       one   two   three at once
//   16 x 200    0.80  1.21  1.06           |  64 x 144    0.77  0.89  2.61
//   28 x 56     0.90  1.18  1.83           |  100 x 100   0.52  1.16  1.67
//   32 x 256    0.96  1.35  0.93           |  128 x 2000  0.63  0.63  1.29
//   33 x 66     1.19  1.82  2.70           |  192 x 1537  0.59  0.57  1.65
//   40 x 80     1.06  1.67  2.66           |  193 x 400   0.52  0.58  1.21
//   41 x 328    1.22  1.80  1.27           |  250 x 333   0.41  0.68  0.99
//   44 x 110    1.07  1.55  2.25           |  256 x 256   0.38  0.75  1.14
//   46 x 115    1.02  1.48  2.26           |  256 x 2100  0.38  0.31  1.12
//   46 x 138    1.07  1.53  1.90           |  320 x 3000  0.36  0.28  1.03
//   48 x 384    1.18  1.53  1.54           |  512 x 512   0.29  0.46  0.87
//   46 x 552    0.99  1.37  1.21           |  1024 x 1024 0.26  0.37  0.72
//   60 x 60     0.81  1.72  2.48           |  50 x 300    1.11  1.46  1.61
// With the rule below the largest of 681 shapes from 2 x 2 to 700 x 5600 is 1.46 (20 x 160).  A step with a larger factor
// is not followed by others: with factors of 8.2, 4.1, 3.9, 3.3, 2.3 two at once had 2.3 (100 x 100), three 1.9 (250 x 333)
// and 2.2 (256 x 256).  Eight steps (1.5, -0.5, 0), which converge: 2.2 to 2.8 times float32's 1.7e-7 to 2.2e-7, however
// many are taken at once.
int steps_until(const MatrixShape &s, const ScheduleBounds &bounds, int steps, int k)
{
    const int m = s.m(), n = s.n();
    int most;
    if (m <= 64 && (n < 2 * m || (m > 32 && m < 46) || (m >= 46 && m <= 48 && 2 * n >= 5 * m && n < 12 * m))) most = 1;
    else if (m <= 32) most = n <= 8 * m ? 2 : 3;
    else if (m <= 192) most = 2;
    else most = m <= 256 && n > 2 * m ? 2 : 3;
    int end = k + 1;
    while (end < steps && end < k + most && bounds.factor[end - 1] <= 3.5f) ++end;
    return end;
}

float pair_scale(double bound) { return (float)exp2(floor(log2(32000.0 / fmax(bound, 0x1p-113)))); }

ChainStep chain_step(const ScheduleBounds &bounds, const float *schedule, int k, double *factor)
{
    const double r = bounds.singular[k], next = bounds.singular[k + 1], most = bounds.factor[k];
    const double gram = pair_scale(r * r), step = pair_scale(most), w = pair_scale(most * r * r), before = pair_scale(*factor);
    *factor *= most;
    ChainStep c;
    c.a = (float)(schedule[3 * k] * step);
    c.b = (float)(schedule[3 * k + 1] * step / gram);
    c.c = (float)(schedule[3 * k + 2] * step / (gram * gram));
    c.to_w = (float)(w / (step * gram));
    c.to_gram = (float)(pair_scale(next * next) / (step * w));
    c.to_p = (float)(pair_scale(*factor) / (step * before));
    c.step_inverse = (float)(1.0 / step), c.p_inverse = (float)(1.0 / before);
    return c;
}

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
        // a + 3 b u + 5 c u^2 = 0 (no root: NaN).  The sum has terms of one sign: the difference would lose the smaller root
        // where c is small.
        const double sum = -0.5 * (3.0 * b + copysign(sqrt(9.0 * b * b - 20.0 * a * c), b));
        if (c != 0.0) visit(sum / (5.0 * c));
        if (sum != 0.0) visit(a / sum);
        if (!(singular <= kMaxSingular) || !(factor <= kMaxFactor)) return false;
        r = singular;
        bounds->factor[k] = (float)factor;
        bounds->singular[k + 1] = (float)singular;
    }
    return true;
}


size_t ortho_workspace_bytes(const MatrixShape &s)
{
    const int64_t most = matrices_at_once(s), left = s.batch % most;
    if (ortho_small_applicable(s, 1)) {
        // (a call without steps sums norms only)
        const size_t small = ortho_small_workspace_bytes(s), norms = align256(most * kNormParts * sizeof(double));
        return small > norms ? small : norms;
    }
    const size_t whole = layout_of(s, most).total, rest = left ? layout_of(s, left).total : 0;
    return whole > rest ? whole : rest;
}

void launch_ortho(const MatrixShape &s, int steps, const float *schedule, const UpdateArgs &u, void *workspace, hipStream_t stream)
{
    if (ortho_small_applicable(s, steps)) return launch_ortho_small(s, steps, schedule, u, workspace, stream);
    ScheduleBounds bounds;
    (void)schedule_bounds(steps, schedule, &bounds);
    const int m = s.m(), n = s.n();
    const int64_t most = matrices_at_once(s);
    for (int64_t first = 0; first < s.batch; first += most) {
        const int64_t count = s.batch - first < most ? s.batch - first : most;
        const Layout l = layout_of(s, count);
        char *ws = static_cast<char *>(workspace);
        const auto pairs = [&](size_t at, int rows, int depth, double bound) {
            const float scale = pair_scale(bound);
            return PairMatrix{ws + at, pair_bytes(rows, depth), rows, depth, scale, 1.0f / scale};
        };
        // of X before step k; the scale and the bits besides end at 2^114
        double grow = 1.0;
        const auto extra_of_x = [&](int k) {
            const int most = 114 - ilogbf(pair_scale(bounds.singular[k]));
            return Extra{(float)grow, bounds.singular[k], most < 0 ? 0 : most};
        };
        double *part = reinterpret_cast<double *>(ws + l.norm);
        const int64_t some = (s.elems() + 4095) / 4096;
        const int parts = (int)(some < kNormParts ? some : kNormParts);
        norm_kernel<<<dim3(parts, (unsigned)count), 256, 0, stream>>>(s, u, first, part);
        if (steps == 0) {
            unscaled_kernel<<<dim3((unsigned)(some < 1024 ? some : 1024), (unsigned)count), 256, 0, stream>>>(s, u, first, part, parts);
            continue;
        }
        const PairMatrix none{};
        float *size = reinterpret_cast<float *>(ws + l.size);
        PairMatrix x = pairs(l.u, m, n, 1.0), xt = pairs(l.v[0], n, m, 1.0);
        int turned = 0;
        const unsigned tiles = (unsigned)(((s.rows + 63) / 64) * (int64_t)((s.cols + 63) / 64));
        split_kernel<<<dim3(tiles, 1, (unsigned)count), 256, 0, stream>>>(SplitArgs{s, u, first, part, parts, s.flip() ? xt : x, s.flip() ? x : xt, extra_of_x(0), size});
        ProductArgs args = {};
        args.matrices = (int)count;
        args.s = s;
        args.u = u;
        args.first = first;
        args.by_four = s.cols % 4 == 0 && reinterpret_cast<uintptr_t>(u.weight ? (const void *)u.weight : u.out) % (u.weight || s.dtype == LMKAN_F32 ? 16 : 8) == 0;
        args.parts = reinterpret_cast<floatx4 *>(ws + l.parts);
        args.size = size;
        args.in = extra_of_x(0);
        const auto one = [&](const Product &p) { args.p[0] = p, args.problems = 1; };
        const auto kept = [&](const PairMatrix &rows, const PairMatrix &cols, const PairMatrix &out, const PairMatrix &mirror, bool symmetric) {
            return Product{rows, cols, out, mirror, none, symmetric, 0, 0, 0, (float)((double)out.scale * rows.inverse * cols.inverse)};
        };
        for (int k = 0; k < steps;) {
            const int end = steps_until(s, bounds, steps, k);
            const double r = bounds.singular[k];
            PairMatrix gram = pairs(l.a, m, m, r * r), so_far = none;
            one(kept(x, x, gram, gram, true));
            args.x_factors = 2, args.out = Extra{};
            launch_product<kKeepX>(args, stream);
            double factor = 1.0;
            if (m <= kSide) {
                ChainArgs chain = {};
                chain.gram = gram;
                chain.steps = end - k;
                for (int i = 0; i < chain.steps; ++i) chain.step[i] = chain_step(bounds, schedule, k + i, &factor);
                chain.p[0] = pairs(l.p[0], m, m, factor), chain.p[1] = pairs(l.p[1], m, m, factor);
                allow_large_lds(reinterpret_cast<const void *>(chain_kernel), 2 * kSideBytes);
                chain_kernel<<<(unsigned)count, 64 * kChainWaves, 2 * kSideBytes, stream>>>(chain);
                so_far = chain.p[(chain.steps - 1) & 1];
                k = end;
            }
            for (const int begin = k; k < end; ++k) {
                const double now = bounds.singular[k], next = bounds.singular[k + 1];
                const PairMatrix step = pairs(l.b[k & 1], m, m, bounds.factor[k]);
                const ChainStep c = chain_step(bounds, schedule, k, &factor);
                one(Product{gram, gram, step, step, gram, true, c.a, c.b, c.c, 0});
                launch_product<kPoly>(args, stream);
                const PairMatrix w = pairs(l.w, m, m, bounds.factor[k] * now * now);
                args.problems = 0;
                if (k + 1 < end) args.p[args.problems++] = kept(step, gram, w, w, true);
                if (k > begin) {
                    const PairMatrix longer = pairs(l.p[k & 1], m, m, factor);
                    args.p[args.problems++] = kept(step, so_far, longer, longer, true);
                    so_far = longer;
                } else {
                    so_far = step;
                }
                if (args.problems) launch_product<kKeep>(args, stream);
                if (k + 1 < end) {
                    gram = pairs(l.a, m, m, next * next);
                    one(kept(w, step, gram, gram, true));
                    launch_product<kKeep>(args, stream);
                }
            }
            if (k < steps) {
                const PairMatrix y = pairs(l.u, m, n, bounds.singular[k]), yt = pairs(l.v[turned ^ 1], n, m, bounds.singular[k]);
                one(kept(so_far, xt, y, yt, false));
                grow *= factor;
                args.x_factors = 1, args.out = extra_of_x(k);
                launch_product<kKeepX>(args, stream);
                args.in = args.out;
                x = y, xt = yt, turned ^= 1;
            } else {
                one(s.flip() ? Product{xt, so_far, none, none, none, false, 0, 0, 0, 0} : Product{so_far, xt, none, none, none, false, 0, 0, 0, 0});
                args.x_factors = 1, args.out = Extra{};
                launch_product<kResult>(args, stream);
            }
        }
    }
}

}  // namespace lmkan
