// Orthogonalisation of matrices whose shorter side is at most 64.
//
// The steps are those of lmkan_ortho.hip: up to three on the m x m Gram matrix, applied together.  Here the Gram
// matrix and its polynomials fit the LDS of one workgroup, so that a matrix costs
//   one launch   where X fits LDS too (whole_kernel): X is read once and the result written once;
//   1 + 2 g      where it is longer, for g groups of steps that share a Gram matrix (steps_until): Gram matrix in parts,
//                then polynomial, and apply with the next Gram matrix in parts; 1 + 3 g where more than 16 parts are summed
//                by a launch of their own.  Five steps: g = 2 up to 32 rows, 5 up to 45, 3 from 46 on.
//                One of 16 x 70001 takes 49 us, one of 48 x 20000 76, one of 64 x 65536 129, four of 64 x 16384 118.
// The products with X take 2 m multiply-adds per element and pass; at m = 64 the float32 instructions (157 TFLOP/s)
// take about as long for that as memory takes for the element, so nothing is gained by splitting factors.  The products
// of the polynomials are a chain in one workgroup: from m = 33 on, pairs of float16 (lmkan_tile.h) make it shorter.
//
// Norms: |X|^2 is the trace of the Gram matrix of the raw direction D, A_0 = D D^T / (|D| + eps)^2 and the first
// polynomial is scaled by 1 / (|D| + eps).  The squares are float32 products, so that D is held times a power of two by its
// largest element: beyond 2^50 times 2^-90, up to 2^-40 times 2^90.  Squares then leave float32's normal range only for
// elements of less than 2^-23 of the largest.  Every workgroup goes by the elements it sees; the trace and the sums of
// parts, in the range of the largest, are taken in float64.
#include "lmkan_dense.h"

#include <math.h>

#include "lmkan_kernels.h"
#include "lmkan_tile.h"

namespace lmkan {

namespace {

// Ranges by the largest element: 0 up to 2^-40, 1 up to 2^50, 2 beyond (or not a number)
constexpr uint32_t kTiny = (127 - 40) << 23, kLarge = (127 + 50) << 23;   // bits of 2^-40 and 2^50
__device__ __forceinline__ float range_scale(int range) { return range == 0 ? 0x1p90f : range == 1 ? 1.0f : 0x1p-90f; }
__device__ __forceinline__ double range_units(int ranges) { return ranges == 0 ? 1.0 : ranges == 1 ? 0x1p-180 : 0x1p-360; }   // of products, so many ranges down
// the bits of a magnitude are ordered like the values, NaN above infinity
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
// The range of what all threads have seen, `before` of what they saw earlier, from each one's largest magnitude
__device__ __forceinline__ int range_of_all(uint32_t top, int before)
{
    if (__syncthreads_or(top > kLarge)) return 2;
    return before > 0 ? before : __syncthreads_or(top > kTiny);
}
constexpr int kSmallLds = 150 * 1024;      // of 160 KiB
constexpr int kMostParts = 512;            // parts of a Gram matrix

// e / d for e < 2^16, d <= 2^12
struct Divide {
    unsigned magic, d;
    __device__ __forceinline__ int quotient(int e) const { return d == 1 ? e : (int)__umulhi((unsigned)e, magic); }
    static Divide by(int d) { return {(unsigned)(((1ull << 32) + d - 1) / d), (unsigned)d}; }
};

struct SmallArgs {
    MatrixShape s;
    UpdateArgs u;
    int steps, from, to;                   // steps [from, to) of the schedule
    float schedule[3 * LMKAN_MAX_ORTHO_STEPS];
    ChainStep step[LMKAN_MAX_ORTHO_STEPS];        // in pairs
    float gram_scale[LMKAN_MAX_ORTHO_STEPS];      // the power of two that pairs of the Gram matrix are held times
    int end[LMKAN_MAX_ORTHO_STEPS];        // the step after those on one Gram matrix, by the first of them
    int columns;                           // of X in LDS at a time, a multiple of 16
    Divide by_fours;                       // columns / 4
    bool whole_fours;                      // four adjacent elements from a multiple of four on are whole and aligned
    int parts;                             // workgroups that share a matrix
    float *gram;                           // [matrices][parts][M][M], upper tiles
    double *sum;                           // [matrices][M][M]: their sums, where they are many
    int *range;                            // [matrices][parts]: of the elements in a part
    float *poly;                           // [matrices][M][M]
    float *unit;                           // [matrices]: what the direction is to be scaled by, by its range
    float *x;                              // [matrices][m][n]: X after a polynomial
};

// element (row, column) of the direction, seen with the shorter side first
__device__ __forceinline__ int64_t stored_at(const MatrixShape &s, int64_t matrix, int row, int column)
{
    return matrix * s.elems() + (s.flip() ? (int64_t)column * s.cols + row : (int64_t)row * s.cols + column);
}

// Four adjacent elements of what is stored, `count` of which exist; `whole`: all four, aligned to their size together
struct Raw4 {
    floatx4 g, m;
};
__device__ __forceinline__ floatx4 load_four(const void *p, int dtype, int64_t at, int count, bool whole)
{
    floatx4 v = {0, 0, 0, 0};
    if (whole) {
        if (dtype == LMKAN_F32) return *reinterpret_cast<const floatx4 *>(static_cast<const float *>(p) + at);
        const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + at);
        const uint16_t h[4] = {(uint16_t)u.x, (uint16_t)(u.x >> 16), (uint16_t)u.y, (uint16_t)(u.y >> 16)};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = load_as_float(h, e, dtype);
        return v;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) v[e] = load_as_float(p, at + e, dtype);
    return v;
}
__device__ __forceinline__ void store_four(void *p, int dtype, int64_t at, int count, bool whole, const floatx4 &v)
{
    if (whole) {
        if (dtype == LMKAN_F32) *reinterpret_cast<floatx4 *>(static_cast<float *>(p) + at) = v;
        else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + at) = make_uint2(two_from_float(dtype, v[0], v[1]), two_from_float(dtype, v[2], v[3]));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) store_from_float(p, at + e, dtype, v[e]);
}
// the direction's, in two halves as fetch() and direction() do one
__device__ __forceinline__ Raw4 fetch_four(const UpdateArgs &u, int dtype, int64_t at, int count, bool whole, bool move)
{
    Raw4 r = {};
    if (!u.momentum || u.nesterov || move) r.g = load_four(u.grad, dtype, at, count, whole);
    if (u.momentum) r.m = load_four(u.momentum, LMKAN_F32, at, count, whole);
    return r;
}
__device__ __forceinline__ floatx4 direction_four(const UpdateArgs &u, Raw4 r, int64_t at, int count, bool whole, bool move)
{
    if (!u.momentum) return r.g;
    if (move) {
        r.m = u.beta * r.m + (1.0f - u.beta) * r.g;
        store_four(u.momentum, LMKAN_F32, at, count, whole, r.m);
    }
    return u.nesterov ? u.beta * r.m + (1.0f - u.beta) * r.g : r.m;
}
__device__ __forceinline__ void store_result_four(const SmallArgs &a, int64_t at, int count, bool whole, const floatx4 &v)
{
    if (a.u.weight) {
        const floatx4 w = load_four(a.u.weight, LMKAN_F32, at, count, whole);
        store_four(a.u.weight, LMKAN_F32, at, count, whole, a.u.keep * w + a.u.add * v);
    } else {
        store_four(a.u.out, a.s.dtype, at, count, whole, v);
    }
}

// M: the shorter side rounded up to 16; WAVES of a workgroup
template <int M_, int WAVES_>
struct Small {
    static constexpr int M = M_, WAVES = WAVES_, THREADS = 64 * WAVES;
    static constexpr int T = M / 16, TILES = T * (T + 1) / 2;                 // tiles of a symmetric matrix
    static constexpr int SHARE = TILES < WAVES && TILES == 1 ? WAVES : 1;     // waves that share a tile's summed axis
    static constexpr int EACH = SHARE > 1 ? 1 : (TILES + WAVES - 1) / WAVES;  // tiles of a wave
    static constexpr int PITCH = M + 4;
    static constexpr int SQUARE = M * PITCH;                                  // floats of an M x M matrix in LDS
    static constexpr bool PAIRS = M >= 48;                                    // products of polynomials in pairs
    static constexpr int LINES = (M + kPanel - 1) / kPanel, PAIR_SQUARE = LINES * M * kLine;   // bytes of one of pairs
    static constexpr int REST = PAIRS ? 3 * PAIR_SQUARE : 2 * SQUARE * (int)sizeof(float);     // bytes that polynomial() needs

    // tile t of the upper triangle, column by column
    static __device__ __forceinline__ void tile(int t, int *i, int *j)
    {
        int c = 0;
        while ((c + 1) * (c + 2) / 2 <= t) ++c;
        *j = c, *i = t - c * (c + 1) / 2;
    }

    // a lane's four values along the summed axis of row `row + (lane & 15)`: 4 (lane >> 4) ..
    static __device__ __forceinline__ floatx4 along(const float *lds, int pitch, int row, int k, int lane)
    {
        return *reinterpret_cast<const floatx4 *>(lds + (row + (lane & 15)) * pitch + k + 4 * (lane >> 4));
    }
    static __device__ __forceinline__ floatx4 multiply(const floatx4 &cols, const floatx4 &rows, floatx4 acc)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(cols[e], rows[e], acc, 0, 0, 0);
        return acc;
    }

    // Calls f(row, column, count) for every four adjacent elements of what is stored of columns [first, first + columns),
    // kAtOnce of them at a time: f(first of them, ...) is for loads, g(...) for what follows.  `count` may be zero or negative.
    template <class F, class G>
    static __device__ __forceinline__ void for_fours(const MatrixShape &s, int first, int columns, const Divide &by_fours, F &&f, G &&g)
    {
        constexpr int kAtOnce = 4;
        const int m = s.m(), n = s.n(), fours = M * columns / 4;
        const bool flip = s.flip();
        for (int e0 = threadIdx.x; e0 < fours; e0 += kAtOnce * THREADS) {
#pragma unroll
            for (int pass = 0; pass < 2; ++pass)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int e = e0 + u * THREADS, q = flip ? e / (M / 4) : by_fours.quotient(e);
                    const int r = flip ? 4 * (e % (M / 4)) : q, c = flip ? q : 4 * (e - q * (columns / 4));
                    const int count = flip ? (first + c < n ? m - r : 0) : (r < m ? n - first - c : 0);
                    if (e >= fours) break;
                    if (pass == 0) f(u, r, c, count);
                    else g(u, r, c, count);
                }
        }
    }

    // X: columns [first, first + columns) of all rows to LDS, zero beyond the matrix; returns the thread's largest magnitude.
    // get(at, count, whole) loads the elements stored from `at` on, use(...) makes the direction of them.
    template <class G, class U>
    static __device__ __forceinline__ uint32_t load(float *x, int pitch, const MatrixShape &s, int64_t matrix, int first, int columns, const Divide &by_fours, bool whole, G &&get, U &&use)
    {
        uint32_t top = 0;
        Raw4 raw[4];
        const bool flip = s.flip();
        for_fours(s, first, columns, by_fours,
            [&](int u, int r, int c, int count) {
                if (count > 0) raw[u] = get(stored_at(s, matrix, r, first + c), count, whole && count >= 4);
            },
            [&](int u, int r, int c, int count) {
                floatx4 v = {0, 0, 0, 0};
                if (count > 0) v = use(raw[u], stored_at(s, matrix, r, first + c), count, whole && count >= 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (e >= count) v[e] = 0.0f;
                    top = max(top, magnitude(v[e]));
                }
                if (!flip) {
                    *reinterpret_cast<floatx4 *>(x + r * pitch + c) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[(r + e) * pitch + c] = v[e];
                }
            });
        return top;
    }

    // Columns [first, first + columns) of X from LDS: put(at, count, whole, values) for every four adjacent stored elements
    template <class P>
    static __device__ __forceinline__ void store(const float *x, int pitch, const MatrixShape &s, int64_t matrix, int first, int columns, const Divide &by_fours, bool whole, P &&put)
    {
        const bool flip = s.flip();
        for_fours(s, first, columns, by_fours, [](int, int, int, int) {},
            [&](int, int r, int c, int count) {
                if (count <= 0) return;
                floatx4 v;
                if (!flip) {
                    v = *reinterpret_cast<const floatx4 *>(x + r * pitch + c);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = x[(r + e) * pitch + c];
                }
                put(stored_at(s, matrix, r, first + c), count, whole && count >= 4, v);
            });
    }

    // acc += X X^T over the columns in LDS, the wave's tiles
    static __device__ __forceinline__ void gram(const float *x, int pitch, int columns, int wave, int lane, floatx4 (&acc)[EACH])
    {
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int t = SHARE > 1 ? 0 : wave + q * WAVES;
            if (t >= TILES) break;
            int i, j;
            tile(t, &i, &j);
            for (int k = SHARE > 1 ? 16 * wave : 0; k < columns; k += 16 * SHARE)
                acc[q] = multiply(along(x, pitch, 16 * j, k, lane), along(x, pitch, 16 * i, k, lane), acc[q]);
        }
    }

    // Calls f(row, col, values): four adjacent columns of a row of the wave's tiles.  SHARE: sums over the waves first,
    // through `scratch` (4 floats a thread); wave 0 goes on.
    template <class F>
    static __device__ __forceinline__ void for_tiles(floatx4 (&acc)[EACH], int wave, int lane, float *scratch, F &&f)
    {
        if (SHARE > 1) {
            *reinterpret_cast<floatx4 *>(scratch + 4 * threadIdx.x) = acc[0];
            __syncthreads();
            if (wave != 0) return;
            for (int w = 1; w < WAVES; ++w) acc[0] += *reinterpret_cast<const floatx4 *>(scratch + 4 * (64 * w + lane));
        }
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int t = SHARE > 1 ? 0 : wave + q * WAVES;
            if (t >= TILES) break;
            int i, j;
            tile(t, &i, &j);
            f(16 * i + (lane & 15), 16 * j + 4 * (lane >> 4), i != j, acc[q]);
        }
    }

    // D = f(L R), all three symmetric; D may be L or R
    template <class F>
    static __device__ __forceinline__ void product(float *d, const float *l, const float *r, int wave, int lane, F &&f)
    {
        floatx4 acc[EACH];
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            acc[q] = floatx4{0, 0, 0, 0};
            const int t = wave + q * WAVES;
            if (t >= TILES) break;
            int i, j;
            tile(t, &i, &j);
#pragma unroll
            for (int k = 0; k < M; k += 16) acc[q] = multiply(along(r, PITCH, 16 * j, k, lane), along(l, PITCH, 16 * i, k, lane), acc[q]);
        }
        // (in place: all have read; f may read d at its own element)
        floatx4 v[EACH];
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int t = wave + q * WAVES;
            if (t >= TILES) break;
            int i, j;
            tile(t, &i, &j);
            v[q] = f(16 * i + (lane & 15), 16 * j + 4 * (lane >> 4), acc[q]);
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            const int t = wave + q * WAVES;
            if (t >= TILES) break;
            int i, j;
            tile(t, &i, &j);
            const int row = 16 * i + (lane & 15), col = 16 * j + 4 * (lane >> 4);
            *reinterpret_cast<floatx4 *>(d + row * PITCH + col) = v[q];
            if (i != j)
#pragma unroll
                for (int e = 0; e < 4; ++e) d[(col + e) * PITCH + row] = v[q][e];
        }
        __syncthreads();
    }

    // The steps [from, to) of the schedule on the Gram matrix `a` in LDS; returns their polynomial.  `rest`: REST bytes.
    static __device__ __forceinline__ float *polynomial(const SmallArgs &s, int from, int to, float *a, char *rest, int wave, int lane)
    {
        if constexpr (PAIRS) {
            polynomial_of_pairs(s, from, to, a, rest, wave, lane);
            return a;
        }
        float *b = reinterpret_cast<float *>(rest), *p = b + SQUARE;
        for (int k = from; k < to; ++k) {
            const float c0 = s.schedule[3 * k], c1 = s.schedule[3 * k + 1], c2 = s.schedule[3 * k + 2];
            float *step = k == from ? p : b;
            product(step, a, a, wave, lane, [&](int row, int col, floatx4 v) {
                const floatx4 g = *reinterpret_cast<const floatx4 *>(a + row * PITCH + col);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = c2 * v[e] + c1 * g[e] + (row == col + e ? c0 : 0.0f);
                return v;
            });
            const auto same = [](int, int, floatx4 v) { return v; };
            if (k + 1 < to) {
                product(a, step, a, wave, lane, same);
                product(a, a, step, wave, lane, same);
            }
            if (k > from) product(p, b, p, wave, lane, same);
        }
        return p;
    }

    // where the four adjacent columns of a lane's row of tile (i, j) lie in a square of pairs, hi; and turned, column
    // 16 j + 4 (lane >> 4) + (lane & 3), four adjacent rows
    static __device__ __forceinline__ int pair_place(int i, int j, int lane, bool lo)
    {
        const int r = 16 * i + (lane & 15), q = lane >> 4, chunk = 2 * (j & 1) + (q >> 1);
        return (j / 2 * M + r) * kLine + slot_of(r, chunk + (lo ? 4 : 0)) * 16 + (q & 1) * 8;
    }
    static __device__ __forceinline__ int turned_place(int i, int j, int lane, bool lo)
    {
        const int r = 16 * j + 4 * (lane >> 4) + (lane & 3), k = (lane & 15) >> 2, chunk = 2 * (i & 1) + (k >> 1);
        return (i / 2 * M + r) * kLine + slot_of(r, chunk + (lo ? 4 : 0)) * 16 + (k & 1) * 8;
    }

    // The same in pairs: `square` holds A and, at the end, the polynomial.  A wave has one tile of the upper triangle; all
    // read, then all write.
    static __device__ __forceinline__ void polynomial_of_pairs(const SmallArgs &s, int from, int to, float *square, char *rest, int wave, int lane)
    {
        static_assert(!PAIRS || TILES <= WAVES, "a tile a wave");
        char *a = rest, *b = a + PAIR_SQUARE, *p = b + PAIR_SQUARE;
        for (int e = threadIdx.x; e < M * LINES * 4; e += THREADS) {
            // eight values a thread, zero beyond the last column
            const int row = e / (LINES * 4), chunk = e % (LINES * 4);
            half8 hi, lo;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float v = chunk * 8 < M ? square[row * PITCH + chunk * 8 + k] * s.gram_scale[from] : 0.0f;
                hi[k] = (_Float16)v, lo[k] = (_Float16)(v - (float)hi[k]);
            }
            char *to = a + (chunk / 4 * M + row) * kLine;
            *reinterpret_cast<half8 *>(to + slot_of(row, chunk % 4) * 16) = hi;
            *reinterpret_cast<half8 *>(to + slot_of(row, 4 + chunk % 4) * 16) = lo;
            if (M % kPanel != 0) {
                // (what products never write of the others)
                const half8 zero = {};
                if (chunk * 8 >= M)
                    for (int t = 1; t < 3; ++t) {
                        *reinterpret_cast<half8 *>(to + t * PAIR_SQUARE + slot_of(row, chunk % 4) * 16) = zero;
                        *reinterpret_cast<half8 *>(to + t * PAIR_SQUARE + slot_of(row, 4 + chunk % 4) * 16) = zero;
                    }
            }
        }
        __syncthreads();
        const bool there = wave < TILES;
        int i = 0, j = 0;
        if (there) tile(wave, &i, &j);
        const FragmentPlace place(lane);
        floatx4 v;
        const auto multiply_pairs = [&](const char *l, const char *r) {
            v = floatx4{0, 0, 0, 0};
            if (!there) return;
#pragma unroll
            for (int k = 0; k < LINES; ++k) {
                Fragment<half8> rows[1], cols;
                place.load(rows[0], l + k * M * kLine, i);
                place.load(cols, r + k * M * kLine, j);
                floatx4 sum[1];
                PairProduct::line(rows, cols, sum);
                v += sum[0];
            }
        };
        const auto keep = [&](char *to, float scale) {
            if (!there) return;
            half4 h, l;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = (_Float16)(v[e] * scale);
#pragma unroll
            for (int e = 0; e < 4; ++e) l[e] = (_Float16)__builtin_fmaf((float)h[e], -1.0f, v[e] * scale);
            const uint2 hi = __builtin_bit_cast(uint2, h), lo = __builtin_bit_cast(uint2, l);
            *reinterpret_cast<uint2 *>(to + pair_place(i, j, lane, false)) = hi;
            *reinterpret_cast<uint2 *>(to + pair_place(i, j, lane, true)) = lo;
            if (i != j) {
                *reinterpret_cast<uint2 *>(to + turned_place(i, j, lane, false)) = turn_quad(hi, lane);
                *reinterpret_cast<uint2 *>(to + turned_place(i, j, lane, true)) = turn_quad(lo, lane);
            }
        };
        const auto result = [&](float first, float second) {
            if (there) put_square(square, 16 * i + (lane & 15), 16 * j + 4 * (lane >> 4), i != j, v * first * second);
        };
        for (int k = from; k < to; ++k) {
            const ChainStep &now = s.step[k];
            char *step = k == from ? p : b;
            multiply_pairs(a, a);
            if (there) {
                const half4 h = *reinterpret_cast<const half4 *>(a + pair_place(i, j, lane, false)), l = *reinterpret_cast<const half4 *>(a + pair_place(i, j, lane, true));
                const int row = 16 * i + (lane & 15), col = 16 * j + 4 * (lane >> 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = now.c * v[e] + now.b * ((float)h[e] + (float)l[e]) + (row == col + e ? now.a : 0.0f);
            }
            if (k + 1 == to && k == from) return result(now.step_inverse, 1.0f), __syncthreads();
            keep(step, 1.0f);   // (B and P are read by nobody at this point)
            __syncthreads();
            if (k > from) {
                multiply_pairs(b, p);
                if (k + 1 == to) {
                    result(now.step_inverse, now.p_inverse);
                } else {
                    __syncthreads();
                    keep(p, now.to_p);
                }
            }
            if (k + 1 < to) {
                multiply_pairs(step, a);
                __syncthreads();
                keep(a, now.to_w);
                __syncthreads();
                multiply_pairs(a, step);
                __syncthreads();
                keep(a, now.to_gram);
            }
            __syncthreads();
        }
    }

    static __device__ __forceinline__ void put_square(float *a, int row, int col, bool mirror, const floatx4 &v)
    {
        *reinterpret_cast<floatx4 *>(a + row * PITCH + col) = v;
        if (mirror)
#pragma unroll
            for (int e = 0; e < 4; ++e) a[(col + e) * PITCH + row] = v[e];
    }

    // X <- P X over the columns in LDS; a wave takes 16 columns at a time, in place
    static __device__ __forceinline__ void apply(const float *p, float *x, int pitch, int columns, int wave, int lane)
    {
        for (int c = 16 * wave; c < columns; c += 16 * WAVES) {
            floatx4 acc[T];
#pragma unroll
            for (int i = 0; i < T; ++i) acc[i] = floatx4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < M; k += 16) {
                floatx4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = x[(k + 4 * (lane >> 4) + e) * pitch + c + (lane & 15)];
#pragma unroll
                for (int i = 0; i < T; ++i) acc[i] = multiply(v, along(p, PITCH, 16 * i, k, lane), acc[i]);
            }
#pragma unroll
            for (int i = 0; i < T; ++i) *reinterpret_cast<floatx4 *>(x + (16 * i + (lane & 15)) * pitch + c + 4 * (lane >> 4)) = acc[i];
        }
    }
};

// The Gram matrix of the scaled direction to that of X_0, in place, from its trace; returns what takes the scaled
// direction to X_0.  `eps`: times the same scale.
template <class S>
__device__ __forceinline__ float normalise(float *a, int m, double eps, double *shared, int lane)
{
    __syncthreads();
    if (threadIdx.x < 64) {
        double trace = lane < m ? (double)a[lane * S::PITCH + lane] : 0.0;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) trace += __shfl_xor(trace, d, 64);
        if (lane == 0) *shared = 1.0 / (sqrt(trace) + eps);
    }
    __syncthreads();
    const double inverse = *shared;
    const double f = inverse * inverse;
    for (int e = threadIdx.x; e < S::SQUARE; e += S::THREADS) a[e] = (float)((double)a[e] * f);
    __syncthreads();
    return (float)inverse;
}

template <class S>
__device__ __forceinline__ void scale_square(float *p, float f)
{
    for (int e = threadIdx.x; e < S::SQUARE; e += S::THREADS) p[e] *= f;
    __syncthreads();
}

template <class S>
__device__ __forceinline__ void scale_columns(float *x, int pitch, int columns, float f)
{
    for (int e = threadIdx.x; e < S::M * pitch; e += S::THREADS) x[e] *= f;
    __syncthreads();
}

// A workgroup per matrix, all of it in LDS: X and three M x M matrices
template <class S>
__global__ __launch_bounds__(S::THREADS) void whole_kernel(SmallArgs a)
{
    extern __shared__ __align__(16) float lds[];
    __shared__ double shared;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t matrix = blockIdx.x;
    const int columns = a.columns, pitch = columns + 4, m = a.s.m();
    float *gram = lds;
    char *rest = reinterpret_cast<char *>(gram + S::SQUARE);
    float *x = reinterpret_cast<float *>(rest + S::REST), *scratch = x + S::M * pitch;
    const uint32_t top = S::load(
        x, pitch, a.s, matrix, 0, columns, a.by_fours, a.whole_fours, [&](int64_t at, int count, bool whole) { return fetch_four(a.u, a.s.dtype, at, count, whole, true); },
        [&](const Raw4 &v, int64_t at, int count, bool whole) { return direction_four(a.u, v, at, count, whole, true); });
    const int range = range_of_all(top, 0);
    const float scale = range_scale(range);
    if (range != 1) scale_columns<S>(x, pitch, columns, scale);
    for (int k = 0; k < a.steps;) {
        const int end = a.end[k];
        floatx4 acc[S::EACH];
#pragma unroll
        for (int q = 0; q < S::EACH; ++q) acc[q] = floatx4{0, 0, 0, 0};
        S::gram(x, pitch, columns, wave, lane, acc);
        S::for_tiles(acc, wave, lane, scratch, [&](int row, int col, bool mirror, const floatx4 &v) { S::put_square(gram, row, col, mirror, v); });
        float inverse = 1.0f;
        if (k == 0) inverse = normalise<S>(gram, m, (double)a.s.eps * scale, &shared, lane);
        else __syncthreads();
        float *p = S::polynomial(a, k, end, gram, rest, wave, lane);
        if (k == 0) scale_square<S>(p, inverse);
        S::apply(p, x, pitch, columns, wave, lane);
        __syncthreads();
        k = end;
    }
    S::store(x, pitch, a.s, matrix, 0, columns, a.by_fours, a.whole_fours, [&](int64_t at, int count, bool whole, const floatx4 &v) { store_result_four(a, at, count, whole, v); });
}

// Part of the Gram matrices of the raw direction: grid (parts, matrices)
template <class S>
__global__ __launch_bounds__(S::THREADS) void gram_kernel(SmallArgs a)
{
    extern __shared__ __align__(16) float lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t matrix = blockIdx.y;
    const int columns = a.columns, pitch = columns + 4, n = a.s.n();
    float *x = lds, *scratch = lds + S::M * pitch;
    floatx4 acc[S::EACH];
#pragma unroll
    for (int q = 0; q < S::EACH; ++q) acc[q] = floatx4{0, 0, 0, 0};
    int range = 0;
    for (int64_t first = (int64_t)blockIdx.x * columns; first < n; first += (int64_t)a.parts * columns) {
        const uint32_t top = S::load(
            x, pitch, a.s, matrix, (int)first, columns, a.by_fours, a.whole_fours, [&](int64_t at, int count, bool whole) { return fetch_four(a.u, a.s.dtype, at, count, whole, true); },
            [&](const Raw4 &v, int64_t at, int count, bool whole) { return direction_four(a.u, v, at, count, whole, true); });
        // (what there is of the sum goes over to a larger range)
        const int now = range_of_all(top, range);
        for (; range < now; ++range)
#pragma unroll
            for (int q = 0; q < S::EACH; ++q) acc[q] *= 0x1p-90f, acc[q] *= 0x1p-90f;
        if (range != 1) scale_columns<S>(x, pitch, columns, range_scale(range));
        S::gram(x, pitch, columns, wave, lane, acc);
        __syncthreads();
    }
    float *to = a.gram + (matrix * a.parts + blockIdx.x) * S::M * S::M;
    S::for_tiles(acc, wave, lane, scratch, [&](int row, int col, bool, const floatx4 &v) { *reinterpret_cast<floatx4 *>(to + row * S::M + col) = v; });
    if (threadIdx.x == 0) a.range[matrix * a.parts + blockIdx.x] = range;
}

// The range of a matrix's direction, from those of the parts (1 for an X between polynomials)
template <class S>
__device__ __forceinline__ int matrix_range(const SmallArgs &a, const int *ranges)
{
    if (a.from != 0) return 1;
    int range = 0;
    for (int k = threadIdx.x; k < a.parts; k += S::THREADS) range = max(range, ranges[k]);
    return __syncthreads_or(range == 2) ? 2 : __syncthreads_or(range == 1);
}

// an element of a part, in float64, in the units of the range `range`; `first`: of the direction
__device__ __forceinline__ double part_element(const float *from, const int *ranges, int range, bool first, int k, int64_t step, int e)
{
    return (double)from[k * step + e] * range_units(first ? range - ranges[k] : 0);
}

constexpr int kFewParts = 16;  // parts that the workgroup of the polynomial sums itself

// Sums of many parts: grid (M M / 64, matrices), 64 elements a workgroup, every WAVES-th part to a wave
template <class S>
__global__ __launch_bounds__(S::THREADS) void sum_kernel(SmallArgs a)
{
    __shared__ double sums[S::WAVES][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t matrix = blockIdx.y;
    const float *from = a.gram + matrix * a.parts * S::M * S::M;
    const int *ranges = a.range + matrix * a.parts;
    const int range = matrix_range<S>(a, ranges);
    const int e = blockIdx.x * 64 + lane;
    double sum = 0.0;
#pragma unroll 8
    for (int k = wave; k < a.parts; k += S::WAVES) sum += part_element(from, ranges, range, a.from == 0, k, S::M * S::M, e);
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < S::WAVES; ++w) sum += sums[w][lane];
    a.sum[matrix * S::M * S::M + e] = sum;
}

// The polynomial of a matrix from the parts of its Gram matrix: a workgroup per matrix.  The first is scaled by the
// inverse of the norm.
template <class S>
__global__ __launch_bounds__(S::THREADS) void polynomial_kernel(SmallArgs a)
{
    extern __shared__ __align__(16) float lds[];
    __shared__ double shared;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t matrix = blockIdx.x;
    float *gram = lds;
    const float *from = a.gram + matrix * a.parts * S::M * S::M;
    const int *ranges = a.range + matrix * a.parts;
    const int range = matrix_range<S>(a, ranges);
#pragma unroll 4
    for (int e = threadIdx.x; e < S::M * S::M; e += S::THREADS) {
        const int i = e / S::M, j = e % S::M;
        if (i / 16 > j / 16) continue;   // (below the diagonal: from above it)
        double sum = 0.0;
        if (a.parts > kFewParts) {
            sum = a.sum[matrix * S::M * S::M + e];
        } else {
#pragma unroll 4
            for (int k = 0; k < a.parts; ++k) sum += part_element(from, ranges, range, a.from == 0, k, S::M * S::M, e);
        }
        gram[i * S::PITCH + j] = (float)sum;
        if (i / 16 != j / 16) gram[j * S::PITCH + i] = (float)sum;
    }
    float inverse = 1.0f;
    if (a.from == 0) inverse = normalise<S>(gram, a.s.m(), (double)a.s.eps * range_scale(range), &shared, lane);
    else __syncthreads();
    const float *p = S::polynomial(a, a.from, a.to, gram, reinterpret_cast<char *>(gram + S::SQUARE), wave, lane);
    if (threadIdx.x == 0) a.unit[matrix] = range_scale(range);
    float *to = a.poly + matrix * S::M * S::M;
    for (int e = threadIdx.x; e < S::M * S::M; e += S::THREADS) to[e] = p[e / S::M * S::PITCH + e % S::M] * inverse;
}

// X <- P X, from the direction (the first time) or from X: with LAST to the result, else to X and to the parts of its
// Gram matrix.  grid (parts, matrices)
template <class S, bool LAST>
__global__ __launch_bounds__(S::THREADS) void apply_kernel(SmallArgs a)
{
    extern __shared__ __align__(16) float lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t matrix = blockIdx.y;
    const int columns = a.columns, pitch = columns + 4, m = a.s.m(), n = a.s.n();
    float *p = lds, *x = p + S::SQUARE, *scratch = x + S::M * pitch;
    for (int e = threadIdx.x; e < S::M * S::M; e += S::THREADS) p[e / S::M * S::PITCH + e % S::M] = a.poly[matrix * S::M * S::M + e];
    floatx4 acc[S::EACH];
#pragma unroll
    for (int q = 0; q < S::EACH; ++q) acc[q] = floatx4{0, 0, 0, 0};
    MatrixShape seen = a.s;   // X itself lies with the shorter side first
    if (a.from != 0) seen.rows = m, seen.cols = n;
    MatrixShape kept = a.s;
    kept.rows = m, kept.cols = n;
    const bool x_fours = n % 4 == 0;
    const float unit = a.unit[matrix];
    for (int64_t first = (int64_t)blockIdx.x * columns; first < n; first += (int64_t)a.parts * columns) {
        S::load(
            x, pitch, seen, matrix, (int)first, columns, a.by_fours, a.from != 0 ? x_fours : a.whole_fours,
            [&](int64_t at, int count, bool whole) {
                return a.from != 0 ? Raw4{load_four(a.x, LMKAN_F32, at, count, whole), {}} : fetch_four(a.u, a.s.dtype, at, count, whole, false);
            },
            [&](const Raw4 &v, int64_t at, int count, bool whole) { return a.from != 0 ? v.g : unit * direction_four(a.u, v, at, count, whole, false); });
        __syncthreads();
        S::apply(p, x, pitch, columns, wave, lane);
        __syncthreads();
        if (LAST) {
            S::store(x, pitch, a.s, matrix, (int)first, columns, a.by_fours, a.whole_fours,
                     [&](int64_t at, int count, bool whole, const floatx4 &v) { store_result_four(a, at, count, whole, v); });
        } else {
            S::store(x, pitch, kept, matrix, (int)first, columns, a.by_fours, x_fours,
                     [&](int64_t at, int count, bool whole, const floatx4 &v) { store_four(a.x, LMKAN_F32, at, count, whole, v); });
            S::gram(x, pitch, columns, wave, lane, acc);
        }
        __syncthreads();
    }
    if (!LAST) {
        float *to = a.gram + (matrix * a.parts + blockIdx.x) * S::M * S::M;
        S::for_tiles(acc, wave, lane, scratch, [&](int row, int col, bool, const floatx4 &v) { *reinterpret_cast<floatx4 *>(to + row * S::M + col) = v; });
    }
}

int round16(int n) { return (n + 15) / 16 * 16; }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

size_t square_bytes(int M) { return (size_t)M * (M + 4) * sizeof(float); }
// one square of float32 and what polynomial() needs
size_t polynomial_lds(int M)
{
    return square_bytes(M) + (M == 16 ? Small<16, 1>::REST : M == 32 ? Small<32, 1>::REST : M == 48 ? Small<48, 8>::REST : Small<64, 12>::REST);
}
size_t whole_lds(const MatrixShape &s)
{
    const size_t M = round16(s.m());
    // (the waves of a matrix of one tile share its sums)
    return polynomial_lds((int)M) + M * (round16(s.n()) + 4) * sizeof(float) + (M == 16 ? 4 * 1024 * sizeof(float) : 0);
}
bool whole(const MatrixShape &s) { return s.n() <= 4096 && whole_lds(s) <= kSmallLds; }

// columns in LDS at a time of a long matrix: 16 KiB of X
int columns_of(int M) { return 4096 / M / 16 * 16; }

int parts_of(const MatrixShape &s, int64_t count)
{
    const int columns = columns_of(round16(s.m()));
    const int64_t blocks = ((int64_t)s.n() + columns - 1) / columns;
    int64_t parts = (1024 + count - 1) / count;   // four workgroups a compute unit
    parts = parts < blocks ? parts : blocks;
    return (int)(parts < kMostParts ? parts : kMostParts);
}

struct Layout {
    size_t gram, range, sum, poly, unit, x, total;
};
Layout layout_of(const MatrixShape &s, int64_t count)
{
    Layout l = {};
    if (whole(s)) return l;
    const size_t M = round16(s.m()), parts = parts_of(s, count);
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += align256(bytes); return here; };
    l.gram = take(count * parts * M * M * sizeof(float));
    l.range = take(count * parts * sizeof(int));
    l.sum = take(parts > kFewParts ? count * M * M * sizeof(double) : 0);
    l.poly = take(count * M * M * sizeof(float));
    l.unit = take(count * sizeof(float));
    l.x = take(count * s.elems() * sizeof(float));
    l.total = at;
    return l;
}

// matrices of a launch; those that share the workspace at a time: 512 M elements, and what a grid takes
int64_t matrices_at_once(const MatrixShape &s)
{
    if (whole(s)) return s.batch < kMostGroups ? s.batch : kMostGroups;
    int64_t most = ((int64_t)512 << 20) / s.elems();
    most = most < 1 ? 1 : most > 32768 ? 32768 : most;
    const int64_t parts = (s.batch + most - 1) / most;
    return (s.batch + parts - 1) / parts;
}

// W: the shape of workgroups that have a matrix to themselves, S: of those that share one
template <class W, class S>
void launch(const MatrixShape &s, const UpdateArgs &update, SmallArgs a, const ScheduleBounds &bounds, char *ws, hipStream_t stream)
{
    double factor = 1.0;
    for (int k = 0, end = 0; k < a.steps; ++k) {
        const double r = bounds.singular[k];
        if (k == end) factor = 1.0, end = a.end[k] = steps_until(s, bounds, a.steps, k);
        a.gram_scale[k] = pair_scale(r * r), a.step[k] = chain_step(bounds, a.schedule, k, &factor);
    }
    const int64_t most_matrices = matrices_at_once(s);
    const size_t item = s.dtype == LMKAN_F32 ? 4 : 2;
    const auto from_matrix = [&](int64_t first) {
        const int64_t skip = first * s.elems();
        a.u.grad = static_cast<const char *>(update.grad) + skip * item;
        a.u.momentum = update.momentum ? update.momentum + skip : nullptr;
        a.u.weight = update.weight ? update.weight + skip : nullptr;
        a.u.out = update.out ? static_cast<char *>(update.out) + skip * item : nullptr;
        return s.batch - first < most_matrices ? s.batch - first : most_matrices;
    };
    if (whole(s)) {
        a.columns = round16(s.n());
        a.by_fours = Divide::by(a.columns / 4);
        const size_t lds = whole_lds(s);
        if (lds > 65536) allow_large_lds(reinterpret_cast<const void *>(whole_kernel<W>), kSmallLds);
        for (int64_t first = 0; first < s.batch; first += most_matrices)
            whole_kernel<W><<<(unsigned)from_matrix(first), W::THREADS, lds, stream>>>(a);
        return;
    }
    typedef Small<S::M, 16> Sum;
    a.columns = columns_of(S::M);
    a.by_fours = Divide::by(a.columns / 4);
    const size_t block = (size_t)S::M * (a.columns + 4) * sizeof(float), scratch = 4 * S::THREADS * sizeof(float), square = square_bytes(S::M);
    for (int64_t first = 0; first < s.batch; first += most_matrices) {
        const int64_t count = from_matrix(first);
        const Layout l = layout_of(s, count);
        a.parts = parts_of(s, count);
        a.gram = reinterpret_cast<float *>(ws + l.gram), a.range = reinterpret_cast<int *>(ws + l.range);
        a.sum = reinterpret_cast<double *>(ws + l.sum);
        a.poly = reinterpret_cast<float *>(ws + l.poly), a.unit = reinterpret_cast<float *>(ws + l.unit), a.x = reinterpret_cast<float *>(ws + l.x);
        const dim3 grid(a.parts, (unsigned)count);
        a.from = 0;
        gram_kernel<S><<<grid, S::THREADS, block + scratch, stream>>>(a);
        for (; a.from < a.steps; a.from = a.to) {
            a.to = a.end[a.from];
            if (polynomial_lds(S::M) > 65536) allow_large_lds(reinterpret_cast<const void *>(polynomial_kernel<W>), (int)polynomial_lds(S::M));
            if (a.parts > kFewParts) sum_kernel<Sum><<<dim3(S::M * S::M / 64, (unsigned)count), Sum::THREADS, 0, stream>>>(a);
            polynomial_kernel<W><<<(unsigned)count, W::THREADS, polynomial_lds(S::M), stream>>>(a);
            if (a.to == a.steps) apply_kernel<S, true><<<grid, S::THREADS, square + block, stream>>>(a);
            else apply_kernel<S, false><<<grid, S::THREADS, square + block + scratch, stream>>>(a);
        }
    }
}

}  // namespace

bool ortho_small_applicable(const MatrixShape &s, int steps) { return s.m() <= 64 && steps > 0; }

size_t ortho_small_workspace_bytes(const MatrixShape &s)
{
    const int64_t most = matrices_at_once(s), left = s.batch % most;
    const size_t full = layout_of(s, most).total, rest = left ? layout_of(s, left).total : 0;
    return full > rest ? full : rest;
}

void launch_ortho_small(const MatrixShape &s, int steps, const float *schedule, const UpdateArgs &u, void *workspace, hipStream_t stream)
{
    SmallArgs a = {};
    a.s = s;
    a.u = u;
    a.steps = steps;
    for (int k = 0; k < 3 * steps; ++k) a.schedule[k] = schedule[k];
    ScheduleBounds bounds;
    (void)schedule_bounds(steps, schedule, &bounds);
    char *ws = static_cast<char *>(workspace);
    const auto aligned = [](const void *p, size_t item) { return reinterpret_cast<uintptr_t>(p) % (4 * item) == 0; };
    const size_t item = s.dtype == LMKAN_F32 ? 4 : 2;
    a.whole_fours = s.cols % 4 == 0 && aligned(u.grad, item) && aligned(u.out, item) && aligned(u.momentum, 4) && aligned(u.weight, 4);
    // Waves of a workgroup that has a matrix to itself: more for longer rows, fewer where one is small enough for several
    // workgroups a compute unit.  Measured (us, 1 / 4 / 8 / 16 waves): 1681 of 8 x 16 8.9 / 14 / 22 / 50; 1000 of
    // 16 x 100 18 / 13 / 19 / 33; 400 of 10 x 300 27 / 20 / 21 / 22; 25 of 12 x 900 68 / 24 / 17 / 15; 1600 of 30 x 60
    // - / 40 / 48 / 79; 441 of 32 x 218 - / 35 / 31 / 41; one of 32 x 500 - / 33 / 26 / 23; 441 of 48 x 100 - / - / 35 / 45;
    // 441 of 48 x 150 - / - / 53 / 66; 441 of 48 x 200 - / - / 76 / 72; 25 of 48 x 500 - / - / 69 / 64; and 1600 of 64 x 64
    // takes 172, 169 of 144 x 64 35 (twelve waves).
    const int m = s.m(), n = s.n();
    if (m <= 16 && n <= 32) launch<Small<16, 1>, Small<16, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 16 && n <= 160) launch<Small<16, 4>, Small<16, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 16 && n <= 512) launch<Small<16, 8>, Small<16, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 16) launch<Small<16, 16>, Small<16, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 32 && n <= 64) launch<Small<32, 4>, Small<32, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 32 && n <= 300) launch<Small<32, 8>, Small<32, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 32) launch<Small<32, 16>, Small<32, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 48 && n <= 200) launch<Small<48, 8>, Small<48, 4>>(s, u, a, bounds, ws, stream);
    else if (m <= 48) launch<Small<48, 16>, Small<48, 4>>(s, u, a, bounds, ws, stream);
    else launch<Small<64, 12>, Small<64, 4>>(s, u, a, bounds, ws, stream);
}

}  // namespace lmkan
