// Orthogonalisation of matrices by Newton-Schulz products, and the optimiser's step round it.
//
//   X_0 = U / (|U|_F + eps),  A_k = X_k X_k^T,  X_{k+1} = B_k X_k,  B_k = a_k I + b_k A_k + c_k A_k^2
//
// with X of m x n, m <= n (the transpose of what is stored where that has more rows than columns).  Everything
// between X_0 and the result is a polynomial of A_0, and polynomials of one symmetric matrix commute, so that
// up to three steps are taken on m x m matrices alone,
//   A_{k+1} = B_k A_k B_k,   P_{k+1} = B_k P_k,
// and then X_{k+3} = P X_k.  All products but that one are symmetric: half their tiles are computed and mirrored.
// For five steps that is 6 m^2 n + 14 m^3 multiply-adds instead of the 15 m^2 n + 5 m^3 of the steps as written,
// and X is read and written twice instead of five times.  Three steps, not all: an error of A is relative to its
// largest eigenvalue and grows by up to a^2 (11.9) a step where the eigenvalue is small; with a new Gram matrix
// after three steps the result is as near to float64 as the steps as written are in float32 (strong directions a
// hundred times the rest: 1.1e-5 and 1.9e-5 of the result; five steps on one Gram matrix: 6e-5).
//
// Factors are pairs of float16 (lmkan_tile.h): three instructions at the rate of float16 keep 22 bits, which
// float32 instructions would do at a sixteenth of that rate.  The power of two that a matrix is scaled by follows
// from the bound of its singular values (schedule_bounds).
#include "lmkan_dense.h"

#include <math.h>

#include "lmkan_kernels.h"
#include "lmkan_tile.h"

namespace lmkan {

namespace {

constexpr int kStepsAtOnce = 3;   // steps on one Gram matrix
constexpr int kNormParts = 64;    // workgroups that sum the norm of one matrix, at most

// A batch of matrices of pairs (lmkan_tile.h); element values are held times `scale`
struct PairMatrix {
    char *base;
    int64_t stride;  // bytes from one matrix to the next
    int rows, depth;
    float scale;
};

// the direction's element i
__device__ __forceinline__ float direction(const UpdateArgs &u, int dtype, int64_t i)
{
    if (!u.momentum) return load_as_float(u.grad, i, dtype);
    const float m = u.momentum[i];
    return u.nesterov ? u.beta * m + (1.0f - u.beta) * load_as_float(u.grad, i, dtype) : m;
}

// Sum of `parts` numbers in a fixed order, for all 256 threads
__device__ __forceinline__ double sum_of_parts(const double *part, int parts, double *shared)
{
    shared[threadIdx.x] = (int)threadIdx.x < parts ? part[threadIdx.x] : 0.0;
    for (int half = kNormParts / 2; half > 0; half >>= 1) {
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
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
        if (u.momentum) u.momentum[base + i] = u.beta * u.momentum[base + i] + (1.0f - u.beta) * load_as_float(u.grad, base + i, s.dtype);
        const double v = direction(u, s.dtype, base + i);
        sum += v * v;
    }
    sums[threadIdx.x] = sum;
    for (int half = 128; half > 0; half >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < half) sums[threadIdx.x] += sums[threadIdx.x + half];
    }
    if (threadIdx.x == 0) part[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = sums[0];
}

__device__ __forceinline__ float inverse_norm(const MatrixShape &s, const double *part, int parts, int64_t matrix, double *shared)
{
    return (float)(1.0 / (sqrt(sum_of_parts(part + matrix * parts, parts, shared)) + (double)s.eps));
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
};
__global__ __launch_bounds__(256) void split_kernel(SplitArgs a)
{
    __shared__ float tile[64][65];
    __shared__ double sums[256];
    const int64_t matrix = blockIdx.z, per = a.s.elems();
    const int across = (a.s.cols + 63) / 64;
    const int r0 = (int)(blockIdx.x / across) * 64, c0 = (int)(blockIdx.x % across) * 64;
    const float f = inverse_norm(a.s, a.part, a.parts, matrix, sums);
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        const int r = e >> 6, c = e & 63;
        const bool in = r0 + r < a.s.rows && c0 + c < a.s.cols;
        // (the scale is a power of two; times the norm's inverse first: the product of both may exceed float32)
        tile[r][c] = in ? direction(a.u, a.s.dtype, (a.first + matrix) * per + (int64_t)(r0 + r) * a.s.cols + c0 + c) * f * a.by_rows.scale : 0.0f;
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

// One value to both halves of a pair, four adjacent columns of a row
__device__ __forceinline__ void store_four(const PairMatrix &d, int64_t matrix, int row, int col, const float (&v)[4])
{
    char *to = d.base + matrix * d.stride;
    const int panel = col / kPanel, in = col % kPanel;
    half4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        _Float16 h, l;
        split(v[e] * d.scale, &h, &l);
        hi[e] = h, lo[e] = l;
    }
    *reinterpret_cast<half4 *>(to + pair_at(d.rows, row, panel, in / 8) + in % 8 * 2) = hi;
    *reinterpret_cast<half4 *>(to + pair_at(d.rows, row, panel, 4 + in / 8) + in % 8 * 2) = lo;
}
__device__ __forceinline__ void store_one(const PairMatrix &d, int64_t matrix, int row, int col, float v)
{
    char *to = d.base + matrix * d.stride;
    const int panel = col / kPanel, in = col % kPanel;
    _Float16 h, l;
    split(v * d.scale, &h, &l);
    *reinterpret_cast<_Float16 *>(to + pair_at(d.rows, row, panel, in / 8) + in % 8 * 2) = h;
    *reinterpret_cast<_Float16 *>(to + pair_at(d.rows, row, panel, 4 + in / 8) + in % 8 * 2) = l;
}

// What becomes of a product
enum Finish {
    kKeep,      // pairs, both ways round
    kPoly,      // a I + b A + c (product), pairs
    kPartial,   // float32 sums of a part of the summed axis
    kResult,    // the result of the call
};

struct Product {
    PairMatrix rows, cols;     // the factors: by the rows and by the columns of the output
    PairMatrix out, mirror;    // mirror: the output's transpose (the same matrix when symmetric); no base: none
    PairMatrix gram;           // kPoly: A
    float a, b, c;
    bool symmetric;
};
struct ProductArgs {
    Product p[2];
    int problems;
    int64_t matrices;
    int tiles_down, tiles_across;
    int64_t tiles;             // of one matrix and problem
    // kPartial
    float *partial;
    int parts;
    // kResult
    MatrixShape s;
    UpdateArgs u;
    int64_t first;
};

// Tile t of the upper triangle of n x n tiles, column by column: (0,0) (0,1) (1,1) (0,2) ...
__device__ __forceinline__ void upper_tile(int t, int *i, int *j)
{
    int c = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while ((c + 1) * (c + 2) / 2 <= t) ++c;
    while (c * (c + 1) / 2 > t) --c;
    *j = c;
    *i = t - c * (c + 1) / 2;
}

template <class T, int FINISH>
__global__ __launch_bounds__(T::THREADS) void product_kernel(ProductArgs a)
{
    extern __shared__ __align__(16) char lds[];
    const int64_t each = a.tiles * (FINISH == kPartial ? a.parts : 1), total = each * a.matrices * a.problems;
    const int64_t place = place_of(blockIdx.x, total);
    if (place >= total) return;
    const int64_t which = place / each;
    const int64_t matrix = which / a.problems;
    const Product &p = a.p[which - matrix * a.problems];
    const int64_t rest = place - which * each;
    const int part = FINISH == kPartial ? (int)(rest / a.tiles) : 0;
    const int tile = (int)(rest - part * a.tiles);
    int ti, tj;
    if (p.symmetric) upper_tile(tile, &ti, &tj);
    else ti = tile / a.tiles_across, tj = tile - ti * a.tiles_across;
    const int i0 = ti * T::ROWS, j0 = tj * T::COLS;
    const auto operand = [&](const PairMatrix &m, int first_row) {
        return Operand{m.base + matrix * m.stride + (int64_t)first_row * kLine, (int64_t)m.rows * kLine, kLine, m.rows - 1 - first_row, true, 0};
    };
    const int stages = panels(p.rows.depth);
    const int begin = FINISH == kPartial ? (int)((int64_t)stages * part / a.parts) : 0;
    const int end = FINISH == kPartial ? (int)((int64_t)stages * (part + 1) / a.parts) : stages;
    floatx16 acc[T::RT][T::CT];
    multiply<T, PairProduct>(operand(p.rows, i0), operand(p.cols, j0), begin, end, lds, acc);
    const float unit = 1.0f / (p.rows.scale * p.cols.scale);
    const int n_rows = p.rows.rows, n_cols = p.cols.rows;
    for_outputs<T>(acc, [&](int r, int c, float v0, float v1, float v2, float v3) {
        const int i = i0 + r, j = j0 + c;
        float v[4] = {v0 * unit, v1 * unit, v2 * unit, v3 * unit};
        if (FINISH == kPartial) {
            float *to = a.partial + ((part * a.matrices + matrix) * n_rows + i) * (int64_t)n_cols + j;
            if (i < n_rows)
                for (int e = 0; e < 4; ++e)
                    if (j + e < n_cols) to[e] = v[e];
            return;
        }
        if (FINISH == kResult) {
            if (i >= n_rows || j >= n_cols) return;
            const int64_t at = (a.first + matrix) * a.s.elems() + (int64_t)i * a.s.cols + j;
            for (int e = 0; e < 4; ++e)
                if (j + e < n_cols) {
                    if (a.u.weight) a.u.weight[at + e] = a.u.keep * a.u.weight[at + e] + a.u.add * v[e];
                    else store_from_float(a.u.out, at + e, a.s.dtype, v[e]);
                }
            return;
        }
        if (FINISH == kPoly && i < n_rows && j < n_cols) {
            const char *from = p.gram.base + matrix * p.gram.stride;
            const half4 hi = *reinterpret_cast<const half4 *>(from + pair_at(p.gram.rows, i, j / kPanel, j % kPanel / 8) + j % 8 * 2);
            const half4 lo = *reinterpret_cast<const half4 *>(from + pair_at(p.gram.rows, i, j / kPanel, 4 + j % kPanel / 8) + j % 8 * 2);
            const float g = 1.0f / p.gram.scale;
            for (int e = 0; e < 4; ++e)
                v[e] = p.c * v[e] + p.b * (((float)hi[e] + (float)lo[e]) * g) + (i == j + e ? p.a : 0.0f);
        }
        // what lies beyond the matrix in a panel is zero
        for (int e = 0; e < 4; ++e)
            if (i >= n_rows || j + e >= n_cols) v[e] = 0.0f;
        if (i < n_rows && j < panels(n_cols) * kPanel) store_four(p.out, matrix, i, j, v);
        if (p.mirror.base && !(p.symmetric && ti == tj) && i < panels(n_rows) * kPanel)
            for (int e = 0; e < 4; ++e)
                if (j + e < n_cols) store_one(p.mirror, matrix, j + e, i, v[e]);
    });
}

// The Gram matrices from their float32 parts (tiles below the diagonal: from above it); a chunk a thread
__global__ __launch_bounds__(256) void sum_parts_kernel(PairMatrix d, const float *partial, int parts, int64_t matrices, int tile)
{
    const int m = d.rows, chunks = panels(m) * 4;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= matrices * m * chunks) return;
    const int chunk = (int)(e % chunks), i = (int)(e / chunks % m);
    const int64_t matrix = e / chunks / m;
    half8 hi, lo;
    for (int k = 0; k < 8; ++k) {
        const int j = chunk * 8 + k;
        float v = 0.0f;
        if (j < m) {
            const bool below = j / tile < i / tile;
            const int64_t at = below ? (int64_t)j * m + i : (int64_t)i * m + j;
            for (int p = 0; p < parts; ++p) v += partial[(p * matrices + matrix) * m * m + at];
        }
        _Float16 h, l;
        split(v * d.scale, &h, &l);
        hi[k] = h, lo[k] = l;
    }
    char *to = d.base + matrix * d.stride;
    *reinterpret_cast<half8 *>(to + pair_at(m, i, chunk / 4, chunk % 4)) = hi;
    *reinterpret_cast<half8 *>(to + pair_at(m, i, chunk / 4, 4 + chunk % 4)) = lo;
}

// No steps: X_0 itself is the result
__global__ __launch_bounds__(256) void unscaled_kernel(MatrixShape s, UpdateArgs u, int64_t first, const double *part, int parts)
{
    __shared__ double sums[256];
    const int64_t per = s.elems(), base = (first + blockIdx.y) * per;
    const float f = inverse_norm(s, part, parts, blockIdx.y, sums);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (int64_t)gridDim.x * 256) {
        const float v = direction(u, s.dtype, base + i) * f;
        if (u.weight) u.weight[base + i] = u.keep * u.weight[base + i] + u.add * v;
        else store_from_float(u.out, base + i, s.dtype, v);
    }
}

typedef TileShape<64, 64, 2, 2> Tile64;
typedef TileShape<128, 128, 2, 2> Tile128;

int64_t upper_tiles(int rows, int tile)
{
    const int64_t n = (rows + tile - 1) / tile;
    return n * (n + 1) / 2;
}

// the larger tile reads half as much per product; the smaller one where the larger leaves compute units without work
bool small_tiles(int64_t large_tiles) { return large_tiles < 256; }

template <class T, int FINISH>
void launch_product_with(ProductArgs &a, hipStream_t stream)
{
    const Product &p = a.p[0];
    a.tiles_down = (p.rows.rows + T::ROWS - 1) / T::ROWS;
    a.tiles_across = (p.cols.rows + T::COLS - 1) / T::COLS;
    a.tiles = p.symmetric ? upper_tiles(p.rows.rows, T::ROWS) : (int64_t)a.tiles_down * a.tiles_across;
    const int64_t total = a.tiles * (FINISH == kPartial ? a.parts : 1) * a.matrices * a.problems;
    if (T::LDS > 65536) allow_large_lds(reinterpret_cast<const void *>(product_kernel<T, FINISH>), T::LDS);
    product_kernel<T, FINISH><<<(unsigned)((total + 7) / 8 * 8), T::THREADS, T::LDS, stream>>>(a);
}

int64_t tiles_of(const Product &p, int tile)
{
    return p.symmetric ? upper_tiles(p.rows.rows, tile) : (int64_t)((p.rows.rows + tile - 1) / tile) * ((p.cols.rows + tile - 1) / tile);
}

template <int FINISH>
void launch_product(ProductArgs &a, hipStream_t stream)
{
    if (small_tiles(tiles_of(a.p[0], 128) * a.matrices * a.problems)) launch_product_with<Tile64, FINISH>(a, stream);
    else launch_product_with<Tile128, FINISH>(a, stream);
}

// parts of the summed axis of a Gram matrix: two tiles a compute unit where there are fewer, four lines at least each
int gram_parts(int m, int n, int64_t matrices)
{
    const int64_t tiles = upper_tiles(m, 64) * matrices;
    const int64_t want = tiles >= 256 ? 1 : (512 + tiles - 1) / tiles, most = panels(n) / 4;
    return (int)(want < most ? want : most < 1 ? 1 : most);
}

// matrices that share the workspace at a time: 128 M elements keep every compute unit busy
int64_t matrices_at_once(const MatrixShape &s)
{
    const int64_t some = ((int64_t)128 << 20) / s.elems();
    return some < 1 ? 1 : some > s.batch ? s.batch : some > 4096 ? 4096 : some;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// the workspace of `count` matrices
struct Layout {
    size_t norm, u, v[2], a, w, b[2], p[2], partial, total;
};
Layout layout_of(const MatrixShape &s, int64_t count)
{
    const size_t u = align256(count * pair_bytes(s.m(), s.n())), v = align256(count * pair_bytes(s.n(), s.m()));
    const size_t g = align256(count * pair_bytes(s.m(), s.m()));
    const int parts = gram_parts(s.m(), s.n(), count);
    Layout l;
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += bytes; return here; };
    l.norm = take(align256(count * kNormParts * sizeof(double)));
    l.u = take(u), l.v[0] = take(v), l.v[1] = take(v);
    l.a = take(g), l.w = take(g), l.b[0] = take(g), l.b[1] = take(g), l.p[0] = take(g), l.p[1] = take(g);
    l.partial = take(parts > 1 ? align256((size_t)parts * count * s.m() * s.m() * sizeof(float)) : 0);
    l.total = at;
    return l;
}

// the power of two that brings values up to `bound` to the upper end of float16's range (65504), with room for rounding
float scale_for(double bound) { return (float)exp2(floor(log2(32000.0 / bound))); }

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
    const int64_t most = matrices_at_once(s), left = s.batch % most;
    const size_t whole = layout_of(s, most).total, rest = left ? layout_of(s, left).total : 0;
    return whole > rest ? whole : rest;
}

void launch_ortho(const MatrixShape &s, int steps, const float *schedule, const UpdateArgs &u, void *workspace, hipStream_t stream)
{
    ScheduleBounds bounds;
    (void)schedule_bounds(steps, schedule, &bounds);
    const int m = s.m(), n = s.n();
    const int64_t most = matrices_at_once(s);
    for (int64_t first = 0; first < s.batch; first += most) {
        const int64_t count = s.batch - first < most ? s.batch - first : most;
        const Layout l = layout_of(s, count);
        char *ws = static_cast<char *>(workspace);
        const auto pairs = [&](size_t at, int rows, int depth, double bound) {
            return PairMatrix{ws + at, pair_bytes(rows, depth), rows, depth, scale_for(bound)};
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
        PairMatrix x = pairs(l.u, m, n, 1.0), xt = pairs(l.v[0], n, m, 1.0);
        int turned = 0;
        const unsigned tiles = (unsigned)(((s.rows + 63) / 64) * (int64_t)((s.cols + 63) / 64));
        split_kernel<<<dim3(tiles, 1, (unsigned)count), 256, 0, stream>>>(SplitArgs{s, u, first, part, parts, s.flip() ? xt : x, s.flip() ? x : xt});
        ProductArgs args = {};
        args.matrices = count;
        args.s = s;
        args.u = u;
        args.first = first;
        const auto one = [&](const Product &p) { args.p[0] = p, args.problems = 1; };
        for (int k = 0; k < steps;) {
            const int end = k + kStepsAtOnce < steps ? k + kStepsAtOnce : steps;
            const double r = bounds.singular[k];
            PairMatrix gram = pairs(l.a, m, m, r * r), so_far = none;
            one(Product{x, x, gram, gram, none, 0, 0, 0, true});
            args.parts = gram_parts(m, n, count);
            if (args.parts > 1) {
                args.partial = reinterpret_cast<float *>(ws + l.partial);
                launch_product_with<Tile64, kPartial>(args, stream);
                const int64_t chunks = count * m * panels(m) * 4;
                sum_parts_kernel<<<(unsigned)((chunks + 255) / 256), 256, 0, stream>>>(gram, args.partial, args.parts, count, Tile64::ROWS);
            } else {
                launch_product<kKeep>(args, stream);
            }
            double factor = 1.0;
            for (const int begin = k; k < end; ++k) {
                const float *abc = schedule + 3 * k;
                const double now = bounds.singular[k], next = bounds.singular[k + 1];
                const PairMatrix step = pairs(l.b[k & 1], m, m, bounds.factor[k]);
                one(Product{gram, gram, step, step, gram, abc[0], abc[1], abc[2], true});
                launch_product<kPoly>(args, stream);
                factor *= bounds.factor[k];
                const PairMatrix w = pairs(l.w, m, m, bounds.factor[k] * now * now);
                args.problems = 0;
                if (k + 1 < end) args.p[args.problems++] = Product{step, gram, w, w, none, 0, 0, 0, true};
                if (k > begin) {
                    const PairMatrix longer = pairs(l.p[k & 1], m, m, factor);
                    args.p[args.problems++] = Product{step, so_far, longer, longer, none, 0, 0, 0, true};
                    so_far = longer;
                } else {
                    so_far = step;
                }
                if (args.problems) launch_product<kKeep>(args, stream);
                if (k + 1 < end) {
                    gram = pairs(l.a, m, m, next * next);
                    one(Product{w, step, gram, gram, none, 0, 0, 0, true});
                    launch_product<kKeep>(args, stream);
                }
            }
            if (k < steps) {
                const PairMatrix y = pairs(l.u, m, n, bounds.singular[k]);
                const PairMatrix yt = pairs(l.v[turned ^ 1], n, m, bounds.singular[k]);
                one(Product{so_far, xt, y, yt, none, 0, 0, 0, false});
                launch_product<kKeep>(args, stream);
                x = y, xt = yt, turned ^= 1;
            } else {
                one(s.flip() ? Product{xt, so_far, none, none, none, 0, 0, 0, false} : Product{so_far, xt, none, none, none, 0, 0, 0, false});
                launch_product<kResult>(args, stream);
            }
        }
    }
}

}  // namespace lmkan
