// Low-rank adapters of many requests beside a shared linear term: y[n] += scale[r] B_r (A_r f(x[n])), r = index[n].
//
// A few rows (one launch): a workgroup takes 512 outputs of a row, works out the row's A f(x) for itself and then its
// outputs; what bounds it is the latency of reading A and B once each.  Many rows (three launches, 32768 rows at a time):
//   order  one workgroup sorts the rows by adapter, by counting, into tiles of up to 32 rows of one adapter
//   down   low = A f(x): a tile and a piece of the inputs a workgroup, whose waves take every fourth 16 inputs
//   up     y += scale B low: a tile and a piece of the outputs a workgroup
// Both products run on float32 matrix instructions, 16 x 16 results of 4 terms: what they read (16 bytes a lane, straight
// into the instruction's operands) bounds them as long as the rank is below a hundred.  A row's result does not depend on
// the rows that share its tile, so that the order within an adapter, which atomics decide, changes nothing.
#include <type_traits>

#include "lmkan_rows.h"
#include "lmkan_tile.h"

namespace lmkan {

namespace {

constexpr int kTileRows = 32;
constexpr int kChunk = 32768;         // rows that are sorted at a time: counters and places of 16 bits hold them
constexpr int kLaneBatch = 4;         // pieces of 16 terms that are under way
constexpr int kFewOutputs = 512;      // outputs of a workgroup of the kernel for a few rows, a thread each

struct Tile {
    int adapter, first, rows;         // places `first` .. in the sorted rows
};

struct AdapterArgs {
    AdapterShape s;
    const void *x;
    const int32_t *index;
    const void *a, *b;
    const float *scale;
    void *y;
    Tile *tiles;        // [most_tiles], those that exist first
    int *tile_count;
    int *rows;          // sorted: row of the chunk
    float *low;         // [splits][place][16 RT]
    int splits, each;   // pieces of the inputs, and their length (a multiple of 64)
    int places;         // rows of the chunk
    int outputs;        // of a workgroup of the kernel `up`
};

// Four elements as they lie in memory, and as float32.  WIDE: float32; else 16 bits, float16 when `half`
template <bool WIDE>
struct Raw;
template <>
struct Raw<true> {
    float4 v;
};
template <>
struct Raw<false> {
    uint2 v;
};
// elements at .. at + 3 of which `left` exist; TOGETHER: all or none do, and they are aligned to their size
template <bool WIDE, bool TOGETHER>
__device__ __forceinline__ Raw<WIDE> fetch_four(const void *row, int at, int left)
{
    Raw<WIDE> r;
    if constexpr (WIDE) {
        const float *p = static_cast<const float *>(row);
        if constexpr (TOGETHER) {
            r.v = *reinterpret_cast<const float4 *>(p + (left > 0 ? at : 0));
        } else {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = p[i < left ? at + i : 0];
            r.v = make_float4(e[0], e[1], e[2], e[3]);
        }
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(row);
        if constexpr (TOGETHER) {
            r.v = *reinterpret_cast<const uint2 *>(p + (left > 0 ? at : 0));
        } else {
            uint32_t e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = p[i < left ? at + i : 0];
            r.v = make_uint2(e[0] | e[1] << 16, e[2] | e[3] << 16);
        }
    }
    return r;
}
// zero for those that do not exist
template <bool WIDE>
__device__ __forceinline__ floatx4 widen(const Raw<WIDE> &r, int left, bool half)
{
    floatx4 f;
    if constexpr (WIDE) {
        f = floatx4{r.v.x, r.v.y, r.v.z, r.v.w};
    } else {
        const uint32_t w[2] = {r.v.x, r.v.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint16_t b = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            const float as_half = (float)__builtin_bit_cast(_Float16, b), as_bf16 = __builtin_bit_cast(float, (uint32_t)b << 16);
            f[i] = half ? as_half : as_bf16;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = i < left ? f[i] : 0.0f;
    return f;
}
__device__ __forceinline__ floatx4 rectify_four(floatx4 f, bool relu)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = rectify(f[i], relu);
    return f;
}

// ---- a few rows ------------------------------------------------------------------------------------------------------

// X, W: x and the adapters are float32
template <bool X, bool W, bool IN4, bool RANK4>
__global__ __launch_bounds__(kFewOutputs) void adapters_few_kernel(AdapterArgs a)
{
    constexpr int kRanks = 16, kAhead = 4;   // values of A f(x) at a time; fours of B that are fetched before they are known
    __shared__ float parts[kFewOutputs / 64][kRanks];
    __shared__ float low[LMKAN_MAX_ADAPTER_RANK];
    const AdapterShape &s = a.s;
    const int64_t n = blockIdx.x;
    const int r = a.index[n];
    if (r < 0 || r >= s.count) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j = blockIdx.y * kFewOutputs + threadIdx.x, seen = j < s.n_out ? j : s.n_out - 1;
    const bool x_half = s.x_dtype == LMKAN_F16, w_half = s.dtype == LMKAN_F16;
    const void *const up = row_at(a.b, ((int64_t)r * s.n_out + seen) * s.rank, s.dtype);
    Raw<W> ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ahead[k] = fetch_four<W, RANK4>(up, 4 * k, s.rank - 4 * k);
    const float before = load_as_float(a.y, n * s.n_out + seen, s.y_dtype);
    const void *const x = row_at(a.x, n * s.n_in, s.x_dtype);
    for (int k0 = 0; k0 < s.rank; k0 += kRanks) {
        const void *const down = row_at(a.a, ((int64_t)r * s.rank + k0) * s.n_in, s.dtype);
        const int most = s.rank - k0 - 1;
        float sum[kRanks] = {};
        for (int c = threadIdx.x * 4; c < s.n_in; c += 4 * kFewOutputs) {
            const int left = s.n_in - c;
            const floatx4 v = rectify_four(widen(fetch_four<X, IN4>(x, c, left), left, x_half), s.relu);
            Raw<W> w[kRanks];
#pragma unroll
            for (int k = 0; k < kRanks; ++k) w[k] = fetch_four<W, IN4>(row_at(down, (int64_t)(k < most ? k : most) * s.n_in, W ? LMKAN_F32 : LMKAN_F16), c, left);
#pragma unroll
            for (int k = 0; k < kRanks; ++k) {
                const floatx4 f = widen(w[k], left, w_half);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[k] = fmaf(f[i], v[i], sum[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < kRanks; ++k) {
            sum[k] = over_lanes(sum[k], 64, [](float p, float q) { return p + q; });
            if (lane == k) parts[wave][k] = sum[k];
        }
        __syncthreads();
        if (threadIdx.x < kRanks) {
            float total = parts[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < kFewOutputs / 64; ++w) total += parts[w][threadIdx.x];
            low[k0 + threadIdx.x] = total;   // (beyond the rank: the last one's again, not used)
        }
        __syncthreads();
    }
    float sum = 0.0f;
    const auto add = [&](const Raw<W> &w, int k) {
        const floatx4 f = widen(w, s.rank - k, w_half);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = fmaf(f[i], k + i < s.rank ? low[k + i] : 0.0f, sum);
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (4 * k < s.rank) add(ahead[k], 4 * k);
#pragma unroll 4
    for (int k = 4 * kAhead; k < s.rank; k += 4) add(fetch_four<W, RANK4>(up, k, s.rank - k), k);
    if (j < s.n_out) store_from_float(a.y, n * s.n_out + j, s.y_dtype, fmaf(a.scale ? a.scale[r] : 1.0f, sum, before));
}

// ---- rows by adapter -------------------------------------------------------------------------------------------------

// Adds one to the counter of every lane's adapter (16 bits, two to a word) and returns what it was.  Lanes of a run of one
// adapter, which is what prompts look like, add once.
__device__ __forceinline__ int count_up(uint32_t *counters, int r, bool valid)
{
    const int lane = threadIdx.x & 63;
    int place = 0;
    uint64_t todo = __ballot(valid);
#pragma unroll 1
    for (int round = 0; round < 2 && todo; ++round) {
        const int leader = __builtin_ctzll(todo), of = __shfl(r, leader, 64);
        const uint64_t same = __ballot(valid && r == of) & todo;
        uint32_t old = 0;
        if (lane == leader) old = atomicAdd(&counters[of >> 1], (uint32_t)__popcll(same) << (16 * (of & 1)));
        old = (uint32_t)__shfl((int)old, leader, 64);
        if (same >> lane & 1) place = (int)(old >> (16 * (of & 1)) & 0xffff) + __popcll(same & ((1ull << lane) - 1));
        todo &= ~same;
    }
    if (todo >> lane & 1) place = (int)(atomicAdd(&counters[r >> 1], 1u << (16 * (r & 1))) >> (16 * (r & 1)) & 0xffff);
    return place;
}

__global__ __launch_bounds__(1024) void adapters_order_kernel(AdapterArgs a, int64_t first)
{
    __shared__ uint32_t counters[LMKAN_MAX_ADAPTERS / 2];
    __shared__ int waves[2][16];
    const int count = a.s.count, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < (count + 1) / 2; i += 1024) counters[i] = 0;
    __syncthreads();
    const int rounds = (a.places + 1023) / 1024;
    const auto index_of = [&](int round) {
        const int i = round * 1024 + threadIdx.x;
        return i < a.places ? a.index[first + i] : -1;
    };
#pragma unroll 8
    for (int k = 0; k < rounds; ++k) {
        const int r = index_of(k);
        count_up(counters, r, r >= 0 && r < count);
    }
    __syncthreads();
    // a thread sums adapters [from, to); sums over the threads before it
    const int span = ((count + 1023) / 1024 + 1) & ~1, from = threadIdx.x * span < count ? threadIdx.x * span : count,
              to = from + span < count ? from + span : count;
    const auto counted = [&](int r) { return (int)(counters[r >> 1] >> (16 * (r & 1)) & 0xffff); };
    int rows = 0, tiles = 0;
    for (int r = from; r < to; ++r) rows += counted(r), tiles += (counted(r) + kTileRows - 1) / kTileRows;
    int rows_before = rows, tiles_before = tiles;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int p = __shfl_up(rows_before, d, 64), q = __shfl_up(tiles_before, d, 64);
        if (lane >= d) rows_before += p, tiles_before += q;
    }
    if (lane == 63) waves[0][wave] = rows_before, waves[1][wave] = tiles_before;
    __syncthreads();
    rows_before -= rows, tiles_before -= tiles;
    for (int w = 0; w < wave; ++w) rows_before += waves[0][w], tiles_before += waves[1][w];
    if (threadIdx.x == 1023) *a.tile_count = tiles_before + tiles;
    // tiles, and the counters become the places where rows go (spans are even: a word belongs to one thread)
    for (int r = from; r < to; r += 2) {
        uint32_t word = 0;
        for (int h = 0; h < 2; ++h) {
            if (r + h >= to) break;
            const int n = counted(r + h);
            for (int t = 0; t < n; t += kTileRows) a.tiles[tiles_before++] = {r + h, rows_before + t, n - t < kTileRows ? n - t : kTileRows};
            word |= (uint32_t)rows_before << (16 * h);
            rows_before += n;
        }
        counters[r >> 1] = word;
    }
    __syncthreads();
#pragma unroll 8
    for (int k = 0; k < rounds; ++k) {
        const int r = index_of(k);
        const bool valid = r >= 0 && r < count;
        const int place = count_up(counters, r, valid);
        if (valid) a.rows[place] = k * 1024 + threadIdx.x;
    }
}

// ---- products --------------------------------------------------------------------------------------------------------

// low[place][k] = sum_e A[k][e] f(x[place][e]) over a piece of the inputs.  A lane's operands: row (rank or place) lane % 16,
// terms 4 (lane / 16) .. of every 16; which of the four goes to which instruction does not matter as both do it alike.
template <bool X, bool W, bool IN4, int RT>
__global__ __launch_bounds__(256) void adapters_down_kernel(AdapterArgs a)
{
    constexpr int kRowTiles = kTileRows / 16;
    if ((int)blockIdx.x >= *a.tile_count) return;
    constexpr int kJoined = RT < 4 ? RT : 4;   // rank tiles that are joined at a time
    __shared__ float sums[3][kRowTiles * kJoined * 4][64];
    const AdapterShape &s = a.s;
    const Tile tile = a.tiles[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, term = 4 * (lane >> 4);
    const bool x_half = s.x_dtype == LMKAN_F16, w_half = s.dtype == LMKAN_F16;
    const void *x[kRowTiles], *w[RT];
#pragma unroll
    for (int i = 0; i < kRowTiles; ++i) {
        const int p = 16 * i + row < tile.rows ? 16 * i + row : tile.rows - 1;   // (rows beyond the last repeat it)
        x[i] = row_at(a.x, (int64_t)a.rows[tile.first + p] * s.n_in, s.x_dtype);
    }
#pragma unroll
    for (int k = 0; k < RT; ++k) {
        const int q = 16 * k + row < s.rank ? 16 * k + row : s.rank - 1;
        w[k] = row_at(a.a, ((int64_t)tile.adapter * s.rank + q) * s.n_in, s.dtype);
    }
    floatx4 acc[kRowTiles][RT];
#pragma unroll
    for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
        for (int k = 0; k < RT; ++k) acc[i][k] = floatx4{0, 0, 0, 0};
    const int begin = blockIdx.y * a.each, end = begin + a.each < s.n_in ? begin + a.each : s.n_in;
    constexpr int kUnder = RT <= 4 ? kLaneBatch : 1;
    for (int c0 = begin + 16 * wave; c0 < end; c0 += 64 * kUnder) {
        Raw<X> vx[kUnder][kRowTiles];
        Raw<W> vw[kUnder][RT];
#pragma unroll
        for (int u = 0; u < kUnder; ++u) {
            const int c = c0 + 64 * u + term;
#pragma unroll
            for (int i = 0; i < kRowTiles; ++i) vx[u][i] = fetch_four<X, IN4>(x[i], c, end - c);
#pragma unroll
            for (int k = 0; k < RT; ++k) vw[u][k] = fetch_four<W, IN4>(w[k], c, end - c);
        }
#pragma unroll
        for (int u = 0; u < kUnder; ++u) {
            const int left = end - (c0 + 64 * u + term);
            floatx4 fx[kRowTiles];
#pragma unroll
            for (int i = 0; i < kRowTiles; ++i) fx[i] = rectify_four(widen(vx[u][i], left, x_half), s.relu);
#pragma unroll
            for (int k = 0; k < RT; ++k) {
                const floatx4 fw = widen(vw[u][k], 16 * k + row < s.rank ? left : 0, w_half);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int i = 0; i < kRowTiles; ++i) acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[e], fx[i][e], acc[i][k], 0, 0, 0);
            }
        }
    }
    // the waves' sums; a lane has ranks 4 (lane / 16) .. + 3 of 16, place lane % 16
    float *const low = a.low + ((int64_t)blockIdx.y * a.places + tile.first) * (16 * RT);
#pragma unroll
    for (int k0 = 0; k0 < RT; k0 += kJoined) {
        if (k0 > 0) __syncthreads();
        if (wave > 0)
#pragma unroll
            for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
                for (int k = 0; k < kJoined; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sums[wave - 1][(i * kJoined + k) * 4 + e][lane] = acc[i][k0 + k][e];
        __syncthreads();
        if (wave > 0) continue;
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
            for (int k = 0; k < kJoined; ++k) {
                floatx4 sum = acc[i][k0 + k];
#pragma unroll
                for (int v = 0; v < 3; ++v)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] += sums[v][(i * kJoined + k) * 4 + e][lane];
                const int at = 16 * (k0 + k) + term;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = at + e < s.rank ? sum[e] : 0.0f;   // (beyond the rank x may have made NaN of zeros)
                if (16 * i + row < tile.rows) *reinterpret_cast<floatx4 *>(low + (16 * i + row) * (16 * RT) + at) = sum;
            }
    }
}

// y[place][j] += scale sum_k B[j][k] low[place][k], 16 outputs of all places of the tile at a time
template <bool W, bool RANK4, int RT>
__global__ __launch_bounds__(256) void adapters_up_kernel(AdapterArgs a, bool by_four)
{
    constexpr int kRowTiles = kTileRows / 16;
    if ((int)blockIdx.x >= *a.tile_count) return;
    const AdapterShape &s = a.s;
    const Tile tile = a.tiles[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, term = 4 * (lane >> 4);
    const bool w_half = s.dtype == LMKAN_F16;
    const float scale = a.scale ? a.scale[tile.adapter] : 1.0f;
    floatx4 low[kRowTiles][RT];
    void *y[kRowTiles];
    bool exists[kRowTiles];
#pragma unroll
    for (int i = 0; i < kRowTiles; ++i) {
        exists[i] = 16 * i + row < tile.rows;
        const int p = tile.first + (exists[i] ? 16 * i + row : tile.rows - 1);
        y[i] = row_at(a.y, (int64_t)a.rows[p] * s.n_out, s.y_dtype);
#pragma unroll
        for (int k = 0; k < RT; ++k) {
            low[i][k] = *reinterpret_cast<const floatx4 *>(a.low + (int64_t)p * (16 * RT) + 16 * k + term);
            for (int d = 1; d < a.splits; ++d) low[i][k] += *reinterpret_cast<const floatx4 *>(a.low + ((int64_t)d * a.places + p) * (16 * RT) + 16 * k + term);
        }
    }
    const int begin = blockIdx.y * a.outputs, end = begin + a.outputs < s.n_out ? begin + a.outputs : s.n_out;
    for (int j0 = begin + 16 * wave; j0 < end; j0 += 64) {
        const int j = j0 + row < s.n_out ? j0 + row : s.n_out - 1;
        const void *const w = row_at(a.b, ((int64_t)tile.adapter * s.n_out + j) * s.rank, s.dtype);
        Raw<W> vw[RT];
#pragma unroll
        for (int k = 0; k < RT; ++k) vw[k] = fetch_four<W, RANK4>(w, 16 * k + term, s.rank - 16 * k - term);
        const int out = j0 + term;   // a lane's results: outputs out .. out + 3, place lane % 16
        float before[kRowTiles][4];
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
            if (by_four) {
                load_piece(y[i], out < s.n_out ? out : 0, s.y_dtype, before[i]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) before[i][e] = load_as_float(y[i], out + e < s.n_out ? out + e : 0, s.y_dtype);
            }
        }
        floatx4 acc[kRowTiles];
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) acc[i] = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < RT; ++k) {
            const floatx4 fw = widen(vw[k], s.rank - 16 * k - term, w_half);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < kRowTiles; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[e], low[i][k][e], acc[i], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(scale, acc[i][e], before[i][e]);
            if (!exists[i]) continue;
            if (by_four) {
                if (out < s.n_out) store_piece(y[i], out, s.y_dtype, o);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (out + e < s.n_out) store_from_float(y[i], out + e, s.y_dtype, o[e]);
            }
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

constexpr int kUnits = 256;   // compute units

size_t item_of(int dtype) { return dtype == LMKAN_F32 ? 4 : 2; }

// One launch while what its workgroups read of A, each for itself, is little
bool few_rows(const AdapterShape &s)
{
    const int64_t a = (int64_t)s.rank * s.n_in * item_of(s.dtype), groups = s.batch * ((s.n_out + kFewOutputs - 1) / kFewOutputs);
    return groups <= 512 && a <= 256 << 10 && a * groups <= 32 << 20;
}

int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : rank <= 128 ? 8 : 16; }

// Pieces of the inputs: as many as keep two workgroups on a compute unit, of 256 inputs at least
void split_inputs(const AdapterShape &s, int rows, int *splits, int *each)
{
    const int tiles = (rows + kTileRows - 1) / kTileRows;
    int n = 1;
    while (n < 32 && tiles * n < 2 * kUnits && s.n_in > 256 * n) n *= 2;
    *each = ((s.n_in + n - 1) / n + 63) / 64 * 64;
    *splits = (s.n_in + *each - 1) / *each;
}

struct Layout {
    size_t tiles, count, rows, low, total;
    int most_tiles, splits, each, chunk;
};
Layout layout_of(const AdapterShape &s)
{
    Layout l = {};
    l.chunk = (int)(s.batch < kChunk ? s.batch : kChunk);
    split_inputs(s, l.chunk, &l.splits, &l.each);
    l.most_tiles = l.chunk / kTileRows + (s.count < l.chunk ? s.count : l.chunk);   // (each adapter has one that is not full at most)
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += align256(bytes); return here; };
    l.tiles = take((size_t)l.most_tiles * sizeof(Tile));
    l.count = take(sizeof(int));
    l.rows = take((size_t)l.chunk * sizeof(int));
    l.low = take((size_t)l.splits * l.chunk * 16 * rank_tiles(s.rank) * sizeof(float));
    l.total = at;
    return l;
}

template <class F>
void with(bool v, F &&f)
{
    if (v) f(std::true_type());
    else f(std::false_type());
}
template <class F>
void with_rank(int rank, F &&f)
{
    switch (rank_tiles(rank)) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    default: return f(std::integral_constant<int, 16>());
    }
}

}  // namespace

size_t adapters_workspace_bytes(const AdapterShape &s) { return few_rows(s) ? 0 : layout_of(s).total; }

void launch_adapters(const AdapterShape &s, const void *x, const int32_t *index, const void *a, const void *b, const float *scale, void *y,
                     void *workspace, hipStream_t stream)
{
    AdapterArgs args{s, x, index, a, b, scale, y};
    const bool in4 = s.n_in % 4 == 0 && aligned_to(x, 4 * item_of(s.x_dtype)) && aligned_to(a, 4 * item_of(s.dtype));
    const bool rank4 = s.rank % 4 == 0 && aligned_to(b, 4 * item_of(s.dtype)), by_four = pieces_ok(4, s.n_out, y, s.y_dtype);
    const bool xw = s.x_dtype == LMKAN_F32, ww = s.dtype == LMKAN_F32;
    if (few_rows(s)) {
        const dim3 groups((unsigned)s.batch, (s.n_out + kFewOutputs - 1) / kFewOutputs);
        with(xw, [&](auto X) {
            with(ww, [&](auto W) {
                with(in4, [&](auto I) {
                    with(rank4, [&](auto R) { adapters_few_kernel<X.value, W.value, I.value, R.value><<<groups, kFewOutputs, 0, stream>>>(args); });
                });
            });
        });
        return;
    }
    const Layout l = layout_of(s);
    char *const ws = static_cast<char *>(workspace);
    args.tiles = reinterpret_cast<Tile *>(ws + l.tiles);
    args.tile_count = reinterpret_cast<int *>(ws + l.count);
    args.rows = reinterpret_cast<int *>(ws + l.rows);
    args.low = reinterpret_cast<float *>(ws + l.low);
    args.splits = l.splits, args.each = l.each;
    // outputs of a workgroup: a multiple of 64, fewer where tiles are few
    const int tiles = (l.chunk + kTileRows - 1) / kTileRows;
    int pieces = 1;
    while (tiles * pieces < 4 * kUnits && pieces * 64 < s.n_out) pieces *= 2;
    args.outputs = ((s.n_out + pieces - 1) / pieces + 63) / 64 * 64;
    const unsigned across = (s.n_out + args.outputs - 1) / args.outputs;
    for (int64_t first = 0; first < s.batch; first += kChunk) {
        args.places = (int)(s.batch - first < kChunk ? s.batch - first : kChunk);
        args.x = static_cast<const char *>(x) + first * s.n_in * item_of(s.x_dtype);
        args.y = static_cast<char *>(y) + first * s.n_out * item_of(s.y_dtype);
        const unsigned most = (unsigned)(args.places / kTileRows + (s.count < args.places ? s.count : args.places));
        adapters_order_kernel<<<1, 1024, 0, stream>>>(args, first);
        with_rank(s.rank, [&](auto RT) {
            with(ww, [&](auto W) {
                with(xw, [&](auto X) {
                    with(in4, [&](auto I) { adapters_down_kernel<X.value, W.value, I.value, RT.value><<<dim3(most, l.splits), 256, 0, stream>>>(args); });
                });
                with(rank4, [&](auto R) { adapters_up_kernel<W.value, R.value, RT.value><<<dim3(most, across), 256, 0, stream>>>(args, by_four); });
            });
        });
    }
}

}  // namespace lmkan
