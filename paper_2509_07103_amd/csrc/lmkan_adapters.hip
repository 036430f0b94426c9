// Low-rank adapters of many requests beside a shared linear term: y[n] += scale[r] B_r (A_r f(x[n])), r = index[n].
//
// A few rows (one launch): a workgroup takes 512 outputs of a row, works out the row's A f(x) for itself and then its
// outputs; what bounds it is the latency of reading A and B once each.  Many rows (three launches, 32768 rows at a time):
//   order  one workgroup sorts the rows by adapter, by counting, into tiles of up to 32 rows of one adapter
//   down   low = A f(x): a tile and a piece of the inputs a workgroup, whose waves take every fourth 16 inputs
//   up     y += scale B low: a tile and a piece of the outputs a workgroup
// Products are those of float32 matrix instructions, 16 x 16 results of 4 terms, or where the types allow it of 16-bit ones.
// Reading x and y once each would bound them as long as the rank is below a hundred; they take twice that at low ranks and three
// times at 128, as every tile of 32 rows reads its adapter again and three launches wait for each other.  A row's result does not
// depend on the rows that share its tile, so that the order within an adapter, which atomics decide, changes nothing.
//
// Measured (us): one row of 4096 -> 4096, rank 16, bfloat16 8.3; 48 rows of 1024 -> 1024, rank 16, 4.2 in a loop of that call (an empty
// launch 3.4); 8192 rows of 1024 -> 1024, rank 32, float32 39: 7.7 for the order (one workgroup, a chain of loads, counters and
// stores), 13.8 down (x at 2.4 TB/s), 16.3 up (y at 4.1 TB/s); 16384 rows of 4096 -> 1024, rank 64, bfloat16 76, float16 80.
#include <type_traits>

#include "lmkan_rows.h"
#include "lmkan_tile.h"

namespace lmkan {

namespace {

constexpr int kTileRows = 32;
constexpr int kChunk = 32768;         // rows that are sorted at a time: counters and places of 16 bits hold them
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
    int splits, each;   // pieces of the inputs, and their length (a multiple of 256)
    int places;         // rows of the chunk
    int outputs;        // of a workgroup of the kernel `up`
};

// Four elements as they lie in memory, and as float32.  WIDE: float32; else 16 bits, float16 when `half`
template <bool WIDE>
struct Raw;
template <>
struct Raw<true> {
    floatx4 v;
};
template <>
struct Raw<false> {
    uintx2 v;
};
// elements at .. at + 3 of which `left` exist; TOGETHER: all or none do, and they are aligned to their size
template <bool WIDE, bool TOGETHER>
__device__ __forceinline__ Raw<WIDE> fetch_four(const void *row, int at, int left)
{
    Raw<WIDE> r;
    if constexpr (WIDE) {
        const float *p = static_cast<const float *>(row);
        if constexpr (TOGETHER) {
            r.v = *reinterpret_cast<const floatx4 *>(p + (left > 0 ? at : 0));
        } else {
            if (left >= 4) {
                r.v = load_words<floatx4, true>(p + at);
                return r;
            }
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = p[i < left ? at + i : 0];
            r.v = floatx4{e[0], e[1], e[2], e[3]};
        }
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(row);
        if constexpr (TOGETHER) {
            r.v = *reinterpret_cast<const uintx2 *>(p + (left > 0 ? at : 0));
        } else {
            if (left >= 4) {
                r.v = load_words<uintx2, true>(p + at);
                return r;
            }
            uint32_t e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = p[i < left ? at + i : 0];
            r.v = uintx2{e[0] | e[1] << 16, e[2] | e[3] << 16};
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
        f = r.v;
    } else {
        const uint32_t w[2] = {r.v[0], r.v[1]};
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
    constexpr int kWaves = kFewOutputs / 64, kRanks = W ? 4 : 8, kPieces = 4, kAhead = 4;   // kAhead: fours of B that are fetched before A f(x) is known
    __shared__ float low[LMKAN_MAX_ADAPTER_RANK];
    const AdapterShape &s = a.s;
    const int64_t n = blockIdx.x;
    const int r = a.index[n];
    if (r < 0 || r >= s.count) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = blockIdx.y * kFewOutputs + threadIdx.x, seen = j < s.n_out ? j : s.n_out - 1;
    const bool x_half = s.x_dtype == LMKAN_F16, w_half = s.dtype == LMKAN_F16;
    const void *const up = row_at(a.b, ((int64_t)r * s.n_out + seen) * s.rank, s.dtype);
    Raw<W> ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ahead[k] = fetch_four<W, RANK4>(up, 4 * k, s.rank - 4 * k);
    const float before = load_as_float(a.y, n * s.n_out + seen, s.y_dtype);
    const void *const x = row_at(a.x, n * s.n_in, s.x_dtype);
    // a wave takes every eighth rank, kRanks of them and kPieces pieces of the row at a time
    for (int k0 = wave; k0 < s.rank; k0 += kWaves * kRanks) {
        const void *const down = row_at(a.a, ((int64_t)r * s.rank + k0) * s.n_in, s.dtype);
        float sum[kRanks] = {};
        for (int c0 = 4 * lane; c0 < s.n_in; c0 += 256 * kPieces) {
            Raw<X> v[kPieces];
            Raw<W> w[kRanks][kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) v[p] = fetch_four<X, IN4>(x, c0 + 256 * p, s.n_in - c0 - 256 * p);
#pragma unroll
            for (int k = 0; k < kRanks; ++k) {
                if (k0 + kWaves * k >= s.rank) break;
#pragma unroll
                for (int p = 0; p < kPieces; ++p)
                    w[k][p] = fetch_four<W, IN4>(row_at(down, (int64_t)(kWaves * k) * s.n_in, W ? LMKAN_F32 : LMKAN_F16), c0 + 256 * p, s.n_in - c0 - 256 * p);
            }
            floatx4 f[kPieces];
#pragma unroll
            for (int p = 0; p < kPieces; ++p) f[p] = rectify_four(widen(v[p], s.n_in - c0 - 256 * p, x_half), s.relu);
#pragma unroll
            for (int k = 0; k < kRanks; ++k) {
                if (k0 + kWaves * k >= s.rank) break;
#pragma unroll
                for (int p = 0; p < kPieces; ++p) {
                    const floatx4 g = widen(w[k][p], s.n_in - c0 - 256 * p, w_half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[k] = fmaf(g[i], f[p][i], sum[k]);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kRanks; ++k) {
            if (k0 + kWaves * k >= s.rank) break;
            sum[k] = over_lanes(sum[k], 64, [](float p, float q) { return p + q; });
            if (lane == 0) low[k0 + kWaves * k] = sum[k];
        }
    }
    __syncthreads();
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

// Adds one to the counter of every lane's adapter (16 bits, two to a word) and returns what it was.  The lanes of a run of
// one adapter, which is what prompts look like, add once.
__device__ __forceinline__ int count_up(uint32_t *counters, int r, bool valid)
{
    const int of = __builtin_amdgcn_readfirstlane(r), shift = 16 * (r & 1);
    if (__ballot(r != of) == 0) {
        if (!__ballot(valid)) return 0;
        const int lane = threadIdx.x & 63;
        uint32_t old = 0;
        if (lane == 0) old = atomicAdd(&counters[of >> 1], 64u << shift);
        return (int)((uint32_t)__builtin_amdgcn_readfirstlane((int)old) >> shift & 0xffff) + lane;
    }
    return valid ? (int)(atomicAdd(&counters[r >> 1], 1u << shift) >> shift & 0xffff) : 0;
}

constexpr int kRead = 16;                 // indices that a thread has in registers
constexpr int kBlockRows = 1024 * kRead;

__global__ __launch_bounds__(1024) void adapters_order_kernel(AdapterArgs a, int64_t first)
{
    __shared__ uint32_t counters[LMKAN_MAX_ADAPTERS / 2];
    __shared__ uint32_t starts[LMKAN_MAX_ADAPTERS + 1];   // of an adapter: its first place, its first tile in the upper half
    __shared__ int waves[2][16];
    const int count = a.s.count, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < (count + 1) / 2; i += 1024) counters[i] = 0;
    int r[kRead];
    const int blocks = (a.places + kBlockRows - 1) / kBlockRows;
    __syncthreads();
    // rows per adapter; block 0 comes last and stays in registers
    for (int b = blocks - 1; b >= 0; --b) {
#pragma unroll
        for (int k = 0; k < kRead; ++k) {
            const int i = b * kBlockRows + k * 1024 + threadIdx.x;
            r[k] = i < a.places ? a.index[first + i] : -1;
        }
#pragma unroll
        for (int k = 0; k < kRead; ++k)
            if (b * kBlockRows + k * 1024 < a.places) count_up(counters, r[k], r[k] >= 0 && r[k] < count);
    }
    __syncthreads();
    // a thread sums adapters [from, to); sums over the threads before it
    const int span = ((count + 1023) / 1024 + 1) & ~1, from = threadIdx.x * span < count ? threadIdx.x * span : count,
              to = from + span < count ? from + span : count;
    const auto counted = [&](int of) { return (int)(counters[of >> 1] >> (16 * (of & 1)) & 0xffff); };
    int rows = 0, tiles = 0;
    for (int of = from; of < to; ++of) rows += counted(of), tiles += (counted(of) + kTileRows - 1) / kTileRows;
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
    if (threadIdx.x == 1023) *a.tile_count = tiles_before + tiles, starts[count] = (uint32_t)(rows_before + rows);
    // the counters become the places where rows go (spans are even: a word belongs to one thread)
    for (int of = from; of < to; of += 2) {
        uint32_t word = 0;
        for (int h = 0; h < 2; ++h) {
            if (of + h >= to) break;
            const int n = counted(of + h);
            starts[of + h] = (uint32_t)rows_before | (uint32_t)tiles_before << 16;
            word |= (uint32_t)rows_before << (16 * h);
            rows_before += n, tiles_before += (n + kTileRows - 1) / kTileRows;
        }
        counters[of >> 1] = word;
    }
    __syncthreads();
    for (int b = 0; b < blocks; ++b) {
        if (b > 0)
#pragma unroll
            for (int k = 0; k < kRead; ++k) {
                const int i = b * kBlockRows + k * 1024 + threadIdx.x;
                r[k] = i < a.places ? a.index[first + i] : -1;
            }
#pragma unroll
        for (int k = 0; k < kRead; ++k) {
            if (b * kBlockRows + k * 1024 >= a.places) break;
            const bool valid = r[k] >= 0 && r[k] < count;
            const int place = count_up(counters, r[k], valid);
            if (!valid) continue;
            a.rows[place] = b * kBlockRows + k * 1024 + threadIdx.x;
            // the row at the start of a tile writes it down
            const uint32_t start = starts[r[k]];
            const int in = place - (int)(start & 0xffff);
            if (in % kTileRows == 0) {
                const int left = (int)(starts[r[k] + 1] & 0xffff) - place;
                a.tiles[(start >> 16) + in / kTileRows] = {r[k], place, left < kTileRows ? left : kTileRows};
            }
        }
    }
}

// ---- products --------------------------------------------------------------------------------------------------------

// Operands come in pieces of 16 bytes, adjacent lanes adjacent pieces of a row (lanes that each take a row of their own
// would cost four times the accesses), and go through LDS, a part of it for every wave, to the lanes that need them: row
// lane % 16 of 16, some terms by lane / 16.  Which terms go to which instruction does not matter, as both operands do it alike.
constexpr int kRowTiles = kTileRows / 16;

// What lanes of a wave have written to LDS is there for the others of the wave (its LDS accesses are in order; the compiler,
// which sees one lane, may not move them over this)
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <bool WIDE>
constexpr int kPerPiece = WIDE ? 4 : 8;

// elements at .. of a row up to `end`, zero beyond; ALIGNED: pieces are whole and aligned
template <bool WIDE, bool ALIGNED>
__device__ __forceinline__ intx4 fetch_piece(const void *row, int at, int end)
{
    constexpr int N = kPerPiece<WIDE>;
    if constexpr (ALIGNED) {
        const intx4 v = *reinterpret_cast<const intx4 *>(static_cast<const char *>(row) + (at < end ? at : 0) * (16 / N));
        return at < end ? v : intx4{0, 0, 0, 0};
    } else {
        if (at + N <= end) return load_words<intx4, true>(static_cast<const char *>(row) + at * (16 / N));
        intx4 v = {0, 0, 0, 0};
        if (at >= end) return v;
        if constexpr (WIDE) {
            const int *p = static_cast<const int *>(row);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = p[at + i < end ? at + i : 0];
                v[i] = at + i < end ? e : 0;
            }
        } else {
            const uint16_t *p = static_cast<const uint16_t *>(row);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = p[at + 2 * i < end ? at + 2 * i : 0], hi = p[at + 2 * i + 1 < end ? at + 2 * i + 1 : 0];
                v[i] = (int)((at + 2 * i < end ? lo : 0) | (at + 2 * i + 1 < end ? hi : 0) << 16);
            }
        }
        return v;
    }
}

// max(., 0) of a piece; NaN stays NaN
template <bool WIDE>
__device__ __forceinline__ intx4 rectify_piece(intx4 v, bool half)
{
    // negative and not NaN: from minus zero up to minus infinity
    const uint32_t most = 0x8000u + (half ? 0x7c00u : 0x7f80u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u = (uint32_t)v[i], lo = u & 0xffffu, hi = u >> 16;
        if (WIDE) v[i] = u >= 0x80000000u && u <= 0xff800000u ? 0 : (int)u;
        else v[i] = (int)((lo >= 0x8000u && lo <= most ? 0 : lo) | (hi >= 0x8000u && hi <= most ? 0 : hi) << 16);
    }
    return v;
}

// four adjacent elements of a line in LDS, as float32
template <bool WIDE>
__device__ __forceinline__ floatx4 four_of(const char *at, bool half)
{
    Raw<WIDE> r;
    r.v = *reinterpret_cast<const decltype(r.v) *>(at);
    return widen(r, 4, half);
}

// low[place][k] = sum_e A[k][e] f(x[place][e]) over a piece of the inputs, for up to 16 RT ranks of a tile.  A wave takes
// every fourth stage of T terms; while a stage is multiplied the next one is on its way.  NATIVE: x and A of one 16-bit type,
// on the instructions of that type (eight times the rate; products are exact and sums float32 as well).
template <bool X, bool W, bool ALIGNED, bool NATIVE, int RT>
__global__ __launch_bounds__(256) void adapters_down_kernel(AdapterArgs a, int held)
{
    constexpr int kLineBytes = RT <= 2 ? 128 : 64, T = kLineBytes / (NATIVE ? 2 : 4), kSlots = kLineBytes / 16;
    constexpr int kRows = kTileRows + 16 * RT, kWave = kRows * kLineBytes, kJoined = RT < 4 ? RT : 4;
    constexpr int kXPieces = T / kPerPiece<X>, kWPieces = T / kPerPiece<W>;                 // of a row
    constexpr int kXLoads = kTileRows * kXPieces / 64, kWLoads = (16 * RT * kWPieces + 63) / 64;
    constexpr int kSums = 3 * kRowTiles * kJoined * 4 * 64 * (int)sizeof(float);
    static_assert(kTileRows * kXPieces % 64 == 0, "");
    if ((int)blockIdx.x >= *a.tile_count) return;
    __shared__ __align__(16) char lds[4 * kWave > kSums ? 4 * kWave : kSums];
    const AdapterShape &s = a.s;
    const Tile tile = a.tiles[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rank0 = blockIdx.z * (16 * RT);
    const bool x_half = s.x_dtype == LMKAN_F16, w_half = s.dtype == LMKAN_F16;
    const int begin = blockIdx.y * a.each, end = begin + a.each < s.n_in ? begin + a.each : s.n_in;
    const void *x[kXLoads];
#pragma unroll
    for (int u = 0; u < kXLoads; ++u) {
        const int p = (u * 64 + lane) / kXPieces;
        x[u] = row_at(a.x, (int64_t)a.rows[tile.first + (p < tile.rows ? p : tile.rows - 1)] * s.n_in, s.x_dtype);   // (the last again)
    }
    const void *const w = row_at(a.a, ((int64_t)tile.adapter * s.rank + rank0) * s.n_in, s.dtype);
    const int ranks = s.rank - rank0;
    struct Stage {
        intx4 x[kXLoads], w[kWLoads];
    };
    const auto fetch = [&](int c) {
        Stage g;
#pragma unroll
        for (int u = 0; u < kXLoads; ++u) g.x[u] = fetch_piece<X, ALIGNED>(x[u], c + lane % kXPieces * kPerPiece<X>, end);
#pragma unroll
        for (int u = 0; u < kWLoads; ++u) {
            const int q = (u * 64 + lane) / kWPieces, at = c + lane % kWPieces * kPerPiece<W>;
            g.w[u] = fetch_piece<W, ALIGNED>(row_at(w, q < ranks ? (int64_t)q * s.n_in : 0, s.dtype), at, q < ranks ? end : 0);   // (beyond the rank: zeros)
        }
        return g;
    };
    // slot of a piece in its line: 16 lanes that read the same piece of 16 rows fall on all banks alike
    const auto slot = [](int row, int piece) { return row * kLineBytes + (piece ^ (kSlots == 8 ? row >> 1 & 7 : row >> 2 & 3)) * 16; };
    char *const mine = lds + wave * kWave, *const mine_w = mine + kTileRows * kLineBytes;
    floatx4 acc[kRowTiles][RT];
#pragma unroll
    for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
        for (int k = 0; k < RT; ++k) acc[i][k] = floatx4{0, 0, 0, 0};
    Stage next = fetch(begin + T * wave);
    for (int c = begin + T * wave; c < end; c += 4 * T) {
        const Stage now = next;
#pragma unroll
        for (int u = 0; u < kXLoads; ++u)
            *reinterpret_cast<intx4 *>(mine + slot((u * 64 + lane) / kXPieces, lane % kXPieces)) = s.relu ? rectify_piece<X>(now.x[u], x_half) : now.x[u];
#pragma unroll
        for (int u = 0; u < kWLoads; ++u)
            if (16 * RT * kWPieces >= 64 || lane < 16 * RT * kWPieces)
                *reinterpret_cast<intx4 *>(mine_w + slot((u * 64 + lane) / kWPieces, lane % kWPieces)) = now.w[u];
        wave_sync();
        if (c + 4 * T < end) next = fetch(c + 4 * T);
        const int row = lane & 15, part = lane >> 4;
        if constexpr (NATIVE) {
#pragma unroll
            for (int h = 0; h < T / 32; ++h) {
                intx4 fx[kRowTiles];
#pragma unroll
                for (int i = 0; i < kRowTiles; ++i) fx[i] = *reinterpret_cast<const intx4 *>(mine + slot(16 * i + row, 4 * h + part));
#pragma unroll
                for (int k = 0; k < RT; ++k) {
                    const intx4 fw = *reinterpret_cast<const intx4 *>(mine_w + slot(16 * k + row, 4 * h + part));
#pragma unroll
                    for (int i = 0; i < kRowTiles; ++i) {
                        if (w_half) acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, fw), __builtin_bit_cast(half8, fx[i]), acc[i][k], 0, 0, 0);
                        else acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw), __builtin_bit_cast(bf16x8, fx[i]), acc[i][k], 0, 0, 0);
                    }
                }
            }
        } else {
            const auto four = [&](const char *base, int r, int q, auto wide, bool half) {   // terms 4 q .. of row r
                constexpr bool kWide = decltype(wide)::value;
                return four_of<kWide>(base + (kWide ? slot(r, q) : slot(r, q >> 1) + 8 * (q & 1)), half);
            };
#pragma unroll
            for (int h = 0; h < T / 16; ++h) {
                floatx4 fx[kRowTiles];
#pragma unroll
                for (int i = 0; i < kRowTiles; ++i) fx[i] = four(mine, 16 * i + row, 4 * h + part, std::bool_constant<X>(), x_half);
#pragma unroll
                for (int k = 0; k < RT; ++k) {
                    const floatx4 fw = four(mine_w, 16 * k + row, 4 * h + part, std::bool_constant<W>(), w_half);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int i = 0; i < kRowTiles; ++i) acc[i][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[e], fx[i][e], acc[i][k], 0, 0, 0);
                }
            }
        }
        wave_sync();
    }
    // the waves' sums; a lane has ranks 4 (lane / 16) .. + 3 of 16, place lane % 16
    float(*const sums)[kRowTiles * kJoined * 4][64] = reinterpret_cast<float(*)[kRowTiles * kJoined * 4][64]>(lds);
    const int row = lane & 15, term = 4 * (lane >> 4);
    float *const low = a.low + ((int64_t)blockIdx.y * a.places + tile.first) * held + rank0;
#pragma unroll
    for (int k0 = 0; k0 < RT; k0 += kJoined) {
        __syncthreads();
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
                for (int e = 0; e < 4; ++e) sum[e] = at + e < ranks ? sum[e] : 0.0f;   // (beyond the rank x may have made NaN of zeros)
                if (16 * i + row < tile.rows) *reinterpret_cast<floatx4 *>(low + (int64_t)(16 * i + row) * held + at) = sum;
            }
    }
}

// Eight values, cut to parts of bfloat16 of 8 bits each: three hold a float32, two a float16, exactly
template <int N>
__device__ __forceinline__ void cut_eight(const float (&v)[8], bf16x8 (&to)[N])
{
    intx4 w[N];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float p = v[i], q = v[i + 1];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t a = __builtin_bit_cast(uint32_t, p), b = __builtin_bit_cast(uint32_t, q);
            w[n][i / 2] = (int)__builtin_amdgcn_perm(b, a, 0x07060302u);   // the upper halves
            if (n + 1 < N) p -= __builtin_bit_cast(float, a & 0xffff0000u), q -= __builtin_bit_cast(float, b & 0xffff0000u);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) to[n] = __builtin_bit_cast(bf16x8, w[n]);
}

// y[place][j] += scale sum_k B[j][k] low[place][k]: 32 outputs of all places of a tile at a time for a wave, while B and y of
// the next 32 are on their way.  The results go through LDS to lanes that lie along the outputs.
// NATIVE: 16-bit adapters, on bfloat16 instructions: low in three parts, B as it is or (float16) in two.  Three or six
// products of 32 terms take 48 or 96 clocks where float32 instructions take 256.
template <bool W, bool Y, bool ALIGNED, bool NATIVE, int RT>
__global__ __launch_bounds__(256) void adapters_up_kernel(AdapterArgs a)
{
    constexpr int kTerms = 16 * RT, kSteps = RT <= 4 ? 1 : RT / 2, T = kTerms / kSteps;   // terms of B at a time: up to 64, or 32 of many
    constexpr int kSize = W ? 4 : 2, kPieces = T / kPerPiece<W>, kLoads = 32 * kPieces / 64;
    constexpr int kBPitch = T * kSize + 16, kLowPitch = (NATIVE && RT == 1 ? 32 : kTerms) + 4, kOutPitch = 36;   // (odd numbers of 16 bytes)
    constexpr int kB = 32 * kBPitch, kOut = 32 * kOutPitch * 4, kWave = kB > kOut ? kB : kOut;
    constexpr int kHalves = NATIVE ? (RT + 1) / 2 : 1, kYLoads = Y ? 4 : 2;
    static_assert(!NATIVE || (!W && ALIGNED && RT <= 8), "");
    if ((int)blockIdx.x >= *a.tile_count) return;
    __shared__ __align__(16) float low[kTileRows * kLowPitch];
    __shared__ __align__(16) char lds[4 * kWave];
    const AdapterShape &s = a.s;
    const Tile tile = a.tiles[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, part = lane >> 4;
    const bool w_half = s.dtype == LMKAN_F16, y_half = s.y_dtype == LMKAN_F16;
    const int begin = blockIdx.y * a.outputs, end = begin + a.outputs < s.n_out ? begin + a.outputs : s.n_out;
    const float scale = a.scale ? a.scale[tile.adapter] : 1.0f;
    const void *const b = row_at(a.b, (int64_t)tile.adapter * s.n_out * s.rank, s.dtype);
    // y: pieces of 16 bytes, 8 or 4 lanes a place
    constexpr int kYPiece = kPerPiece<Y>, kYLanes = 32 / kYPiece;
    void *y[kYLoads];
#pragma unroll
    for (int u = 0; u < kYLoads; ++u) {
        const int p = (u * 64 + lane) / kYLanes;
        y[u] = row_at(a.y, (int64_t)a.rows[tile.first + (p < tile.rows ? p : tile.rows - 1)] * s.n_out, s.y_dtype);
    }
    struct Held {
        intx4 b[kLoads], y[kYLoads];
    };
    const auto fetch_b = [&](int j0, int k0, intx4 (&to)[kLoads]) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int j = j0 + (u * 64 + lane) / kPieces;
            to[u] = fetch_piece<W, ALIGNED>(row_at(b, (int64_t)(j < s.n_out ? j : 0) * s.rank, s.dtype), k0 + lane % kPieces * kPerPiece<W>, j < s.n_out ? s.rank : 0);
        }
    };
    const auto fetch = [&](int j0) {
        Held h;
        if (kSteps == 1) fetch_b(j0, 0, h.b);
#pragma unroll
        for (int u = 0; u < kYLoads; ++u) h.y[u] = fetch_piece<Y, ALIGNED>(y[u], j0 + lane % kYLanes * kYPiece, s.n_out);
        return h;
    };
    Held next = fetch(begin + 32 * wave);
    // the splits' sums
    constexpr int kLow = kLowPitch - 4;
    for (int q = threadIdx.x; q < kTileRows * kLow / 4; q += 256) {
        const int p = q / (kLow / 4), k = q % (kLow / 4) * 4;
        floatx4 sum = {0, 0, 0, 0};
        if (p < tile.rows && k < kTerms)
            for (int d = 0; d < a.splits; ++d) sum += *reinterpret_cast<const floatx4 *>(a.low + ((int64_t)d * a.places + tile.first + p) * kTerms + k);
        *reinterpret_cast<floatx4 *>(low + p * kLowPitch + k) = sum;
    }
    __syncthreads();
    bf16x8 parts[kRowTiles][kHalves][3];
    if constexpr (NATIVE)
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
            for (int k = 0; k < kHalves; ++k) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; e += 4) *reinterpret_cast<floatx4 *>(v + e) = *reinterpret_cast<const floatx4 *>(low + (16 * i + row) * kLowPitch + 32 * k + 8 * part + e);
                cut_eight(v, parts[i][k]);
            }
    char *const mine = lds + wave * kWave;
    for (int j0 = begin + 32 * wave; j0 < end; j0 += 128) {
        const Held now = next;
        floatx4 acc[2][kRowTiles];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kRowTiles; ++i) acc[t][i] = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int step = 0; step < kSteps; ++step) {
            intx4 pieces[kLoads];
            if constexpr (kSteps == 1) {
#pragma unroll
                for (int u = 0; u < kLoads; ++u) pieces[u] = now.b[u];
            } else {
                fetch_b(j0, step * T, pieces);
            }
#pragma unroll
            for (int u = 0; u < kLoads; ++u) *reinterpret_cast<intx4 *>(mine + (u * 64 + lane) / kPieces * kBPitch + lane % kPieces * 16) = pieces[u];
            wave_sync();
            if (step == 0 && j0 + 128 < end) next = fetch(j0 + 128);
            if constexpr (NATIVE) {
                constexpr int kParts = 2;
#pragma unroll
                for (int k = 0; k < (T + 31) / 32; ++k)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        // (16 terms: lanes of the others have zeros of low, and read what they need not)
                        const intx4 w = *reinterpret_cast<const intx4 *>(mine + (16 * t + row) * kBPitch + (T < 32 ? part & 1 : 4 * k + part) * 16);
                        bf16x8 f[kParts];
                        const int at = step * ((T + 31) / 32) + k;
                        if (w_half) {
                            const half8 h = __builtin_bit_cast(half8, w);
                            float v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = T < 32 && part > 1 ? 0.0f : (float)h[e];
                            cut_eight(v, f);
                        } else {
                            f[0] = __builtin_bit_cast(bf16x8, T < 32 && part > 1 ? intx4{0, 0, 0, 0} : w);
                        }
                        // small products first, all of them: the last part of low times the second of B is up to 2^-22 of the whole
#pragma unroll
                        for (int q = 2; q >= 0; --q) {
                            if (w_half)
#pragma unroll
                                for (int i = 0; i < kRowTiles; ++i) acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[1], parts[i][at][q], acc[t][i], 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < kRowTiles; ++i) acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[0], parts[i][at][q], acc[t][i], 0, 0, 0);
                        }
                    }
            } else {
#pragma unroll
                for (int k = 0; k < T / 16; ++k) {
                    floatx4 fl[kRowTiles];
#pragma unroll
                    for (int i = 0; i < kRowTiles; ++i) fl[i] = *reinterpret_cast<const floatx4 *>(low + (16 * i + row) * kLowPitch + step * T + 16 * k + 4 * part);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const floatx4 fw = four_of<W>(mine + (16 * t + row) * kBPitch + (16 * k + 4 * part) * kSize, w_half);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
#pragma unroll
                            for (int i = 0; i < kRowTiles; ++i) acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[e], fl[i][e], acc[t][i], 0, 0, 0);
                    }
                }
            }
            wave_sync();
        }
        // a lane has outputs 4 part .. + 3 of 16, place lane % 16
        float *const out = reinterpret_cast<float *>(mine);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < kRowTiles; ++i) *reinterpret_cast<floatx4 *>(out + (16 * i + row) * kOutPitch + 16 * t + 4 * part) = acc[t][i];
        wave_sync();
#pragma unroll
        for (int u = 0; u < kYLoads; ++u) {
            const int p = (u * 64 + lane) / kYLanes, in = lane % kYLanes * kYPiece, j = j0 + in;
            float o[kYPiece];
#pragma unroll
            for (int e = 0; e < kYPiece; ++e) {
                float old;
                if constexpr (Y) {
                    const int bits = now.y[u][e];   // (a cast of the vector's element itself takes the first)
                    old = __builtin_bit_cast(float, bits);
                } else {
                    const uint16_t bits = (uint16_t)((uint32_t)now.y[u][e / 2] >> (16 * (e & 1)));
                    old = y_half ? (float)__builtin_bit_cast(_Float16, bits) : __builtin_bit_cast(float, (uint32_t)bits << 16);
                }
                o[e] = fmaf(scale, out[p * kOutPitch + in + e], old);
            }
            if (p >= tile.rows) continue;
            if (ALIGNED) {
                if (j < s.n_out) store_piece<kYPiece>(y[u], j, s.n_out, s.y_dtype, o);
            } else {
#pragma unroll
                for (int e = 0; e < kYPiece; e += 4) {
                    const float four[4] = {o[e], o[e + 1], o[e + 2], o[e + 3]};
                    if (j + e < s.n_out) store_piece<-4>(y[u], j + e, s.n_out, s.y_dtype, four);
                }
            }
        }
        wave_sync();
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

constexpr int kUnits = 256;   // compute units

size_t item_of(int dtype) { return dtype == LMKAN_F32 ? 4 : 2; }

// One launch while what its workgroups read of A, each for itself, is little.  Measured (us, one launch / three; bfloat16 adapters):
// 48 rows of 1024 -> 1024, rank 16, 4.2 / 12.9; 512 rows 9.3 / 13.5; 2000 of 333 -> 100, rank 20, 24 / 17; 128 of 2048 -> 2048, rank
// 64, 26 / 17; one of 4096 -> 4096, rank 128, in float32 29 / 24.
bool few_rows(const AdapterShape &s)
{
    const int64_t a = (int64_t)s.rank * s.n_in * item_of(s.dtype), groups = s.batch * ((s.n_out + kFewOutputs - 1) / kFewOutputs);
    return groups <= 1024 && a <= 256 << 10 && a * groups <= 32 << 20;
}

int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : rank <= 128 ? 8 : 16; }

// Pieces of the inputs: as many as keep two workgroups on a compute unit, of 256 inputs at least; of the outputs (below) for four.
// Measured (us, for half as many / as they are / twice as many): 8192 rows of 1024 -> 1024, rank 32, float32 41 / 39 / 44; bfloat16
// 16384 of 4096 -> 1024, rank 64, 79 / 76 / 67; 4096 of 4096 -> 4096, rank 128, 66 / 68 / 87.
constexpr int kMostSplits = 32;
void split_inputs(const AdapterShape &s, int rows, int *splits, int *each)
{
    const int tiles = (rows + kTileRows - 1) / kTileRows;
    int n = 1;
    while (n < kMostSplits && tiles * n < 2 * kUnits && s.n_in > 256 * n) n *= 2;
    *each = ((s.n_in + n - 1) / n + 255) / 256 * 256;
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

// (fewer tiles have more pieces of the inputs: of each number of pieces the batch with the most rows)
size_t adapters_workspace_most(const AdapterShape &s)
{
    size_t most = adapters_workspace_bytes(s);
    for (int n = 2; n <= kMostSplits; n *= 2) {
        AdapterShape smaller = s;
        const int64_t rows = (2 * 2 * kUnits - 1) / n * kTileRows;   // tiles n / 2 < 2 kUnits: the last that `split_inputs` cuts in n
        if (rows < s.batch) smaller.batch = rows;
        const size_t bytes = adapters_workspace_bytes(smaller);
        if (bytes > most) most = bytes;
    }
    return most;
}

void launch_adapters(const AdapterShape &s, const void *x, const int32_t *index, const void *a, const void *b, const float *scale, void *y,
                     void *workspace, hipStream_t stream)
{
    AdapterArgs args{s, x, index, a, b, scale, y};
    const bool in4 = s.n_in % 4 == 0 && aligned_to(x, 4 * item_of(s.x_dtype)) && aligned_to(a, 4 * item_of(s.dtype));
    const bool rank4 = s.rank % 4 == 0 && aligned_to(b, 4 * item_of(s.dtype));
    // pieces of 16 bytes
    const auto whole = [](int n, const void *p, int dtype) { return n % (16 / item_of(dtype)) == 0 && aligned_to(p, 16); };
    const bool in_whole = whole(s.n_in, x, s.x_dtype) && whole(s.n_in, a, s.dtype), out_whole = whole(s.rank, b, s.dtype) && whole(s.n_out, y, s.y_dtype);
    // 16-bit instructions here and on the way up.  Measured (us, float32 / 16-bit): 16384 rows of 4096 -> 1024, rank 64, bfloat16
    // 172 / 76; 4096 of 4096 -> 4096, rank 128, 136 / 69; 16384 of 1024 -> 1024, rank 16, 49 / 41
    const bool native = s.x_dtype == s.dtype && s.dtype != LMKAN_F32;
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
    // outputs of a workgroup: a multiple of 128, fewer where tiles are few
    const int tiles = (l.chunk + kTileRows - 1) / kTileRows;
    int pieces = 1;
    while (tiles * pieces < 4 * kUnits && pieces * 128 < s.n_out) pieces *= 2;
    args.outputs = ((s.n_out + pieces - 1) / pieces + 127) / 128 * 128;
    const unsigned across = (s.n_out + args.outputs - 1) / args.outputs;
    for (int64_t first = 0; first < s.batch; first += kChunk) {
        args.places = (int)(s.batch - first < kChunk ? s.batch - first : kChunk);
        args.x = static_cast<const char *>(x) + first * s.n_in * item_of(s.x_dtype);
        args.y = static_cast<char *>(y) + first * s.n_out * item_of(s.y_dtype);
        const unsigned most = (unsigned)(args.places / kTileRows + (s.count < args.places ? s.count : args.places));
        adapters_order_kernel<<<1, 1024, 0, stream>>>(args, first);
        with_rank(s.rank, [&](auto R) {
            constexpr int RT = R.value, kDown = RT < 8 ? RT : 8;   // (more than 128 ranks take two workgroups on the way down)
            const dim3 down(most, l.splits, RT / kDown), up(most, across);
            if (native) {
                with(in_whole, [&](auto A) { adapters_down_kernel<false, false, A.value, true, kDown><<<down, 256, 0, stream>>>(args, 16 * RT); });
            } else {
                with(ww, [&](auto W) {
                    with(xw, [&](auto X) {
                        with(in_whole, [&](auto A) { adapters_down_kernel<X.value, W.value, A.value, false, kDown><<<down, 256, 0, stream>>>(args, 16 * RT); });
                    });
                });
            }
            with(s.y_dtype == LMKAN_F32, [&](auto Y) {
                if (RT <= 8 && out_whole && s.dtype != LMKAN_F32) {
                    adapters_up_kernel<false, Y.value, true, true, kDown><<<up, 256, 0, stream>>>(args);
                } else {
                    with(ww, [&](auto W) {
                        with(out_whole, [&](auto A) { adapters_up_kernel<W.value, Y.value, A.value, false, RT><<<up, 256, 0, stream>>>(args); });
                    });
                }
            });
        });
    }
}

}  // namespace lmkan
