// Tiles of matrix products on the matrix cores: operands whose rows lie along the summed axis, staged through
// LDS in lines of 128 bytes a row, 16-byte fragments, 16 x 16 matrix instructions.
//
// Two kinds of operands:
//   pairs   a float32 value v held as two float16, v s = hi + lo (s a power of two, 22 bits of v): a line of
//           128 bytes holds 32 values, eight at a time: chunks 0..3 the hi parts, 4..7 the lo parts.  A product
//           is hi hi + hi lo + lo hi, summed in float32 (lo lo, 2^-22 of it, is left out).  Matrices of pairs
//           lie panel by panel, [depth / 32][rows][128 bytes]: what a tile reads at a time is one piece.
//   codes   int8, 128 of them a line, rows `pitch` bytes apart.
// Chunk c of row r sits in slot c ^ ((r >> 1) & 7) of its line, in LDS and in panels: the 16-byte reads of the
// lanes of a wave (16 rows, four chunks) then fall on all banks alike.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lmkan {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));

constexpr int kLine = 128;       // bytes of a row in LDS
constexpr int kPanel = 32;       // values of a line of pairs

__host__ __device__ __forceinline__ int panels(int depth) { return (depth + kPanel - 1) / kPanel; }
__host__ __device__ __forceinline__ int64_t pair_bytes(int rows, int depth) { return (int64_t)panels(depth) * rows * kLine; }

__device__ __forceinline__ int slot_of(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

// where chunk `chunk` of values k .. k + 7 of a row lies in a matrix of pairs
__device__ __forceinline__ int64_t pair_at(int rows, int row, int panel, int chunk)
{
    return ((int64_t)panel * rows + row) * kLine + slot_of(row, chunk) * 16;
}

// The value of the first lane, for one that is the same in all of them but that the compiler cannot tell to be
template <class V>
__device__ __forceinline__ V uniform(V v)
{
    static_assert(sizeof(V) == 4 || sizeof(V) == 8, "");
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)u), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32));
        return __builtin_bit_cast(V, (uint64_t)hi << 32 | lo);
    }
}

// 16 bytes per lane from global memory (a wave-uniform base, 32 bits of offset per lane) to LDS at lds + 16 lane.
// The compiler does not know of the load (it cannot make reads of the other buffer wait for it); it is awaited
// with landed().  m0 is a reserved register to the compiler, which sets it before any use of its own.  The instruction
// set asks for one wait state between a scalar write of m0 and a load that takes its place from it; the compiler adds
// none inside a statement of ours (s_nop: without it a line may go to the place of the one before).
__device__ __forceinline__ void load_to_lds(const void *base, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :
                 : "v"(offset), "s"(uniform(base)), "s"(uniform(lds)) : "memory");
}

__device__ __forceinline__ unsigned lds_offset(const void *p)
{
    return (unsigned)(size_t)(__attribute__((address_space(3))) const void *)p;
}

// All but the wave's last `LEFT` loads have landed and its own reads are done; with several waves, then all waves' have
template <int LEFT, int WAVES>
__device__ __forceinline__ void landed()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
    if (WAVES > 1) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Tile shape: ROWS x COLS outputs of one workgroup, WR x WC waves, stages in BUFFERS buffers
template <int ROWS_, int COLS_, int WR_, int WC_, int BUFFERS_>
struct TileShape {
    static constexpr int ROWS = ROWS_, COLS = COLS_, WR = WR_, WC = WC_, BUFFERS = BUFFERS_;
    static constexpr int WAVES = WR * WC, THREADS = 64 * WAVES;
    static constexpr int RT = ROWS / WR / 16, CT = COLS / WC / 16;   // 16 x 16 tiles of a wave
    static constexpr int STAGE = (ROWS + COLS) * kLine;              // bytes of a stage
    static constexpr int LOADS = (ROWS + COLS) / 8 / WAVES;          // loads of a wave a stage
    static constexpr int LDS = BUFFERS * STAGE;
    static constexpr int GROUPS = RT * CT;                           // groups of four outputs of a lane
};

// One operand of a tile: the lines of stage s of its rows start at base + s * step
struct Operand {
    const char *base;
    int64_t step;
    int last;        // last row of the tile that exists (for rows beyond, others are read: their outputs are dropped)
    bool panels;     // lines are adjacent, slots in place (pairs); else rows of codes, `pitch` bytes apart
    unsigned pitch;
    int limit;       // codes: the last 16 bytes of a row; lines that end beyond read them there (the other operand is zero)
};

// Where a lane's 16 bytes of the eight lines from row r0 on lie in a panel, for a tile of N rows that exist up to row
// `last`; lanes beyond the last line read its last bytes.  (A panel may have 2^26 lines, a tile no more than N.)
template <int N>
__host__ __device__ __forceinline__ unsigned panel_offset(int last, int r0, int lane)
{
    const unsigned end = (unsigned)(last < N - 1 ? last : N - 1) * kLine + kLine - 16, at = (unsigned)(r0 * kLine + lane * 16);
    return at < end ? at : end;
}

// Brings the lines of a stage of one operand to LDS, N rows, from wave `wave` of WAVES.
template <int N, int WAVES>
__device__ __forceinline__ void stage_operand(const Operand &o, int stage, unsigned lds, int wave, int lane)
{
    const char *base = o.base + stage * o.step;
    asm volatile("" : "+v"(lane));   // (offsets are worked out again every stage: kept, they take the registers of sums)
#pragma unroll
    for (int g = 0; g < N / 8 / WAVES; ++g) {
        const int r0 = (g * WAVES + wave) * 8;
        unsigned at;
        if (o.panels) {
            at = panel_offset<N>(o.last, r0, lane);
        } else {
            const int r = r0 + (lane >> 3), c = slot_of(r, lane & 7) * 16, most = o.limit - stage * kLine;
            at = (unsigned)(r < o.last ? r : o.last) * o.pitch + (unsigned)(c < most ? c : most);
        }
        load_to_lds(base, at, lds + r0 * kLine);
    }
}

// What a lane holds of a line of 16 rows: row lane & 15, chunk lane >> 4 of the four of each half of the line.
// (16 rows further on the slots are the same.)
template <class V>
struct Fragment {
    V half[2];
};
struct FragmentPlace {
    unsigned at[2];   // of the first 16 rows
    __device__ __forceinline__ FragmentPlace(int lane)
    {
        const int row = lane & 15, chunk = lane >> 4;
        at[0] = row * kLine + slot_of(row, chunk) * 16;
        at[1] = row * kLine + slot_of(row, 4 + chunk) * 16;
    }
    template <class V>
    __device__ __forceinline__ void load(Fragment<V> &f, const char *lds, int sixteens) const
    {
        f.half[0] = *reinterpret_cast<const V *>(lds + at[0] + sixteens * 16 * kLine);
        f.half[1] = *reinterpret_cast<const V *>(lds + at[1] + sixteens * 16 * kLine);
    }
};

// acc[i] += the products of row fragments i and one column fragment over a line.  The instruction's first operand
// gives the columns of the output (four adjacent ones to a lane), its second the rows (a row a lane).
struct PairProduct {
    typedef half8 Element;
    typedef floatx4 Acc;
    // The 96 products of a line are summed by themselves first: one rounding at the size of the whole sum a line
    // instead of three (over a depth of 1024 the sum is then off by 2^-24 * 6, not * 10)
    template <int N>
    static __device__ __forceinline__ void line(const Fragment<half8> (&rows)[N], const Fragment<half8> &cols, Acc (&sum)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(cols.half[1], rows[i].half[0], Acc{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(cols.half[0], rows[i].half[1], sum[i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(cols.half[0], rows[i].half[0], sum[i], 0, 0, 0);
    }
    static constexpr bool kBySum = true;
};

struct CodeProduct {
    typedef intx4 Element;
    typedef intx4 Acc;
    template <int N>
    static __device__ __forceinline__ void line(const Fragment<intx4> (&rows)[N], const Fragment<intx4> &cols, Acc (&sum)[N])
    {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cols.half[h], rows[i].half[h], sum[i], 0, 0, 0);
    }
    static constexpr bool kBySum = false;
};

// The main loop: stages from, from + step .. below `to` of both operands, by wave `wave` of T's.  While one buffer is
// multiplied the others fill; the last columns of a stage are multiplied after the barrier that ends it, while the first
// fragments of the next are on their way.
template <class T, class Product>
__device__ __forceinline__ void multiply_stages(const Operand &rows, const Operand &cols, int from, int to, int step, char *lds, int wave,
                                                typename Product::Acc (&acc)[T::CT][T::RT])
{
    typedef typename Product::Acc Acc;
    typedef Fragment<typename Product::Element> Frag;
    constexpr int kAhead = T::BUFFERS - 1;
    const int lane = threadIdx.x & 63;
    const unsigned at = lds_offset(lds);
    const int wr = wave / T::WC, wc = wave % T::WC;
    const int n = (to - from + step - 1) / step;
#pragma unroll
    for (int j = 0; j < T::CT; ++j)
#pragma unroll
        for (int i = 0; i < T::RT; ++i) acc[j][i] = Acc{0, 0, 0, 0};
    if (n <= 0) return;
    const auto fill = [&](int k, int buffer) {
        const int stage = from + k * step;
        stage_operand<T::ROWS, T::WAVES>(rows, stage, at + buffer * T::STAGE, wave, lane);
        stage_operand<T::COLS, T::WAVES>(cols, stage, at + buffer * T::STAGE + T::ROWS * kLine, wave, lane);
    };
    // stage k has landed (near the end fewer loads are under way: then all of them are awaited)
    const auto await = [&](int k) {
        if (k + kAhead <= n) landed<(kAhead - 1) * T::LOADS, T::WAVES>();
        else landed<0, T::WAVES>();
    };
    const FragmentPlace place(lane);
    for (int b = 0; b < kAhead; ++b)
        if (b < n) fill(b, b);
    int buffer = 0;
    Frag r[T::RT], c[2];
    // the first fragments of a stage that has landed
    const auto begin = [&]() {
        const char *p = lds + buffer * T::STAGE;
        place.load(c[0], p + (T::ROWS + wc * T::CT * 16) * kLine, 0);
#pragma unroll
        for (int i = 0; i < T::RT; ++i) place.load(r[i], p + wr * T::RT * 16 * kLine, i);
    };
    // sums of columns j are added while columns j + 1 are multiplied
    Acc sum[T::RT];
    const auto multiply_by = [&](const Frag (&rows)[T::RT], const Frag &cols, Acc (&to)[T::RT], Acc (&before)[T::RT]) {
        if (Product::kBySum) {
            Acc now[T::RT];
            Product::line(rows, cols, now);
#pragma unroll
            for (int i = 0; i < T::RT; ++i) {
                before[i] += sum[i], sum[i] = now[i];
                asm volatile("" : "+v"(before[i]));   // (added here, not when the sum is next needed: that keeps them all)
            }
#pragma unroll
            for (int i = 0; i < T::RT; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 3, 0);   // matrix instructions
                __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);   // vector instructions
            }
        } else {
            Product::line(rows, cols, to);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int i = 0; i < T::RT; ++i) sum[i] = Acc{0, 0, 0, 0};
    await(0);
    if (kAhead < n) fill(kAhead, kAhead);
    begin();
    for (int k = 0; k < n; ++k) {
        const char *p = lds + buffer * T::STAGE + (T::ROWS + wc * T::CT * 16) * kLine;
#pragma unroll
        for (int j = 0; j + 1 < T::CT; ++j) {
            place.load(c[(j + 1) & 1], p, j + 1);
            multiply_by(r, c[j & 1], acc[j], acc[j == 0 ? T::CT - 1 : j - 1]);
        }
        // own reads are done (told to the compiler: it would wait for the next stage's before the products below)
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
        static_assert(T::CT % 2 == 0, "the last columns of a stage are the second of two");
        const Frag last = c[1];
        Frag held[T::RT];
#pragma unroll
        for (int i = 0; i < T::RT; ++i) held[i] = r[i];
        if (k + 1 < n) {
            await(k + 1);
            const int done = buffer;
            buffer = buffer == kAhead ? 0 : buffer + 1;
            if (k + 1 + kAhead < n) fill(k + 1 + kAhead, done);
            begin();
        }
        multiply_by(held, last, acc[T::CT - 1], acc[T::CT - 2]);
    }
    if (Product::kBySum)
#pragma unroll
        for (int i = 0; i < T::RT; ++i) acc[T::CT - 1][i] += sum[i];
}

// Stages [from, to), from < to, by all waves of the workgroup together; LDS is free when it returns
template <class T, class Product>
__device__ __forceinline__ void multiply(const Operand &rows, const Operand &cols, int from, int to, char *lds,
                                         typename Product::Acc (&acc)[T::CT][T::RT])
{
    multiply_stages<T, Product>(rows, cols, from, to, 1, lds, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), acc);
    __syncthreads();
}

// The same for a tile that has a compute unit to itself: each wave takes every WAVES-th stage of the whole tile, in
// buffers of its own and without a barrier, and the sums are added up at the end, a quarter of the tile to a wave.
// Half as much is read from LDS per product as where the waves share the tile.
template <class T>
struct Alone {
    typedef TileShape<T::ROWS, T::COLS, 1, 1, T::BUFFERS> Whole;
    static constexpr int LDS = T::WAVES * Whole::LDS;
};
template <class T, class Product>
__device__ __forceinline__ void multiply_alone(const Operand &rows, const Operand &cols, int from, int to, char *lds,
                                               typename Product::Acc (&acc)[T::CT][T::RT])
{
    typedef typename Product::Acc Acc;
    typedef typename Alone<T>::Whole W;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    Acc own[W::CT][W::RT];
    char *place = lds + wave * W::LDS;
    multiply_stages<W, Product>(rows, cols, from + wave, to, T::WAVES, place, 0, own);
    static_assert(W::LDS >= W::GROUPS * 64 * (int)sizeof(Acc), "the sums fit the buffers");
    Acc *sums = reinterpret_cast<Acc *>(place) + lane;
#pragma unroll
    for (int j = 0; j < W::CT; ++j)
#pragma unroll
        for (int i = 0; i < W::RT; ++i) sums[(j * W::RT + i) * 64] = own[j][i];
    __syncthreads();
    const int wr = wave / T::WC, wc = wave % T::WC;
#pragma unroll
    for (int j = 0; j < T::CT; ++j)
#pragma unroll
        for (int i = 0; i < T::RT; ++i) acc[j][i] = Acc{0, 0, 0, 0};
    for (int w = 0; w < T::WAVES; ++w) {
        const Acc *from_wave = reinterpret_cast<const Acc *>(lds + w * W::LDS) + lane;
#pragma unroll
        for (int j = 0; j < T::CT; ++j)
#pragma unroll
            for (int i = 0; i < T::RT; ++i) acc[j][i] += from_wave[((wc * T::CT + j) * W::RT + wr * T::RT + i) * 64];
    }
    __syncthreads();
}

// The order of tiles: neighbours in the order, which run on one die, share rows and columns of their operands.
// Rows are taken eight at a time, column by column.
__host__ __device__ __forceinline__ void grouped_tile(int t, int down, int across, int *i, int *j)
{
    constexpr int kRows = 8;
    const int group = t / (kRows * across), rest = t - group * kRows * across;
    const int height = down - group * kRows < kRows ? down - group * kRows : kRows;
    *j = rest / height;
    *i = group * kRows + rest - *j * height;
}
// The upper triangle of n x n tiles, in blocks of 4 x 4, column of blocks by column of blocks
__host__ __device__ __forceinline__ void upper_tile(int t, int n, int *i, int *j)
{
    int block = 0;
    while (8 * (block + 1) * (block + 1) + 2 * (block + 1) <= t) ++block;   // (tiles in the columns of blocks before it: 8 b^2 + 2 b)
    const int rest = t - 8 * block * block - 2 * block, width = n - 4 * block < 4 ? n - 4 * block : 4;
    if (rest < 16 * block * width / 4) {
        const int above = rest / (4 * width), in = rest - above * 4 * width;
        *i = 4 * above + (in & 3), *j = 4 * block + (in >> 2);
    } else {
        int in = rest - 4 * width * block, c = 0;
        while (in > c) in -= ++c;
        *i = 4 * block + in, *j = 4 * block + c;
    }
}

// A launch of W workgroups on `tiles` products of `stages` stages each.  Each takes whole tiles round by round; the
// tiles left over for less than a round are cut along the summed axis so that all workgroups get the same number
// of stages.  What a workgroup has of a tile that it does not own whole goes to one of its two slots of a buffer,
// where a second kernel joins the parts in order.
// (Tiles are counted in 32 bits: a tile that is not at the end of a row of tiles stands for at least 64 x 64 results.)
struct WorkSplit {
    int whole;     // tiles [0, whole) are taken whole, a multiple of `workers`
    int tiles;
    int stages;
    int workers;   // workgroups, a multiple of 8
    int cutters;   // workgroups that share the tiles left over
    int each, more;   // their stages, counted through: `each` a workgroup, one more for the first `more`
    __host__ __device__ int left() const { return tiles - whole; }
    __host__ __device__ bool cut() const { return cutters > left(); }
    __host__ __device__ int begin(int w) const { return w * each + (w < more ? w : more); }
    __host__ __device__ int owner(int stage) const
    {
        const int first = more * (each + 1);
        return stage < first ? stage / (each + 1) : more + (stage - first) / each;
    }
    // `join`: what writing and joining parts takes, in stages; tiles are cut where that is less than the stages that
    // the fullest workgroup is spared.  Parts have four stages at least.
    static WorkSplit of(int tiles, int stages, int workers, int join)
    {
        WorkSplit w;
        w.tiles = tiles, w.stages = stages;
        w.whole = tiles / workers * workers;
        const int left = w.left();
        const int64_t total = (int64_t)left * stages, pieces = total / 4;
        const bool cut = (int64_t)stages * (workers - left) > (int64_t)workers * join && pieces > left;
        w.cutters = (int)(!cut ? left : pieces < workers ? pieces : workers);
        w.each = left ? (int)(total / w.cutters) : 0, w.more = left ? (int)(total % w.cutters) : 0;
        w.workers = w.whole ? workers : (w.cutters + 7) / 8 * 8;
        return w;
    }
};

// Calls f(tile, from, to, slot) for everything workgroup `id` takes; slot < 0: the whole tile.  Ids that run on the
// same die (every eighth) take neighbouring tiles.
template <class F>
__device__ __forceinline__ void for_work(const WorkSplit &w, int id, F &&f)
{
    const int place = (id & 7) * (w.workers / 8) + (id >> 3);
    const bool cuts = place < w.cutters;
    int t = place, s = cuts ? w.begin(place) : 0;
    const int end = cuts ? w.begin(place + 1) : 0;
    while (true) {   // (one call: the body is long)
        int tile, from = 0, to = w.stages, slot = -1;
        if (t < w.whole) {
            tile = t, t += w.workers;
        } else if (s < end) {
            const int k = s / w.stages, left = end - s;
            tile = w.whole + k, from = s - k * w.stages;
            to = left < w.stages - from ? from + left : w.stages;
            if (from > 0 || to < w.stages) slot = 2 * place + (from == 0);
            s += to - from;
        } else {
            break;
        }
        f(tile, uniform(from), uniform(to), slot);
    }
}

template <class T, class Acc>
__device__ __forceinline__ void store_part(Acc *parts, int slot, const Acc (&acc)[T::CT][T::RT])
{
    Acc *to = parts + (int64_t)slot * T::GROUPS * 64 * T::WAVES + threadIdx.x;
#pragma unroll
    for (int j = 0; j < T::CT; ++j)
#pragma unroll
        for (int i = 0; i < T::RT; ++i) to[(j * T::RT + i) * 64 * T::WAVES] = acc[j][i];
}

// A wave's share of the parts of tile `tile` (counted from the first that is cut), summed in a fixed order by the
// JOINERS waves of the workgroup; false when the tile was taken whole, or to all but the first of the waves.
// `shared`: GROUPS * 64 * (JOINERS - 1) accumulators.
template <class T, int JOINERS, class Acc>
__device__ __forceinline__ bool join_parts(const WorkSplit &w, int tile, int wave, const Acc *parts, Acc *shared, Acc (&acc)[T::CT][T::RT])
{
    const int first = tile * w.stages;
    const int from = w.owner(first), to = w.owner(first + w.stages - 1);
    if (from == to) return false;
    const int lane = threadIdx.x & 63, joiner = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int j = 0; j < T::CT; ++j)
#pragma unroll
        for (int i = 0; i < T::RT; ++i) acc[j][i] = Acc{0, 0, 0, 0};
    for (int k = from + joiner; k <= to; k += JOINERS) {
        const Acc *at = parts + (int64_t)(2 * k + (w.begin(k) <= first)) * T::GROUPS * 64 * T::WAVES + wave * 64 + lane;
#pragma unroll
        for (int j = 0; j < T::CT; ++j)
#pragma unroll
            for (int i = 0; i < T::RT; ++i) acc[j][i] += at[(j * T::RT + i) * 64 * T::WAVES];
    }
    if (JOINERS == 1) return true;
    if (joiner > 0)
#pragma unroll
        for (int j = 0; j < T::CT; ++j)
#pragma unroll
            for (int i = 0; i < T::RT; ++i) shared[((joiner - 1) * T::GROUPS + j * T::RT + i) * 64 + lane] = acc[j][i];
    __syncthreads();
    if (joiner > 0) return false;
    for (int k = 0; k < JOINERS - 1; ++k)
#pragma unroll
        for (int j = 0; j < T::CT; ++j)
#pragma unroll
            for (int i = 0; i < T::RT; ++i) acc[j][i] += shared[(k * T::GROUPS + j * T::RT + i) * 64 + lane];
    return true;
}

// Waves that join a wave's share: several where parts are small and may be many
template <class T>
constexpr int joiners() { return T::GROUPS <= 4 ? 8 : 1; }
template <class T>
constexpr int join_lds() { return T::GROUPS * 64 * 16 * (joiners<T>() - 1); }

// Calls f(row, col, values) for every 32 x 32 tile of the wave, one after the other: row and col of its corner within
// the workgroup's tile.  values[2 i + j][e] of a lane is at row 16 i + (lane & 15), column 16 j + 4 (lane >> 4) + e.
// ahead(row, col) is called one tile early, where registers allow; what it returns (loads under way) is passed to f.
template <class T, class Acc, class A, class F>
__device__ __forceinline__ void for_wave_tiles(const Acc (&acc)[T::CT][T::RT], int wave, A &&ahead, F &&f)
{
    constexpr int kTiles = T::CT / 2 * (T::RT / 2);
    const int row = wave / T::WC * T::RT * 16, col = wave % T::WC * T::CT * 16;
    const auto values = [&](int i, int j, Acc (&v)[4]) { v[0] = acc[j][i], v[1] = acc[j + 1][i], v[2] = acc[j][i + 1], v[3] = acc[j + 1][i + 1]; };
    if constexpr (T::GROUPS <= 16) {
        auto next = ahead(row, col);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int i = t % (T::RT / 2) * 2, j = t / (T::RT / 2) * 2;
            const auto now = next;
            if (t + 1 < kTiles) next = ahead(row + (t + 1) % (T::RT / 2) * 32, col + (t + 1) / (T::RT / 2) * 32);
            Acc v[4];
            values(i, j, v);
            f(row + 16 * i, col + 16 * j, v, now);
            __builtin_amdgcn_sched_barrier(0);   // (one tile's values at a time in registers)
        }
    } else {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int i = t % (T::RT / 2) * 2, j = t / (T::RT / 2) * 2;
            Acc v[4];
            values(i, j, v);
            f(row + 16 * i, col + 16 * j, v, ahead(row + 16 * i, col + 16 * j));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Four rows of a lane quad, four 16-bit values of adjacent columns each -> the lane's column (its place in the quad),
// four adjacent rows
__device__ __forceinline__ uint2 turn_quad(uint2 x, int lane)
{
    constexpr int kXor1 = 0xb1, kXor2 = 0x4e;   // quad_perm
    const bool upper = lane & 2;
    const int got = __builtin_amdgcn_mov_dpp((int)(upper ? x.x : x.y), kXor2, 0xf, 0xf, true);
    const int y0 = upper ? got : (int)x.x, y1 = upper ? (int)x.y : got;
    const int r0 = __builtin_amdgcn_mov_dpp(y0, kXor1, 0xf, 0xf, true), r1 = __builtin_amdgcn_mov_dpp(y1, kXor1, 0xf, 0xf, true);
    const unsigned pick = lane & 1 ? 0x03020706u : 0x05040100u;
    return make_uint2(__builtin_amdgcn_perm((unsigned)r0, (unsigned)y0, pick), __builtin_amdgcn_perm((unsigned)r1, (unsigned)y1, pick));
}

}  // namespace lmkan
