// Tiles of matrix products on the matrix cores: operands whose rows lie along the summed axis, staged through
// LDS in lines of 128 bytes a row, 16-byte fragments, 32 x 32 matrix instructions.
//
// Two kinds of operands:
//   pairs   a float32 value v held as two float16, v s = hi + lo (s a power of two, 22 bits of v): a line of
//           128 bytes holds 32 values, eight at a time: chunks 0..3 the hi parts, 4..7 the lo parts.  A product
//           is hi hi + hi lo + lo hi, summed in float32 (lo lo, 2^-22 of it, is left out).  Matrices of pairs
//           lie panel by panel, [depth / 32][rows][128 bytes]: what a tile reads at a time is one piece.
//   codes   int8, 128 of them a line, rows `pitch` bytes apart.
// Chunk c of row r sits in slot c ^ ((r >> 1) & 7) of its line, in LDS and in panels: the 16-byte reads of the
// lanes of a wave (32 rows, two chunks) then fall on all banks alike.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lmkan {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int intx16 __attribute__((ext_vector_type(16)));
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

// 16 bytes per lane from global memory (a wave-uniform base, 32 bits of offset per lane) to LDS at lds + 16 lane.
// The compiler does not know of the load (it cannot make reads of the other buffer wait for it); it is awaited
// with landed().  m0 is a reserved register to the compiler, which sets it before any use of its own.
__device__ __forceinline__ void load_to_lds(const void *base, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(lds) : "memory");
}

__device__ __forceinline__ unsigned lds_offset(const void *p)
{
    return (unsigned)(size_t)(__attribute__((address_space(3))) const void *)p;
}

// own loads have landed and own reads are done; then all waves' have
__device__ __forceinline__ void landed()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Tile shape: ROWS x COLS outputs of one workgroup, WR x WC waves.
template <int ROWS_, int COLS_, int WR_, int WC_>
struct TileShape {
    static constexpr int ROWS = ROWS_, COLS = COLS_, WR = WR_, WC = WC_;
    static constexpr int WAVES = WR * WC, THREADS = 64 * WAVES;
    static constexpr int RT = ROWS / WR / 32, CT = COLS / WC / 32;   // 32 x 32 tiles of a wave
    static constexpr int STAGE = (ROWS + COLS) * kLine;              // bytes of a stage
    static constexpr int LDS = 2 * STAGE;
};

// One operand of a tile: its lines of stage s start at base + s * step, row r of the tile `row_step` bytes apart
struct Operand {
    const char *base;
    int64_t step;
    unsigned row_step;
    int last;        // last row of the tile that exists (rows beyond it repeat it: their outputs are dropped)
    bool swizzled;   // slots are chunks already (panels of pairs)
    int limit;       // codes: bytes of a row; a chunk beyond reads the row's last one (the other operand is zero there)
};

// Brings the lines of a stage of one operand to LDS, N rows, from wave `wave` of WAVES.
template <int N, int WAVES>
__device__ __forceinline__ void stage_operand(const Operand &o, int stage, unsigned lds, int wave, int lane)
{
    const char *base = o.base + stage * o.step;
#pragma unroll
    for (int g = 0; g < N / 8 / WAVES; ++g) {
        const int r0 = (g * WAVES + wave) * 8, r = r0 + (lane >> 3), slot = lane & 7;
        const unsigned row = (unsigned)(r < o.last ? r : o.last);
        unsigned at;
        if (o.swizzled) {
            at = row * o.row_step + slot * 16;
        } else {
            const int c = slot_of(r, slot) * 16, most = o.limit - stage * kLine;
            at = row * o.row_step + (unsigned)(c < most ? c : most);
        }
        load_to_lds(base, at, lds + r0 * kLine);
    }
}

__device__ __forceinline__ const char *fragment_at(const char *lds, int row, int chunk) { return lds + row * kLine + slot_of(row, chunk) * 16; }

// acc[r][c] += the tile's products over one stage in LDS, which are summed by themselves first: one rounding at the
// size of the whole sum for 32 values instead of six (a sum over 1024 is then off by 2^-24 * 6, not * 14).  The instruction's first operand gives the columns of the
// output (four adjacent ones to a lane), its second the rows (a row a lane).
template <class T>
struct PairProduct {
    typedef floatx16 Acc;
    static __device__ __forceinline__ void stage(const char *rows, const char *cols, int lane, Acc (&acc)[T::RT][T::CT])
    {
        const int r = lane & 31, h = lane >> 5;
        half8 rh[T::RT][2], rl[T::RT][2];
#pragma unroll
        for (int i = 0; i < T::RT; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                rh[i][k] = *reinterpret_cast<const half8 *>(fragment_at(rows, 32 * i + r, 2 * k + h));
                rl[i][k] = *reinterpret_cast<const half8 *>(fragment_at(rows, 32 * i + r, 4 + 2 * k + h));
            }
#pragma unroll
        for (int j = 0; j < T::CT; ++j) {
            half8 ch[2], cl[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ch[k] = *reinterpret_cast<const half8 *>(fragment_at(cols, 32 * j + r, 2 * k + h));
                cl[k] = *reinterpret_cast<const half8 *>(fragment_at(cols, 32 * j + r, 4 + 2 * k + h));
            }
#pragma unroll
            for (int i = 0; i < T::RT; ++i) {
                Acc t = {};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    t = __builtin_amdgcn_mfma_f32_32x32x16_f16(ch[k], rl[i][k], t, 0, 0, 0);
                    t = __builtin_amdgcn_mfma_f32_32x32x16_f16(cl[k], rh[i][k], t, 0, 0, 0);
                    t = __builtin_amdgcn_mfma_f32_32x32x16_f16(ch[k], rh[i][k], t, 0, 0, 0);
                }
                acc[i][j] += t;
            }
        }
    }
};

template <class T>
struct CodeProduct {
    typedef intx16 Acc;
    static __device__ __forceinline__ void stage(const char *rows, const char *cols, int lane, Acc (&acc)[T::RT][T::CT])
    {
        const int r = lane & 31, h = lane >> 5;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            intx4 rf[T::RT];
#pragma unroll
            for (int i = 0; i < T::RT; ++i) rf[i] = *reinterpret_cast<const intx4 *>(fragment_at(rows, 32 * i + r, 2 * k + h));
#pragma unroll
            for (int j = 0; j < T::CT; ++j) {
                const intx4 cf = *reinterpret_cast<const intx4 *>(fragment_at(cols, 32 * j + r, 2 * k + h));
#pragma unroll
                for (int i = 0; i < T::RT; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(cf, rf[i], acc[i][j], 0, 0, 0);
            }
        }
    }
};

// The main loop: stages [from, to) of both operands.  Two buffers: while one is multiplied the other fills.
template <class T, template <class> class Product>
__device__ __forceinline__ void multiply(const Operand &rows, const Operand &cols, int from, int to, char *lds,
                                         typename Product<T>::Acc (&acc)[T::RT][T::CT])
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const unsigned at = lds_offset(lds);
    const int wr = wave / T::WC, wc = wave % T::WC;
#pragma unroll
    for (int i = 0; i < T::RT; ++i)
#pragma unroll
        for (int j = 0; j < T::CT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const auto fill = [&](int stage, int buffer) {
        stage_operand<T::ROWS, T::WAVES>(rows, stage, at + buffer * T::STAGE, wave, lane);
        stage_operand<T::COLS, T::WAVES>(cols, stage, at + buffer * T::STAGE + T::ROWS * kLine, wave, lane);
    };
    if (from >= to) return;
    fill(from, 0);
    for (int s = from; s < to; ++s) {
        const int buffer = (s - from) & 1;
        landed();
        if (s + 1 < to) fill(s + 1, buffer ^ 1);
        const char *p = lds + buffer * T::STAGE;
        Product<T>::stage(p + wr * T::RT * 32 * kLine, p + T::ROWS * kLine + wc * T::CT * 32 * kLine, lane, acc);
    }
}

// Calls f(row, col, values) for every group of four adjacent columns a lane holds; row and col within the tile
template <class T, class Acc, class F>
__device__ __forceinline__ void for_outputs(Acc (&acc)[T::RT][T::CT], F &&f)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int row = wave / T::WC * T::RT * 32 + (lane & 31), col = wave % T::WC * T::CT * 32 + 4 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < T::RT; ++i)
#pragma unroll
        for (int j = 0; j < T::CT; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const auto &a = acc[i][j];
                f(row + 32 * i, col + 32 * j + 8 * g, a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]);
            }
}

// Workgroup id -> place in the order of work: the ids of one die (every eighth) take neighbouring places
__device__ __forceinline__ int64_t place_of(unsigned id, int64_t total)
{
    const int64_t each = (total + 7) / 8;
    return (int64_t)(id & 7) * each + (id >> 3);
}

}  // namespace lmkan
