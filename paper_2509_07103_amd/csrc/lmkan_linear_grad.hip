// Gradients of the linear term's weights and bias from a checkpoint of its input:
//   grad_weight[j][e] = sum_n g[n][j] f(value[n][e]),  grad_bias[j] = sum_n g[n][j].
//
// A value has 7 bits and a power of two: it is exact in bfloat16.  A gradient is cut into parts of 8 bits, three of a float32, two of
// a float16, which are exact as well, so that 32 x 32 x 16 bfloat16 instructions make exact products and float32 sums: three of
// them take a third of the time of float32 instructions.  The axis that is summed is the batch, across which neither matrix is
// contiguous: gradients go from memory to the instruction's operands directly (a lane has two adjacent outputs of eight rows),
// codes are turned on their way through LDS.  A tile of 64 to 256 outputs and 128 inputs a workgroup; the batch is cut where tiles are
// few, and a second launch adds the parts.
//
// Measured (us; TFLOP/s counted with the parts, where the library's bfloat16 product reaches 1225): 16384 of 4096 -> 4096 float32
// 1330 (1240), 8192 of 1024 -> 1024 float32 58 (890), of which 8.8 add the parts, float16 47 (730); 4096 of 4096 -> 4096 bfloat16 143
// (960), bound by reads of four bytes a lane; 5000 of 500 -> 333 float32 24, 131072 of 64 -> 10 bfloat16 22 with the bias and 18
// without, bound by the start of a workgroup (3 to 4) and the second launch.
#include <type_traits>

#include "lmkan_rows.h"
#include "lmkan_tile.h"

namespace lmkan {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int kDepth = 64;            // rows of the batch in a stage
constexpr int kCols = 128;            // inputs of a tile
constexpr int kWaveRows = 64;         // outputs of a wave
constexpr int kStageBytes = kCols * kLine;
constexpr int kScalePitch = kDepth + 4, kScaleFloats = kCols / kBlock * kScalePitch;   // powers of two of a stage

// slot of chunk `chunk` (eight rows of the batch) in the line of input `e`
__device__ __forceinline__ int grad_slot(int e, int chunk) { return chunk ^ ((e >> 1) & 7) ^ ((e >> 4) & 1); }

struct GradArgs {
    int64_t batch;
    int n_in, n_out;
    bool relu, accumulate;
    const int8_t *codes;
    const uint8_t *exps;
    const void *grad_y;
    float *grad_weight, *grad_bias;
    int down, across;      // tiles
    int first;             // of the launch, counted through tiles and splits
    int splits, stages;    // stages: of 64 rows in all
    int each, more;        // of a split: `each`, one more for the first `more`
    floatx4 *parts;        // [splits][tiles][wave][GROUPS][lane], or null: one split
    double *bias_parts;    // [splits][n_out]
    bool out_by_four;
    __host__ __device__ int begin(int s) const { return s * each + (s < more ? s : more); }
};

// WJ waves lie along the outputs, 4 / WJ along the inputs: a tile of 64 WJ outputs and 128 inputs.  H = 2: twice as many, and of a
// stage's four steps of 16 rows each half takes two, so that two waves share a matrix unit, one making parts while the other
// multiplies.  H = 1: two workgroups on a unit do the same for each other, where tiles are that many; float32 gradients then need 6
// to 11 registers more than the 256 that a lane has, which go to memory and back in every stage
template <int WJ, int H>
struct GradTile {
    static constexpr int HALF = 4, WAVES = H * HALF, THREADS = 64 * WAVES, WE = HALF / WJ, ROWS = kWaveRows * WJ, TE = kCols / WE / 32;   // TE: tiles of 32 inputs of a wave
    static constexpr int OUT = 2 / H, GROUPS = OUT * TE * 4;                              // outputs of a pair and groups of four results that a lane ends with
    static constexpr int STEPS = kDepth / 16 / H;                                         // of a wave in a stage
    static constexpr int CODED = kDepth * kCols / 4 / THREADS;                            // rows of codes of a thread in a stage
};

// Group q of a lane's results: adjacent inputs e .. e + 3 of output j, within the workgroup's tile
template <int WJ, int H>
__device__ __forceinline__ void place_of(int wave, int lane, int q, int *j, int *e)
{
    typedef GradTile<WJ, H> T;
    const int wj = wave % T::HALF / T::WE, we = wave % T::WE, part = q & 3, et = (q >> 2) % T::TE, jt = (q >> 2) / T::TE;
    *j = wj * kWaveRows + 2 * (lane & 31) + (H == 2 ? wave / T::HALF : jt);
    *e = (we * T::TE + et) * 32 + 8 * part + 4 * (lane >> 5);
}

__device__ __forceinline__ void store_group(const GradArgs &a, int j, int e, floatx4 v)
{
    if (j >= a.n_out || e >= a.n_in) return;
    float *to = a.grad_weight + (int64_t)j * a.n_in + e;
    if (a.out_by_four) {
        floatx4 *p = reinterpret_cast<floatx4 *>(to);
        *p = a.accumulate ? *p + v : v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e + i < a.n_in) to[i] = a.accumulate ? to[i] + v[i] : v[i];
    }
}

// Eight adjacent rows of two adjacent outputs, as they lie in memory
template <int DTYPE>
struct RawPair {
    floatx2 v[8];
};
template <>
struct RawPair<LMKAN_F16> {
    uint32_t v[8];
};
template <>
struct RawPair<LMKAN_BF16> {
    uint32_t v[8];
};
template <int DTYPE>
constexpr int parts_of() { return DTYPE == LMKAN_F32 ? 3 : DTYPE == LMKAN_F16 ? 2 : 1; }

// the upper halves of two words, `a` in the lower half
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t bits(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float cut(float v) { return __builtin_bit_cast(float, bits(v) & 0xffff0000u); }

// Eight values to parts of bfloat16, of 8 bits each, cut off one after the other: their sum is the value, exactly
template <int N>
__device__ __forceinline__ void to_parts(const float (&v)[8], bf16x8 (&to)[N])
{
    uint32_t w[N][4];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        float a = v[i], b = v[i + 1];
#pragma unroll
        for (int p = 0; p < N; ++p) {
            w[p][i / 2] = upper_halves(bits(a), bits(b));
            if (p + 1 < N) a -= cut(a), b -= cut(b);
        }
    }
#pragma unroll
    for (int p = 0; p < N; ++p) to[p] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const intx4 *>(w[p]));
}

// Those of output t (0 or 1) of a pair
template <int DTYPE>
__device__ __forceinline__ float value_in(const RawPair<DTYPE> &r, int i, int t)
{
    if constexpr (DTYPE == LMKAN_F32) return r.v[i][t];
    else if constexpr (DTYPE == LMKAN_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)(r.v[i] >> (16 * t)));
    else return __builtin_bit_cast(float, t ? r.v[i] & 0xffff0000u : r.v[i] << 16);
}
template <int DTYPE>
__device__ __forceinline__ float sum_of(const RawPair<DTYPE> &r, int t)
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = value_in(r, i, t);
    return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}
template <int DTYPE, int N>
__device__ __forceinline__ void to_parts(const RawPair<DTYPE> &r, bf16x8 (&to)[2][N])
{
    if constexpr (DTYPE == LMKAN_BF16) {
        intx4 w[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[0][i] = (int)__builtin_amdgcn_perm(r.v[2 * i + 1], r.v[2 * i], 0x05040100u);
            w[1][i] = (int)upper_halves(r.v[2 * i], r.v[2 * i + 1]);
        }
        to[0][0] = __builtin_bit_cast(bf16x8, w[0]), to[1][0] = __builtin_bit_cast(bf16x8, w[1]);
    } else {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = value_in(r, i, t);
            to_parts(v, to[t]);
        }
    }
}

// max(., 0) of four codes (a block that stands for NaN has codes of zero and a scale of NaN)
__device__ __forceinline__ uint32_t positive_codes(uint32_t four)
{
    const uint32_t sign = four & 0x80808080u;
    return four & ~(sign | (sign - (sign >> 7)));
}

// Reads of `bytes` of memory: beyond its end, and everywhere where `bytes` is negative, they give zero
struct Buffer {
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ Buffer(const char *p, int bytes)
        : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p), 0, bytes > 0 ? bytes : 0, 0x00027000))
    {
    }
    __device__ __forceinline__ uint32_t word(unsigned at) const { return __builtin_amdgcn_raw_buffer_load_b32(rsrc, at, 0, 0); }
    __device__ __forceinline__ uint32_t half(unsigned at) const { return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rsrc, at, 0, 0); }
    __device__ __forceinline__ uint32_t byte(unsigned at) const { return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(rsrc, at, 0, 0); }
    __device__ __forceinline__ floatx2 two_floats(unsigned at) const
    {
        return __builtin_bit_cast(floatx2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, 0, 0));
    }
};

// The rows of one matrix, stage by stage: 64 rows take at most 2^30 + 2^11 bytes
struct Stages {
    const char *base;
    int64_t left;   // bytes
    int pitch;
    __device__ __forceinline__ Stages(const void *p, int64_t batch, int bytes, int stage)
        : base(static_cast<const char *>(p) + (int64_t)stage * kDepth * bytes), left((batch - (int64_t)stage * kDepth) * bytes), pitch(bytes)
    {
    }
    __device__ __forceinline__ void next()
    {
        base += (int64_t)(kDepth * pitch), left -= (int64_t)(kDepth * pitch);
    }
    // rows from `row` of the stage on
    __device__ __forceinline__ Buffer at(int row) const
    {
        const int most = left < 0x7fffffff ? (int)left : 0x7fffffff;
        return Buffer(base + row * pitch, most - row * pitch);
    }
};

// How pairs of 16-bit gradients and fours of codes are read: as words (at any address, but then inside the matrix: at its end
// a word may be there in part), or element by element
enum Reads { kWords, kElements };

// ALIGNED: pairs of 16-bit outputs and fours of codes lie at multiples of their size
template <int DTYPE, int WJ, int H, bool ALIGNED>
__global__ __launch_bounds__((GradTile<WJ, H>::THREADS), H == 1 ? 2 : 1) void linear_grad_kernel(GradArgs a)
{
    typedef GradTile<WJ, H> T;
    constexpr int P = parts_of<DTYPE>();
    constexpr int kSteps = T::STEPS, AHEAD = 2;   // AHEAD: steps whose gradients are under way
    __shared__ __align__(16) char lds[2 * kStageBytes + 2 * kScaleFloats * (int)sizeof(float)];
    const int tiles = a.down * a.across, total = tiles * a.splits;
    const int id = a.first + (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);   // (workgroups on one die: adjacent tiles of the same rows)
    if (id >= total) return;
    const int split = id / tiles, tile = id - split * tiles;
    int ti, tj;
    grouped_tile(tile, a.down, a.across, &ti, &tj);
    const int j0 = ti * T::ROWS, e0 = tj * kCols;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = wave / T::HALF, wj = wave % T::HALF / T::WE, we = wave % T::WE;
    const int from = a.begin(split), to = a.begin(split + 1);

    // Gradients: outputs j, j + 1, rows 8 (lane / 32) on of every 16.  What lies beyond the last row reads as zero; what lies
    // beyond the last column belongs to results that are dropped.
    constexpr unsigned kSize = DTYPE == LMKAN_F32 ? 4 : 2;
    const int j = j0 + wj * kWaveRows + 2 * (lane & 31);
    const int pitch = a.n_out * (int)kSize;
    const unsigned at = (unsigned)(lane >> 5) * 8 * (unsigned)pitch + (unsigned)j * kSize;
    const auto load_pair = [&](auto reads, const Stages &rows, int step) {
        constexpr Reads kReads = decltype(reads)::value;
        RawPair<DTYPE> r;
        const Buffer b = rows.at(16 * step);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned to = at + i * (unsigned)pitch;
            if constexpr (DTYPE == LMKAN_F32) r.v[i] = b.two_floats(to);
            else r.v[i] = kReads == kWords ? b.word(to) : b.half(to) | b.half(to + 2) << 16;
        }
        return r;
    };

    // codes: inputs e .. e + 3, some adjacent rows of a stage
    const int per_row = exp_blocks(a.n_in);
    const int row0 = (threadIdx.x >> 5) * T::CODED, ec = 4 * (threadIdx.x & 31), e = e0 + ec;
    struct Codes {
        uint32_t v[T::CODED];
    };
    const auto load_codes = [&](auto reads, const Stages &rows) {
        constexpr Reads kReads = decltype(reads)::value;
        Codes c;
        const Buffer b = rows.at(0);
#pragma unroll
        for (int i = 0; i < T::CODED; ++i) {
            const unsigned f = (unsigned)(row0 + i) * (unsigned)a.n_in + (unsigned)e;
            c.v[i] = kReads == kWords ? b.word(f) : b.byte(f) | b.byte(f + 1) << 8 | b.byte(f + 2) << 16 | b.byte(f + 3) << 24;
        }
        return c;
    };
    const auto rectified = [&](Codes c) {
        if (a.relu)
#pragma unroll
            for (int i = 0; i < T::CODED; ++i) c.v[i] = positive_codes(c.v[i]);
        return c;
    };
    // powers of two: a row and a block of inputs a thread, for all threads in LDS [block][row]
    float *const scales = reinterpret_cast<float *>(lds + 2 * kStageBytes);
    const bool scaling = threadIdx.x < kDepth * 4;
    const auto load_exp = [&](const Stages &rows) {
        return scaling ? rows.at(0).byte((threadIdx.x >> 2) * (unsigned)per_row + (unsigned)e0 / kBlock + (threadIdx.x & 3)) : 0;
    };
    const auto store_scale = [&](uint32_t byte, float *to) {
        if (scaling) to[(threadIdx.x & 3) * kScalePitch + (threadIdx.x >> 2)] = value_of(1, (int)byte);
    };
    // column k of a thread's codes, as bfloat16
    const auto store_column = [&](const Codes &c, int k, const float *scale, char *buffer) {
        float v[T::CODED], by[T::CODED];
#pragma unroll
        for (int i = 0; i < T::CODED; i += 4)
            *reinterpret_cast<floatx4 *>(by + i) = *reinterpret_cast<const floatx4 *>(scale + (ec / kBlock) * kScalePitch + row0 + i);
#pragma unroll
        for (int i = 0; i < T::CODED; ++i) v[i] = (float)(int8_t)(c.v[i] >> (8 * k)) * by[i];
        uint32_t w[T::CODED / 2];
#pragma unroll
        for (int i = 0; i < T::CODED / 2; ++i) w[i] = upper_halves(bits(v[2 * i]), bits(v[2 * i + 1]));
        char *to = buffer + (ec + k) * kLine + grad_slot(ec + k, row0 / 8) * 16 + row0 % 8 * 2;
        if constexpr (T::CODED == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
    };

    const auto load_fragments = [&](const char *buffer, int step, bf16x8 (&v)[T::TE]) {
#pragma unroll
        for (int k = 0; k < T::TE; ++k) {
            const int row = (we * T::TE + k) * 32 + (lane & 31);
            v[k] = *reinterpret_cast<const bf16x8 *>(buffer + row * kLine + grad_slot(row, 2 * step + (lane >> 5)) * 16);
        }
    };

    floatx16 acc[2][T::TE];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int k = 0; k < T::TE; ++k) acc[t][k] = floatx16{};
    const bool with_bias = a.grad_bias && tj == 0 && we == 0;
    double bias[2] = {};
    const auto run = [&](int from, int to) {
        if (from >= to) return;
        const auto reads = std::integral_constant<Reads, kWords>();
        // (powers of two are read two stages ahead, as zeros beyond the last row; what else would be beyond the last stage is that
        // stage again, and not used)
        Stages rows(a.grad_y, a.batch, pitch, from), codes(a.codes, a.batch, a.n_in, from), exps(a.exps, a.batch, per_row, from);
        // (loads in the order in which the loop leaves them under way: a wait counts back from the last one)
        Codes first = load_codes(reads, codes);
        const uint32_t byte0 = load_exp(exps);
        exps.next();
        const uint32_t byte1 = load_exp(exps);
        if (from + 1 < to) codes.next();
        Codes c = load_codes(reads, codes);
        __builtin_amdgcn_sched_barrier(0);
        RawPair<DTYPE> raw[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) raw[k] = load_pair(reads, rows, kSteps * half + k);
        __builtin_amdgcn_sched_barrier(0);
        store_scale(byte0, scales);
        store_scale(byte1, scales + kScaleFloats);
        first = rectified(first);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) store_column(first, k, scales, lds);
        __syncthreads();
        for (int s = from; s < to; ++s) {
            const int now = s - from & 1;
            const char *buffer = lds + now * kStageBytes;
            exps.next();
            if (s + 2 < to) codes.next();
            Stages ahead = rows;
            if (s + 1 < to) ahead.next();
            const Codes later = load_codes(reads, codes);
            c = rectified(c);
            const uint32_t byte = load_exp(exps);
            bf16x8 v[T::TE];
            load_fragments(buffer, kSteps * half, v);
#pragma unroll
            for (int step = 0; step < kSteps; ++step) {
                bf16x8 g[2][P];
                to_parts(raw[step % AHEAD], g);
                if (with_bias)
#pragma unroll
                    for (int t = 0; t < 2; ++t) bias[t] += (double)sum_of(raw[step % AHEAD], t);
                raw[step % AHEAD] = load_pair(reads, step + AHEAD < kSteps ? rows : ahead, kSteps * half + (step + AHEAD) % kSteps);
#pragma unroll
                for (int k = 0; k < 4 / kSteps; ++k)
                    store_column(c, 4 / kSteps * step + k, scales + (now ^ 1) * kScaleFloats, lds + (now ^ 1) * kStageBytes);
                bf16x8 then[T::TE];
                if (step + 1 < kSteps) load_fragments(buffer, kSteps * half + step + 1, then);
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
#pragma unroll
                    for (int k = 0; k < T::TE; ++k)
#pragma unroll
                        for (int t = 0; t < 2; ++t) acc[t][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[k], g[t][p], acc[t][k], 0, 0, 0);
                if (step + 1 < kSteps)
#pragma unroll
                    for (int k = 0; k < T::TE; ++k) v[k] = then[k];
            }
            rows = ahead;
            c = later;
            store_scale(byte, scales + now * kScaleFloats);
            __syncthreads();
        }
    };
    // the last stages, one thing after the other
    const auto run_elements = [&](int from, int to) {
        const auto reads = std::integral_constant<Reads, kElements>();
        for (int s = from; s < to; ++s) {
            const Stages rows(a.grad_y, a.batch, pitch, s);
            store_scale(load_exp(Stages(a.exps, a.batch, per_row, s)), scales);
            __syncthreads();
            const Codes c = rectified(load_codes(reads, Stages(a.codes, a.batch, a.n_in, s)));
#pragma unroll
            for (int k = 0; k < 4; ++k) store_column(c, k, scales, lds);
            __syncthreads();
#pragma unroll 1
            for (int step = kSteps * half; step < kSteps * (half + 1); ++step) {
                const RawPair<DTYPE> raw = load_pair(reads, rows, step);
                bf16x8 g[2][P], v[T::TE];
                to_parts(raw, g);
                if (with_bias)
#pragma unroll
                    for (int t = 0; t < 2; ++t) bias[t] += (double)sum_of(raw, t);
                load_fragments(lds, step, v);
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
#pragma unroll
                    for (int k = 0; k < T::TE; ++k)
#pragma unroll
                        for (int t = 0; t < 2; ++t) acc[t][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[k], g[t][p], acc[t][k], 0, 0, 0);
            }
            __syncthreads();
        }
    };
    if constexpr (ALIGNED) {
        run(from, to);
    } else {
        // stages whose reads of whole tiles stay inside both matrices
        const auto inside = [&](int bytes, int past) {
            const int64_t rows = a.batch - (past + bytes - 1) / bytes;
            return rows > 0 ? (int)(rows / kDepth) : 0;
        };
        const int both = min(inside(pitch, 2 * T::ROWS + 4), inside(a.n_in, kCols + 4)), middle = both < from ? from : both < to ? both : to;
        run(from, middle);
        run_elements(middle, to);
    }
    // the halves' sums: each ends with one output of a pair, and gives the other
    floatx16 sum[T::OUT][T::TE];
    if constexpr (H == 1) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < T::TE; ++k) sum[t][k] = acc[t][k];
    } else {
        floatx4 *const given = reinterpret_cast<floatx4 *>(lds);
        static_assert(T::WAVES * 64 * 16 * (int)sizeof(float) <= 2 * kStageBytes, "");
#pragma unroll
        for (int k = 0; k < T::TE; ++k) {
            sum[0][k] = half ? acc[1][k] : acc[0][k];
            const floatx16 give = half ? acc[0][k] : acc[1][k];
            __syncthreads();
#pragma unroll
            for (int p = 0; p < 4; ++p) given[(wave * 4 + p) * 64 + lane] = floatx4{give[4 * p], give[4 * p + 1], give[4 * p + 2], give[4 * p + 3]};
            __syncthreads();
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const floatx4 v = given[((wave ^ T::HALF) * 4 + p) * 64 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[0][k][4 * p + i] += v[i];
            }
        }
    }
    if (a.grad_bias && tj == 0) {
        double *const halves = reinterpret_cast<double *>(lds);
#pragma unroll
        for (int t = 0; t < 2; ++t) bias[t] += __shfl_xor(bias[t], 32, 64);
        if constexpr (H == 2) {
            __syncthreads();
#pragma unroll
            for (int t = 0; t < 2; ++t)
                if (half && with_bias && lane < 32) halves[(wj * 2 + t) * 32 + lane] = bias[t];
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if (!half && with_bias && lane < 32 && j + t < a.n_out) {
                const double both = H == 2 ? bias[t] + halves[(wj * 2 + t) * 32 + lane] : bias[t];
                if (a.parts) a.bias_parts[(int64_t)split * a.n_out + j + t] = both;
                else a.grad_bias[j + t] = a.accumulate ? a.grad_bias[j + t] + (float)both : (float)both;
            }
    }
#pragma unroll
    for (int q = 0; q < T::GROUPS; ++q) {
        const floatx16 &t = sum[(q >> 2) / T::TE][(q >> 2) % T::TE];
        const floatx4 v = {t[4 * (q & 3)], t[4 * (q & 3) + 1], t[4 * (q & 3) + 2], t[4 * (q & 3) + 3]};
        if (H == 2 && a.parts) {
            a.parts[(((int64_t)split * tiles + tile) * T::WAVES + wave) * (T::GROUPS * 64) + q * 64 + lane] = v;
        } else {
            int jo, eo;
            place_of<WJ, H>(wave, lane, q, &jo, &eo);
            store_group(a, j0 + jo, e0 + eo, v);
        }
    }
}

// The sums of 64 groups' parts a workgroup: a wave takes every fourth split, and the waves' sums meet in LDS
template <int WJ>
__global__ __launch_bounds__(256) void linear_grad_join_kernel(GradArgs a)
{
    typedef GradTile<WJ, 2> T;
    __shared__ floatx4 sums[3][64];
    __shared__ double bias_sums[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t groups = (int64_t)a.down * a.across * T::WAVES * T::GROUPS * 64, i = (int64_t)blockIdx.x * 64 + lane;
    const bool biased = a.grad_bias && i < a.n_out;
    floatx4 sum = {0, 0, 0, 0};
    double bias = 0.0;
#pragma unroll 8
    for (int s = wave; s < a.splits; s += 4) sum += a.parts[s * groups + i];
    if (biased)
#pragma unroll 8
        for (int s = wave; s < a.splits; s += 4) bias += a.bias_parts[(int64_t)s * a.n_out + i];
    if (wave > 0) sums[wave - 1][lane] = sum, bias_sums[wave - 1][lane] = bias;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w) sum += sums[w][lane], bias += bias_sums[w][lane];
    const int tile = (int)(blockIdx.x / (T::WAVES * T::GROUPS)), rest = (int)(blockIdx.x % (T::WAVES * T::GROUPS));
    int ti, tj, j, e;
    grouped_tile(tile, a.down, a.across, &ti, &tj);
    place_of<WJ, 2>(rest / T::GROUPS, lane, rest % T::GROUPS, &j, &e);
    store_group(a, ti * T::ROWS + j, tj * kCols + e, sum);
    if (biased) a.grad_bias[i] = a.accumulate ? a.grad_bias[i] + (float)bias : (float)bias;
}

// ---- host ------------------------------------------------------------------------------------------------------------

constexpr int kUnits = 256;   // compute units

struct Plan {
    int wj, halves, down, across, splits, stages;
};

// Workgroups that a unit takes one after the other
int64_t turns_of(int64_t workgroups) { return (workgroups + kUnits - 1) / kUnits; }

// Tile and splits by what a call takes in us: stages of a workgroup, fitted to 18 shapes, one and a half of them to begin with, and
// parts, which are written and joined.  Workgroups of two halves have a unit for themselves; of one half two are on a unit, which
// takes that many tiles without splits.  Measured (us, as chosen / next other tile / next other number of splits): 8192 rows of
// 1024 -> 1024 float32 62 / 71 / 73; 5000 of 500 -> 333 25 / 24 / 26; 65536 of 128 -> 128 21 / 22 / 23; 20000 of 1000 -> 1000 bfloat16
// 61 / 78 / 72; 1000 of 100 -> 4000 float32 18 / 19 / 20.  Halves (one / two): 4096 of 4096 -> 4096 bfloat16 150 / 167, 16384 of
// 4096 -> 4096 float32 1300 / 1353, 64 of 4096 -> 4096 20 / 28, 8192 of 1024 -> 1024 72 / 62.
// Calls f(plan, cost) with every tile and number of splits that is considered.
template <class F>
void candidates(const LinearShape &s, F &&f)
{
    const int stages = (int)((s.batch + kDepth - 1) / kDepth);
    const int parts = s.y_dtype == LMKAN_F32 ? 3 : s.y_dtype == LMKAN_F16 ? 2 : 1;
    for (int wj = 4; wj >= 1; wj /= 2) {
        const int down = (s.n_out + kWaveRows * wj - 1) / (kWaveRows * wj), across = (s.n_in + kCols - 1) / kCols;
        const int64_t tiles = (int64_t)down * across;
        if (wj == 4 && tiles > kUnits) {
            const int64_t turns = turns_of(tiles);
            const double cost = ((turns / 2) * (0.75 + 1.43 * parts) + (turns % 2) * (0.4 + 1.1 * parts)) * (stages + 1.5);
            f(Plan{wj, 1, down, across, 1, stages}, cost);
        }
        const double stage = wj == 4 ? 0.72 + 0.71 * parts : wj == 2 ? 0.43 + 0.47 * parts : 0.75 + 0.27 * parts;
        for (int splits = 1; splits <= 512 && splits <= (stages > 0 ? stages : 1); splits *= 2) {
            if (splits > 1 && tiles * splits > 4 * kUnits) break;
            const double bytes = (double)tiles * splits * wj * kWaveRows * kCols * sizeof(float);
            const double cost = turns_of(tiles * splits) * ((stages + splits - 1) / splits + 1.5) * stage + (splits > 1 ? 3.0 + bytes / 3.5e6 : 0.0);
            f(Plan{wj, 2, down, across, splits, stages}, cost);
        }
    }
}

Plan plan_of(const LinearShape &s)
{
    Plan best = {};
    double least = 1e300;
    candidates(s, [&](const Plan &p, double cost) {
        if (cost < least) least = cost, best = p;
    });
    return best;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

size_t parts_bytes(const Plan &p) { return align256((size_t)p.splits * p.down * p.across * p.wj * kWaveRows * kCols * sizeof(float)); }

size_t plan_bytes(const LinearShape &s, const Plan &p)
{
    return p.splits > 1 ? parts_bytes(p) + align256((size_t)p.splits * s.n_out * sizeof(double)) : 0;
}

// (two float32 need no more than their own alignment)
bool whole_shape(const LinearShape &s) { return (s.y_dtype == LMKAN_F32 || s.n_out % 2 == 0) && s.n_in % 4 == 0; }

template <int DTYPE, int WJ, int H>
void launch(GradArgs a, bool whole, hipStream_t stream)
{
    typedef GradTile<WJ, H> T;
    const int64_t total = (int64_t)a.down * a.across * a.splits;
    for (int64_t first = 0; first < total; first += kMostGroups) {
        const unsigned groups = (unsigned)((total - first < kMostGroups ? total - first : kMostGroups) + 7) / 8 * 8;
        a.first = (int)first;
        if (whole) linear_grad_kernel<DTYPE, WJ, H, true><<<groups, T::THREADS, 0, stream>>>(a);
        else linear_grad_kernel<DTYPE, WJ, H, false><<<groups, T::THREADS, 0, stream>>>(a);
    }
    if (!a.parts) return;
    // (a group of the join for every four results of the tiles, which are at least as many as the outputs)
    if constexpr (H == 2) linear_grad_join_kernel<WJ><<<(unsigned)(a.down * a.across * T::WAVES * T::GROUPS), 256, 0, stream>>>(a);
}

template <int DTYPE>
void launch_type(const Plan &p, const GradArgs &a, bool whole, hipStream_t stream)
{
    if (p.halves == 1) launch<DTYPE, 4, 1>(a, whole, stream);
    else if (p.wj == 4) launch<DTYPE, 4, 2>(a, whole, stream);
    else if (p.wj == 2) launch<DTYPE, 2, 2>(a, whole, stream);
    else launch<DTYPE, 1, 2>(a, whole, stream);
}

bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace

size_t linear_grad_workspace_bytes(const LinearShape &s) { return plan_bytes(s, plan_of(s)); }

// The most that this and any smaller batch needs.  A smaller one considers no plan that this one does not; of those that cut the
// batch none is taken that has more splits than another of its tile but no fewer turns a split (s = m s' splits with
// turns(s) >= m turns(s') take ceil(n / s) turns(s) >= ceil(n / s') turns(s') for any n stages, and have more parts).
size_t linear_grad_workspace_most(const LinearShape &s)
{
    size_t most = 0;
    candidates(s, [&](const Plan &p, double) {
        const int64_t tiles = (int64_t)p.down * p.across;
        for (int fewer = 1; fewer < p.splits; fewer *= 2)
            if (turns_of(tiles * p.splits) >= p.splits / fewer * turns_of(tiles * fewer)) return;
        const size_t bytes = plan_bytes(s, p);
        if (bytes > most) most = bytes;
    });
    return most;
}

void launch_linear_grad(const LinearShape &s, bool accumulate, const int8_t *codes, const uint8_t *exps, const void *grad_y,
                        float *grad_weight, float *grad_bias, void *workspace, hipStream_t stream)
{
    const bool whole = whole_shape(s) && aligned_to(grad_y, 4) && aligned_to(codes, 4);
    const Plan p = plan_of(s);
    GradArgs a{s.batch, s.n_in, s.n_out, s.relu, accumulate, codes, exps, grad_y, grad_weight, grad_bias, p.down, p.across, 0, p.splits, p.stages,
               p.stages / p.splits, p.stages % p.splits, nullptr, nullptr, s.n_in % 4 == 0 && aligned_to(grad_weight, 16)};
    if (p.splits > 1) {
        a.parts = static_cast<floatx4 *>(workspace);
        a.bias_parts = reinterpret_cast<double *>(static_cast<char *>(workspace) + parts_bytes(p));
    }
    if (s.y_dtype == LMKAN_F32) launch_type<LMKAN_F32>(p, a, whole, stream);
    else if (s.y_dtype == LMKAN_F16) launch_type<LMKAN_F16>(p, a, whole, stream);
    else launch_type<LMKAN_BF16>(p, a, whole, stream);
}

}  // namespace lmkan
