// The linear term in 8-bit whole numbers: rows scaled to codes one by one, products of codes summed exactly,
//   y = beta y + xscale wscale sum(xcode wcode) + bias.
//
// quantize_kernel reads rows once and writes codes and scales; linear_kernel multiplies tiles of codes on the matrix
// cores (lmkan_tile.h), few tiles with a long summed axis cut along it and joined.  Calls of few rows are bound by
// launches and by reading the weights: one_row_kernel and some_rows_kernel (up to 64 short rows) take one launch, in
// which every workgroup scales the rows for itself while its weights are on their way.
#include "lmkan_dense.h"

#include "lmkan_kernels.h"
#include "lmkan_tile.h"

namespace lmkan {

namespace {

// ---- rows to codes ---------------------------------------------------------------------------------------------------

// What scales a row to codes, and the codes back: from the bits of its largest magnitude (ordered like the values for
// non-negative floats, NaN above infinity).  A row with a NaN or an infinity ends with a scale that is not finite.
struct RowScale {
    float factor, scale;
    bool finite;
    __device__ __forceinline__ explicit RowScale(uint32_t top)
    {
        const float r = __builtin_bit_cast(float, top), f = 127.0f / r;
        finite = top < 0x7f800000u;
        factor = finite && f < __builtin_inff() ? f : 0.0f;
        scale = r / 127.0f;
    }
    __device__ __forceinline__ int code(float v) const { return finite ? (int)rintf(v * factor) : 0; }
};

// A sum of codes to the term.  (The sum first: the product of both scales may lie below float32's range where the term
// does not; rows may have any magnitude, the scale of an output is that of weights)
__device__ __forceinline__ float scaled(int sum, float w_scale, float x_scale) { return (float)sum * w_scale * x_scale; }

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ float rectified(float v, bool relu) { return relu && v < 0.0f ? 0.0f : v; }

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = larger(v, (uint32_t)__shfl_xor((int)v, d, 64));
    return v;
}

__device__ __forceinline__ uint32_t packed(const int (&c)[4])
{
    return (uint32_t)(c[0] & 255) | (uint32_t)(c[1] & 255) << 8 | (uint32_t)(c[2] & 255) << 16 | (uint32_t)(c[3] & 255) << 24;
}

// four adjacent elements; `whole`: they exist and are aligned to their size together
template <int DTYPE>
__device__ __forceinline__ void load_four(const void *x, int64_t at, int left, bool whole, float (&v)[4])
{
    if (whole) {
        if (DTYPE == LMKAN_F32) {
            const float4 f = *reinterpret_cast<const float4 *>(static_cast<const float *>(x) + at);
            v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
        } else {
            const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(x) + at);
            const uint16_t b[4] = {(uint16_t)u.x, (uint16_t)(u.x >> 16), (uint16_t)u.y, (uint16_t)(u.y >> 16)};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = load_as_float(b, e, DTYPE);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < left ? load_as_float(x, at + e, DTYPE) : 0.0f;
    }
}

// Weights whose rows are not a multiple of 16 bytes, or start anywhere, to rows that are; a dword a thread
struct AlignArgs {
    const int8_t *w;
    int n_in, n_out, pitch;
    int8_t *to;
    int64_t first;   // block of the launch's first
};
__device__ __forceinline__ void align_rows(const AlignArgs &a, unsigned block)
{
    const int64_t e = (a.first + block) * 256 + threadIdx.x;
    const int64_t row = e / (a.pitch / 4);
    const int k = (int)(e - row * (a.pitch / 4)) * 4;
    if (row >= a.n_out) return;
    int c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = k + i < a.n_in ? a.w[row * a.n_in + k + i] : 0;
    *reinterpret_cast<uint32_t *>(a.to + row * a.pitch + k) = packed(c);
}

constexpr int kHeld = 8;   // fours of a row that a thread keeps; longer rows are read again (from the L2)

struct QuantizeArgs {
    int64_t rows;
    int cols, pitch;   // pitch: bytes from one row of codes to the next; what lies between is zeroed when `pad`
    bool relu, pad, by_four, codes_by_four;
    const void *x;
    int8_t *codes;
    float *scale;
    unsigned row_blocks;
    AlignArgs align;   // the workgroups beyond row_blocks
};

// LANES threads a row (a wave, or a workgroup of 256)
template <int DTYPE, int LANES>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs a)
{
    __shared__ uint32_t tops[4];
    if (blockIdx.x >= a.row_blocks) return align_rows(a.align, blockIdx.x - a.row_blocks);
    const int64_t row = LANES == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (LANES == 64 && row >= a.rows) return;
    const int t = LANES == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int fours = (a.cols + 3) / 4;
    float v[kHeld][4];
    uint32_t top = 0;
    const auto load = [&](int f, float (&to)[4]) {
        const int left = a.cols - 4 * f;
        load_four<DTYPE>(a.x, row * a.cols + 4 * f, left, a.by_four && left >= 4, to);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = rectified(to[e], a.relu);
    };
    const auto see = [&](const float (&from)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) top = larger(top, magnitude(from[e]));
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
        if (t + h * LANES < fours) load(t + h * LANES, v[h]);
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
        if (t + h * LANES < fours) see(v[h]);
    for (int f = t + kHeld * LANES; f < fours; f += LANES) {
        float w[4];
        load(f, w);
        see(w);
    }
    top = wave_max(top);
    if (LANES == 256) {
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
        top = larger(larger(tops[0], tops[1]), larger(tops[2], tops[3]));
    }
    const RowScale s(top);
    int8_t *to = a.codes + row * a.pitch;
    const auto store = [&](int f, const float (&from)[4]) {
        int c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = s.code(from[e]);
        if (a.codes_by_four) {
            *reinterpret_cast<uint32_t *>(to + 4 * f) = packed(c);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (4 * f + e < a.cols) to[4 * f + e] = (int8_t)c[e];
        }
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h)
        if (t + h * LANES < fours) store(t + h * LANES, v[h]);
    for (int f = t + kHeld * LANES; f < fours; f += LANES) {
        float w[4];
        load(f, w);
        store(f, w);
    }
    if (a.pad)
        for (int f = fours + t; f < a.pitch / 4; f += LANES) *reinterpret_cast<uint32_t *>(to + 4 * f) = 0;
    if (t == 0) a.scale[row] = s.scale;
}

// ---- products of tiles -----------------------------------------------------------------------------------------------

constexpr int kPitch = 36;                                // floats of a row of a wave's tile in LDS
constexpr int kWaveScratch = 32 * kPitch * (int)sizeof(float);

struct LinearArgs {
    const int8_t *x, *w;       // codes
    int64_t x_pitch, w_pitch;
    const float *x_scale, *w_scale, *bias;
    float beta;
    void *y;
    int64_t batch;
    int n_in, n_out, y_dtype;
    bool by_four;              // rows of y take accesses of four elements
    int tiles_down, tiles_across;
    WorkSplit work;
    intx4 *parts;
};

template <class T>
__device__ __forceinline__ void finish_tile(const LinearArgs &a, int tile, const intx4 (&acc)[T::CT][T::RT], char *scratch, int wave)
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // (the addresses below are worked out here, not kept in registers through the main loop)
    const int r = lane & 15, q = lane >> 4;
    int ti, tj;
    grouped_tile(tile, a.tiles_down, a.tiles_across, &ti, &tj);
    const int64_t i0 = (int64_t)ti * T::ROWS;
    const int j0 = tj * T::COLS;
    // what a lane finishes of a 32 x 32 tile, after the tile went through LDS: rows 8 t + lane / 8, four columns
    const int fr = lane >> 3, fc = (lane & 7) * 4;
    struct Held {
        floatx4 y[4];   // of 16-bit elements: two words
        float scale[4];
    };
    // (rows and columns beyond the end: others are loaded, and not used)
    const auto ahead = [&](int row, int col) {
        Held h;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            int64_t i = i0 + row + 8 * t + fr;
            i = i < a.batch ? i : a.batch - 1;
            h.scale[t] = a.x_scale[i];
            if (a.by_four && a.beta != 0.0f) {
                const int64_t at = i * a.n_out + min(j0 + col + fc, a.n_out - 4);
                if (a.y_dtype == LMKAN_F32) {
                    h.y[t] = *reinterpret_cast<const floatx4 *>(static_cast<const float *>(a.y) + at);
                } else {
                    const uint2 u = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(a.y) + at);
                    h.y[t][0] = __builtin_bit_cast(float, u.x), h.y[t][1] = __builtin_bit_cast(float, u.y);
                }
            }
        }
        return h;
    };
    for_wave_tiles<T>(acc, wave, ahead, [&](int row, int col, const intx4 (&v)[4], const Held &held) {
        if (i0 + row >= a.batch || j0 + col >= a.n_out) return;
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<intx4 *>(scratch + ((16 * (g >> 1) + r) * kPitch + 16 * (g & 1) + 4 * q) * 4) = v[g];
        if (a.by_four) {
            const int j = j0 + col + fc, seen = min(j, a.n_out - 4);
            const floatx4 zero = {0, 0, 0, 0};
            floatx4 ws, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) ws[e] = a.w_scale[seen + e];
            b = zero;
            if (a.bias)
#pragma unroll
                for (int e = 0; e < 4; ++e) b[e] = a.bias[seen + e];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int64_t i = i0 + row + 8 * t + fr;
                const intx4 sum = *reinterpret_cast<const intx4 *>(scratch + ((8 * t + fr) * kPitch + fc) * 4);
                if (i >= a.batch || j >= a.n_out) continue;
                const int64_t at = i * a.n_out + j;
                floatx4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = scaled(sum[e], ws[e], held.scale[t]) + b[e];
                if (a.y_dtype == LMKAN_F32) {
                    if (a.beta != 0.0f) o += a.beta * held.y[t];
                    *reinterpret_cast<floatx4 *>(static_cast<float *>(a.y) + at) = o;
                } else {
                    if (a.beta != 0.0f) {
                        const uint32_t u[2] = {__builtin_bit_cast(uint32_t, (float)held.y[t][0]), __builtin_bit_cast(uint32_t, (float)held.y[t][1])};
                        const uint16_t h[4] = {(uint16_t)u[0], (uint16_t)(u[0] >> 16), (uint16_t)u[1], (uint16_t)(u[1] >> 16)};
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] += a.beta * load_as_float(h, e, a.y_dtype);
                    }
                    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.y) + at) =
                        make_uint2(two_from_float(a.y_dtype, o[0], o[1]), two_from_float(a.y_dtype, o[2], o[3]));
                }
            }
        } else {
            // element by element, 32 adjacent ones of two rows at a time
            const int j = j0 + col + (lane & 31);
            if (j >= a.n_out) return;
            const float ws = a.w_scale[j], b = a.bias ? a.bias[j] : 0.0f;
#pragma unroll 8
            for (int k = lane >> 5; k < 32; k += 2) {
                const int64_t i = i0 + row + k;
                if (i >= a.batch) break;
                const int sum = *reinterpret_cast<const int *>(scratch + (k * kPitch + (lane & 31)) * 4);
                float o = scaled(sum, ws, a.x_scale[i]) + b;
                if (a.beta != 0.0f) o += a.beta * load_as_float(a.y, i * a.n_out + j, a.y_dtype);
                store_from_float(a.y, i * a.n_out + j, a.y_dtype, o);
            }
        }
    });
}

template <class T>
__global__ __launch_bounds__(T::THREADS) void linear_kernel(LinearArgs a)
{
    extern __shared__ __align__(16) char lds[];
    for_work(a.work, blockIdx.x, [&](int tile, int from, int to, int slot) {
        int ti, tj;
        grouped_tile(tile, a.tiles_down, a.tiles_across, &ti, &tj);
        const int64_t i0 = (int64_t)uniform(ti) * T::ROWS;
        const int j0 = uniform(tj) * T::COLS;
        const int64_t last = a.batch - 1 - i0;
        const Operand x{reinterpret_cast<const char *>(uniform(a.x + i0 * a.x_pitch)), kLine, uniform((int)(last < T::ROWS ? last : T::ROWS)), false,
                        (unsigned)a.x_pitch, (int)a.x_pitch - 16};
        const Operand w{reinterpret_cast<const char *>(uniform(a.w + j0 * a.w_pitch)), kLine, uniform(a.n_out - 1 - j0), false, (unsigned)a.w_pitch,
                        (int)a.w_pitch - 16};
        intx4 acc[T::CT][T::RT];
        multiply<T, CodeProduct>(x, w, from, to, lds, acc);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (slot < 0) finish_tile<T>(a, tile, acc, lds + wave * kWaveScratch, wave);
        else store_part<T>(a.parts, slot, acc);
        __syncthreads();
    });
}

// A wave's share of a tile that was cut, a workgroup each
template <class T>
__global__ __launch_bounds__(64 * joiners<T>()) void linear_join_kernel(LinearArgs a)
{
    __shared__ __align__(16) char lds[kWaveScratch + join_lds<T>()];
    const int tile = blockIdx.x / T::WAVES, wave = blockIdx.x % T::WAVES;
    intx4 acc[T::CT][T::RT];
    if (!join_parts<T, joiners<T>()>(a.work, tile, wave, a.parts, reinterpret_cast<intx4 *>(lds + kWaveScratch), acc)) return;
    finish_tile<T>(a, a.work.whole + tile, acc, lds, wave);
}

// ---- one row ---------------------------------------------------------------------------------------------------------

constexpr int kRowHeld = 4;              // fours of the row that a thread keeps

struct RowsArgs {
    const void *x;
    const int8_t *w;
    const float *w_scale, *bias;
    float beta;
    void *y;
    int n_in, n_out, y_dtype;
    bool relu, w_aligned, x_by_four;
};

// 16 codes of a row from k on, zero beyond its end
__device__ __forceinline__ intx4 load_codes(const int8_t *row, int k, int n_in, bool aligned)
{
    if (k + 16 <= n_in) {
        if (aligned) return *reinterpret_cast<const intx4 *>(row + k);
        intx4 v;
        __builtin_memcpy(&v, row + k, 16);
        return v;
    }
    intx4 v = {0, 0, 0, 0};
    for (int e = 0; k + e < n_in; ++e) v[e >> 2] |= (int)((uint32_t)(uint8_t)row[k + e] << (8 * (e & 3)));
    return v;
}

// A wave takes OUTS outputs; CHUNKS pieces of 1024 codes of each are on their way at a time, the first before the row
// is scaled.  `padded`: n_in rounded up to pieces.
template <int DTYPE, int OUTS, int CHUNKS>
__global__ __launch_bounds__(256) void one_row_kernel(RowsArgs a, int padded)
{
    extern __shared__ __align__(16) char lds[];
    __shared__ uint32_t tops[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j0 = (blockIdx.x * 4 + wave) * OUTS;
    intx4 w[OUTS][CHUNKS];
    const auto fetch = [&](int k0) {
#pragma unroll
        for (int o = 0; o < OUTS; ++o)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int k = k0 + c * 1024 + lane * 16, j = j0 + o;
                w[o][c] = j < a.n_out && k < a.n_in ? load_codes(a.w + (int64_t)j * a.n_in, k, a.n_in, a.w_aligned) : intx4{0, 0, 0, 0};
            }
    };
    fetch(0);
    // the row's codes, in LDS; a thread keeps the first kRowHeld fours that it sees
    const int fours = (a.n_in + 3) / 4;
    float v[kRowHeld][4];
    const auto load = [&](int f, float (&to)[4]) {
        const int left = a.n_in - 4 * f;
        load_four<DTYPE>(a.x, 4 * f, left, a.x_by_four && left >= 4, to);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = rectified(to[e], a.relu);
    };
    uint32_t top = 0;
    const auto see = [&](const float (&from)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) top = larger(top, magnitude(from[e]));
    };
#pragma unroll
    for (int h = 0; h < kRowHeld; ++h)
        if ((int)threadIdx.x + h * 256 < fours) load(threadIdx.x + h * 256, v[h]);
#pragma unroll
    for (int h = 0; h < kRowHeld; ++h)
        if ((int)threadIdx.x + h * 256 < fours) see(v[h]);
#pragma unroll 4
    for (int f = threadIdx.x + kRowHeld * 256; f < fours; f += 256) {
        float t[4];
        load(f, t);
        see(t);
    }
    top = wave_max(top);
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    const RowScale s(larger(larger(tops[0], tops[1]), larger(tops[2], tops[3])));
    const auto store = [&](int f, const float (&from)[4]) {
        int c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = s.code(from[e]);   // (beyond the row's end: of zero)
        *reinterpret_cast<uint32_t *>(lds + 4 * f) = packed(c);
    };
#pragma unroll
    for (int h = 0; h < kRowHeld; ++h)
        if ((int)threadIdx.x + h * 256 < fours) store(threadIdx.x + h * 256, v[h]);
#pragma unroll 4
    for (int f = threadIdx.x + kRowHeld * 256; f < fours; f += 256) {
        float t[4];
        load(f, t);
        store(f, t);
    }
    for (int f = fours + threadIdx.x; f < padded / 4; f += 256) *reinterpret_cast<uint32_t *>(lds + 4 * f) = 0;
    __syncthreads();
    int sum[OUTS] = {};
    for (int k0 = 0; k0 < a.n_in; k0 += CHUNKS * 1024) {
        if (k0) fetch(k0);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (k0 + c * 1024 >= a.n_in) break;
            const intx4 x = *reinterpret_cast<const intx4 *>(lds + k0 + c * 1024 + lane * 16);
#pragma unroll
            for (int o = 0; o < OUTS; ++o)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[o] = __builtin_amdgcn_sdot4(x[e], w[o][c][e], sum[o], false);
        }
    }
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
        int t = sum[o];
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) t += __shfl_xor(t, d, 64);
        const int j = j0 + o;
        if (lane == 0 && j < a.n_out) {
            float y = scaled(t, a.w_scale[j], s.scale) + (a.bias ? a.bias[j] : 0.0f);
            if (a.beta != 0.0f) y += a.beta * load_as_float(a.y, j, a.y_dtype);
            store_from_float(a.y, j, a.y_dtype, y);
        }
    }
}

// ---- some rows -------------------------------------------------------------------------------------------------------

constexpr int kSomeRows = 64;                // rows of a call that some_rows_kernel takes
constexpr int kSomeWaves = 16;
constexpr int kSomeLds = 128 * 1024;         // bytes of LDS for their codes
constexpr int kSomeFetched = 4;              // pieces of 64 codes that a wave has on their way at the start

// 64 codes are a piece of the summed axis; rows of codes are a piece apart from a multiple of LDS's banks
int some_pitch(int n_in) { return (n_in + 63) / 64 * 64 + 16; }

// A workgroup takes 16 outputs of all rows, RT tiles of 16.  A wave scales every sixteenth row, then multiplies every
// sixteenth piece; the waves' sums meet in LDS, as whole numbers in any order.
template <int DTYPE, int RT>
__global__ __launch_bounds__(64 * kSomeWaves) void some_rows_kernel(RowsArgs a, int rows, int pitch)
{
    extern __shared__ __align__(16) char lds[];
    __shared__ int sums[RT * 16][17];
    __shared__ float scales[RT * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j0 = blockIdx.x * 16, pieces = (a.n_in + 63) / 64;
    // weights: row lane & 15 of the 16 outputs, 16 codes from 16 (lane >> 4) on of a piece
    const int8_t *w = a.w + (int64_t)min(j0 + (lane & 15), a.n_out - 1) * a.n_in;
    const auto fetch = [&](int piece) { return load_codes(w, min(64 * piece + 16 * (lane >> 4), a.n_in), a.n_in, a.w_aligned); };
    intx4 fetched[kSomeFetched];
#pragma unroll
    for (int k = 0; k < kSomeFetched; ++k)
        if (wave + k * kSomeWaves < pieces) fetched[k] = fetch(wave + k * kSomeWaves);
    for (int e = threadIdx.x; e < RT * 16 * 17; e += 64 * kSomeWaves) (&sums[0][0])[e] = 0;
    const int fours = (a.n_in + 3) / 4;
    for (int r = wave; r < rows; r += kSomeWaves) {
        float v[kHeld][4];
        uint32_t top = 0;
        const auto load = [&](int f, float (&to)[4]) {
            const int left = a.n_in - 4 * f;
            load_four<DTYPE>(a.x, (int64_t)r * a.n_in + 4 * f, left, a.x_by_four && left >= 4, to);
#pragma unroll
            for (int e = 0; e < 4; ++e) to[e] = rectified(to[e], a.relu);
        };
        const auto see = [&](const float (&from)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) top = larger(top, magnitude(from[e]));
        };
#pragma unroll
        for (int h = 0; h < kHeld; ++h)
            if (lane + h * 64 < fours) load(lane + h * 64, v[h]);
#pragma unroll
        for (int h = 0; h < kHeld; ++h)
            if (lane + h * 64 < fours) see(v[h]);
#pragma unroll 4
        for (int f = lane + kHeld * 64; f < fours; f += 64) {
            float t[4];
            load(f, t);
            see(t);
        }
        const RowScale s(wave_max(top));
        if (lane == 0) scales[r] = s.scale;
        char *to = lds + r * pitch;
        const auto store = [&](int f, const float (&from)[4]) {
            int c[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = s.code(from[e]);   // (beyond the row's end: of zero)
            *reinterpret_cast<uint32_t *>(to + 4 * f) = packed(c);
        };
#pragma unroll
        for (int h = 0; h < kHeld; ++h)
            if (lane + h * 64 < fours) store(lane + h * 64, v[h]);
#pragma unroll 4
        for (int f = lane + kHeld * 64; f < fours; f += 64) {
            float t[4];
            load(f, t);
            store(f, t);
        }
        if (lane < 16 * pieces - fours) *reinterpret_cast<uint32_t *>(to + 4 * (fours + lane)) = 0;
    }
    __syncthreads();
    intx4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = intx4{0, 0, 0, 0};
    const auto multiply = [&](int piece, const intx4 &cols) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            // (rows beyond the last repeat it: their outputs are dropped)
            const intx4 x = *reinterpret_cast<const intx4 *>(lds + min(16 * i + (lane & 15), rows - 1) * pitch + 64 * piece + 16 * (lane >> 4));
            acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cols, x, acc[i], 0, 0, 0);
        }
    };
#pragma unroll
    for (int k = 0; k < kSomeFetched; ++k)
        if (wave + k * kSomeWaves < pieces) multiply(wave + k * kSomeWaves, fetched[k]);
    for (int piece = wave + kSomeFetched * kSomeWaves; piece < pieces; piece += kSomeWaves) multiply(piece, fetch(piece));
    if (wave < pieces)
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) atomicAdd(&sums[16 * i + (lane & 15)][4 * (lane >> 4) + e], acc[i][e]);
    __syncthreads();
    const int r = threadIdx.x >> 4, j = j0 + (threadIdx.x & 15);
    if (r < rows && j < a.n_out) {
        const int64_t at = (int64_t)r * a.n_out + j;
        float y = scaled(sums[r][threadIdx.x & 15], a.w_scale[j], scales[r]) + (a.bias ? a.bias[j] : 0.0f);
        if (a.beta != 0.0f) y += a.beta * load_as_float(a.y, at, a.y_dtype);
        store_from_float(a.y, at, a.y_dtype, y);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int padded_row(int n_in) { return (n_in + kLine - 1) / kLine * kLine; }
int padded_one(int n_in) { return (n_in + 1023) / 1024 * 1024; }

// One launch, in which every workgroup scales all rows, or three.  The former takes 3.5 us and 0.14 for every 1024
// elements of x and turn of a compute unit (a workgroup of 16 outputs at a time), the latter 7 to 17 us.  Measured (us, one
// launch / three): 16 rows of 1024 -> 1024 5.7 / 10.7; 48 of 1024 -> 1024 10.1 / 11.4; 64 of 1024 -> 4096 13.1 / 11.4;
// 64 of 256 -> 16384 30 / 8.3.
bool some_rows(const LinearShape &s)
{
    const int64_t turns = (s.n_out + 16 * 256 - 1) / (16 * 256);
    return s.batch > 1 && s.batch <= kSomeRows && s.batch * some_pitch(s.n_in) <= kSomeLds && s.batch * s.n_in * turns <= 50 * 1024;
}

typedef TileShape<64, 64, 2, 2, 3> Tile64;
typedef TileShape<128, 128, 2, 2, 2> Tile128;

constexpr int kUnits = 256;   // compute units

template <class T>
WorkSplit split_work(const LinearShape &s)
{
    const int tiles = (int)(((s.batch + T::ROWS - 1) / T::ROWS) * ((s.n_out + T::COLS - 1) / T::COLS));
    const int stages = padded_row(s.n_in) / kLine, workers = kUnits * (160 * 1024 / T::LDS);
    // (joining takes 5 us, a stage of the smaller tile 0.3: 48 rows of 1024 -> 1024, eight stages, 17 us cut, 11 whole)
    return WorkSplit::of(tiles, stages, workers, T::ROWS == 64 ? 16 : 12);
}

// The larger tile reads half as much per product, and needs two tiles a compute unit to keep them busy.  Measured
// (us, tiles of 64 / 128): 4096 rows of 4096 -> 4096 174 / 104; 8192 of 1024 -> 1024 38 / 35; 5000 of 500 -> 333 16 / 24.
bool large_tiles(const LinearShape &s) { return ((s.batch + 127) / 128) * ((s.n_out + 127) / 128) >= 2 * kUnits; }

WorkSplit split_work(const LinearShape &s) { return large_tiles(s) ? split_work<Tile128>(s) : split_work<Tile64>(s); }

// the workspace: codes of the rows, their scales, weights in aligned rows, parts of tiles that are cut
struct Layout {
    size_t codes, scale, w, parts, total;
};
Layout layout_of(const LinearShape &s)
{
    Layout l = {};
    if (s.batch == 1 || some_rows(s)) return l;
    const WorkSplit w = split_work(s);
    const size_t tile = (large_tiles(s) ? Tile128::ROWS * Tile128::COLS : Tile64::ROWS * Tile64::COLS) * sizeof(int);
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += align256(bytes); return here; };
    l.codes = take((size_t)s.batch * padded_row(s.n_in));
    l.scale = take((size_t)s.batch * sizeof(float));
    l.w = take((size_t)s.n_out * padded_row(s.n_in));   // (whether it is needed depends on a pointer)
    l.parts = take(w.cut() ? 2 * w.cutters * tile : 0);
    l.total = at;
    return l;
}

template <class T>
void launch_tiles(LinearArgs &a, hipStream_t stream)
{
    a.tiles_down = (int)((a.batch + T::ROWS - 1) / T::ROWS);
    a.tiles_across = (a.n_out + T::COLS - 1) / T::COLS;
    if (T::LDS > 65536) allow_large_lds(reinterpret_cast<const void *>(linear_kernel<T>), T::LDS);
    linear_kernel<T><<<a.work.workers, T::THREADS, T::LDS, stream>>>(a);
    if (a.work.cut()) linear_join_kernel<T><<<a.work.left() * T::WAVES, 64 * joiners<T>(), 0, stream>>>(a);
}

template <int DTYPE>
void launch_one(const RowsArgs &a, hipStream_t stream)
{
    // one output a wave where four would leave compute units idle
    const int padded = padded_one(a.n_in);
    if (padded > 56 * 1024) {
        allow_large_lds(reinterpret_cast<const void *>(one_row_kernel<DTYPE, 1, 8>), padded_one(LMKAN_MAX_N_IN));
        allow_large_lds(reinterpret_cast<const void *>(one_row_kernel<DTYPE, 4, 4>), padded_one(LMKAN_MAX_N_IN));
    }
    if (a.n_out < 2048) one_row_kernel<DTYPE, 1, 8><<<(a.n_out + 3) / 4, 256, padded, stream>>>(a, padded);
    else one_row_kernel<DTYPE, 4, 4><<<(a.n_out + 15) / 16, 256, padded, stream>>>(a, padded);
}

template <int DTYPE, int RT>
void launch_some_rows(int rows, const RowsArgs &a, hipStream_t stream)
{
    const int pitch = some_pitch(a.n_in), lds = rows * pitch;
    if (lds > 56 * 1024) allow_large_lds(reinterpret_cast<const void *>(some_rows_kernel<DTYPE, RT>), kSomeLds);
    some_rows_kernel<DTYPE, RT><<<(a.n_out + 15) / 16, 64 * kSomeWaves, lds, stream>>>(a, rows, pitch);
}
template <int DTYPE>
void launch_some(int rows, const RowsArgs &a, hipStream_t stream)
{
    if (rows <= 16) launch_some_rows<DTYPE, 1>(rows, a, stream);
    else if (rows <= 32) launch_some_rows<DTYPE, 2>(rows, a, stream);
    else launch_some_rows<DTYPE, 4>(rows, a, stream);
}

template <int DTYPE>
void launch_quantize(QuantizeArgs a, hipStream_t stream)
{
    // a wave a row while the row fits what its lanes hold
    const bool wave = a.cols <= 64 * 4 * kHeld;
    const int64_t rows = a.rows, most = kMostGroups * (wave ? 4 : 1), item = DTYPE == LMKAN_F32 ? 4 : 2;
    const int64_t aligning = a.align.w ? ((int64_t)a.align.n_out * (a.align.pitch / 4) + 255) / 256 : 0;
    for (int64_t row = 0, block = 0; row < rows || block < aligning; row += a.rows) {
        a.rows = rows - row < most ? rows - row : most;
        a.row_blocks = (unsigned)(wave ? (a.rows + 3) / 4 : a.rows);
        const int64_t room = kMostGroups - a.row_blocks, now = aligning - block < room ? aligning - block : room;
        const unsigned blocks = a.row_blocks + (unsigned)now;
        if (wave) quantize_kernel<DTYPE, 64><<<blocks, 256, 0, stream>>>(a);
        else quantize_kernel<DTYPE, 256><<<blocks, 256, 0, stream>>>(a);
        a.x = static_cast<const char *>(a.x) + a.rows * a.cols * item;
        a.codes += a.rows * a.pitch, a.scale += a.rows;
        block += now, a.align.first = block;
    }
}

void quantize(int64_t rows, int cols, int pitch, int dtype, bool relu, const void *x, int8_t *codes, float *scale, const AlignArgs &align,
              hipStream_t stream)
{
    QuantizeArgs a{rows, cols, pitch, relu, pitch > cols, false, false, x, codes, scale, 0, align};
    a.by_four = cols % 4 == 0 && aligned_to(x, dtype == LMKAN_F32 ? 16 : 8);
    a.codes_by_four = pitch % 4 == 0 && aligned_to(codes, 4);
    if (dtype == LMKAN_F32) launch_quantize<LMKAN_F32>(a, stream);
    else if (dtype == LMKAN_F16) launch_quantize<LMKAN_F16>(a, stream);
    else launch_quantize<LMKAN_BF16>(a, stream);
}

}  // namespace

void launch_quantize_rows(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, float *scale, hipStream_t stream)
{
    quantize(rows, cols, cols, dtype, relu, x, codes, scale, AlignArgs{}, stream);
}

size_t linear_i8_workspace_bytes(const LinearShape &s) { return layout_of(s).total; }

void launch_linear_i8(const LinearShape &s, const void *x, const int8_t *w, const float *w_scale, const float *bias,
                      float beta, void *y, void *workspace, hipStream_t stream)
{
    if (s.batch == 1 || some_rows(s)) {
        const RowsArgs a{x, w, w_scale, bias, beta, y, s.n_in, s.n_out, s.y_dtype, s.relu, s.n_in % 16 == 0 && aligned_to(w, 16),
                         s.n_in % 4 == 0 && aligned_to(x, s.x_dtype == LMKAN_F32 ? 16 : 8)};
        const int rows = (int)s.batch;
        if (s.x_dtype == LMKAN_F32) rows == 1 ? launch_one<LMKAN_F32>(a, stream) : launch_some<LMKAN_F32>(rows, a, stream);
        else if (s.x_dtype == LMKAN_F16) rows == 1 ? launch_one<LMKAN_F16>(a, stream) : launch_some<LMKAN_F16>(rows, a, stream);
        else rows == 1 ? launch_one<LMKAN_BF16>(a, stream) : launch_some<LMKAN_BF16>(rows, a, stream);
        return;
    }
    const Layout l = layout_of(s);
    char *ws = static_cast<char *>(workspace);
    int8_t *codes = reinterpret_cast<int8_t *>(ws + l.codes);
    float *scale = reinterpret_cast<float *>(ws + l.scale);
    const int pitch = padded_row(s.n_in);
    LinearArgs a = {};
    a.x = codes, a.x_pitch = pitch;
    a.w = w, a.w_pitch = s.n_in;
    AlignArgs align = {};
    if (s.n_in % 16 != 0 || !aligned_to(w, 16)) {
        align = {w, s.n_in, s.n_out, pitch, reinterpret_cast<int8_t *>(ws + l.w)};
        a.w = align.to, a.w_pitch = pitch;
    }
    quantize(s.batch, s.n_in, pitch, s.x_dtype, s.relu, x, codes, scale, align, stream);
    a.x_scale = scale, a.w_scale = w_scale, a.bias = bias, a.beta = beta;
    a.y = y, a.batch = s.batch, a.n_in = s.n_in, a.n_out = s.n_out, a.y_dtype = s.y_dtype;
    a.by_four = s.n_out % 4 == 0 && aligned_to(y, s.y_dtype == LMKAN_F32 ? 16 : 8);
    a.parts = reinterpret_cast<intx4 *>(ws + l.parts);
    a.work = split_work(s);
    if (large_tiles(s)) launch_tiles<Tile128>(a, stream);
    else launch_tiles<Tile64>(a, stream);
}

}  // namespace lmkan
