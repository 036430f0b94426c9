// What the operators on rows share (lmkan_norm.hip, lmkan_checkpoint.hip, lmkan_linear_grad.hip, lmkan_adapters.hip):
// their launchers, the blocks of a checkpoint.
// Every launcher enqueues on the given stream and returns; arguments have been validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lmkan_dense.h"

namespace lmkan {

constexpr int kBlock = LMKAN_CHECKPOINT_BLOCK;
constexpr int kExpBias = 133, kMostExp = 121;   // a block's byte is its exponent + 133
constexpr int kExpNan = 255;

__host__ __device__ __forceinline__ int exp_blocks(int cols) { return (cols + kBlock - 1) / kBlock; }

// The byte of a block whose largest magnitude has the bits `top` (ordered like the values; NaN above infinity)
__device__ __forceinline__ int block_byte(uint32_t top)
{
    if (top >= 0x7f800000u) return kExpNan;
    if (top == 0) return 0;
    const float t = __builtin_bit_cast(float, top);
    int e = __builtin_amdgcn_frexp_expf(t) - 7;                        // t / 2^e in [64, 128)
    e += rintf(__builtin_amdgcn_ldexpf(t, -e)) > 127.0f;
    e = e < -kExpBias ? -kExpBias : e > kMostExp ? kMostExp : e;
    return e + kExpBias;
}

// Code of an element of a block that has no NaN or infinity, in the lowest byte, and the value that a code stands for.
// Both scalings are exact, so that rounding to a whole number is the only one: the sum with 1.5 2^23 has no bits behind
// the point, and the whole number's two's complement in its last bits.
__device__ __forceinline__ uint32_t code_bits(float v, int byte)
{
    const float scaled = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(v, kExpBias - byte), -127.0f, 127.0f);
    return __builtin_bit_cast(uint32_t, scaled + 12582912.0f);
}
__device__ __forceinline__ float value_of(int code, int byte)
{
    return byte == kExpNan ? __builtin_nanf("") : __builtin_amdgcn_ldexpf((float)code, byte - kExpBias);
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
// max(v, 0); a NaN stays one
__device__ __forceinline__ float rectify(float v, bool relu) { return relu && v < 0.0f ? 0.0f : v; }

// ---- across lanes ----------------------------------------------------------------------------------------------------

constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;   // DPP: within 2, 4, 8 and 16 lanes

template <int CTRL, class V>
__device__ __forceinline__ V from_lane(V v)
{
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)u, CTRL, 0xf, 0xf, true), hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(u >> 32), CTRL, 0xf, 0xf, true);
        return __builtin_bit_cast(V, (uint64_t)hi << 32 | lo);
    }
}

// The values of both halves of 32 (16: HALF) lanes, in all of them
template <int HALF, class V>
__device__ __forceinline__ void halves(V v, V *a, V *b)
{
    const auto swap = [](uint32_t w) {
        if constexpr (HALF == 16) return __builtin_amdgcn_permlane16_swap(w, w, false, false);
        else return __builtin_amdgcn_permlane32_swap(w, w, false, false);
    };
    if constexpr (sizeof(V) == 4) {
        const auto s = swap(__builtin_bit_cast(uint32_t, v));
        *a = __builtin_bit_cast(V, (uint32_t)s[0]), *b = __builtin_bit_cast(V, (uint32_t)s[1]);
    } else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const auto lo = swap((uint32_t)u), hi = swap((uint32_t)(u >> 32));
        *a = __builtin_bit_cast(V, (uint64_t)hi[0] << 32 | lo[0]), *b = __builtin_bit_cast(V, (uint64_t)hi[1] << 32 | lo[1]);
    }
}

// What `f` makes of the values of 4 to 64 adjacent lanes (a power of two, the same for the wave), in all of them
template <class V, class F>
__device__ __forceinline__ V over_lanes(V v, int lanes, F &&f)
{
    v = f(v, from_lane<kXor1>(v));
    v = f(v, from_lane<kXor2>(v));
    if (lanes > 4) v = f(v, from_lane<kHalfMirror>(v));
    if (lanes > 8) v = f(v, from_lane<kMirror>(v));
    V a, b;
    if (lanes > 16) halves<16>(v, &a, &b), v = f(a, b);
    if (lanes > 32) halves<32>(v, &a, &b), v = f(a, b);
    return v;
}

// ---- pieces of a row -------------------------------------------------------------------------------------------------

// A row that starts at element `first`
__device__ __forceinline__ const void *row_at(const void *p, int64_t first, int dtype) { return static_cast<const char *>(p) + first * (dtype == LMKAN_F32 ? 4 : 2); }
__device__ __forceinline__ void *row_at(void *p, int64_t first, int dtype) { return static_cast<char *>(p) + first * (dtype == LMKAN_F32 ? 4 : 2); }

// Pieces of adjacent elements, of kind K:
//   4, 8   aligned to their size together; a row is a whole number of them
//   -4     four that start anywhere (the loads take any address that elements may have); at the end of a row the last four
//          elements are read and moved down, and the rest is zero.  Rows of four elements at least
//   1      one by one
constexpr int elements_of(int kind) { return kind < 0 ? -kind : kind; }

template <class V>
struct __attribute__((packed, aligned(1))) Anywhere {
    V v;
};
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
template <class V, bool ANYWHERE>
__device__ __forceinline__ V load_words(const void *p)
{
    if constexpr (ANYWHERE) return reinterpret_cast<const Anywhere<V> *>(p)->v;
    else return *static_cast<const V *>(p);
}
template <bool ANYWHERE, class V>
__device__ __forceinline__ void store_words(void *p, V v)
{
    if constexpr (ANYWHERE) reinterpret_cast<Anywhere<V> *>(p)->v = v;
    else *static_cast<V *>(p) = v;
}

// Where the elements of the piece at column `at` are read: in the row in any case
template <int K>
__device__ __forceinline__ unsigned read_at(int at, int cols)
{
    return (unsigned)(K < 0 ? (at + 4 <= cols ? at : cols - 4) : (at < cols ? at : 0));
}
// What belongs to the columns at .. of what was read (beyond the end: zeros)
template <int K, int E>
__device__ __forceinline__ void settle(float (&v)[E], int at, int cols)
{
    if constexpr (K < 0) {
        const int move = at + 4 - cols;
        if (move > 0) {
            if (move & 1) v[0] = v[1], v[1] = v[2], v[2] = v[3], v[3] = 0.0f;
            if (move & 2) v[0] = v[2], v[1] = v[3], v[2] = v[3] = 0.0f;
            if (move >= 4) v[0] = v[1] = v[2] = v[3] = 0.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = at < cols ? v[i] : 0.0f;
    }
}
template <int K>
__device__ __forceinline__ bool exists(int at, int i, int cols) { return K < 0 ? at + i < cols : at < cols; }

// A piece as it lies in memory (WIDE: float32), and then as float32
template <int K, bool WIDE, int E>
__device__ __forceinline__ void load_raw(const void *row, int at, int cols, uint32_t (&w)[E])
{
    const unsigned from = read_at<K>(at, cols);
    if constexpr (E == 1) {
        w[0] = WIDE ? static_cast<const uint32_t *>(row)[from] : static_cast<const uint16_t *>(row)[from];
    } else {
        const char *p = static_cast<const char *>(row) + from * (WIDE ? 4u : 2u);
        constexpr int kWords = WIDE ? E : E / 2;
        if constexpr (kWords == 2) {
            const uintx2 u = load_words<uintx2, K < 0>(p);
            w[0] = u[0], w[1] = u[1];
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uintx4 u = load_words<uintx4, K < 0>(p + 4 * i);
                w[i] = u[0], w[i + 1] = u[1], w[i + 2] = u[2], w[i + 3] = u[3];
            }
        }
#pragma unroll
        for (int i = kWords; i < E; ++i) w[i] = 0;
    }
}
template <int DTYPE, int E>
__device__ __forceinline__ void convert(const uint32_t (&w)[E], float (&v)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const uint32_t word = E == 1 || DTYPE == LMKAN_F32 ? w[i] : w[i / 2];
        if (DTYPE == LMKAN_F32) v[i] = __builtin_bit_cast(float, word);
        else if (DTYPE == LMKAN_F16) v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(word >> (16 * (i & 1))));
        else v[i] = __builtin_bit_cast(float, i & 1 ? word & 0xffff0000u : word << 16);
    }
}
// (what was read; `settle` makes columns of it)
template <int K, int DTYPE, int E>
__device__ __forceinline__ void load_piece_as(const void *row, int at, int cols, float (&v)[E])
{
    uint32_t w[E];
    load_raw<K, DTYPE == LMKAN_F32>(row, at, cols, w);
    convert<DTYPE>(w, v);
}
template <int K, int E>
__device__ __forceinline__ void load_piece(const void *row, int at, int cols, int dtype, float (&v)[E])
{
    if (dtype == LMKAN_F32) load_piece_as<K, LMKAN_F32>(row, at, cols, v);
    else if (dtype == LMKAN_F16) load_piece_as<K, LMKAN_F16>(row, at, cols, v);
    else load_piece_as<K, LMKAN_BF16>(row, at, cols, v);
}

// Two adjacent 16-bit elements, the first in the lower half (bfloat16 by the instruction that rounds two at a time)
__device__ __forceinline__ uint32_t two_narrow(int dtype, float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if (dtype == LMKAN_F16) return two_from_float(LMKAN_F16, a, b);
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// A piece that exists, in part at the end of a row
template <int K, int E>
__device__ __forceinline__ void store_piece(void *row, int at, int cols, int dtype, const float (&v)[E])
{
    if constexpr (E == 1) {
        store_from_float(row, at, dtype, v[0]);
        return;
    }
    if (K < 0 && at + E > cols) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (at + i < cols) store_from_float(row, at + i, dtype, v[i]);
    } else if (dtype == LMKAN_F32) {
#pragma unroll
        for (int i = 0; i + 3 < E; i += 4) {
            uintx4 u;
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = __builtin_bit_cast(uint32_t, v[i + e]);
            store_words<K < 0>(static_cast<float *>(row) + at + i, u);
        }
    } else {
        char *to = reinterpret_cast<char *>(static_cast<uint16_t *>(row) + at);
        if constexpr (E == 8) store_words<false>(to, uintx4{two_narrow(dtype, v[0], v[1]), two_narrow(dtype, v[2], v[3]), two_narrow(dtype, v[4], v[5]), two_narrow(dtype, v[6], v[7])});
        else if constexpr (E == 4) store_words<K < 0>(to, uintx2{two_narrow(dtype, v[0], v[1]), two_narrow(dtype, v[2], v[3])});
    }
}

// A piece of codes as it was read, four to a word; then the values, which `settle` puts in place
template <int K, int W>
__device__ __forceinline__ void load_codes_piece(const int8_t *row, int at, int cols, uint32_t (&w)[W])
{
    const int8_t *p = row + read_at<K>(at, cols);
    if constexpr (K == 1) {
        w[0] = (uint8_t)*p;
    } else if constexpr (K == 8) {
        const uintx2 u = load_words<uintx2, false>(p);
        w[0] = u[0], w[1] = u[1];
    } else {
        w[0] = load_words<uint32_t, K < 0>(p);
    }
}
// (a code times its block's power of two is exact, 2^-133 times 127 too; the power is NaN for 255)
template <int E>
__device__ __forceinline__ void values_of(const uint32_t (&w)[(E + 3) / 4], int byte, float (&v)[E])
{
    const float power = value_of(1, byte);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i & 3))) * power;
}

// A piece of a block to codes: its byte, from the largest magnitude over the lanes of the block, and the codes.  All lanes of
// the block take part.
template <int E>
__device__ __forceinline__ int encode_piece(const float (&v)[E], uint32_t (&w)[(E + 3) / 4])
{
    const auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    uint32_t top = magnitude_bits(v[0]);
#pragma unroll
    for (int i = 1; i < E; ++i) top = larger(top, magnitude_bits(v[i]));
    top = over_lanes(top, kBlock / E, larger);
    const int byte = block_byte(top);
    uint32_t c[E];
#pragma unroll
    for (int i = 0; i < E; ++i) c[i] = code_bits(v[i], byte);
    if constexpr (E == 1) {
        w[0] = byte == kExpNan ? 0 : c[0];
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const uint32_t ab = __builtin_amdgcn_perm(c[i + 1], c[i], 0x0c0c0400u), cd = __builtin_amdgcn_perm(c[i + 3], c[i + 2], 0x0c0c0400u);
            w[i / 4] = byte == kExpNan ? 0 : ab | cd << 16;
        }
    }
    return byte;
}
template <int K, int W>
__device__ __forceinline__ void store_codes_piece(int8_t *row, int at, int cols, const uint32_t (&w)[W])
{
    if constexpr (K == 1) {
        row[at] = (int8_t)w[0];
    } else if constexpr (K == 8) {
        store_words<false>(row + at, uintx2{w[0], w[1]});
    } else if (K < 0 && at + 4 > cols) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (at + i < cols) row[at + i] = (int8_t)(w[0] >> (8 * i));
    } else {
        store_words<K < 0>(row + at, w[0]);
    }
}

// Whether pieces of 4 or 8 elements of a matrix of rows of `cols` are aligned
inline bool pieces_ok(int e, int cols, const void *p, int dtype)
{
    const size_t size = dtype == LMKAN_F32 ? 16 : 2 * e;
    return cols % e == 0 && reinterpret_cast<uintptr_t>(p) % size == 0;
}
inline int unaligned_kind(int cols) { return cols < 4 ? 1 : -4; }

struct NormShape {
    int64_t rows;
    int cols;
    int x_dtype, y_dtype;
    float eps;
    bool accumulate;
};

struct NormBackwardArgs {
    const void *x;          // or null, and the checkpoint
    const int8_t *codes;
    const uint8_t *exps;
    const float *stats, *weight;
    const void *grad_y;
    void *grad_x;
    float *grad_weight, *grad_bias;
};

void launch_checkpoint(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, uint8_t *exps, hipStream_t stream);
void launch_restore(int64_t rows, int cols, int dtype, bool relu, const int8_t *codes, const uint8_t *exps, const float *weight,
                    const float *bias, void *y, hipStream_t stream);

void launch_layer_norm(const NormShape &s, const void *x, const float *weight, const float *bias, void *y, float *stats, int8_t *codes,
                       uint8_t *exps, hipStream_t stream);
size_t layer_norm_backward_workspace_bytes(const NormShape &s);
void launch_layer_norm_backward(const NormShape &s, const NormBackwardArgs &a, void *workspace, hipStream_t stream);

// y_dtype: of grad_y
size_t linear_grad_workspace_bytes(const LinearShape &s);   // of this batch
size_t linear_grad_workspace_most(const LinearShape &s);    // of this and every smaller batch
void launch_linear_grad(const LinearShape &s, bool accumulate, const int8_t *codes, const uint8_t *exps, const void *grad_y,
                        float *grad_weight, float *grad_bias, void *workspace, hipStream_t stream);

struct AdapterShape {
    int64_t batch;
    int count, rank, n_in, n_out;
    int dtype, x_dtype, y_dtype;
    bool relu;
};
size_t adapters_workspace_bytes(const AdapterShape &s);   // of this batch
size_t adapters_workspace_most(const AdapterShape &s);    // of this and every smaller batch
void launch_adapters(const AdapterShape &s, const void *x, const int32_t *index, const void *a, const void *b, const float *scale, void *y,
                     void *workspace, hipStream_t stream);

}  // namespace lmkan
