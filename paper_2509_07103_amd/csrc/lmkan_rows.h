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

// E adjacent elements of a row: 1, or 4 or 8 that are aligned to their size together
template <int E, int DTYPE>
__device__ __forceinline__ void load_piece(const void *p, unsigned at, float (&v)[E])
{
    if constexpr (E == 1) {
        v[0] = load_as_float(p, at, DTYPE);
    } else if constexpr (DTYPE == LMKAN_F32) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at + i);
            v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
        }
    } else {
        uint32_t w[E / 2];
        const uint16_t *from = static_cast<const uint16_t *>(p) + at;
        if constexpr (E == 8) {
            const uint4 u = *reinterpret_cast<const uint4 *>(from);
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        } else {
            const uint2 u = *reinterpret_cast<const uint2 *>(from);
            w[0] = u.x, w[1] = u.y;
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const uint16_t b = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
            v[i] = load_as_float(&b, 0, DTYPE);
        }
    }
}
template <int E>
__device__ __forceinline__ void load_piece(const void *p, unsigned at, int dtype, float (&v)[E])
{
    if (dtype == LMKAN_F32) load_piece<E, LMKAN_F32>(p, at, v);
    else if (dtype == LMKAN_F16) load_piece<E, LMKAN_F16>(p, at, v);
    else load_piece<E, LMKAN_BF16>(p, at, v);
}
template <int E>
__device__ __forceinline__ void store_piece(void *p, unsigned at, int dtype, const float (&v)[E])
{
    if constexpr (E == 1) {
        store_from_float(p, at, dtype, v[0]);
    } else if (dtype == LMKAN_F32) {
#pragma unroll
        for (int i = 0; i < E; i += 4) *reinterpret_cast<float4 *>(static_cast<float *>(p) + at + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
        uint32_t w[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) w[i] = two_from_float(dtype, v[2 * i], v[2 * i + 1]);
        uint16_t *to = static_cast<uint16_t *>(p) + at;
        if constexpr (E == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
    }
}

// E adjacent codes as they lie in memory, four to a word
template <int E>
__device__ __forceinline__ void load_codes_piece(const int8_t *p, uint32_t (&w)[(E + 3) / 4])
{
    if constexpr (E == 1) {
        w[0] = (uint8_t)*p;
    } else if constexpr (E == 4) {
        w[0] = *reinterpret_cast<const uint32_t *>(p);
    } else {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        w[0] = u.x, w[1] = u.y;
    }
}
// The power of two of a block in float32 (NaN for 255); times a code it is the value, exactly, where it is not below 2^-126
// (there the value itself is worked out)
template <int E>
__device__ __forceinline__ void values_of(const uint32_t (&w)[(E + 3) / 4], int byte, float (&v)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i & 3)));
    const int e = byte - kExpBias;
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = __builtin_amdgcn_ldexpf(byte == kExpNan ? __builtin_nanf("") : v[i], e);
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
template <int E>
__device__ __forceinline__ void store_codes_piece(int8_t *p, const uint32_t (&w)[(E + 3) / 4])
{
    if constexpr (E == 1) *p = (int8_t)w[0];
    else if constexpr (E == 4) *reinterpret_cast<uint32_t *>(p) = w[0];
    else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}

// Whether pieces of E elements of a matrix of rows of `cols` may be taken together
inline bool pieces_ok(int e, int cols, const void *p, int dtype)
{
    const size_t size = dtype == LMKAN_F32 ? 16 : 2 * e;
    return cols % e == 0 && reinterpret_cast<uintptr_t>(p) % size == 0;
}

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
size_t linear_grad_workspace_bytes(const LinearShape &s);
void launch_linear_grad(const LinearShape &s, bool accumulate, const int8_t *codes, const uint8_t *exps, const void *grad_y,
                        float *grad_weight, float *grad_bias, void *workspace, hipStream_t stream);

struct AdapterShape {
    int64_t batch;
    int count, rank, n_in, n_out;
    int dtype, x_dtype, y_dtype;
    bool relu;
};
size_t adapters_workspace_bytes(const AdapterShape &s);
void launch_adapters(const AdapterShape &s, const void *x, const int32_t *index, const void *a, const void *b, const float *scale, void *y,
                     void *workspace, hipStream_t stream);

}  // namespace lmkan
