// Activations to 8-bit checkpoints and back.  A block of 32 columns shares a power of two, so that both directions are
// exact but for the one rounding to a whole number, and a value (7 bits and a sign) is exact in 16-bit types too (float16: within
// its range).
//
// Both are bound by memory.  A lane takes pieces of 4 or 8 adjacent elements (16 bytes), 8 or 4 lanes a block, whose largest
// magnitude they find without LDS; a row goes to as many lanes as give each a few pieces, which are under way together.
// 16384 x 4096 float32, each in a loop of its own: to codes 62 us (5.4 TB/s of what is read and written; a copy reaches 5.2 to 5.4),
// back 61 (5.5).  One after the other, on rows that the last cache no longer holds in part, 83 and 57, 140 in all (4.8); 5000 x 500
// float16 9.5, two launches that take hardly more than empty ones.
#include "lmkan_rows.h"

namespace lmkan {

namespace {

// Pieces of a lane that are under way.  Measured (us, 2 / 4 / 8 of them): to codes 8192 x 1024 float32 8.8 / 7.8 / 8.0, 65536 x 1024
// 59 / 62 / 63, 100000 x 333 bfloat16 (unaligned) 31 / 23 / 22; back 60000 x 1000 float32 50 / 59 / 57, 262144 x 128 bfloat16
// 16.8 / 17.9 / 18.5, 100000 x 333 30 / 23 / 22
constexpr int kTaken = 4;
constexpr int restored_together(int kind) { return kind > 0 ? 2 : 4; }

struct RowsArgs {
    int64_t rows;
    int cols, dtype;
    bool relu;
    int lanes_log;   // of a row
    const void *x;
    int8_t *codes;
    uint8_t *exps;
    const float *weight, *bias;
    void *y;
};

template <int K, int DTYPE>
__global__ __launch_bounds__(256) void checkpoint_kernel(RowsArgs a)
{
    constexpr int E = elements_of(K);
    const int lanes = 1 << a.lanes_log, per_row = exp_blocks(a.cols), pieces = per_row * (kBlock / E);
    const int lane = threadIdx.x & (lanes - 1), rows = 256 >> a.lanes_log;
    for (int64_t row = (int64_t)blockIdx.x * rows + (threadIdx.x >> a.lanes_log); row < a.rows; row += (int64_t)gridDim.x * rows) {
        const void *x = row_at(a.x, row * a.cols, DTYPE);
        int8_t *codes = a.codes + row * a.cols;
        uint8_t *exps = a.exps + row * per_row;
        for (int p0 = lane; p0 < pieces; p0 += kTaken * lanes) {
            float v[kTaken][E];
#pragma unroll
            for (int k = 0; k < kTaken; ++k) load_piece_as<K, DTYPE>(x, (p0 + k * lanes) * E, a.cols, v[k]);
#pragma unroll
            for (int k = 0; k < kTaken; ++k) {
                const int c = (p0 + k * lanes) * E;
                if (p0 + k * lanes >= pieces) break;
                settle<K>(v[k], c, a.cols);
#pragma unroll
                for (int i = 0; i < E; ++i) v[k][i] = rectify(v[k][i], a.relu);
                uint32_t w[(E + 3) / 4];
                const int byte = encode_piece(v[k], w);
                if (c < a.cols) {
                    store_codes_piece<K>(codes, c, a.cols, w);
                    if (c % kBlock == 0) exps[c / kBlock] = (uint8_t)byte;
                }
            }
        }
    }
}

template <int K>
__global__ __launch_bounds__(256) void restore_kernel(RowsArgs a)
{
    constexpr int E = elements_of(K), kTogether = restored_together(K);
    const int lanes = 1 << a.lanes_log, per_row = exp_blocks(a.cols);
    const int lane = threadIdx.x & (lanes - 1), rows = 256 >> a.lanes_log;
    for (int64_t row = (int64_t)blockIdx.x * rows + (threadIdx.x >> a.lanes_log); row < a.rows; row += (int64_t)gridDim.x * rows) {
        const int8_t *codes = a.codes + row * a.cols;
        void *y = row_at(a.y, row * a.cols, a.dtype);
        const uint8_t *exps = a.exps + row * per_row;
        for (int c0 = lane * E; c0 < a.cols; c0 += kTogether * lanes * E) {
            uint32_t w[kTogether][(E + 3) / 4];
            int byte[kTogether];
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                const int c = c0 + k * lanes * E;
                load_codes_piece<K>(codes, c, a.cols, w[k]);
                byte[k] = exps[(c < a.cols ? c : 0) / kBlock];
            }
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                const int c = c0 + k * lanes * E;
                if (c >= a.cols) break;
                float v[E];
                values_of<E>(w[k], byte[k], v);
                settle<K>(v, c, a.cols);
                if (a.weight || a.bias) {
                    float m[E], b[E];
                    if (a.weight) load_piece_as<K, LMKAN_F32>(a.weight, c, a.cols, m), settle<K>(m, c, a.cols);
                    if (a.bias) load_piece_as<K, LMKAN_F32>(a.bias, c, a.cols, b), settle<K>(b, c, a.cols);
#pragma unroll
                    for (int i = 0; i < E; ++i) v[i] = fmaf(a.weight ? m[i] : 1.0f, v[i], a.bias ? b[i] : 0.0f);
                }
#pragma unroll
                for (int i = 0; i < E; ++i) v[i] = rectify(v[i], a.relu);
                store_piece<K>(y, c, a.cols, a.dtype, v);
            }
        }
    }
}

// Lanes of a row: each has up to `taken` pieces, and blocks are whole
int lanes_log(int cols, int e, int taken)
{
    int log = e == 1 ? 5 : e == 4 ? 3 : 2;
    while (log < 8 && cols > (taken * e) << log) ++log;
    return log;
}

unsigned groups(int64_t rows, int log)
{
    const int64_t n = (rows + (256 >> log) - 1) / (256 >> log);
    return (unsigned)(n < kMostGroups ? n : kMostGroups);
}

template <int K>
void launch_checkpoint_type(const RowsArgs &a, hipStream_t stream)
{
    const unsigned n = groups(a.rows, a.lanes_log);
    if (a.dtype == LMKAN_F32) {
        if constexpr (K < 8) checkpoint_kernel<K, LMKAN_F32><<<n, 256, 0, stream>>>(a);
    } else if (a.dtype == LMKAN_F16) {
        checkpoint_kernel<K, LMKAN_F16><<<n, 256, 0, stream>>>(a);
    } else {
        checkpoint_kernel<K, LMKAN_BF16><<<n, 256, 0, stream>>>(a);
    }
}

}  // namespace

void launch_checkpoint(int64_t rows, int cols, int dtype, bool relu, const void *x, int8_t *codes, uint8_t *exps, hipStream_t stream)
{
    RowsArgs a{rows, cols, dtype, relu, 0, x, codes, exps};
    const auto fits = [&](int e) { return pieces_ok(e, cols, x, dtype) && reinterpret_cast<uintptr_t>(codes) % e == 0; };
    // (262144 x 128 bfloat16: eight together 20.4 us, four 21.6)
    const int kind = dtype != LMKAN_F32 && fits(8) ? 8 : fits(4) ? 4 : unaligned_kind(cols);
    a.lanes_log = lanes_log(cols, elements_of(kind), kTaken);
    if (kind == 8) launch_checkpoint_type<8>(a, stream);
    else if (kind == 4) launch_checkpoint_type<4>(a, stream);
    else if (kind == -4) launch_checkpoint_type<-4>(a, stream);
    else launch_checkpoint_type<1>(a, stream);
}

void launch_restore(int64_t rows, int cols, int dtype, bool relu, const int8_t *codes, const uint8_t *exps, const float *weight,
                    const float *bias, void *y, hipStream_t stream)
{
    RowsArgs a{rows, cols, dtype, relu, 0, nullptr, const_cast<int8_t *>(codes), const_cast<uint8_t *>(exps), weight, bias, y};
    // (65536 x 1024 bfloat16: pieces of eight 32 us, of four 36)
    const auto fits = [&](int e) {
        return pieces_ok(e, cols, y, dtype) && reinterpret_cast<uintptr_t>(codes) % e == 0 && pieces_ok(4, 4, weight, LMKAN_F32) && pieces_ok(4, 4, bias, LMKAN_F32);
    };
    const int kind = dtype != LMKAN_F32 && fits(8) ? 8 : fits(4) ? 4 : unaligned_kind(cols);
    a.lanes_log = lanes_log(cols, elements_of(kind), restored_together(kind));
    const unsigned n = groups(rows, a.lanes_log);
    if (kind == 8) restore_kernel<8><<<n, 256, 0, stream>>>(a);
    else if (kind == 4) restore_kernel<4><<<n, 256, 0, stream>>>(a);
    else if (kind == -4) restore_kernel<-4><<<n, 256, 0, stream>>>(a);
    else restore_kernel<1><<<n, 256, 0, stream>>>(a);
}

}  // namespace lmkan
