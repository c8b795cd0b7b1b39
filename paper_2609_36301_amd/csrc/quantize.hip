// Rows of bf16 in 8-bit integers for gfx950: with a_t the largest magnitude of row t,
//   inv = RN32(127 / a_t)    q_ti = RNE(x_ti inv)    scale_t = RN32(a_t / 127)
// x_ti inv is rounded once, straight to the integer: fma(x, inv, 1.5 2^23) keeps the sum's last integer bit, so q is
// defined to the bit.  Gated, x_ti is silu(g_ti) u_ti of the row's two halves [g u], in fp32.
// A row stays in registers between its maximum and its rounding, so it is read once; memory-bound: 32768 gated rows of
// 2 x 1024 values 27.5 us, 6.1 TB/s; one token 2.3 us in a graph.  (A rounding by bits, not by a conversion: it needs no clamp,
// since |x inv| is at most 127.00002.)
// Rows below 2^-100 count as zero (their inverse might not be finite); a row with an infinity or NaN gets the scale
// NaN, so that what is made of it is NaN.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ffn_device.h"
#include "linear.h"

namespace more {

namespace {

constexpr float kTinyRow = 0x1p-100f;

// A group of THREADS threads takes a row, R pieces of eight values to a thread.
template <int THREADS, int R, bool GATED>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void quantize_rows_kernel(const uint16_t* __restrict__ x,
                                                                                    int32_t T, int32_t width,
                                                                                    uint2* __restrict__ q,
                                                                                    float* __restrict__ scale) {
    constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;  // rows of a workgroup
    constexpr int kWaves = THREADS / 64;
    __shared__ uint32_t part[kWaves];
    const int32_t pieces = width / 8;
    const int tid = threadIdx.x % THREADS;
    const int64_t row_stride = GATED ? 2 * (int64_t)width : width;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS; row < T; row += (int64_t)gridDim.x * kRows) {
        const uint16_t* in = x + row * row_stride;
        float v[R][8];
        u32x4 g[R], u[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int32_t at = tid + r * THREADS;
            g[r] = u[r] = u32x4{0u, 0u, 0u, 0u};
            if (at < pieces) {
                g[r] = *reinterpret_cast<const u32x4*>(in + 8 * at);
                if constexpr (GATED) u[r] = *reinterpret_cast<const u32x4*>(in + width + 8 * at);
            }
        }
        // magnitudes order as their bits do, NaN above infinity
        uint32_t most = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t w = g[r][i / 2];
                float f = bf16_bits_to_f32(i % 2 ? w >> 16 : w & 0xFFFFu);
                if constexpr (GATED) {
                    const uint32_t w2 = u[r][i / 2];
                    f = f * ffn_sigmoid(f) * bf16_bits_to_f32(i % 2 ? w2 >> 16 : w2 & 0xFFFFu);
                }
                v[r][i] = f;
                most = max(most, __builtin_bit_cast(uint32_t, f) & 0x7FFFFFFFu);
            }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
        if constexpr (kWaves > 1) {
            if ((tid & 63) == 0) part[tid >> 6] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) most = max(most, part[w]);
            __syncthreads();  // the next row's maxima may be written
        }
        const float a = __builtin_bit_cast(float, most);
        const bool some = a >= kTinyRow && most < 0x7F800000u;
        const float inv = some ? 127.0f / a : 0.0f;
        if (tid == 0) scale[row] = some ? a / 127.0f : most >= 0x7F800000u ? __builtin_nanf("") : 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int32_t at = tid + r * THREADS;
            if (at >= pieces) continue;
            uint32_t b[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t whole = __builtin_bit_cast(uint32_t, __builtin_fmaf(v[r][i], inv, 12582912.0f));
                b[i / 4] |= (some ? whole & 0xFFu : 0u) << (8 * (i % 4));
            }
            q[row * pieces + at] = uint2{b[0], b[1]};
        }
    }
}

template <int THREADS, int R>
void launch(const uint16_t* x, int32_t T, int32_t width, bool gated, int8_t* q, float* scale, hipStream_t stream) {
    const int rows = THREADS < 256 ? 256 / THREADS : 1, threads = THREADS < 256 ? 256 : THREADS;
    const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)T + rows - 1) / rows, 1 << 20);
    uint2* out = reinterpret_cast<uint2*>(q);
    if (gated)
        quantize_rows_kernel<THREADS, R, true><<<blocks, threads, 0, stream>>>(x, T, width, out, scale);
    else
        quantize_rows_kernel<THREADS, R, false><<<blocks, threads, 0, stream>>>(x, T, width, out, scale);
}

}  // namespace

hipError_t quantize_rows_launch(const uint16_t* x, int64_t T, int32_t width, bool gated, int8_t* q, float* scale,
                                hipStream_t stream) {
    const int32_t pieces = width / 8, t = (int32_t)T;
    if (pieces <= 64)
        launch<64, 1>(x, t, width, gated, q, scale, stream);
    else if (pieces <= 128)
        launch<64, 2>(x, t, width, gated, q, scale, stream);
    else if (pieces <= 256)
        launch<64, 4>(x, t, width, gated, q, scale, stream);
    else if (pieces <= 1024)
        launch<256, 4>(x, t, width, gated, q, scale, stream);
    else if (pieces <= 4096)
        launch<1024, 4>(x, t, width, gated, q, scale, stream);
    else
        launch<1024, 8>(x, t, width, gated, q, scale, stream);
    return hipGetLastError();
}

}  // namespace more
