// The experts' up kernel, shared by the forward and the backward pass (ffn.hip, ffn_backward.hip).
//
// What bounds it, and what it takes: with few rows per expert the weights' way from memory (4096 experts
// of h = 512, s = 64 with one row each: 79 us, 6.8 TB/s; with 32 rows 118 us, 4.8 TB/s of weights or 5.8 with the
// gathered token rows; 1800 experts of h = 4096 with one row: 280 us, 6.8 TB/s); with many rows the stages of the matrix product (32 experts of h = 2048, s = 1024 with 1024 rows: 317
// us, 867 TFLOP/s, backward 358 us): 1.14 us for 256 rows and 2 x 128 units with everything in LDS, 1.5 to 1.7 with
// the loads, and by the card's power with both.  Hence tiles as large as the rows allow, and no tile larger
// (256 x 256 of rows and hidden units would need 256 accumulators a lane for the two projections).
#pragma once

#include "ffn.h"
#include "ffn_device.h"

namespace more {

// A workgroup computes A of one tile and kUnits hidden units: the gate rows and up rows of W1t are the
// M side of the matrix product, the tile's token rows the N side.  A wave holds kS times 16 hidden units
// (both projections) and kN times 16 tokens, so the activation meets both its factors in the same lane.
template <int BM>
struct UpShape {
    static constexpr int kWaves = BM == 256 ? 8 : 4;
    static constexpr int kThreads = 64 * kWaves;
    // an expert has one tile, mostly, so its weights are read once (nontemporal: 1800 experts of h = 4096,
    // s = 64 with one row 465 us for both kernels against 520)
    static constexpr bool kOnce = BM == 32;
    static constexpr int kWavesS = BM >= 64 ? 2 : 4;      // waves along the hidden units
    static constexpr int kUnits = BM == 256 ? 128 : 64;
    static constexpr int kS = kUnits / kWavesS / 16;      // 16-unit tiles per wave
    static constexpr int kN = BM / (kWaves / kWavesS) / 16;
    static constexpr int kStages = BM >= 128 ? 2 : 3;
    static constexpr int kRowsAt = 2 * kUnits * 128;      // the token rows' place in a stage
    static constexpr int kStageBytes = kRowsAt + BM * 128;
    static constexpr int kLoads = (2 * kUnits + BM) / kWaves / 8;
};

// What the backward pass adds.
struct UpBackward {
    const float* dA0;  // [n][s], sorted order
    uint16_t* dgu;     // [n][2s]
    float* dgp;        // [workgroups along s][n], or NULL
};

// Forward: hidden = A.  BACKWARD (of one plane only): hidden = gate A, dgu = [dG dU], dgp = this workgroup's
// share of dgate.
template <int BM, bool BACKWARD>
__global__ __launch_bounds__(UpShape<BM>::kThreads, 2) void ffn_up_kernel(FfnArgs a, const void* __restrict__ list,
                                                             uint16_t* __restrict__ hidden, UpBackward back) {
    using S = UpShape<BM>;
    static_assert(!BACKWARD || S::kS == 4, "a wave's hidden units are a line of the results");
    __shared__ float dsum[BACKWARD ? S::kWavesS : 1][BACKWARD ? BM : 1];
    __shared__ __attribute__((aligned(1024))) char smem_raw[S::kStages * S::kStageBytes];
    LdsChar* smem = (LdsChar*)smem_raw;
    __shared__ __attribute__((aligned(16))) char scratch_raw[BACKWARD ? S::kWaves * kFfnScratch : 16];
    LdsChar* scratch = (LdsChar*)scratch_raw + (BACKWARD ? ffn_wave() * kFfnScratch : 0);
    const FfnTile* tiles = ffn_tile_list(list);
    const int32_t s = a.s, h = a.h;
    const int32_t n = a.T * a.k;
    const int32_t cols = (s + S::kUnits - 1) / S::kUnits;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int ws = wave % S::kWavesS, wn = wave / S::kWavesS;
    const int64_t total = (int64_t)*static_cast<const int32_t*>(list) * cols;
    ffn_for_each(total, [&](int64_t item) {
        const FfnTile tile = tiles[item / cols];
        if (tile.expert < 0) return;
        const int32_t s0 = (int32_t)(item % cols) * S::kUnits;
        RowTileLoader<2 * S::kUnits, S::kWaves, S::kOnce> weights;
        const uint16_t* W = a.W1t + (int64_t)tile.expert * 2 * s * h;
        weights.init([&](int i) {
            const int32_t u = min(s0 + i % S::kUnits, s - 1);
            return W + (int64_t)(i / S::kUnits * s + u) * h;
        });
        RowTileLoader<BM, S::kWaves> tokens;
        tokens.init([&](int i) {
            const uint32_t p = a.sorted[tile.row0 + min(i, tile.rows - 1)];
            return a.x + (int64_t)(p < (uint32_t)n ? p / (uint32_t)a.k : 0) * h;
        });
        f32x4 g[S::kS][S::kN], u[S::kS][S::kN];
#pragma unroll
        for (int i = 0; i < S::kS; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) g[i][j] = u[i][j] = zero_f32x4();
        // the gate rows are one group of M-side fragments, the up rows the other
        using M = FfnFragments<S::kS>;
        using N = FfnFragments<S::kN>;
        ffn_pipeline<S::kStages, S::kLoads, 2, BM == 256, M, N>(
            (h + kFfnBK - 1) / kFfnBK, 16 * wn * S::kN < tile.rows,
            [&](int step, int slot) { weights.load(smem + slot * S::kStageBytes, step * kFfnBK, h); },
            [&](int step, int slot) { tokens.load(smem + slot * S::kStageBytes + S::kRowsAt, step * kFfnBK, h); },
            ffn_work(
                [&](int slot, int kk, int group, M& m) {
#pragma unroll
                    for (int i = 0; i < S::kS; ++i)
                        m.v[i] = row_fragment(smem + slot * S::kStageBytes,
                                              group * S::kUnits + 16 * (ws * S::kS + i), kk);
                },
                [&](int slot, int kk, N& f) {
#pragma unroll
                    for (int j = 0; j < S::kN; ++j)
                        f.v[j] = row_fragment(smem + slot * S::kStageBytes + S::kRowsAt, 16 * (wn * S::kN + j), kk);
                },
                [&](int group, const M& m, const N& f) {
#pragma unroll
                    for (int i = 0; i < S::kS; ++i)
#pragma unroll
                        for (int j = 0; j < S::kN; ++j) {
                            f32x4& c = group ? u[i][j] : g[i][j];
                            c = mfma_16x16x32(m.v[i], f.v[j], c);
                        }
                },
                [] {}));
        // lane l holds token l % 16 and hidden units 4 (l / 16) .. + 3 of each 16 x 16 tile
        if constexpr (!BACKWARD) {
#pragma unroll
            for (int j = 0; j < S::kN; ++j) {
                const int32_t row = 16 * (wn * S::kN + j) + (lane & 15);
                if (row >= tile.rows) continue;
                uint16_t* out = hidden + (int64_t)(tile.row0 + row) * s;
#pragma unroll
                for (int i = 0; i < S::kS; ++i) {
                    const int32_t c = s0 + 16 * (ws * S::kS + i) + 4 * (lane >> 4);
                    if (c >= s) continue;
                    float v[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = g[i][j][q] * ffn_sigmoid(g[i][j][q]) * u[i][j][q];
                    *reinterpret_cast<uint2*>(out + c) = pack_bf16x4(v[0], v[1], v[2], v[3]);
                    if (a.planes > 1)
                        *reinterpret_cast<uint2*>(out + (int64_t)n * s + c) = pack_bf16_rest(v[0], v[1], v[2], v[3]);
                }
            }
        } else {
            // the row's dA0 is read a group of 16 rows ahead of the stores
            f32x4 d[S::kS], ahead[S::kS];
            float gate = 1.0f, gate_ahead;
            auto fetch = [&](int j) {
                const int32_t row = 16 * (wn * S::kN + j) + (lane & 15);
                const bool in = row < tile.rows;
                const uint32_t p = in ? (uint32_t)a.sorted[tile.row0 + row] : 0xFFFFFFFFu;
                gate_ahead = a.gate && p < (uint32_t)n ? a.gate[p] : 1.0f;
#pragma unroll
                for (int i = 0; i < S::kS; ++i) {
                    const int32_t c = s0 + 16 * (ws * S::kS + i) + 4 * (lane >> 4);
                    ahead[i] = zero_f32x4();
                    if (in && c < s)
                        ahead[i] = *reinterpret_cast<const f32x4*>(back.dA0 + (int64_t)(tile.row0 + row) * s + c);
                }
            };
            fetch(0);
#pragma unroll
            for (int j = 0; j < S::kN; ++j) {
                const int32_t row0 = 16 * (wn * S::kN + j), c0 = s0 + 16 * ws * S::kS;
                gate = gate_ahead;
#pragma unroll
                for (int i = 0; i < S::kS; ++i) d[i] = ahead[i];
                if (j + 1 < S::kN) fetch(j + 1);
                float dot = 0.0f;
#pragma unroll
                for (int i = 0; i < S::kS; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float sig = ffn_sigmoid(g[i][j][q]);
                        const float silu = g[i][j][q] * sig;
                        const float A = silu * u[i][j][q];
                        // units past s repeat unit s - 1 and have no share
                        dot = c0 + 16 * i + 4 * (lane >> 4) < s ? __builtin_fmaf(A, d[i][q], dot) : dot;
                        const float dA = gate * d[i][q];
                        g[i][j][q] = dA * u[i][j][q] * (sig + silu * (1.0f - sig));
                        u[i][j][q] = dA * silu;
                        d[i][q] = gate * A;
                    }
                dot += __shfl_xor(dot, 16, 64);
                dot += __shfl_xor(dot, 32, 64);
                if (lane < 16) dsum[ws][row0 + lane] = dot;
                auto store = [&](auto value, uint16_t* out, int32_t stride) {
#pragma unroll
                    for (int i = 0; i < S::kS; ++i) place_bf16(scratch, i, value(i));
                    flush_rows(scratch, (s - c0) * 2, [&](int row) {
                        return row0 + row < tile.rows ? out + (int64_t)(tile.row0 + row0 + row) * stride + c0 : nullptr;
                    });
                };
                store([&](int i) { return g[i][j]; }, back.dgu, 2 * s);
                store([&](int i) { return u[i][j]; }, back.dgu + s, 2 * s);
                store([&](int i) { return d[i]; }, hidden, s);
            }
            if (back.dgp) {
                ffn_barrier<63>();
                for (int32_t row = threadIdx.x; row < tile.rows; row += S::kThreads) {
                    float v = 0.0f;
#pragma unroll
                    for (int w = 0; w < S::kWavesS; ++w) v += dsum[w][row];
                    back.dgp[(int64_t)(s0 / S::kUnits) * n + tile.row0 + row] = v;
                }
            }
        }
    });
}

}  // namespace more
