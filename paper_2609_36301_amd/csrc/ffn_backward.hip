// Backward pass of the experts' gated feed-forward block (ffn.hip) for gfx950, with recompute.  Given
// du [T][h], the gradient with respect to sum_j y[t k + j], for every entry p = t k + j of expert e:
//   G = x_t Wg^T, U = x_t Wu^T, sigma = 1 / (1 + e^-G), A = G sigma U         (recomputed)
//   dA0 = du_t W2,  dgate_p = A . dA0,  dA = gate_p dA0
//   dG = dA U sigma (1 + G (1 - sigma)),  dU = dA G sigma
//   dx_t = sum_j [dG dU] W1t[e]
//   dW1t[e] = sum_p [dG dU]^T x_t,  dW2t[e] = sum_p du_t^T (gate_p A)
//
// Kernels of one call (entries in the order of Sort + Count, cut into tiles of one expert):
//   ffn_tiles     lists the tiles
//   ffn_bwd_up    G, U and dA0 of one tile and 64 hidden units: [dG dU] and gate A (bf16, sorted order) and
//                 the partial sums of dgate; tiles of 256 rows take two kernels instead,
//   ffn_bwd_rows  dA0 = du_t W2t[e] (fp32, sorted order), and
//   ffn_up        G and U, with the same results from them and dA0
//   ffn_bwd_rows  [dG dU] W1t[e] per entry (fp32, entry order)
//   ffn_bwd_sum   dx: the k entries of a token added in order; dgate: the partials added in order
//   ffn_bwd_dw    dW1t and dW2t: contractions over the rows of an expert; an expert without rows gets
//                 zeros
// Every sum runs in a fixed order: nothing is added atomically, and a call gives the same bits on every
// run.  Numerics: bf16 operands with fp32 accumulation; [dG dU] and gate A are rounded to bf16 once (the
// matrix cores' operand type), or to two bf16 addends (FfnPlan::planes), the entries' shares of dx stay in fp32
// until they are summed, dgate comes from unrounded fp32 values.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "ffn.h"
#include "ffn_device.h"
#include "ffn_up.h"

namespace more {

// ------------------------------------------------------------------------------ up, tiles of up to 128 rows
// (Two kernels for tiles of 256 rows: there the matrix products count, a tile of 128 hidden units halves
// what the caches deliver, and three sets of accumulators do not fit; 32 experts of s = 1024, h = 2048 with
// 1024 rows 565 us against 820.  For 4096 experts of s = 64, h = 512 with 32 rows, where the weights' way from
// memory counts, this one kernel takes 213 us (805 MB of weights: 4.1 TB/s) against 235.)
// A workgroup computes one tile and kUnits hidden units: first G and U (x rows against the gate and up
// rows of W1t), then dA0 (du rows against a column tile of W2t) into other accumulators.  In turn rather
// than side by side: a stage is smaller by the second pair of operands, so twice as many workgroups fit
// a CU (or a tile twice as large).
template <int BM>
struct BwdUpShape {
    static_assert(BM <= 128, "");
    static constexpr int kWaves = 4;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kWavesS = BM >= 64 ? 2 : 4;
    static constexpr int kUnits = 64;
    static constexpr int kS = kUnits / kWavesS / 16;
    static constexpr int kN = BM / (kWaves / kWavesS) / 16;
    static constexpr int kStages = 2;
    static constexpr int kRowsAt = 2 * kUnits * 128;
    static constexpr int kStageBytes = kRowsAt + BM * 128;
};

template <int BM>
__global__ __launch_bounds__(BwdUpShape<BM>::kThreads, 2) void ffn_bwd_up_kernel(
    FfnArgs a, const void* __restrict__ list, uint16_t* __restrict__ hidden, uint16_t* __restrict__ dgu,
    float* __restrict__ dgp) {
    using S = BwdUpShape<BM>;
    __shared__ __attribute__((aligned(1024))) char smem_raw[S::kStages * S::kStageBytes];
    LdsChar* smem = (LdsChar*)smem_raw;
    __shared__ float dsum[S::kWavesS][BM];
    const FfnTile* tiles = ffn_tile_list(list);
    const int32_t s = a.s, h = a.h;
    const int32_t n = a.T * a.k;
    const int32_t cols = (s + S::kUnits - 1) / S::kUnits;
    const int32_t hsteps = (h + kFfnBK - 1) / kFfnBK;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int ws = wave % S::kWavesS, wn = wave / S::kWavesS;
    const int64_t total = (int64_t)*static_cast<const int32_t*>(list) * cols;
    ffn_for_each(total, [&](int64_t item) {
        const FfnTile tile = tiles[item / cols];
        if (tile.expert < 0) return;
        const int32_t col = (int32_t)(item % cols), s0 = col * S::kUnits;
        RowTileLoader<2 * S::kUnits, S::kWaves> weights;
        const uint16_t* W1 = a.W1t + (int64_t)tile.expert * 2 * s * h;
        const uint16_t* W2 = a.W2t + (int64_t)tile.expert * h * s;
        weights.init([&](int i) {
            const int32_t u = min(s0 + i % S::kUnits, s - 1);
            return W1 + (int64_t)(i / S::kUnits * s + u) * h;
        });
        ColTileLoader<S::kUnits, S::kWaves> down;
        down.init();
        RowTileLoader<BM, S::kWaves> rows;
        rows.init([&](int i) {
            const uint32_t p = a.sorted[tile.row0 + min(i, tile.rows - 1)];
            return a.x + (int64_t)(p < (uint32_t)n ? p / (uint32_t)a.k : 0) * h;
        });
        f32x4 g[S::kS][S::kN], u[S::kS][S::kN], d[S::kS][S::kN];
#pragma unroll
        for (int i = 0; i < S::kS; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) g[i][j] = u[i][j] = zero_f32x4();
        const bool live = 16 * wn * S::kN < tile.rows;  // (per wave) some of its rows are wanted
        // the gate rows are one group of M-side fragments, the up rows the other
        using M = FfnFragments<S::kS>;
        using N = FfnFragments<S::kN>;
        ffn_pipeline<S::kStages, 0, 2, false, M, N>(
            (h + kFfnBK - 1) / kFfnBK, live,
            [&](int step, int slot) { rows.load(smem + slot * S::kStageBytes + S::kRowsAt, step * kFfnBK, h); },
            [&](int step, int slot) { weights.load(smem + slot * S::kStageBytes, step * kFfnBK, h); },
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
#pragma unroll
        for (int i = 0; i < S::kS; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) d[i][j] = zero_f32x4();
        const int64_t to_du = a.du - a.x;  // (elements; the same rows of the other tensor)
#pragma unroll
        for (int i = 0; i < rows.kLoads; ++i) rows.p[i] += to_du;
        using G = FfnGroups<S::kS>;
        using M2 = FfnFragments<G::kSize>;
        using Stage = StagePair<decltype(rows), decltype(down)>;
        ffn_pipeline_staged<Stage, 2, M2, N>(
            hsteps, live,
            [&](int step, Stage& st) {
                const int32_t k0 = step * kFfnBK;
                rows.fetch(st.a, k0, h);
                down.fetch(st.b, s - s0, [&](int i) {
                    const int kappa = k0 + down.row(i);
                    return kappa < h ? W2 + (int64_t)kappa * s + s0 : nullptr;
                });
            },
            [&](int slot, const Stage& st) {
                rows.put(smem + slot * S::kStageBytes + S::kRowsAt, st.a);
                down.put(smem + slot * S::kStageBytes, st.b);
            },
            ffn_work(
                [&](int slot, int kk, int group, M2& m) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < S::kS)
                            m.v[i] = col_fragment(smem + slot * S::kStageBytes, 16 * (ws * S::kS + G::tile(group, i)), kk);
                },
                [&](int slot, int kk, N& f) {
#pragma unroll
                    for (int j = 0; j < S::kN; ++j)
                        f.v[j] = row_fragment(smem + slot * S::kStageBytes + S::kRowsAt, 16 * (wn * S::kN + j), kk);
                },
                [&](int group, const M2& m, const N& f) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < S::kS)
#pragma unroll
                            for (int j = 0; j < S::kN; ++j) {
                                f32x4& c = d[G::tile(group, i)][j];
                                c = mfma_16x16x32(m.v[i], f.v[j], c);
                            }
                },
                [] {}));
        // lane l holds token l % 16 and hidden units 4 (l / 16) .. + 3 of each 16 x 16 tile
#pragma unroll
        for (int j = 0; j < S::kN; ++j) {
            const int32_t row = 16 * (wn * S::kN + j) + (lane & 15);
            const bool live = row < tile.rows;
            const uint32_t p = live ? (uint32_t)a.sorted[tile.row0 + row] : 0xFFFFFFFFu;
            const float gate = a.gate && p < (uint32_t)n ? a.gate[p] : 1.0f;
            const int64_t at = tile.row0 + row;
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < S::kS; ++i) {
                const int32_t c = s0 + 16 * (ws * S::kS + i) + 4 * (lane >> 4);
                float A[4], dG[4], dU[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float sig = ffn_sigmoid(g[i][j][q]);
                    const float silu = g[i][j][q] * sig;
                    A[q] = silu * u[i][j][q];
                    const float dA = gate * d[i][j][q];
                    dG[q] = dA * u[i][j][q] * (sig + silu * (1.0f - sig));
                    dU[q] = dA * silu;
                    // units past s repeat unit s - 1 and have no share
                    dot = c < s ? __builtin_fmaf(A[q], d[i][j][q], dot) : dot;
                    A[q] *= gate;
                }
                if (live && c < s) {
                    *reinterpret_cast<uint2*>(hidden + at * s + c) = pack_bf16x4(A[0], A[1], A[2], A[3]);
                    *reinterpret_cast<uint2*>(dgu + at * 2 * s + c) = pack_bf16x4(dG[0], dG[1], dG[2], dG[3]);
                    *reinterpret_cast<uint2*>(dgu + at * 2 * s + s + c) = pack_bf16x4(dU[0], dU[1], dU[2], dU[3]);
                    if (a.planes > 1) {
                        uint16_t *h1 = hidden + (int64_t)n * s, *g1 = dgu + (int64_t)n * 2 * s;
                        *reinterpret_cast<uint2*>(h1 + at * s + c) = pack_bf16_rest(A[0], A[1], A[2], A[3]);
                        *reinterpret_cast<uint2*>(g1 + at * 2 * s + c) = pack_bf16_rest(dG[0], dG[1], dG[2], dG[3]);
                        *reinterpret_cast<uint2*>(g1 + at * 2 * s + s + c) = pack_bf16_rest(dU[0], dU[1], dU[2], dU[3]);
                    }
                }
            }
            dot += __shfl_xor(dot, 16, 64);
            dot += __shfl_xor(dot, 32, 64);
            if (lane < 16) dsum[ws][row] = dot;
        }
        if (dgp) {
            ffn_barrier<63>();
            for (int32_t row = threadIdx.x; row < tile.rows; row += S::kThreads) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < S::kWavesS; ++w) v += dsum[w][row];
                dgp[(int64_t)col * n + tile.row0 + row] = v;
            }
        }
    });
}

// ------------------------------------------------------------------------------ rows times weights
// out = rows W[e] with fp32 results, for the two products whose weights lie with the contraction axis
// slowest: dA0 = du W2t[e] (the token's row of du, contraction over h, results in sorted order) and the
// entries' shares of dx = [dG dU] W1t[e] (contraction over 2s, results in entry order).  The weights are a
// column tile (M side), the rows a row tile (N side).  A workgroup computes `span` columns in steps of
// kCols; the pipeline runs over (column step, contraction step) pairs.  Bound like the forward pass: 32 experts
// of h = 2048, s = 1024 with 1024 rows, dA0 213 us (645 TFLOP/s), dx 367 us (749 TFLOP/s) on tiles of 256 rows
// and 476 us on tiles of 128; 4096 experts of h = 512, s = 64 with 32 rows, dx 164 us (840 MB, 5.1 TB/s).
// The shares of dx go through memory in fp32, a third of that traffic: in bf16 dx would carry k + 1 roundings
// for one.
constexpr int rows_threads(int bm) { return bm == 256 ? 512 : 256; }
template <int BM>
struct RowsShape {
    static constexpr int kThreads = rows_threads(BM);
    static constexpr int kWaves = kThreads / 64;
    static constexpr int kCols = BM == 256 ? 256 : 128;
    static constexpr int kWavesM = BM >= 64 ? 2 : 4;
    static constexpr int kM = kCols / kWavesM / 16;
    static constexpr int kN = BM / (kWaves / kWavesM) / 16;
    static constexpr int kRowsAt = kCols * 128;
    static constexpr int kStageBytes = kRowsAt + BM * 128;
};

template <int BM, bool TOKENS>
__global__ __launch_bounds__(rows_threads(BM), 2) void ffn_bwd_rows_kernel(
    FfnArgs a, const void* __restrict__ list, const uint16_t* __restrict__ rows_in, const uint16_t* __restrict__ W,
    int32_t len, int32_t cols, int32_t span, float* __restrict__ out) {
    using S = RowsShape<BM>;
    __shared__ __attribute__((aligned(1024))) char smem_raw[2 * S::kStageBytes];
    LdsChar* smem = (LdsChar*)smem_raw;
    const FfnTile* tiles = ffn_tile_list(list);
    const int32_t n = a.T * a.k;
    const int32_t spans = (cols + span - 1) / span;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int wm = wave % S::kWavesM, wn = wave / S::kWavesM;
    const int64_t total = (int64_t)*static_cast<const int32_t*>(list) * spans;
    ffn_for_each(total, [&](int64_t item) {
        const FfnTile tile = tiles[item / spans];
        if (tile.expert < 0) return;  // dropped entries have no share (ffn_bwd_sum leaves them out)
        const int32_t c0 = (int32_t)(item % spans) * span, c1 = min(cols, c0 + span);
        const uint16_t* We = W + (int64_t)tile.expert * len * cols;
        RowTileLoader<BM, S::kWaves> rows;
        rows.init([&](int i) {
            const int32_t at = tile.row0 + min(i, tile.rows - 1);
            if constexpr (!TOKENS) return rows_in + (int64_t)at * len;
            const uint32_t p = a.sorted[at];
            return rows_in + (int64_t)(p < (uint32_t)n ? p / (uint32_t)a.k : 0) * len;
        });
        ColTileLoader<S::kCols, S::kWaves> weights;
        weights.init();
        int64_t place[S::kN];  // of the lane's rows in out; -1: not wanted
#pragma unroll
        for (int j = 0; j < S::kN; ++j) {
            const int32_t row = 16 * (wn * S::kN + j) + (lane & 15);
            place[j] = row < tile.rows ? tile.row0 + row : -1;
            if (!TOKENS && row < tile.rows) {
                const uint32_t p = (uint32_t)a.sorted[tile.row0 + row];
                place[j] = p < (uint32_t)n ? (int64_t)p : -1;
            }
        }
        f32x4 acc[S::kM][S::kN];
#pragma unroll
        for (int i = 0; i < S::kM; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) acc[i][j] = zero_f32x4();
        const int32_t ksteps = (len + kFfnBK - 1) / kFfnBK, kall = TOKENS ? ksteps : ksteps * a.planes;
        const int32_t csteps = (c1 - c0 + S::kCols - 1) / S::kCols;
        // (column step, contraction step) of the next load and of the next product
        int32_t lc = c0, lk = 0, cc = c0, ck = 0;
        using G = FfnGroups<S::kM, S::kM == 8 ? 4 : 2>;
        using M = FfnFragments<G::kSize>;
        using N = FfnFragments<S::kN>;
        auto weight_row = [&](int i) -> const uint16_t* {
            const int kappa = (lk < ksteps ? lk : lk - ksteps) * kFfnBK + weights.row(i);
            return kappa < len ? We + (int64_t)kappa * cols + lc : nullptr;
        };
        auto advance = [&] {
            if (++lk < kall) return;
            lk = 0;
            lc += S::kCols;
        };
        auto read_n = [&](int slot, int kk, N& f) {
#pragma unroll
            for (int j = 0; j < S::kN; ++j)
                f.v[j] = row_fragment(smem + slot * S::kStageBytes + S::kRowsAt, 16 * (wn * S::kN + j), kk);
        };
        auto multiply = [&](int group, const M& m, const N& f) {
#pragma unroll
            for (int i = 0; i < G::kSize; ++i)
                if (G::tile(group, i) < S::kM)
#pragma unroll
                    for (int j = 0; j < S::kN; ++j) {
                        f32x4& c = acc[G::tile(group, i)][j];
                        c = mfma_16x16x32(m.v[i], f.v[j], c);
                    }
        };
        auto done = [&] {
            if (++ck < kall) return;
#pragma unroll
            for (int j = 0; j < S::kN; ++j) {
#pragma unroll
                for (int i = 0; i < S::kM; ++i) {
                    const int32_t c = cc + 16 * (wm * S::kM + i) + 4 * (lane >> 4);
                    if (place[j] >= 0 && c < c1)
                        *reinterpret_cast<f32x4*>(out + place[j] * cols + c) = acc[i][j];
                    acc[i][j] = zero_f32x4();
                }
            }
            ck = 0;
            cc += S::kCols;
        };
        if constexpr (BM == 256) {
            constexpr int kLoads = weights.kLoads + rows.kLoads;
            ffn_pipeline<2, kLoads, G::kGroups, true, M, N>(
                kall * csteps, 16 * wn * S::kN < tile.rows,
                [&](int, int slot) { weights.load(smem + slot * S::kStageBytes, cols - lc, weight_row); },
                [&](int, int slot) {
                    const int32_t k0 = (lk < ksteps ? lk : lk - ksteps) * kFfnBK;
                    rows.load(smem + slot * S::kStageBytes + S::kRowsAt, k0, len, lk < ksteps ? 0 : (int64_t)n * len);
                    advance();
                },
                ffn_work(
                    [&](int slot, int kk, int group, M& m) {
                        col_fragments2(smem + slot * S::kStageBytes, 16 * (wm * S::kM + G::tile(group, 0)), kk, m.v[0],
                                       m.v[1]);
                    },
                    read_n, multiply, done));
        } else {
            using Stage = StagePair<decltype(weights), decltype(rows)>;
            ffn_pipeline_staged<Stage, G::kGroups, M, N>(
                kall * csteps, 16 * wn * S::kN < tile.rows,
                [&](int, Stage& st) {
                    weights.fetch(st.a, cols - lc, weight_row);
                    const int32_t k0 = (lk < ksteps ? lk : lk - ksteps) * kFfnBK;
                    rows.fetch(st.b, k0, len, lk < ksteps ? 0 : (int64_t)n * len);
                    advance();
                },
                [&](int slot, const Stage& st) {
                    weights.put(smem + slot * S::kStageBytes, st.a);
                    rows.put(smem + slot * S::kStageBytes + S::kRowsAt, st.b);
                },
                ffn_work(
                    [&](int slot, int kk, int group, M& m) {
#pragma unroll
                        for (int i = 0; i < G::kSize; ++i)
                            if (G::tile(group, i) < S::kM)
                                m.v[i] = col_fragment(smem + slot * S::kStageBytes,
                                                      16 * (wm * S::kM + G::tile(group, i)), kk);
                    },
                    read_n, multiply, done));
        }
    });
}

// ------------------------------------------------------------------------------ sums over the entries
// A thread adds eight columns of a token's k rows in order; dropped entries (id outside [0, M)) are left
// out.  The threads past the columns add the partials of dgate.  Memory-bound: 302 MB (h = 2048, 32768 entries)
// in 55 us, 5.5 TB/s.
__global__ __launch_bounds__(256) void ffn_bwd_sum_kernel(const float* __restrict__ dxs, const int32_t* __restrict__ idx,
                                                       int32_t T, int32_t h, int32_t M, int32_t k,
                                                       uint16_t* __restrict__ dx, int64_t colblocks,
                                                       const float* __restrict__ dgp, int32_t parts,
                                                       const int32_t* __restrict__ sorted,
                                                       float* __restrict__ dgate) {
    const int32_t n = T * k;
    const int32_t h8 = h / 8;
    if ((int64_t)blockIdx.x < colblocks) {
        const int64_t total = (int64_t)T * h8;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += colblocks * 256) {
            const int64_t t = i / h8;
            const int32_t c = (int32_t)(i - t * h8) * 8;
            f32x4 a = zero_f32x4(), b = zero_f32x4();
            for (int32_t j = 0; j < k; ++j) {
                const int64_t p = t * k + j;
                if ((uint32_t)idx[p] >= (uint32_t)M) continue;
                const f32x4* v = reinterpret_cast<const f32x4*>(dxs + p * h + c);
                a += v[0];
                b += v[1];
            }
            const uint2 lo = pack_bf16x4(a[0], a[1], a[2], a[3]), hi = pack_bf16x4(b[0], b[1], b[2], b[3]);
            *reinterpret_cast<u32x4*>(dx + t * h + c) = u32x4{lo.x, lo.y, hi.x, hi.y};
        }
        return;
    }
    const int64_t blocks = (int64_t)gridDim.x - colblocks;
    for (int64_t i = ((int64_t)blockIdx.x - colblocks) * 256 + threadIdx.x; i < n; i += blocks * 256) {
        const uint32_t p = (uint32_t)sorted[i];
        if (p >= (uint32_t)n) continue;
        float v = 0.0f;
        if ((uint32_t)idx[p] < (uint32_t)M)
            for (int32_t c = 0; c < parts; ++c) v += dgp[(int64_t)c * n + i];
        dgate[p] = v;
    }
}

// ------------------------------------------------------------------------------ weight gradients
// out[e] [rows_out][cols_out] = sum over the entries i of expert e of Q[i][row] P[i][col], both operands
// column tiles (the contraction runs over rows).  dW1t: P = x of the entry's token (cols h), Q = [dG dU]
// (rows 2s).  dW2t: P = gate A (cols s), Q = du of the entry's token (rows h).  The gathered operand is the
// one along h; a workgroup computes a tile of RT rows and CT columns after the other over `hspan` of h, and
// the pipeline runs over (tile, 64 entries) pairs, so that the few rows of a small expert do not drain it.
// PARTS: the entries of an expert are cut into `parts` runs and a workgroup takes one tile and one run; the
// fp32 results of run i go to parts_out + i part_stride, and ffn_bwd_dw_sum adds them.  ONCE: nontemporal
// stores.
// Bound by the gradients' way to memory where experts are small (4096 of h = 512, s = 64 with 32 rows 236 us, 805 MB
// written, 134 read: 4.0 TB/s), by the products' stages where they are large (32 of h = 2048, s = 1024 with
// 1024 rows 540 us, 763 TFLOP/s).
struct DwArgs {
    const uint16_t *P, *Q;
    int32_t rows_out, cols_out, hspan, blocks;  // workgroups of this product
    uint16_t* out;
    int32_t planes, parts;
    float* parts_out;
    int64_t part_stride;
};

template <int CT, int RT, int WAVES, bool GATHER_P, bool PARTS, bool ONCE>
__device__ __forceinline__ void ffn_bwd_dw(const DwArgs& d, const int32_t* __restrict__ offsets,
                                           const int32_t* __restrict__ sorted, int32_t n, int32_t k, int32_t M,
                                           LdsChar* smem, LdsChar* scratch, int32_t block) {
    const uint16_t *P = d.P, *Q = d.Q;
    const int32_t rows_out = d.rows_out, cols_out = d.cols_out, hspan = d.hspan;
    uint16_t* out = d.out;
    constexpr int kStageBytes = (CT + RT) * 128;
    constexpr int kWavesM = CT >= 128 ? 2 : 1, kWavesN = WAVES / kWavesM;
    constexpr int kM = CT / kWavesM / 16, kN = RT / kWavesN / 16;  // 16 x 16 tiles per wave
    static_assert(kM % 4 == 0, "whole lines of out: 64 columns");
    using PLoader = ColTileLoader<CT, WAVES>;
    using QLoader = ColTileLoader<RT, WAVES>;
    constexpr int kGathered = PLoader::kGroups;  // rows per lane of either operand
    const int wm = ffn_wave() % kWavesM, wn = ffn_wave() / kWavesM;
    constexpr int kStep = GATHER_P ? CT : RT;  // of h
    const int32_t h = GATHER_P ? cols_out : rows_out;
    const int32_t spans = (h + hspan - 1) / hspan;
    const int32_t others = GATHER_P ? (rows_out + RT - 1) / RT : (cols_out + CT - 1) / CT;
    // Items in turn over the XCDs: the parts of an expert run on all of them, so that experts with many
    // entries load them alike.
    const int32_t runs = PARTS ? d.parts : 1;
    for (int64_t work = block; work < (int64_t)M * spans * others * runs; work += d.blocks) {
        const int32_t run = PARTS ? (int32_t)(work % runs) : 0;
        const int64_t item = PARTS ? work / runs : work;
        const int32_t e = (int32_t)(item / (spans * others)), q = (int32_t)(item % (spans * others));
        const int32_t h0 = (q % spans) * hspan, h1 = min(h, h0 + hspan);
        const int32_t other = (q / spans) * (GATHER_P ? RT : CT);  // first row (column) of the other side
        int32_t begin = min(max(offsets[e], 0), n), end = min(max(offsets[e + 1], begin), n);
        if constexpr (PARTS) {  // whole stages
            const int32_t len = ((end - begin + runs - 1) / runs + kFfnBK - 1) / kFfnBK * kFfnBK;
            begin = (int32_t)min((int64_t)begin + (int64_t)run * len, (int64_t)end);
            end = (int32_t)min((int64_t)begin + len, (int64_t)end);
        }
        PLoader pl;
        QLoader ql;
        pl.init();
        ql.init();
        const int32_t ksteps = (end - begin + kFfnBK - 1) / kFfnBK, kall = ksteps * d.planes;
        const int32_t hsteps = (h1 - h0 + kStep - 1) / kStep;
        // the gathered operand's entries of the next load (read one load ahead)
        int32_t entry[kGathered];
        auto fetch = [&](int32_t step) {
#pragma unroll
            for (int i = 0; i < kGathered; ++i) {
                const int32_t at = begin + step * kFfnBK + pl.row(i);
                entry[i] = at < end ? sorted[at] : -1;
            }
        };
        auto gathered = [&](int i, const uint16_t* base, int32_t stride) -> const uint16_t* {
            const uint32_t p = (uint32_t)entry[i];
            return p < (uint32_t)n ? base + (int64_t)(p / (uint32_t)k) * stride : nullptr;
        };
        f32x4 acc[kM][kN];
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j) acc[i][j] = zero_f32x4();
        int32_t lh = h0, lk = 0, ch = h0, ck = 0;
        auto store = [&] {
            if constexpr (PARTS) {
                float* o = d.parts_out + run * d.part_stride + (int64_t)e * rows_out * cols_out;
#pragma unroll
                for (int j = 0; j < kN; ++j)
#pragma unroll
                    for (int i = 0; i < kM; ++i) {
                        const int32_t c = (GATHER_P ? ch : other) + 16 * (wm * kM + i) + 4 * (ffn_lane() >> 4);
                        const int32_t r = (GATHER_P ? other : ch) + 16 * (wn * kN + j) + (ffn_lane() & 15);
                        if (c < (GATHER_P ? h1 : cols_out) && r < (GATHER_P ? rows_out : h1))
                            *reinterpret_cast<f32x4*>(o + (int64_t)r * cols_out + c) = acc[i][j];
                        acc[i][j] = zero_f32x4();
                    }
                ch += kStep;
                return;
            }
            uint16_t* o = out + (int64_t)e * rows_out * cols_out;
#pragma unroll
            for (int j = 0; j < kN; ++j)
#pragma unroll
                for (int i0 = 0; i0 < kM; i0 += 4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        place_bf16(scratch, i, acc[i0 + i][j]);
                        acc[i0 + i][j] = zero_f32x4();
                    }
                    const int32_t c = (GATHER_P ? ch : other) + 16 * (wm * kM + i0);
                    const int32_t r = (GATHER_P ? other : ch) + 16 * (wn * kN + j);
                    flush_rows<ONCE>(scratch, ((GATHER_P ? h1 : cols_out) - c) * 2, [&](int row) {
                        return r + row < (GATHER_P ? rows_out : h1) ? o + (int64_t)(r + row) * cols_out + c : nullptr;
                    });
                }
            ch += kStep;
        };
        if (ksteps == 0) {  // no entries: zeros
            if constexpr (PARTS) {
                for (int32_t step = 0; step < hsteps; ++step) store();
            } else {  // the expert's items share its matrix in runs of whole lines
                const int64_t pieces = (int64_t)rows_out * cols_out / 8;
                const int64_t share = (pieces / (spans * others) + 8) / 8 * 8;
                u32x4* o = reinterpret_cast<u32x4*>(out + (int64_t)e * rows_out * cols_out);
                const int64_t last = min(pieces, (q + 1) * share);
                for (int64_t i = q * share + threadIdx.x; i < last; i += 64 * WAVES)
                    __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, o + i);
            }
            continue;
        }
        using G = FfnGroups<kM, kM == 8 ? 4 : 2>;
        using MF = FfnFragments<G::kSize>;
        using NF = FfnFragments<kN>;
        using Stage = StagePair<PLoader, QLoader>;
        fetch(0);
        ffn_pipeline_staged<Stage, G::kGroups, MF, NF>(
            kall * hsteps, true,
            [&](int, Stage& st) {
                const bool rest = lk >= ksteps;  // the second plane of the operand that is not gathered
                const int32_t i0 = begin + (rest ? lk - ksteps : lk) * kFfnBK;
                const int64_t first = rest ? n : 0;
                const int32_t c = GATHER_P ? lh : other, r = GATHER_P ? other : lh;
                pl.fetch(st.a, cols_out - c, [&](int i) -> const uint16_t* {
                    if constexpr (GATHER_P) return gathered(i, P + c, cols_out);
                    const int32_t row = i0 + pl.row(i);
                    return row < end ? P + (first + row) * cols_out + c : nullptr;
                });
                ql.fetch(st.b, rows_out - r, [&](int i) -> const uint16_t* {
                    if constexpr (!GATHER_P) return gathered(i, Q + r, rows_out);
                    const int32_t row = i0 + ql.row(i);
                    return row < end ? Q + (first + row) * rows_out + r : nullptr;
                });
                if (++lk == kall) {
                    lk = 0;
                    lh += kStep;
                }
                if (ksteps > 1) fetch(lk < ksteps ? lk : lk - ksteps);
            },
            [&](int slot, const Stage& st) {
                pl.put(smem + slot * kStageBytes, st.a);
                ql.put(smem + slot * kStageBytes + CT * 128, st.b);
            },
            ffn_work(
                [&](int slot, int kk, int group, MF& m) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < kM)
                            m.v[i] = col_fragment(smem + slot * kStageBytes, 16 * (wm * kM + G::tile(group, i)), kk);
                },
                [&](int slot, int kk, NF& f) {
#pragma unroll
                    for (int j = 0; j < kN; ++j)
                        f.v[j] = col_fragment(smem + slot * kStageBytes + CT * 128, 16 * (wn * kN + j), kk);
                },
                [&](int group, const MF& m, const NF& f) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < kM)
#pragma unroll
                            for (int j = 0; j < kN; ++j) {
                                f32x4& c = acc[G::tile(group, i)][j];
                                c = mfma_16x16x32(m.v[i], f.v[j], c);
                            }
                },
                [&] {
                    if (++ck < kall) return;
                    ck = 0;
                    store();
                }));
    }
}

// Both products in one launch (the second one's workgroups follow the first one's, so that the last of one
// and the first of the other share the chip).
template <int CT1, int CT2, int RT, int WAVES, bool PARTS, bool ONCE2>
__global__ __launch_bounds__(64 * WAVES, 2) void ffn_bwd_dw_kernel(DwArgs w1, DwArgs w2,
                                                                const int32_t* __restrict__ offsets,
                                                                const int32_t* __restrict__ sorted, int32_t n,
                                                                int32_t k, int32_t M) {
    __shared__ __attribute__((aligned(1024))) char smem_raw[2 * (CT1 + RT) * 128];
    __shared__ __attribute__((aligned(16))) char scratch_raw[WAVES * kFfnScratch];
    LdsChar* smem = (LdsChar*)smem_raw;
    LdsChar* scratch = (LdsChar*)scratch_raw + ffn_wave() * kFfnScratch;
    const int32_t block = (int32_t)blockIdx.x;
    if (block < w1.blocks)
        ffn_bwd_dw<CT1, RT, WAVES, true, PARTS, true>(w1, offsets, sorted, n, k, M, smem, scratch, block);
    else
        ffn_bwd_dw<CT2, RT, WAVES, false, PARTS, ONCE2>(w2, offsets, sorted, n, k, M, smem, scratch, block - w1.blocks);
}

// Adds the runs' partial gradients in order: a thread takes eight values, of dW1t and behind them of dW2t.
__global__ __launch_bounds__(256) void ffn_bwd_dw_sum_kernel(const float* __restrict__ parts, int32_t count,
                                                          int64_t stride, int64_t size1, uint16_t* __restrict__ dW1t,
                                                          uint16_t* __restrict__ dW2t) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < stride; i += (int64_t)gridDim.x * 256 * 8) {
        f32x4 a = zero_f32x4(), b = zero_f32x4();
#pragma unroll 4
        for (int32_t q = 0; q < count; ++q) {
            const f32x4* v = reinterpret_cast<const f32x4*>(parts + q * stride + i);
            a += v[0];
            b += v[1];
        }
        const uint2 lo = pack_bf16x4(a[0], a[1], a[2], a[3]), hi = pack_bf16x4(b[0], b[1], b[2], b[3]);
        *reinterpret_cast<u32x4*>(i < size1 ? dW1t + i : dW2t + (i - size1)) = u32x4{lo.x, lo.y, hi.x, hi.y};
    }
}

// ------------------------------------------------------------------------------ host
namespace {

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }
constexpr int64_t kMaxBlocks = 1 << 19;
unsigned grid_of(int64_t items) {
    return (unsigned)(std::min<int64_t>((items + 7) / 8, kMaxBlocks / 8) * 8);
}

// Elements of both weight gradients.
int64_t dw_size(int32_t h, int32_t s, int32_t M) { return (int64_t)M * 3 * s * h; }

// Workgroups along the hidden units: a partial sum of dgate each.
int32_t dgate_parts(const FfnPlan& p, int32_t s) {
    const int32_t units = p.bm == 256 ? UpShape<256>::kUnits : BwdUpShape<128>::kUnits;
    return (s + units - 1) / units;
}

template <int BM>
void rows_launch(const FfnPlan& p, const FfnArgs& a, char* ws, hipStream_t stream) {
    using R = RowsShape<BM>;
    const void* list = ws + p.off_tiles;
    uint16_t* hidden = reinterpret_cast<uint16_t*>(ws + p.off_hidden);
    uint16_t* dgu = reinterpret_cast<uint16_t*>(ws + p.off_dgu);
    float* dgp = a.dgate ? reinterpret_cast<float*>(ws + p.off_dgp) : nullptr;
    const unsigned up_blocks = grid_of(p.tiles * dgate_parts(p, a.s));
    if constexpr (BM == 256) {
        float* dA0 = reinterpret_cast<float*>(ws + p.off_da0);
        const int32_t span = p.da0_span;
        ffn_bwd_rows_kernel<BM, true><<<grid_of(p.tiles * ((a.s + span - 1) / span)), R::kThreads, 0, stream>>>(
            a, list, a.du, a.W2t, a.h, a.s, span, dA0);
        ffn_up_kernel<BM, true><<<up_blocks, UpShape<BM>::kThreads, 0, stream>>>(a, list, hidden,
                                                                              UpBackward{dA0, dgu, dgp});
    } else {
        ffn_bwd_up_kernel<BM><<<up_blocks, BwdUpShape<BM>::kThreads, 0, stream>>>(a, list, hidden, dgu, dgp);
    }
    ffn_bwd_rows_kernel<BM, false><<<grid_of(p.tiles * ((a.h + p.span - 1) / p.span)), R::kThreads, 0, stream>>>(
        a, list, dgu, a.W1t, 2 * a.s, a.h, p.span, reinterpret_cast<float*>(ws + p.off_dxs));
}

// One weight gradient: `others` tiles across h, `hspan` of h to a workgroup.
DwArgs dw_args(const FfnPlan& p, const FfnArgs& a, const uint16_t* P, const uint16_t* Q, int32_t rows, int32_t cols,
               int32_t others, int32_t hspan, uint16_t* out, float* parts_out) {
    DwArgs d;
    d.P = P;
    d.Q = Q;
    d.rows_out = rows;
    d.cols_out = cols;
    d.planes = p.planes;
    d.parts = p.dw_parts;
    d.parts_out = parts_out;
    d.part_stride = dw_size(a.h, a.s, a.M);
    d.hspan = hspan;
    d.blocks = (int32_t)grid_of((int64_t)a.M * others * ((a.h + hspan - 1) / hspan) * d.parts);
    d.out = out;
    return d;
}

template <int CT1, int CT2, int RT, int WAVES, bool PARTS, bool ONCE2>
void dw_launch(const FfnPlan& p, const FfnArgs& a, char* ws, hipStream_t stream) {
    const uint16_t* hidden = reinterpret_cast<const uint16_t*>(ws + p.off_hidden);
    const uint16_t* dgu = reinterpret_cast<const uint16_t*>(ws + p.off_dgu);
    float* parts = reinterpret_cast<float*>(ws + p.off_dwp);
    const int64_t size1 = (int64_t)a.M * 2 * a.s * a.h;
    const DwArgs w1 = dw_args(p, a, a.x, dgu, 2 * a.s, a.h, (2 * a.s + RT - 1) / RT, p.dw1_span, a.dW1t, parts);
    const DwArgs w2 = dw_args(p, a, hidden, a.du, a.h, a.s, (a.s + CT2 - 1) / CT2, p.dw2_span, a.dW2t, parts + size1);
    ffn_bwd_dw_kernel<CT1, CT2, RT, WAVES, PARTS, ONCE2><<<(unsigned)(w1.blocks + w2.blocks), 64 * WAVES, 0, stream>>>(
        w1, w2, a.offsets, a.sorted, (int32_t)p.n, a.k, a.M);
    if (PARTS) {
        const int64_t size = dw_size(a.h, a.s, a.M);
        ffn_bwd_dw_sum_kernel<<<(unsigned)std::min<int64_t>((size / 8 + 255) / 256, 1 << 14), 256, 0, stream>>>(
            parts, p.dw_parts, size, size1, a.dW1t, a.dW2t);
    }
}

// Tile size of the weight gradients, by the same cost as the rows' tiles (call in us, 256 : 128, 32 experts of
// h = 2048, s = 1024 with 1024 rows 1402 : 1658, a dense block of 16384 rows 854 : 697, whose 96 large tiles leave
// most CUs idle), and the runs into which an expert's entries are cut: as many as bring the tiles to 512, of
// four stages at least, and at most 32 (runs : us of the call, a dense block of h = 512, s = 128, 16384 rows 1 : 343,
// 8 : 97, 32 : 76, 64 : 85; 1024 rows 1 : 49, 4 : 41, 16 : 43; four experts of h = 2016, s = 8, 12000 rows 1 : 509,
// 2 : 407, 4 : 383, 16 : 400; two of h = 1024, s = 512, 4096 rows 1 : 191, 2 : 162, 8 : 186; and where there are
// 512 tiles and more, h = 2048, s = 1024, 16384 rows 1 : 697, 2 : 715).  The means of all experts decide: an expert
// that far more tokens select than others belongs to few workgroups (4096 experts of h = 512, s = 64, 16384
// tokens, k = 8: 622 us with experts chosen evenly, 1699 where every token selects one of them).
void dw_plan(int64_t n, int32_t h, int32_t s, int32_t M, FfnPlan* p) {
    const int64_t steps = std::max<int64_t>(1, n / M / kFfnBK);
    auto tiles = [&](int32_t a, int32_t b) { return (int64_t)((a + b - 1) / b); };
    const int64_t large = M * tiles(h, 256) * (tiles(2 * s, 256) + tiles(s, 256));
    const int64_t small = M * tiles(h, 128) * (tiles(2 * s, 128) + (tiles(s, 64) + 1) / 2);
    p->dw_tile = ffn_cost(large, steps, 256) < ffn_cost(small, steps, 128) ? 256 : 128;
    p->dw_parts = 1;
    if (p->dw_tile == 128) p->dw_parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>({512 / small, steps / 4, 32}));
    const int32_t step = p->dw_tile, len = (int32_t)std::min<int64_t>(n / M, 1 << 20);
    const int64_t groups1 = M * tiles(2 * s, step), groups2 = M * tiles(s, step == 256 ? 256 : 64);
    p->dw1_span = p->dw_parts > 1 ? step : ffn_span(len, step, groups1, h);
    p->dw2_span = p->dw_parts > 1 ? step : ffn_span(len, step, groups2, h);
}

// Rows of a tile, as in the forward pass (over the same 196 shapes 0.6% off the best on geometric mean, at
// most 18%; us for 64 : 128 : 256 rows, 32 experts of h = 2048, s = 1024, 96 rows 357 : 294 : 338, 384 rows 775 :
// 719 : 594; 4096 experts of h = 512, s = 64, 32 rows 622 : 663 : 1030).
int32_t backward_rows(int64_t n, int32_t h, int32_t s, int32_t M, int32_t planes) {
    if (n / std::max<int64_t>(1, std::min<int64_t>(n, M)) < 24) return 32;
    const int32_t most = planes == 2 ? 128 : 256;  // (the kernels of 256 rows write one plane)
    int32_t best = 64;
    int64_t least = INT64_MAX;
    const int64_t hsteps = (h + kFfnBK - 1) / kFfnBK, ssteps = (2 * s + kFfnBK - 1) / kFfnBK;
    auto parts = [](int32_t v, int32_t size) { return (int64_t)((v + size - 1) / size); };
    for (int32_t bm = 64; bm <= most; bm *= 2) {
        const int64_t tiles2 = ffn_expected_tiles2(n, M, bm);
        int64_t cost;
        if (bm == 256) {
            cost = ffn_cost(tiles2 * parts(s, RowsShape<256>::kCols) / 2, hsteps, bm) +
                   ffn_cost(tiles2 * parts(s, UpShape<256>::kUnits) / 2, hsteps, bm) +
                   ffn_cost(tiles2 * parts(h, RowsShape<256>::kCols) / 2, ssteps, bm);
        } else {
            cost = ffn_cost(tiles2 * parts(s, BwdUpShape<128>::kUnits) / 2, 2 * hsteps, bm) +
                   ffn_cost(tiles2 * parts(h, RowsShape<128>::kCols) / 2, ssteps, bm);
        }
        if (cost < least) {
            least = cost;
            best = bm;
        }
    }
    return best;
}

}  // namespace

void ffn_backward_make_plan(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends, FfnPlan* p) {
    const int32_t planes = addends == 2 || T * k * s <= kFfnTwoPlanes ? 2 : 1;
    ffn_tiles_plan(T * k, M, backward_rows(T * k, h, s, M, planes), p);
    p->planes = planes;
    dw_plan(p->n, h, s, M, p);
    const int32_t cols = p->bm == 256 ? RowsShape<256>::kCols : RowsShape<128>::kCols;
    p->span = ffn_span(2 * s, cols, p->tiles, h);
    p->da0_span = ffn_span(h, cols, p->tiles, s);
    size_t at = p->workspace_bytes;
    p->off_hidden = at;
    at += align256((size_t)p->n * s * 2 * p->planes);
    p->off_dgu = at;
    at += align256((size_t)p->n * 2 * s * 2 * p->planes);
    p->off_da0 = at;
    at += p->bm == 256 ? align256((size_t)p->n * s * 4) : 0;
    p->off_dxs = at;
    at += align256((size_t)p->n * h * 4);
    p->off_dgp = at;
    at += align256((size_t)p->n * dgate_parts(*p, s) * 4);
    p->off_dwp = at;
    at += p->dw_parts > 1 ? align256((size_t)p->dw_parts * dw_size(h, s, M) * 4) : 0;
    p->workspace_bytes = at;
}

hipError_t ffn_backward_launch(const FfnPlan& p, FfnArgs a, void* workspace, hipStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    a.planes = p.planes;
    const int32_t n = (int32_t)p.n;
    if (n > 0) {
        hipError_t e = ffn_tiles_launch(p, a, ws, stream);
        if (e != hipSuccess) return e;
        switch (p.bm) {
            case 256: rows_launch<256>(p, a, ws, stream); break;
            case 128: rows_launch<128>(p, a, ws, stream); break;
            case 64: rows_launch<64>(p, a, ws, stream); break;
            default: rows_launch<32>(p, a, ws, stream);
        }
        const int64_t colblocks = std::min<int64_t>(((int64_t)a.T * (a.h / 8) + 255) / 256, 1 << 16);
        const int64_t gateblocks = a.dgate ? std::min<int64_t>(((int64_t)n + 255) / 256, 1 << 14) : 0;
        ffn_bwd_sum_kernel<<<(unsigned)(colblocks + gateblocks), 256, 0, stream>>>(
            reinterpret_cast<const float*>(ws + p.off_dxs), a.idx, a.T, a.h, a.M, a.k, a.dx, colblocks,
            reinterpret_cast<const float*>(ws + p.off_dgp), dgate_parts(p, a.s), a.sorted, a.dgate);
    }
    // Nontemporal stores keep what the next kernels read in the caches (h = 512, s = 64, 4096 experts of 32
    // rows, experts chosen evenly: 623 us for the call against 651; s = 72, 1024 experts of 16 rows: 180 with dW1t alone against 209).
    // Not for dW2t where a row takes several tiles of 64 columns that split a line (s = 72: 188 with both).
    if (p.dw_tile == 256)
        dw_launch<256, 256, 256, 8, false, true>(p, a, ws, stream);
    else if (p.dw_parts > 1)
        dw_launch<128, 64, 128, 4, true, false>(p, a, ws, stream);
    else if (a.s <= 64 || a.s % 64 == 0)
        dw_launch<128, 64, 128, 4, false, true>(p, a, ws, stream);
    else
        dw_launch<128, 64, 128, 4, false, false>(p, a, ws, stream);
    return hipGetLastError();
}

}  // namespace more
