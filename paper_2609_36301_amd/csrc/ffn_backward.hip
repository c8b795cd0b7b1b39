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
//   ffn_bwd_up    G, U and dA0 of one tile and 64 hidden units, all three contracted over h in one loop:
//                 [dG dU] and gate A (bf16, sorted order) and the partial sums of dgate
//   ffn_bwd_dx    [dG dU] W1t[e] per entry (fp32, entry order)
//   ffn_bwd_sum   dx: the k entries of a token added in order; dgate: the partials added in order
//   ffn_bwd_dw    dW1t and dW2t: contractions over the rows of an expert, one launch each; an expert
//                 without rows gets zeros
// Every sum runs in a fixed order: nothing is added atomically, and a call gives the same bits on every
// run.  Numerics: bf16 operands with fp32 accumulation; [dG dU] and gate A are rounded to bf16 once (the
// matrix cores' operand type), the entries' shares of dx stay in fp32 until they are summed, dgate comes
// from unrounded fp32 values.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ffn.h"
#include "ffn_device.h"

namespace more {

// ------------------------------------------------------------------------------ up
template <int BM>
struct BwdUpShape {
    static constexpr int kWavesS = BM >= 64 ? 2 : 4;
    static constexpr int kS = 64 / kWavesS / 16;
    static constexpr int kN = BM / (4 / kWavesS) / 16;
    static constexpr int kStages = 2;
    // x rows, du rows, gate and up rows, a column tile of W2t
    static constexpr int kOffDu = BM * 128, kOffW1 = 2 * BM * 128, kOffW2 = kOffW1 + 128 * 128;
    static constexpr int kStageBytes = kOffW2 + 64 * 128;
    static constexpr int kLoads = 2 * (BM / 32) + 4 + 2;
};

template <int BM>
__global__ __launch_bounds__(kFfnThreads) void ffn_bwd_up_kernel(FfnArgs a, const void* __restrict__ list,
                                                              uint16_t* __restrict__ hidden,
                                                              uint16_t* __restrict__ dgu, float* __restrict__ dgp) {
    using S = BwdUpShape<BM>;
    __shared__ __attribute__((aligned(1024))) char smem_raw[S::kStages * S::kStageBytes];
    __shared__ float dsum[S::kWavesS][BM];
    LdsChar* smem = (LdsChar*)smem_raw;
    const FfnTile* tiles = ffn_tile_list(list);
    const int32_t s = a.s, h = a.h;
    const int32_t n = a.T * a.k;
    const int32_t cols = (s + 63) / 64;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int ws = wave % S::kWavesS, wn = wave / S::kWavesS;
    const int64_t total = (int64_t)*static_cast<const int32_t*>(list) * cols;
    ffn_for_each(total, [&](int64_t item) {
        const FfnTile tile = tiles[item / cols];
        if (tile.expert < 0) return;
        const int32_t col = (int32_t)(item % cols), s0 = col * 64;
        RowTileLoader<128> weights;
        const uint16_t* W1 = a.W1t + (int64_t)tile.expert * 2 * s * h;
        const uint16_t* W2 = a.W2t + (int64_t)tile.expert * h * s;
        weights.init([&](int i) {
            const int32_t u = min(s0 + (i & 63), s - 1);
            return W1 + (int64_t)((i >> 6) * s + u) * h;
        });
        ColTileLoader<64> down;
        down.init();
        RowTileLoader<BM> tokens, grads;
        auto token_of = [&](int i) {
            const uint32_t p = a.sorted[tile.row0 + min(i, tile.rows - 1)];
            return (int64_t)(p < (uint32_t)n ? p / (uint32_t)a.k : 0) * h;
        };
        tokens.init([&](int i) { return a.x + token_of(i); });
        grads.init([&](int i) { return a.du + token_of(i); });
        f32x4 g[S::kS][S::kN], u[S::kS][S::kN], d[S::kS][S::kN];
#pragma unroll
        for (int i = 0; i < S::kS; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) g[i][j] = u[i][j] = d[i][j] = zero_f32x4();
        ffn_pipeline<S::kStages, S::kLoads>(
            (h + kFfnBK - 1) / kFfnBK,
            [&](int step, int slot) {
                LdsChar* at = smem + slot * S::kStageBytes;
                const int32_t k0 = step * kFfnBK;
                tokens.load(at, k0, h);
                grads.load(at + S::kOffDu, k0, h);
                weights.load(at + S::kOffW1, k0, h);
                down.load(at + S::kOffW2, s - s0, [&](int, int kappa) {
                    return k0 + kappa < h ? W2 + (int64_t)(k0 + kappa) * s + s0 : nullptr;
                });
            },
            [&](int, int slot) {
                LdsChar* at = smem + slot * S::kStageBytes;
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    bf16x8 b[S::kN], c[S::kN];
#pragma unroll
                    for (int j = 0; j < S::kN; ++j) {
                        b[j] = row_fragment(at, 16 * (wn * S::kN + j), kk);
                        c[j] = row_fragment(at + S::kOffDu, 16 * (wn * S::kN + j), kk);
                    }
#pragma unroll
                    for (int i = 0; i < S::kS; ++i) {
                        const int row = 16 * (ws * S::kS + i);
                        const bf16x8 fg = row_fragment(at + S::kOffW1, row, kk);
                        const bf16x8 fu = row_fragment(at + S::kOffW1, 64 + row, kk);
                        const bf16x8 fd = col_fragment<64>(at + S::kOffW2, row, kk);
#pragma unroll
                        for (int j = 0; j < S::kN; ++j) {
                            g[i][j] = mfma_16x16x32(fg, b[j], g[i][j]);
                            u[i][j] = mfma_16x16x32(fu, b[j], u[i][j]);
                            d[i][j] = mfma_16x16x32(fd, c[j], d[i][j]);
                        }
                    }
                }
            });
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
                }
            }
            dot += __shfl_xor(dot, 16, 64);
            dot += __shfl_xor(dot, 32, 64);
            if (lane < 16) dsum[ws][row] = dot;
        }
        if (a.dgate) {
            ffn_barrier<63>();
            for (int32_t row = threadIdx.x; row < tile.rows; row += kFfnThreads) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < S::kWavesS; ++w) v += dsum[w][row];
                dgp[(int64_t)col * n + tile.row0 + row] = v;
            }
        }
    });
}

// ------------------------------------------------------------------------------ dx of the entries
// As ffn_down with [dG dU] as the rows and W1t[e] [2s][h] as a column tile (contraction over 2s).
template <int BM>
struct BwdDxShape {
    static constexpr int kWavesM = BM >= 64 ? 2 : 4;
    static constexpr int kM = 128 / kWavesM / 16;
    static constexpr int kN = BM / (4 / kWavesM) / 16;
    static constexpr int kStages = BM >= 128 ? 2 : 3;
    static constexpr int kStageBytes = (128 + BM) * 128;
    static constexpr int kLoads = 4 + BM / 32;
};

template <int BM>
__global__ __launch_bounds__(kFfnThreads, 2) void ffn_bwd_dx_kernel(FfnArgs a, const void* __restrict__ list,
                                                                 const uint16_t* __restrict__ dgu, int32_t hspan,
                                                                 float* __restrict__ dxs) {
    using S = BwdDxShape<BM>;
    __shared__ __attribute__((aligned(1024))) char smem_raw[S::kStages * S::kStageBytes];
    LdsChar* smem = (LdsChar*)smem_raw;
    const FfnTile* tiles = ffn_tile_list(list);
    const int32_t h = a.h, s2 = 2 * a.s;
    const int32_t n = a.T * a.k;
    const int32_t spans = (h + hspan - 1) / hspan;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int wm = wave % S::kWavesM, wn = wave / S::kWavesM;
    const int64_t total = (int64_t)*static_cast<const int32_t*>(list) * spans;
    ffn_for_each(total, [&](int64_t item) {
        const FfnTile tile = tiles[item / spans];
        if (tile.expert < 0) return;  // dropped entries have no share (ffn_bwd_sum leaves them out)
        const int32_t h0 = (int32_t)(item % spans) * hspan, h1 = min(h, h0 + hspan);
        const uint16_t* W = a.W1t + (int64_t)tile.expert * s2 * h;
        RowTileLoader<BM> rows;
        rows.init([&](int i) { return dgu + (int64_t)(tile.row0 + min(i, tile.rows - 1)) * s2; });
        ColTileLoader<128> weights;
        weights.init();
        uint32_t place[S::kN];
#pragma unroll
        for (int j = 0; j < S::kN; ++j) {
            const int32_t row = 16 * (wn * S::kN + j) + (lane & 15);
            place[j] = row < tile.rows ? (uint32_t)a.sorted[tile.row0 + row] : 0xFFFFFFFFu;
        }
        f32x4 acc[S::kM][S::kN];
#pragma unroll
        for (int i = 0; i < S::kM; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) acc[i][j] = zero_f32x4();
        const int32_t ksteps = (s2 + kFfnBK - 1) / kFfnBK;
        const int32_t hsteps = (h1 - h0 + 127) / 128;
        int32_t lh = h0, lk = 0, ch = h0, ck = 0;
        ffn_pipeline<S::kStages, S::kLoads>(
            ksteps * hsteps,
            [&](int, int slot) {
                LdsChar* at = smem + slot * S::kStageBytes;
                const int32_t k0 = lk * kFfnBK;
                weights.load(at, h - lh, [&](int, int kappa) {
                    return k0 + kappa < s2 ? W + (int64_t)(k0 + kappa) * h + lh : nullptr;
                });
                rows.load(at + 128 * 128, k0, s2);
                if (++lk == ksteps) {
                    lk = 0;
                    lh += 128;
                }
            },
            [&](int, int slot) {
                LdsChar* at = smem + slot * S::kStageBytes;
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    bf16x8 b[S::kN];
#pragma unroll
                    for (int j = 0; j < S::kN; ++j) b[j] = row_fragment(at + 128 * 128, 16 * (wn * S::kN + j), kk);
#pragma unroll
                    for (int i = 0; i < S::kM; ++i) {
                        const bf16x8 f = col_fragment<128>(at, 16 * (wm * S::kM + i), kk);
#pragma unroll
                        for (int j = 0; j < S::kN; ++j) acc[i][j] = mfma_16x16x32(f, b[j], acc[i][j]);
                    }
                }
                if (++ck < ksteps) return;
#pragma unroll
                for (int j = 0; j < S::kN; ++j) {
#pragma unroll
                    for (int i = 0; i < S::kM; ++i) {
                        const int32_t c = ch + 16 * (wm * S::kM + i) + 4 * (lane >> 4);
                        if (place[j] < (uint32_t)n && c < h1)
                            *reinterpret_cast<f32x4*>(dxs + (int64_t)place[j] * h + c) = acc[i][j];
                        acc[i][j] = zero_f32x4();
                    }
                }
                ck = 0;
                ch += 128;
            });
    });
}

// ------------------------------------------------------------------------------ sums over the entries
// A thread adds eight columns of a token's k rows in order; dropped entries (id outside [0, M)) are left
// out.  The threads past the columns add the partials of dgate.
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
// (rows 2s).  dW2t: P = gate A (cols s), Q = du of the entry's token (rows h).
template <int CT, int RT, bool GATHER_P, bool GATHER_Q>
__global__ __launch_bounds__(kFfnThreads, 2) void ffn_bwd_dw_kernel(const uint16_t* __restrict__ P,
                                                                 const uint16_t* __restrict__ Q,
                                                                 const int32_t* __restrict__ offsets,
                                                                 const int32_t* __restrict__ sorted, int32_t n,
                                                                 int32_t k, int32_t M, int32_t rows_out,
                                                                 int32_t cols_out, uint16_t* __restrict__ out) {
    constexpr int kStages = 2;
    constexpr int kStageBytes = (CT + RT) * 128;
    constexpr int kM = CT / 32, kN = RT / 32;  // 16 x 16 tiles per wave (2 x 2 waves)
    __shared__ __attribute__((aligned(1024))) char smem_raw[kStages * kStageBytes];
    LdsChar* smem = (LdsChar*)smem_raw;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int wm = wave & 1, wn = wave >> 1;
    const int32_t ct = (cols_out + CT - 1) / CT, rt = (rows_out + RT - 1) / RT;
    ffn_for_each((int64_t)M * ct * rt, [&](int64_t item) {
        const int32_t e = (int32_t)(item / (ct * rt)), q = (int32_t)(item % (ct * rt));
        const int32_t c0 = (q % ct) * CT, r0 = (q / ct) * RT;
        const int32_t begin = min(max(offsets[e], 0), n), end = min(max(offsets[e + 1], begin), n);
        ColTileLoader<CT> pl;
        ColTileLoader<RT> ql;
        pl.init();
        ql.init();
        auto token_of = [&](int32_t i) {
            const uint32_t p = (uint32_t)sorted[i];
            return p < (uint32_t)n ? p / (uint32_t)k : 0u;
        };
        f32x4 acc[kM][kN];
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j) acc[i][j] = zero_f32x4();
        ffn_pipeline<kStages, ColTileLoader<CT>::kLoads + ColTileLoader<RT>::kLoads>(
            (end - begin + kFfnBK - 1) / kFfnBK,
            [&](int step, int slot) {
                LdsChar* at = smem + slot * kStageBytes;
                const int32_t i0 = begin + step * kFfnBK;
                pl.load(at, cols_out - c0, [&](int, int kappa) -> const uint16_t* {
                    if (i0 + kappa >= end) return nullptr;
                    return P + (int64_t)(GATHER_P ? token_of(i0 + kappa) : i0 + kappa) * cols_out + c0;
                });
                ql.load(at + CT * 128, rows_out - r0, [&](int, int kappa) -> const uint16_t* {
                    if (i0 + kappa >= end) return nullptr;
                    return Q + (int64_t)(GATHER_Q ? token_of(i0 + kappa) : i0 + kappa) * rows_out + r0;
                });
            },
            [&](int, int slot) {
                LdsChar* at = smem + slot * kStageBytes;
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    bf16x8 b[kN];
#pragma unroll
                    for (int j = 0; j < kN; ++j) b[j] = col_fragment<RT>(at + CT * 128, 16 * (wn * kN + j), kk);
#pragma unroll
                    for (int i = 0; i < kM; ++i) {
                        const bf16x8 f = col_fragment<CT>(at, 16 * (wm * kM + i), kk);
#pragma unroll
                        for (int j = 0; j < kN; ++j) acc[i][j] = mfma_16x16x32(f, b[j], acc[i][j]);
                    }
                }
            });
        uint16_t* o = out + (int64_t)e * rows_out * cols_out;
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            const int32_t r = r0 + 16 * (wn * kN + j) + (lane & 15);
#pragma unroll
            for (int i = 0; i < kM; ++i) {
                const int32_t c = c0 + 16 * (wm * kM + i) + 4 * (lane >> 4);
                if (r < rows_out && c < cols_out)
                    *reinterpret_cast<uint2*>(o + (int64_t)r * cols_out + c) =
                        pack_bf16x4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
            }
        }
    });
}

// ------------------------------------------------------------------------------ host
namespace {

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }
constexpr int64_t kMaxBlocks = 1 << 19;
unsigned grid_of(int64_t items) {
    return (unsigned)(std::min<int64_t>((items + 7) / 8, kMaxBlocks / 8) * 8);
}

template <int BM>
void rows_launch(const FfnPlan& p, const FfnArgs& a, char* ws, hipStream_t stream) {
    uint16_t* hidden = reinterpret_cast<uint16_t*>(ws + p.off_hidden);
    uint16_t* dgu = reinterpret_cast<uint16_t*>(ws + p.off_dgu);
    ffn_bwd_up_kernel<BM><<<grid_of(p.tiles * ((a.s + 63) / 64)), kFfnThreads, 0, stream>>>(
        a, ws + p.off_tiles, hidden, dgu, reinterpret_cast<float*>(ws + p.off_dgp));
    const int32_t hspan = 512;
    ffn_bwd_dx_kernel<BM><<<grid_of(p.tiles * ((a.h + hspan - 1) / hspan)), kFfnThreads, 0, stream>>>(
        a, ws + p.off_tiles, dgu, hspan, reinterpret_cast<float*>(ws + p.off_dxs));
}

}  // namespace

void ffn_backward_make_plan(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, FfnPlan* p) {
    ffn_make_plan(T, h, s, M, k, p);
    size_t at = p->workspace_bytes;
    p->off_dgu = at;
    at += align256((size_t)p->n * 2 * s * 2);
    p->off_dxs = at;
    at += align256((size_t)p->n * h * 4);
    p->off_dgp = at;
    at += align256((size_t)p->n * ((s + 63) / 64) * 4);
    p->workspace_bytes = at;
}

hipError_t ffn_backward_launch(const FfnPlan& p, const FfnArgs& a, void* workspace, hipStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    const int32_t n = (int32_t)p.n;
    if (n > 0) {
        hipError_t e = ffn_tiles_launch(p, a, ws + p.off_tiles, stream);
        if (e != hipSuccess) return e;
        switch (p.bm) {
            case 128: rows_launch<128>(p, a, ws, stream); break;
            case 64: rows_launch<64>(p, a, ws, stream); break;
            default: rows_launch<32>(p, a, ws, stream);
        }
        const int64_t colblocks = std::min<int64_t>(((int64_t)a.T * (a.h / 8) + 255) / 256, 1 << 16);
        const int64_t gateblocks = a.dgate ? std::min<int64_t>(((int64_t)n + 255) / 256, 1 << 14) : 0;
        ffn_bwd_sum_kernel<<<(unsigned)(colblocks + gateblocks), 256, 0, stream>>>(
            reinterpret_cast<const float*>(ws + p.off_dxs), a.idx, a.T, a.h, a.M, a.k, a.dx, colblocks,
            reinterpret_cast<const float*>(ws + p.off_dgp), (a.s + 63) / 64, a.sorted, a.dgate);
    }
    const uint16_t* hidden = reinterpret_cast<const uint16_t*>(ws + p.off_hidden);
    const uint16_t* dgu = reinterpret_cast<const uint16_t*>(ws + p.off_dgu);
    auto tiles = [](int32_t v, int32_t t) { return (int64_t)((v + t - 1) / t); };
    ffn_bwd_dw_kernel<128, 128, true, false>
        <<<grid_of(a.M * tiles(a.h, 128) * tiles(2 * a.s, 128)), kFfnThreads, 0, stream>>>(
            a.x, dgu, a.offsets, a.sorted, n, a.k, a.M, 2 * a.s, a.h, a.dW1t);
    ffn_bwd_dw_kernel<64, 128, false, true>
        <<<grid_of(a.M * tiles(a.s, 64) * tiles(a.h, 128)), kFfnThreads, 0, stream>>>(
            hidden, a.du, a.offsets, a.sorted, n, a.k, a.M, a.h, a.s, a.dW2t);
    return hipGetLastError();
}

}  // namespace more
