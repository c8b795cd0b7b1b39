// Backward pass of the experts' linear maps (linear.hip) for gfx950: for every entry p = t k + j of expert
// e = idx[t][j],
//   dx_t = sum_j dy_p W_e       dW_e = sum_{p of e} dy_p^T x_t
//
// Kernels of one call (entries in the order of Sort + Count, cut into tiles of one expert; either gradient may be
// left out; small calls make both in one launch, linear_both):
//   ffn_tiles         lists the tiles (where they are many)
//   linear_dx         dy_p W_e of one tile: with one entry per token dx itself (bf16), else the entries' shares
//                     (fp32, entry order), which linear_sum adds in the entries' order
//   linear_dw         dW: contractions over the rows of an expert; an expert without rows gets zeros.  Long
//                     rows of few experts are cut into runs whose fp32 sums ffn_parts_sum adds
// Every sum runs in a fixed order: nothing is added atomically, and a call gives the same bits on every run.
// Numerics: exact products of bf16 and fp32 sums, one rounding to bf16.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ffn_device.h"
#include "linear.h"
#include "linear_device.h"

namespace more {

// ------------------------------------------------------------------------------ dx
// The weights lie with the contraction axis (N) slowest: they are a column tile (M side), the entries' rows of dy
// a row tile (N side).  A workgroup computes `span` columns in steps of COLS; the pipeline runs over (column
// step, contraction step) pairs.  4096 experts of K = 64, N = 512 with 32 rows 79 us, 419 MB at 5.3 TB/s; 32 of
// 2048 x 2048 with 1024 rows 322 us in calls one after the other (352 to 380 in a trace), 850 TFLOP/s, and 53 for the fp32
// shares' sum; the matrix cores work in 36 % of the cycles, waves wait in 39 %.  Up to 128 rows the weights, read
// across their rows, come by way of registers; tiles of 256 rows load straight to LDS.
constexpr int dx_threads(int bm) { return bm == 256 ? 512 : 256; }
template <int BM, int COLS>
struct DxShape {
    static constexpr int kThreads = dx_threads(BM);
    static constexpr int kWaves = kThreads / 64;
    static constexpr int kWavesM = BM >= 64 ? 2 : 4;
    static constexpr int kM = COLS / kWavesM / 16;
    static constexpr int kN = BM / (kWaves / kWavesM) / 16;
    static constexpr int kRowsAt = COLS * 128;
    static constexpr int kStageBytes = kRowsAt + BM * 128;
    static constexpr int kRing = 2 * kStageBytes;
    static constexpr bool kLines = kM % 4 == 0;  // a wave's columns are whole lines of dx
    static constexpr int kLds = kRing + (kLines ? kWaves * kLinesScratch : 0);
    // An expert has one tile, mostly, and its weights lie one line after the other: nontemporal (4096 experts, K = 64,
    // N = 512, 32 rows 68 us, without 88; of wider weights, taken 128 columns at a time, 262 : 227).
    static constexpr bool kOnce = BM <= 64 && COLS == 64;
};

// DIRECT: one entry per token, `out` is dx (bf16); else the shares (fp32).
template <int BM, int COLS, bool DIRECT, bool OWN>
__device__ __forceinline__ void linear_dx(const LinearArgs& a, const void* __restrict__ list, int32_t bound, int32_t span,
                                          void* __restrict__ out, LdsChar* smem) {
    using S = DxShape<BM, COLS>;
    LdsChar* lines = smem + (S::kLines ? S::kRing + ffn_wave() * kLinesScratch : 0);
    const int32_t n = a.T * a.k, len = a.N, cols = a.len;
    const int32_t spans = (cols + span - 1) / span;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int wm = wave % S::kWavesM, wn = wave / S::kWavesM;
    linear_for_each<BM, S::kThreads, OWN>(a, list, bound, spans, smem, [&](const FfnTile& tile, int32_t turn) {
        const int32_t c0 = turn * span, c1 = min(cols, c0 + span);
        if (tile.expert < 0) {  // dropped entries: zero rows of dx; the sum leaves their shares out
            if constexpr (DIRECT) {
                const int32_t pieces = (c1 - c0) / 8;
                for (int32_t i = threadIdx.x; i < tile.rows * pieces; i += S::kThreads) {
                    const uint32_t p = a.sorted[tile.row0 + i / pieces];
                    if (p < (uint32_t)n)
                        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + (int64_t)p * cols + c0 + 8 * (i % pieces)) =
                            u32x4{0u, 0u, 0u, 0u};
                }
            }
            return;
        }
        const uint16_t* We = a.W + (int64_t)tile.expert * len * cols;
        RowTileLoader<BM, S::kWaves> rows;
        rows.init([&](int i) {
            const uint32_t p = a.sorted[tile.row0 + min(i, tile.rows - 1)];
            return a.dy + (int64_t)(p < (uint32_t)n ? p : 0) * len;
        });
        ColTileLoader<COLS, S::kWaves> weights;
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
        const int32_t ksteps = (len + kFfnBK - 1) / kFfnBK;
        const int32_t csteps = (c1 - c0 + COLS - 1) / COLS;
        // (column step, contraction step) of the next load and of the next product
        int32_t lc = c0, lk = 0, cc = c0, ck = 0;
        using G = FfnGroups<S::kM, S::kM == 8 ? 4 : 2>;
        using M = FfnFragments<G::kSize>;
        using F = FfnFragments<S::kN>;
        auto weight_row = [&](int i) -> const uint16_t* {
            const int kappa = lk * kFfnBK + weights.row(i);
            return kappa < len ? We + (int64_t)kappa * cols + lc : nullptr;
        };
        auto advance = [&] {
            if (++lk < ksteps) return;
            lk = 0;
            lc += COLS;
        };
        auto read_n = [&](int slot, int kk, F& f) {
#pragma unroll
            for (int j = 0; j < S::kN; ++j)
                f.v[j] = row_fragment(smem + slot * S::kStageBytes + S::kRowsAt, 16 * (wn * S::kN + j), kk);
        };
        auto multiply = [&](int group, const M& m, const F& f) {
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
            if (++ck < ksteps) return;
            if constexpr (S::kLines) {
                using L = Lines<!DIRECT>;
                using Out = typename L::Element;
#pragma unroll
                for (int j = 0; j < S::kN; ++j)
#pragma unroll
                    for (int i0 = 0; i0 < S::kM; i0 += L::kTiles) {
#pragma unroll
                        for (int i = 0; i < L::kTiles; ++i) L::place(lines, i, acc[i0 + i][j]);
                        const int32_t c = cc + 16 * (wm * S::kM + i0);
                        L::store(lines, c1 - c, a.whole, [&](int r) -> Out* {
                            const uint32_t p = (uint32_t)__shfl((int)place[j], r, 64);
                            return p < (uint32_t)n ? static_cast<Out*>(out) + (int64_t)p * cols + c : nullptr;
                        });
                    }
            } else if constexpr (DIRECT && S::kM % 2 == 0) {
#pragma unroll
                for (int j = 0; j < S::kN; ++j)
#pragma unroll
                    for (int i = 0; i < S::kM; i += 2) {
                        const int32_t c = cc + 16 * (wm * S::kM + i) + 8 * (lane >> 4);
                        const u32x4 v = linear_pair(acc[i][j], acc[i + 1][j]);
                        if (place[j] < (uint32_t)n && c < c1)
                            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + (int64_t)place[j] * cols + c) = v;
                    }
            } else {
#pragma unroll
                for (int j = 0; j < S::kN; ++j)
#pragma unroll
                    for (int i = 0; i < S::kM; ++i) {
                        const int32_t c = cc + 16 * (wm * S::kM + i) + 4 * (lane >> 4);
                        if (place[j] < (uint32_t)n && c < c1) linear_put(out, !DIRECT, (int64_t)place[j] * cols + c, acc[i][j]);
                    }
            }
#pragma unroll
            for (int i = 0; i < S::kM; ++i)
#pragma unroll
                for (int j = 0; j < S::kN; ++j) acc[i][j] = zero_f32x4();
            ck = 0;
            cc += COLS;
        };
        if constexpr (BM == 256) {
            constexpr int kLoads = weights.kLoads + rows.kLoads;
            ffn_pipeline<2, kLoads, G::kGroups, true, M, F>(
                ksteps * csteps, 16 * wn * S::kN < tile.rows,
                [&](int, int slot) { weights.load(smem + slot * S::kStageBytes, cols - lc, weight_row); },
                [&](int, int slot) {
                    rows.load(smem + slot * S::kStageBytes + S::kRowsAt, lk * kFfnBK, len);
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
            ffn_pipeline_staged<Stage, G::kGroups, M, F>(
                ksteps * csteps, 16 * wn * S::kN < tile.rows,
                [&](int, Stage& st) {
                    weights.template fetch<S::kOnce>(st.a, cols - lc, weight_row);
                    rows.fetch(st.b, lk * kFfnBK, len);
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

template <int BM, int COLS, bool DIRECT, bool OWN>
__global__ __launch_bounds__(dx_threads(BM), 2) void linear_dx_kernel(LinearArgs a, const void* __restrict__ list,
                                                                  int32_t bound, int32_t span, void* __restrict__ out) {
    __shared__ __attribute__((aligned(1024))) char smem[DxShape<BM, COLS>::kLds];
    linear_dx<BM, COLS, DIRECT, OWN>(a, list, bound, span, out, (LdsChar*)smem);
}

// A thread adds eight columns of a token's k shares in order; dropped entries are left out.  The shares and ids of four
// entries are read at a time, whether wanted or not: one after the other their reads would wait for the ids.  8192 tokens,
// k = 4, K = 2048 53 us, 5.7 TB/s.
__global__ __launch_bounds__(256) void linear_sum_kernel(LinearArgs a, const float* __restrict__ shares) {
    constexpr int kAhead = 4;
    const int32_t pieces = a.len / 8, k = a.k;
    const int64_t total = (int64_t)a.T * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = i / pieces;
        const int32_t c = (int32_t)(i - t * pieces) * 8;
        f32x4 lo = zero_f32x4(), hi = zero_f32x4();
        for (int32_t j0 = 0; j0 < k; j0 += kAhead) {
            uint32_t id[kAhead];
            f32x4 v[kAhead][2];
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int64_t p = t * k + min(j0 + q, k - 1);
                id[q] = j0 + q < k ? (uint32_t)a.idx[p] : 0xFFFFFFFFu;
                const f32x4* s = reinterpret_cast<const f32x4*>(shares + p * a.len + c);
                v[q][0] = s[0];
                v[q][1] = s[1];
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                if (id[q] >= (uint32_t)a.M) continue;
                lo += v[q][0];
                hi += v[q][1];
            }
        }
        const uint2 x = pack_bf16x4(lo[0], lo[1], lo[2], lo[3]), y = pack_bf16x4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<u32x4*>(a.dx + t * a.len + c) = u32x4{x.x, x.y, y.x, y.y};
    }
}

// ------------------------------------------------------------------------------ dW
// dW_e [N][K] = sum over the entries p of e of dy_p^T x_t: both operands are column tiles (the contraction runs over
// rows), dy the N side and x the M side, and both are gathered.  A workgroup computes tiles of RT rows (of N) and CT
// columns (of K) one after the other over `span` of one side (BY_COLS: of K), and the pipeline runs over (tile, 64
// entries) pairs, so that the few rows of a small expert do not drain it.
// Small experts are bound by memory (4096 of K = 64, N = 512, 32 entries 84 to 90 us, 419 MB at 5.0 TB/s), large ones by the
// transposing reads of both operands, which come by way of registers: 32 of 2048 x 2048, 1024 entries 328 us in calls one
// after the other (368 to 422 in a trace), 840 TFLOP/s; the matrix cores work in 32 % of the cycles, waves wait in 39 %.
// PARTS: the entries of an expert are cut into `runs` runs and a workgroup takes one tile and one run; the fp32
// results of run i go to parts + i M N K.
struct LinearDw {
    int32_t span, runs;
    float* parts;
};

// Narrow tiles (64 rows or columns) do with one stage in LDS, so that four workgroups fit on a CU instead of two (us, two
// stages : one, 4096 experts of K = 64, N = 512, 32 entries 99 : 84; 2000 of K = 40, N = 520, 30 entries 62 : 38; wide tiles,
// whose registers leave room for three, 4096 of K = 512, N = 128 109 : 115).
template <int CT, int RT>
constexpr int dw_slots() {
    return CT + RT <= 192 ? 1 : 2;
}
template <int CT, int RT, int WAVES>
constexpr int dw_lds() {
    return dw_slots<CT, RT>() * (CT + RT) * 128 + WAVES * kLinesScratch;
}

// The pipeline by way of registers with one stage in LDS (the arguments are ffn_pipeline_staged's): the next stage is read
// into registers while the present one is multiplied.
template <typename S, int GROUPS, typename M, typename N, typename F, typename P, typename W>
__device__ __forceinline__ void pipeline_single(int steps, F fetch, P put, W w) {
    S s;
    M m;
    N n;
    fetch(0, s);
    for (int step = 0; step < steps; ++step) {
        ffn_barrier<63>();  // the stage before has been read
        put(0, s);
        if (step + 1 < steps) fetch(step + 1, s);
        ffn_barrier<63>();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            w.read_n(0, kk, n);
#pragma unroll
            for (int group = 0; group < GROUPS; ++group) {
                w.read_m(0, kk, group, m);
                w.multiply(group, m, n);
            }
        }
        w.done();
    }
}

// The work of workgroup `block` of `blocks`.
template <int CT, int RT, int WAVES, bool BY_COLS, bool PARTS>
__device__ __forceinline__ void linear_dw(const LinearArgs& a, const LinearDw& d, uint32_t block, uint32_t blocks, LdsChar* smem) {
    constexpr int kStageBytes = (CT + RT) * 128;
    LdsChar* lines = smem + dw_slots<CT, RT>() * kStageBytes + ffn_wave() * kLinesScratch;
    constexpr int kWavesM = CT >= 128 ? 2 : 1, kWavesN = WAVES / kWavesM;
    constexpr int kM = CT / kWavesM / 16, kN = RT / kWavesN / 16;  // 16 x 16 tiles per wave
    static_assert(kM % 4 == 0, "whole lines of dW: 64 columns");
    using XLoader = ColTileLoader<CT, WAVES>;
    using YLoader = ColTileLoader<RT, WAVES>;
    constexpr int kGroups = XLoader::kGroups;  // entries per lane (the same ones of both operands)
    const int wm = ffn_wave() % kWavesM, wn = ffn_wave() / kWavesM;
    constexpr int kStep = BY_COLS ? CT : RT;
    const int32_t n = a.T * a.k, K = a.len, N = a.N;
    const int32_t side = BY_COLS ? K : N;
    const int32_t spans = (side + d.span - 1) / d.span;
    const int32_t others = BY_COLS ? (N + RT - 1) / RT : (K + CT - 1) / CT;
    const int32_t runs = PARTS ? d.runs : 1;
    for (int64_t work = block; work < (int64_t)a.M * spans * others * runs; work += blocks) {
        const int32_t run = PARTS ? (int32_t)(work % runs) : 0;
        const int64_t item = PARTS ? work / runs : work;
        const int64_t per = (int64_t)spans * others;
        const int32_t e = (int32_t)(item / per), q = (int32_t)(item % per);
        const int32_t s0 = (q % spans) * d.span, s1 = min(side, s0 + d.span);
        const int32_t other = (q / spans) * (BY_COLS ? RT : CT);  // first row (column) of the other side
        int32_t begin = min(max(a.offsets[e], 0), n), end = min(max(a.offsets[e + 1], begin), n);
        if constexpr (PARTS) {  // whole stages
            const int32_t len = ((end - begin + runs - 1) / runs + kFfnBK - 1) / kFfnBK * kFfnBK;
            begin = (int32_t)min((int64_t)begin + (int64_t)run * len, (int64_t)end);
            end = (int32_t)min((int64_t)begin + len, (int64_t)end);
        }
        XLoader xl;
        YLoader yl;
        xl.init();
        yl.init();
        const int32_t ksteps = (end - begin + kFfnBK - 1) / kFfnBK;
        const int32_t ssteps = (s1 - s0 + kStep - 1) / kStep;
        uint32_t entry[kGroups];  // of the next load (read one load ahead)
        auto fetch = [&](int32_t step) {
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const int32_t at = begin + step * kFfnBK + xl.row(i);
                entry[i] = at < end ? (uint32_t)a.sorted[at] : 0xFFFFFFFFu;
            }
        };
        f32x4 acc[kM][kN];
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j) acc[i][j] = zero_f32x4();
        int32_t ls = s0, lk = 0, cs = s0, ck = 0;
        auto store = [&] {
            if constexpr (PARTS) {
                float* o = d.parts + ((int64_t)run * a.M + e) * N * K;
#pragma unroll
                for (int j = 0; j < kN; ++j)
#pragma unroll
                    for (int i0 = 0; i0 < kM; i0 += 2) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            Lines<true>::place(lines, i, acc[i0 + i][j]);
                            acc[i0 + i][j] = zero_f32x4();
                        }
                        const int32_t c = (BY_COLS ? cs : other) + 16 * (wm * kM + i0);
                        const int32_t r = (BY_COLS ? other : cs) + 16 * (wn * kN + j);
                        Lines<true>::store(lines, (BY_COLS ? s1 : K) - c, false, [&](int row) {
                            return r + row < (BY_COLS ? N : s1) ? o + (int64_t)(r + row) * K + c : nullptr;
                        });
                    }
                cs += kStep;
                return;
            }
            uint16_t* o = a.dW + (int64_t)e * N * K;
#pragma unroll
            for (int j = 0; j < kN; ++j)
#pragma unroll
                for (int i0 = 0; i0 < kM; i0 += 4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        Lines<false>::place(lines, i, acc[i0 + i][j]);
                        acc[i0 + i][j] = zero_f32x4();
                    }
                    const int32_t c = (BY_COLS ? cs : other) + 16 * (wm * kM + i0);
                    const int32_t r = (BY_COLS ? other : cs) + 16 * (wn * kN + j);
                    Lines<false>::store(lines, (BY_COLS ? s1 : K) - c, true, [&](int row) {
                        return r + row < (BY_COLS ? N : s1) ? o + (int64_t)(r + row) * K + c : nullptr;
                    });
                }
            cs += kStep;
        };
        if (ksteps == 0) {  // no entries: zeros
            if constexpr (PARTS) {
                for (int32_t step = 0; step < ssteps; ++step) store();
            } else {  // the expert's items share its matrix in runs of whole lines
                const int64_t pieces = (int64_t)N * K / 8;
                const int64_t share = (pieces / per + 8) / 8 * 8;
                u32x4* o = reinterpret_cast<u32x4*>(a.dW + (int64_t)e * N * K);
                const int64_t last = min(pieces, (q + 1) * share);
                for (int64_t i = q * share + threadIdx.x; i < last; i += 64 * WAVES)
                    __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, o + i);
            }
            continue;
        }
        using G = FfnGroups<kM, kM == 8 ? 4 : 2>;
        using MF = FfnFragments<G::kSize>;
        using NF = FfnFragments<kN>;
        using Stage = StagePair<XLoader, YLoader>;
        fetch(0);
        auto load = [&](int, Stage& st) {
            const int32_t c = BY_COLS ? ls : other, r = BY_COLS ? other : ls;
            xl.fetch(st.a, K - c, [&](int i) -> const uint16_t* {
                return entry[i] < (uint32_t)n ? a.x + (int64_t)(entry[i] / (uint32_t)a.k) * K + c : nullptr;
            });
            yl.fetch(st.b, N - r, [&](int i) -> const uint16_t* {
                return entry[i] < (uint32_t)n ? a.dy + (int64_t)entry[i] * N + r : nullptr;
            });
            if (++lk == ksteps) {
                lk = 0;
                ls += kStep;
            }
            if (ksteps > 1) fetch(lk);
        };
        auto put = [&](int slot, const Stage& st) {
            xl.put(smem + slot * kStageBytes, st.a);
            yl.put(smem + slot * kStageBytes + CT * 128, st.b);
        };
        auto products = ffn_work(
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
                if (++ck < ksteps) return;
                ck = 0;
                store();
            });
        if constexpr (dw_slots<CT, RT>() == 1)
            pipeline_single<Stage, G::kGroups, MF, NF>(ksteps * ssteps, load, put, products);
        else
            ffn_pipeline_staged<Stage, G::kGroups, MF, NF>(ksteps * ssteps, true, load, put, products);
    }
}

template <int CT, int RT, int WAVES, bool BY_COLS, bool PARTS>
__global__ __launch_bounds__(64 * WAVES, 2) void linear_dw_kernel(LinearArgs a, LinearDw d) {
    __shared__ __attribute__((aligned(1024))) char smem[dw_lds<CT, RT, WAVES>()];
    linear_dw<CT, RT, WAVES, BY_COLS, PARTS>(a, d, blockIdx.x, gridDim.x, (LdsChar*)smem);
}

// Both gradients of a small call at once: the first `dx_blocks` workgroups take dx, the others dW.  Neither fills the chip
// or hides its latency alone (us, apart : at once, a dense map of 1024 x 1024, 300 rows 21.6 : 12.4; 16 experts of
// 512 x 512, 4096 rows 25.5 : 18.5).
template <int BM, int COLS, bool DIRECT, int CT, int RT, bool BY_COLS, bool PARTS>
__global__ __launch_bounds__(256, 2) void linear_both_kernel(LinearArgs a, int32_t bound, int32_t span, void* __restrict__ out,
                                                             uint32_t dx_blocks, LinearDw d) {
    constexpr int kDx = DxShape<BM, COLS>::kLds, kDw = dw_lds<CT, RT, 4>();
    __shared__ __attribute__((aligned(1024))) char smem[kDx > kDw ? kDx : kDw];
    if (blockIdx.x < dx_blocks)
        linear_dx<BM, COLS, DIRECT, true>(a, nullptr, bound, span, out, (LdsChar*)smem);
    else
        linear_dw<CT, RT, 4, BY_COLS, PARTS>(a, d, blockIdx.x - dx_blocks, gridDim.x - dx_blocks, (LdsChar*)smem);
}

// ------------------------------------------------------------------------------ host
namespace {

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }
constexpr int64_t kMaxBlocks = 1 << 19;
unsigned grid_of(int64_t items) { return (unsigned)(std::min<int64_t>((items + 7) / 8, kMaxBlocks / 8) * 8); }

unsigned dx_blocks(const LinearPlan& p, const LinearArgs& a) {
    return grid_of(p.tiles.tiles * ((a.len + p.span - 1) / p.span));
}

template <int BM, int COLS, bool OWN>
void dx_launch(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream) {
    const unsigned blocks = dx_blocks(p, a);
    const void* list = OWN ? nullptr : ws + p.tiles.off_tiles;
    const int32_t bound = (int32_t)p.tiles.tiles;
    if (a.k == 1)
        linear_dx_kernel<BM, COLS, true, OWN><<<blocks, dx_threads(BM), 0, stream>>>(a, list, bound, p.span, a.dx);
    else
        linear_dx_kernel<BM, COLS, false, OWN><<<blocks, dx_threads(BM), 0, stream>>>(a, list, bound, p.span, ws + p.off_shares);
}
template <int BM, int COLS>
void dx_launch(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream) {
    if (p.listed)
        dx_launch<BM, COLS, false>(p, a, ws, stream);
    else if constexpr (BM < 256)
        dx_launch<BM, COLS, true>(p, a, ws, stream);
}

int64_t dw_items(const LinearPlan& p, int32_t K, int32_t N, int32_t M, bool by_cols) {
    const int32_t side = by_cols ? K : N, other = by_cols ? N : K, step = by_cols ? p.dw_rows : p.dw_cols;
    return (int64_t)M * ((side + p.dw_span - 1) / p.dw_span) * ((other + step - 1) / step);
}

LinearDw dw_args(const LinearPlan& p, char* ws) {
    return LinearDw{p.dw_span, p.dw_parts, reinterpret_cast<float*>(ws + p.off_parts)};
}

template <int CT, int RT, int WAVES, bool BY_COLS>
void dw_launch(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream) {
    const LinearDw d = dw_args(p, ws);
    const unsigned blocks = grid_of(dw_items(p, a.len, a.N, a.M, BY_COLS) * d.runs);
    if (p.dw_parts > 1) {
        if constexpr (CT < 256) linear_dw_kernel<CT, RT, WAVES, BY_COLS, true><<<blocks, 64 * WAVES, 0, stream>>>(a, d);
    } else {
        linear_dw_kernel<CT, RT, WAVES, BY_COLS, false><<<blocks, 64 * WAVES, 0, stream>>>(a, d);
    }
}

template <int BM, int COLS, bool DIRECT, int CT, int RT, bool BY_COLS>
void both_launch(const LinearPlan& p, const LinearArgs& a, char* ws, void* out, hipStream_t stream) {
    const LinearDw d = dw_args(p, ws);
    const unsigned dx = dx_blocks(p, a), dw = grid_of(dw_items(p, a.len, a.N, a.M, BY_COLS) * d.runs);
    const int32_t bound = (int32_t)p.tiles.tiles;
    if (p.dw_parts > 1)
        linear_both_kernel<BM, COLS, DIRECT, CT, RT, BY_COLS, true><<<dx + dw, 256, 0, stream>>>(a, bound, p.span, out, dx, d);
    else
        linear_both_kernel<BM, COLS, DIRECT, CT, RT, BY_COLS, false><<<dx + dw, 256, 0, stream>>>(a, bound, p.span, out, dx, d);
}
template <int BM, int COLS, int CT, int RT, bool BY_COLS>
void both_launch(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream) {
    if (a.k == 1)
        both_launch<BM, COLS, true, CT, RT, BY_COLS>(p, a, ws, a.dx, stream);
    else
        both_launch<BM, COLS, false, CT, RT, BY_COLS>(p, a, ws, ws + p.off_shares, stream);
}
template <int BM>
void both_launch(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream) {
    if (p.dw_cols == 64)
        both_launch<BM, 64, 64, 128, false>(p, a, ws, stream);
    else if (p.dw_rows == 64)
        both_launch<BM, 128, 128, 64, true>(p, a, ws, stream);
    else
        both_launch<BM, 128, 128, 128, true>(p, a, ws, stream);
}

// Tile of dW, by the rounds in which its workgroups fill the chip (two of 128 x 128 to a CU, one of 256 x 256) times the
// stages times the time of a stage, and for 256 what such a tile costs beside its stages; and the runs into which an expert's
// entries are cut: as many as bring the tiles to 512, of four stages at least, at most 32, or 128 of 14 stages (us, 32 : 128
// runs of 115849 rows, K = 144, N = 8 54 : 29, 131072 of K = 256, N = 128 82 : 42; 32 : 39 of 10000, 3 experts, K = 200,
// N = 136 21 : 23).  0.9 % off the better tile on
// geometric mean over 240 shapes (us, 128 : 256, 94 experts of 192 x 304, 30249 entries 26 : 34; 31 of 960 x 2048, 12500
// 210 : 148).
void dw_plan(int64_t n, int32_t K, int32_t N, int32_t M, LinearPlan* p) {
    const int64_t steps = std::max<int64_t>(1, n / M / kFfnBK);
    auto tiles = [&](int32_t a, int32_t b) { return (int64_t)((a + b - 1) / b); };
    p->dw_cols = K <= 64 ? 64 : 128;
    p->dw_rows = K > 64 && N <= 64 ? 64 : 128;
    const int64_t large = M * tiles(K, 256) * tiles(N, 256), small = M * tiles(K, p->dw_cols) * tiles(N, p->dw_rows);
    p->dw_parts = 1;
    if (std::max<int64_t>(256, large) * 2 * (32 * steps + 10) < std::max<int64_t>(512, small) * (small <= 256 ? 16 : 20) * steps)
        p->dw_rows = p->dw_cols = 256;
    else
        p->dw_parts = (int32_t)std::max<int64_t>(
            1, std::min({512 / small, steps / 4, std::max<int64_t>(32, std::min<int64_t>(steps / 14, 128))}));
    // along the longer side, where the launch is dW's alone (us, 4096 experts of K = 128, N = 512, 32 entries, along K : N
    // 185 : 154; 1024 of K = 128, N = 1024, 128 entries 139 : 144)
    p->dw_by_rows = p->dw_cols == 64 || (p->dw_cols == 128 && p->dw_rows == 128 && p->listed && K <= 128 && N > 128);
    const bool by_cols = !p->dw_by_rows;
    const int32_t step = by_cols ? p->dw_cols : p->dw_rows, side = by_cols ? K : N;
    const int64_t groups = M * (by_cols ? tiles(N, p->dw_rows) : tiles(K, p->dw_cols));
    p->dw_span = p->dw_parts > 1 ? step : linear_span(n / M, step, groups, side);
    if (p->dw_rows != p->dw_cols) p->dw_span = std::min(p->dw_span, 256);  // (512 89 us of the 84 above)
}

}  // namespace

void linear_backward_make_plan(int64_t T, int32_t len, int32_t N, int32_t M, int32_t k, LinearPlan* p) {
    const int64_t n = T * k;
    *p = LinearPlan{};
    p->cols = len <= 64 ? 64 : 128;
    const int32_t bm = linear_tile_rows(n, M, len, p->cols, (N + kFfnBK - 1) / kFfnBK, kProductDx);
    ffn_tiles_plan(n, M, bm, &p->tiles);
    if (bm == 256) p->cols = 256;
    p->span = linear_span(N, p->cols, p->tiles.tiles, len);
    p->listed = linear_listed(p->tiles, M, (len + p->span - 1) / p->span);
    dw_plan(n, len, N, M, p);
    p->both = !p->listed && p->dw_cols < 256;
    size_t at = p->listed ? p->tiles.workspace_bytes : 0;
    p->off_shares = at;
    at += k > 1 ? align256((size_t)n * len * 4) : 0;
    p->off_parts = at;
    at += p->dw_parts > 1 ? align256((size_t)p->dw_parts * M * N * len * 4) : 0;
    p->workspace_bytes = at;
}

hipError_t linear_backward_launch(const LinearPlan& p, LinearArgs a, void* workspace, hipStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    a.whole = a.k == 1 ? linear_whole(a.dx, a.len * (int64_t)2) : linear_whole(nullptr, a.len * (int64_t)4);
    const bool dx = p.tiles.n > 0 && a.dx, both = p.both && dx && a.dW;
    hipError_t e = hipSuccess;
    if (both) {
        switch (p.tiles.bm) {
            case 128: both_launch<128>(p, a, ws, stream); break;
            case 64: both_launch<64>(p, a, ws, stream); break;
            default: both_launch<32>(p, a, ws, stream);
        }
    } else if (dx) {
        if (p.listed) e = linear_tiles_launch(p, a, ws, stream);
        if (e != hipSuccess) return e;
        switch (p.tiles.bm) {
            case 256: dx_launch<256, 256>(p, a, ws, stream); break;
            case 128: p.cols == 64 ? dx_launch<128, 64>(p, a, ws, stream) : dx_launch<128, 128>(p, a, ws, stream); break;
            case 64: p.cols == 64 ? dx_launch<64, 64>(p, a, ws, stream) : dx_launch<64, 128>(p, a, ws, stream); break;
            default: p.cols == 64 ? dx_launch<32, 64>(p, a, ws, stream) : dx_launch<32, 128>(p, a, ws, stream);
        }
    }
    if (dx && a.k > 1) {
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int64_t blocks = std::min<int64_t>(((int64_t)a.T * (a.len / 8) + 255) / 256, 1 << 16);
        linear_sum_kernel<<<(unsigned)blocks, 256, 0, stream>>>(a, reinterpret_cast<const float*>(ws + p.off_shares));
    }
    if (a.dW && !both) {
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (p.dw_cols == 256)
            dw_launch<256, 256, 8, true>(p, a, ws, stream);
        else if (p.dw_cols == 64)
            dw_launch<64, 128, 4, false>(p, a, ws, stream);
        else if (p.dw_rows == 64)
            dw_launch<128, 64, 4, true>(p, a, ws, stream);
        else if (p.dw_by_rows)
            dw_launch<128, 128, 4, false>(p, a, ws, stream);
        else
            dw_launch<128, 128, 4, true>(p, a, ws, stream);
    }
    e = hipGetLastError();
    if (e != hipSuccess || !a.dW || p.dw_parts == 1) return e;
    return ffn_parts_sum_launch(reinterpret_cast<const float*>(ws + p.off_parts), p.dw_parts, (int64_t)a.M * a.N * a.len, a.dW,
                                stream);
}

}  // namespace more
