// The experts' linear maps for gfx950: for every entry p = t k + j of a selection with expert e = idx[t][j],
//   y_p = x_t W_e^T      [N]
// in bf16, or in int8 with a scale per row of x and per row of W:
//   y_p = gate_p xs_t ws_e[c] (sum_i q_t[i] Wq_e[c][i])
// The entries are taken in the order of Sort + Count and cut into tiles of rows of one expert (ffn_tiles);
// linear_kernel multiplies a tile, linear_few_kernel does without tiles where there are few entries.  y goes to the
// entry's row, so nothing is scattered afterwards; dropped entries get rows of zeros.
// Numerics: bf16, exact products and fp32 sums; int8, exact 32-bit integer sums (at most 2^16 values of at most 2^14),
// converted to fp32 and multiplied by three fp32 factors.  One rounding to y's type.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ffn_device.h"
#include "linear.h"
#include "linear_device.h"

namespace more {

// ------------------------------------------------------------------------------ tiles
// A workgroup computes a tile's rows of y, `span` columns in steps of COLS: the rows of W are the M side, the
// entries' rows of x the N side.  The pipeline runs over (column step, contraction step) pairs, so that a
// short contraction does not drain it.  Small experts are bound by their weights' way from memory (4096 experts of K = 512,
// N = 128 with 32 rows 117 us, 587 MB at 5.0 TB/s beside the gathered rows of x; 8-bit, 8192 of K = 4096, N = 128 with a
// quarter row 140 us), large ones by how well the matrix cores are fed: 32 experts of 2048 x 2048 with 1024 rows 282 us a call,
// 975 TFLOP/s, the kernel 291 to 325 in a trace.  Counters there: the matrix cores work in 44 % of the cycles, waves wait in
// 38 %, CUs have no tile in 16 % (4.5 rounds of tiles, the last ones of an expert partly empty), the clock is 2.1 GHz.  Full
// tiles in eight whole rounds (65536 rows) reach 1120 TFLOP/s, a dense library product of 8192^3 1600.
// LINES: y is stored in whole lines by way of LDS, where a wave has whole lines of a row (us, in halves of lines : whole,
// 65536 rows, N = 2048, 16 experts, bf16 K = 128 115 : 78, K = 512 194 : 173; 32 experts of 2048 x 2048, 32768 entries 290 : 280).
template <int BM, int COLS, int STAGES>
struct LinearShape {
    static constexpr int kWaves = BM == 256 ? 8 : 4;
    static constexpr int kThreads = 64 * kWaves;
    // an expert has one tile, mostly: nontemporal weights (4096 experts, K = 64, N = 512, 32 rows 83 us, without 89)
    static constexpr bool kOnce = BM <= 64;
    static constexpr int kWavesM = BM >= 64 ? 2 : 4;
    static constexpr int kM = COLS / kWavesM / 16;
    static constexpr int kN = BM / (kWaves / kWavesM) / 16;
    static constexpr int kRowsAt = COLS * 128;
    static constexpr int kStageBytes = kRowsAt + BM * 128;
    static constexpr int kLoads = (COLS + BM) / kWaves / 8;
};

constexpr int linear_threads(int bm) { return bm == 256 ? 512 : 256; }
template <bool I8, int BM, int COLS, int STAGES, bool LINES, bool OWN>
__global__ __launch_bounds__(linear_threads(BM), 2) void linear_kernel(LinearArgs a, const void* __restrict__ list,
                                                                    int32_t bound, int32_t span) {
    using S = LinearShape<BM, COLS, STAGES>;
    using Type = LinearType<I8>;
    static_assert(S::kThreads == linear_threads(BM) && (!LINES || S::kM % 4 == 0), "");
    constexpr int kRing = STAGES * S::kStageBytes;
    __shared__ __attribute__((aligned(1024))) char smem_raw[kRing + (LINES ? S::kWaves * kLinesScratch : 0)];
    LdsChar* smem = (LdsChar*)smem_raw;
    LdsChar* lines = smem + (LINES ? kRing + ffn_wave() * kLinesScratch : 0);
    const int32_t len = a.len, N = a.N;
    const int32_t n = a.T * a.k;
    const int32_t spans = (N + span - 1) / span;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int wm = wave % S::kWavesM, wn = wave / S::kWavesM;
    linear_for_each<BM, S::kThreads, OWN>(a, list, bound, spans, smem, [&](const FfnTile& tile, int32_t turn) {
        const int32_t c0 = turn * span, c1 = min(N, c0 + span);
        if (tile.expert < 0) {  // dropped entries: zero rows
            const int32_t pieces = (c1 - c0) / 8;
            for (int32_t i = threadIdx.x; i < tile.rows * pieces; i += S::kThreads) {
                const uint32_t p = a.sorted[tile.row0 + i / pieces];
                if (p < (uint32_t)n) linear_zero(a, p, c0 + 8 * (i % pieces));
            }
            return;
        }
        const uint16_t* W = a.W + (int64_t)tile.expert * N * len;
        const float* w_scale = I8 ? a.w_scale + (int64_t)tile.expert * N : nullptr;
        RowTileLoader<COLS, S::kWaves, S::kOnce> weights;
        RowTileLoader<BM, S::kWaves> rows;
        rows.init([&](int i) {
            const uint32_t p = a.sorted[tile.row0 + min(i, tile.rows - 1)];
            return a.x + (int64_t)(p < (uint32_t)n ? p / (uint32_t)a.k : 0) * len;
        });
        uint32_t place[S::kN];
        float row_scale[S::kN];
#pragma unroll
        for (int j = 0; j < S::kN; ++j) {
            const int32_t row = 16 * (wn * S::kN + j) + (lane & 15);
            place[j] = row < tile.rows ? (uint32_t)a.sorted[tile.row0 + row] : 0xFFFFFFFFu;
            row_scale[j] = linear_row_scale<I8>(a, place[j], n);
        }
        typename Type::Acc acc[S::kM][S::kN];
#pragma unroll
        for (int i = 0; i < S::kM; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) acc[i][j] = Type::zero();
        const int32_t ksteps = (len + kFfnBK - 1) / kFfnBK;
        const int32_t csteps = (c1 - c0 + COLS - 1) / COLS;
        // (column step, contraction step) of the next load and of the next product
        int32_t lc = c0, lk = 0, cc = c0, ck = 0;
        using G = FfnGroups<S::kM, S::kM == 8 ? 4 : 2>;
        using M = FfnFragments<G::kSize>;
        using F = FfnFragments<S::kN>;
        ffn_pipeline<STAGES, S::kLoads, G::kGroups, BM == 256, M, F>(
            ksteps * csteps, 16 * wn * S::kN < tile.rows,
            [&](int, int slot) {
                if (lk == 0) weights.init([&](int i) { return W + (int64_t)min(lc + i, N - 1) * len; });
                weights.load(smem + slot * S::kStageBytes, lk * kFfnBK, len);
            },
            [&](int, int slot) {
                rows.load(smem + slot * S::kStageBytes + S::kRowsAt, lk * kFfnBK, len);
                if (++lk == ksteps) {
                    lk = 0;
                    lc += COLS;
                }
            },
            ffn_work(
                [&](int slot, int kk, int group, M& m) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < S::kM)
                            m.v[i] = row_fragment(smem + slot * S::kStageBytes, 16 * (wm * S::kM + G::tile(group, i)), kk);
                },
                [&](int slot, int kk, F& f) {
#pragma unroll
                    for (int j = 0; j < S::kN; ++j)
                        f.v[j] = row_fragment(smem + slot * S::kStageBytes + S::kRowsAt, 16 * (wn * S::kN + j), kk);
                },
                [&](int group, const M& m, const F& f) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < S::kM)
#pragma unroll
                            for (int j = 0; j < S::kN; ++j) {
                                auto& c = acc[G::tile(group, i)][j];
                                c = Type::multiply(m.v[i], f.v[j], c);
                            }
                },
                [&] {
                    if (++ck < ksteps) return;
                    auto store_lines = [&](auto wide) {
                        using L = Lines<decltype(wide)::value>;
                        using Out = typename L::Element;
#pragma unroll
                        for (int i0 = 0; i0 < S::kM; i0 += L::kTiles) {
                            const int32_t c = cc + 16 * (wm * S::kM + i0);
                            f32x4 ws[L::kTiles];
#pragma unroll
                            for (int i = 0; i < L::kTiles; ++i) ws[i] = linear_w_scale<I8>(w_scale, c + 16 * i, N);
#pragma unroll
                            for (int j = 0; j < S::kN; ++j) {
#pragma unroll
                                for (int i = 0; i < L::kTiles; ++i)
                                    L::place(lines, i, linear_value<I8>(acc[i0 + i][j], row_scale[j], ws[i]));
                                L::store(lines, c1 - c, a.whole, [&](int r) -> Out* {
                                    const uint32_t p = (uint32_t)__shfl((int)place[j], r, 64);
                                    return p < (uint32_t)n ? static_cast<Out*>(a.y) + (int64_t)p * N + c : nullptr;
                                });
                            }
                        }
                    };
                    if constexpr (LINES) {
                        if (a.wide) store_lines(std::true_type{});
                        else store_lines(std::false_type{});
                    } else if (S::kM % 2 == 0 && !a.wide) {
#pragma unroll
                        for (int i = 0; i + 1 < S::kM; i += 2) {
                            const int32_t c = cc + 16 * (wm * S::kM + i), mine = c + 8 * (lane >> 4);
                            const f32x4 ws0 = linear_w_scale<I8>(w_scale, c, N), ws1 = linear_w_scale<I8>(w_scale, c + 16, N);
#pragma unroll
                            for (int j = 0; j < S::kN; ++j) {
                                const u32x4 v = linear_pair(linear_value<I8>(acc[i][j], row_scale[j], ws0),
                                                            linear_value<I8>(acc[i + 1][j], row_scale[j], ws1));
                                if (place[j] < (uint32_t)n && mine < c1)
                                    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + (int64_t)place[j] * N + mine) = v;
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < S::kM; ++i) {
                            const int32_t c = cc + 16 * (wm * S::kM + i), mine = c + 4 * (lane >> 4);
                            const f32x4 ws = linear_w_scale<I8>(w_scale, c, N);
#pragma unroll
                            for (int j = 0; j < S::kN; ++j)
                                if (place[j] < (uint32_t)n && mine < c1)
                                    linear_put(a.y, a.wide, (int64_t)place[j] * N + mine,
                                               linear_value<I8>(acc[i][j], row_scale[j], ws));
                        }
                    }
#pragma unroll
                    for (int i = 0; i < S::kM; ++i)
#pragma unroll
                        for (int j = 0; j < S::kN; ++j) acc[i][j] = Type::zero();
                    ck = 0;
                    cc += COLS;
                }));
    });
}

// ------------------------------------------------------------------------------ few entries
// Where there are few entries, the weights' way from memory is all that counts: they go straight into the
// registers of the matrix instruction (16 weight rows against 16 entries), with no LDS, no tile list and no
// barrier on the way.  Workgroups are laid over the sorted entries; the one whose entry is the first, 17th, ...
// of its expert takes that and the next 15 entries, the others end at once.
// Bound by the dependent reads sorted -> idx -> operands and the launch: one token, 8 experts of K = 2048, N = 128 4.7 us in a
// graph, 6.3 by calls (in 8 bits 4.1).
// SPLIT: the waves share 16 columns, take pieces of 64 words of the contraction in turn, and their sums are
// added in wave order; else each wave has 32 columns of its own.
constexpr int kFewWaves = 8;
template <bool SPLIT>
constexpr int few_span() {
    return SPLIT ? 16 : 32 * kFewWaves;
}

template <bool I8, bool SPLIT>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(LinearArgs a) {
    using Type = LinearType<I8>;
    using Acc = typename Type::Acc;
    constexpr int kR = SPLIT ? 1 : 2;      // groups of 16 columns per wave
    constexpr int kAhead = SPLIT ? 4 : 2;  // pieces of 64 words in flight per wave
    constexpr int kStep = SPLIT ? 64 * kFewWaves : 64;
    constexpr int kSpan = few_span<SPLIT>();
    __shared__ Acc part[SPLIT ? kFewWaves : 1][64];
    const int32_t len = a.len, N = a.N, n = a.T * a.k;
    const int32_t spans = (N + kSpan - 1) / kSpan;
    const int wave = ffn_wave(), lane = ffn_lane();
    for (int64_t item = blockIdx.x; item < (int64_t)n * spans; item += gridDim.x) {
        const int32_t i = (int32_t)(item / spans);
        const int32_t c0 = (int32_t)(item % spans) * kSpan + (SPLIT ? 0 : 32 * wave);
        if (c0 >= N) continue;  // (SPLIT: never)
        const FewRows f = few_rows(a.sorted, a.idx, a.offsets, a.M, n, i);
        if (f.rows == 0) continue;
        const bool mine = (lane & 15) < f.rows && f.p < (uint32_t)n;
        if (f.expert < 0) {  // a dropped entry
            const int32_t c = c0 + 8 * (lane >> 4);
            if (mine && (!SPLIT || (wave == 0 && lane < 32)) && c < N) linear_zero(a, f.p, c);
            continue;
        }
        const int32_t at = 8 * (lane >> 4);
        const uint16_t* w[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r)
            w[r] = a.W + ((int64_t)f.expert * N + min(c0 + 16 * r + (lane & 15), N - 1)) * len + at;
        // (the columns of lanes past the rows are not stored)
        const uint16_t* x = a.x + (int64_t)(f.p < (uint32_t)n ? f.p / (uint32_t)a.k : 0) * len + at;
        Acc acc[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) acc[r] = Type::zero();
        for (int32_t k0 = SPLIT ? 64 * wave : 0; k0 < len; k0 += kStep * kAhead) {
            bf16x8 fw[kR][kAhead][2], fx[kAhead][2];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int32_t k = k0 + kStep * q + 32 * c;
                    const bool in = k + at < len;
                    fx[q][c] = few_load(x + k, in);
#pragma unroll
                    for (int r = 0; r < kR; ++r) fw[r][q][c] = few_load(w[r] + k, in);
                }
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int r = 0; r < kR; ++r) acc[r] = Type::multiply(fw[r][q][c], fx[q][c], acc[r]);
        }
        if constexpr (SPLIT) {
            __syncthreads();  // the item before has been read
            part[wave][lane] = acc[0];
            __syncthreads();
            if (wave > 0) continue;
#pragma unroll
            for (int v = 1; v < kFewWaves; ++v) acc[0] += part[v][lane];
        }
        if (!mine) continue;
        const float row_scale = linear_row_scale<I8>(a, f.p, n);
        const float* w_scale = I8 ? a.w_scale + (int64_t)f.expert * N : nullptr;
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const int32_t c = c0 + 16 * r, at_c = c + 4 * (lane >> 4);
            const f32x4 v = linear_value<I8>(acc[r], row_scale, linear_w_scale<I8>(w_scale, c, N));
            if (at_c < N) linear_put(a.y, a.wide, (int64_t)f.p * N + at_c, v);
        }
    }
}

// ------------------------------------------------------------------------------ host
namespace {

constexpr int64_t kMaxBlocks = 1 << 19;
unsigned grid_of(int64_t items) { return (unsigned)(std::min<int64_t>((items + 7) / 8, kMaxBlocks / 8) * 8); }
unsigned few_grid(int64_t items) { return (unsigned)std::min<int64_t>(items, 1 << 22); }

template <bool I8, int BM, int COLS, int STAGES>
void tiled(const LinearPlan& p, const LinearArgs& a, const char* ws, hipStream_t stream) {
    constexpr bool kLines = BM >= 64 && COLS >= 128;
    constexpr bool kOwn = BM < 256 && !(BM == 32 && STAGES == 2);  // (else there is always a list)
    const unsigned blocks = grid_of(p.tiles.tiles * ((a.N + p.span - 1) / p.span));
    const void* list = ws + p.tiles.off_tiles;
    const int32_t bound = (int32_t)p.tiles.tiles;
    if (p.listed)
        linear_kernel<I8, BM, COLS, STAGES, kLines, false><<<blocks, linear_threads(BM), 0, stream>>>(a, list, bound, p.span);
    else if constexpr (kOwn)
        linear_kernel<I8, BM, COLS, STAGES, kLines, true><<<blocks, linear_threads(BM), 0, stream>>>(a, nullptr, bound, p.span);
}

template <bool I8>
void forward(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream) {
    if (p.few) {
        const unsigned blocks = few_grid(p.tiles.n * ((a.N + p.span - 1) / p.span));
        if (p.split)
            linear_few_kernel<I8, true><<<blocks, 64 * kFewWaves, 0, stream>>>(a);
        else
            linear_few_kernel<I8, false><<<blocks, 64 * kFewWaves, 0, stream>>>(a);
        return;
    }
    switch (p.tiles.bm) {
        case 256:  // (8 bits: linear_stream_launch)
            if constexpr (!I8) tiled<I8, 256, 256, 2>(p, a, ws, stream);
            return;
        case 128: return p.cols == 64 ? tiled<I8, 128, 64, 2>(p, a, ws, stream) : tiled<I8, 128, 128, 2>(p, a, ws, stream);
        case 64: return p.cols == 64 ? tiled<I8, 64, 64, 3>(p, a, ws, stream) : tiled<I8, 64, 128, 3>(p, a, ws, stream);
        default:
            if (p.cols == 64) return tiled<I8, 32, 64, 3>(p, a, ws, stream);
            return p.stages == 2 ? tiled<I8, 32, 128, 2>(p, a, ws, stream) : tiled<I8, 32, 128, 3>(p, a, ws, stream);
    }
}

}  // namespace

// Rows of a tile: 32 where experts have less than 8 rows (then mostly one tile, whose weights are not read again), else
// what costs least: the rounds in which the workgroups fill the chip (two of up to 128 rows to a CU, one of 256), beyond three
// with half a round of rest, times the stages times the time of a stage and what a tile costs beside its stages.
// Fitted to 800 shapes (1 to 8192 experts, 4 to 16384 rows each, contractions and columns of 16 to 4096, of which half are not
// multiples of 64): 2.0 % off the best on geometric mean, five in a hundred more than 14 %.  Bf16 rows that split lines have
// costs of their own: small tiles touch more lines for a product (27 experts of K = 2952, N = 152 with 552 rows, 64 : 128 rows
// 73 : 40).  us for 32 : 64 : 128 : 256 rows, one expert of K = 2912, N = 1160 with 1976 rows 83 : 65 : 34 : 76; 8 bits,
// 15 of K = 3200, N = 3008 with 225 rows 174 : 105 : 55 : 89; dx, 11 of K = 3648, N = 576 with 2523 rows 287 : 234 : 174 : 148.
namespace {
struct TileCost {
    int32_t alone, two;  // time of a stage, one workgroup and two to a CU
    int32_t fixed;       // of a tile beside its stages
    int32_t narrow;      // sixteenths of a stage's time where a step has 64 columns
};
constexpr TileCost kTileCost[4][4] = {{{7, 18, 18, 13}, {14, 17, 30, 14}, {14, 17, 46, 13}, {25, 25, 119, 16}},
                                      {{7, 25, 18, 13}, {14, 20, 30, 14}, {17, 17, 46, 13}, {25, 25, 119, 16}},
                                      {{7, 10, 8, 14}, {9, 12, 26, 10}, {16, 16, 27, 10}, {21, 21, 87, 16}},
                                      {{14, 21, 31, 17}, {8, 18, 43, 16}, {12, 16, 61, 8}, {14, 14, 163, 16}}};
}  // namespace
int32_t linear_tile_rows(int64_t n, int32_t M, int32_t cols, int32_t cols_of, int64_t steps, LinearProduct product) {
    if (n / std::max<int64_t>(1, std::min<int64_t>(n, M)) < 8) return 32;
    int32_t best = 64;
    int64_t least = INT64_MAX;
    for (int32_t i = 0, bm = 32; bm <= 256; bm *= 2, ++i) {
        if (bm == 256 && product == kProductQ8 && steps < kStreamSteps) break;  // (linear_stream_kernel needs them)
        const TileCost c = kTileCost[product][i];
        const int32_t step = bm == 256 ? 256 : cols_of;
        const int64_t slots = bm == 256 ? 256 : 512;
        const int64_t items = ffn_expected_tiles2(n, M, bm) * ((cols + step - 1) / step) / 2;
        const int64_t stage = (items <= 256 ? c.alone : c.two) * (step == 64 ? c.narrow : 16);
        const int64_t item = steps * stage + 16 * c.fixed;
        const int64_t cost = items <= 3 * slots ? (items + slots - 1) / slots * 2 * item : items * 2 * item / slots + item;
        if (cost < least) {
            least = cost;
            best = bm;
        }
    }
    return best;
}

// A single step where the contraction alone fills the pipeline (three stages), where the groups are too few to fill the chip
// with more, or where the workgroups would be uneven; else 256, or 512 of very many groups.  Fitted to 200 shapes: the map 2.5 %,
// in 8 bits 3.6 %, dx 2.4 % and dW 5.7 % off the best of the three on geometric mean (us, a step of 128 : 256 : 512, dx of
// 5338 groups, K = 736, N = 48 73 : 56 : 65; dW of 64 experts of 1024 x 1024, 31 entries 34 : 29 : 37; of 4096, K = 64,
// N = 512, 32 entries 99 : 79 : 66; of 32, 1024 x 520, 250 entries 31 : 33 : 59).
int32_t linear_span(int64_t len, int32_t step, int64_t groups, int32_t side) {
    if (len > 3 * kFfnBK) return step;
    const int32_t steps = (side + step - 1) / step;
    if ((steps % 4 == 0 || steps >= 18) && groups * ((side + 511) / 512) >= 2048) return std::max(step, 512);
    if ((steps % 2 == 0 || steps >= 9) && groups * ((side + 255) / 256) >= 512) return std::max(step, 256);
    return step;
}

// A workgroup finds its tile itself while few of them do the same: up to kLinearOwn experts and three workgroups to a
// place (two to a CU).  us, found : listed by a launch ahead, 240 shapes of up to 512 workgroups 2.9 less, of up to 1024 2.4,
// to 2048 0.6, to 4096 -0.3 (T = 200, k = 4, 64 experts of 512 x 512 10.3 : 13.6; T = 16384, 256 experts 80.6 : 77.3).  With
// 256 rows to a tile it would take registers that the products want.
bool linear_listed(const FfnPlan& tiles, int32_t M, int64_t spans) {
    return M > kLinearOwn || tiles.bm == 256 || tiles.tiles * spans > 1536;
}

// Upper bound on the workgroups along the entries that have work in the kernel without tiles.
static int64_t few_starts(int64_t n, int32_t M) { return std::min<int64_t>(n, std::min<int64_t>(n, M) + n / kFewRows); }

void linear_make_plan(int64_t T, int32_t len, int32_t N, int32_t M, int32_t k, bool q8, LinearPlan* p) {
    const int64_t n = T * k;
    *p = LinearPlan{};
    p->cols = N <= 64 ? 64 : 128;
    const int32_t bm = linear_tile_rows(n, M, N, p->cols, (len + kFfnBK - 1) / kFfnBK,
                                        q8 ? kProductQ8 : len % kFfnBK ? kProductSplit : kProductMap);
    ffn_tiles_plan(n, M, bm, &p->tiles);
    // The kernel without tiles has a short way to its first operands, but reads the weights again for every 16 entries, the
    // rows of x in every workgroup, and starts a workgroup for each entry, of which most end at once: it is taken
    // while these are few, fewer where the other one does without a launch for its list.  Its waves share the columns of
    // contractions beyond 256, up to 512 only while that leaves few workgroups.  Fitted to 500 shapes of both types (1 to 4096
    // entries, 1 to 8192 experts): 2.4 % off the best of the three on geometric mean, 3.7 % beyond kLinearOwn experts.  us with
    // tiles : own columns : shared, bf16, one dense map of K = 192, N = 480, 180 rows 6.3 : 11.4 : 12.9; 8-bit, one entry of
    // K = 2048, N = 128 18.9 : 19.2 : 7.6; bf16, 93 entries in 3107 experts of K = 96, N = 432 9.3 : 6.0 : 10.6.
    const int64_t starts = few_starts(n, M), spans = (N + few_span<false>() - 1) / few_span<false>();
    const bool own = M <= kLinearOwn;
    p->few = n * len <= (int64_t)1 << 20 && n * spans <= (own ? 256 : 2048) &&
             starts * N <= 12000 + (own ? 0 : ((int64_t)1 << 24) / len);
    if (p->few) {
        p->split = len > 512 || (len > 256 && starts * spans < 64);
        p->span = p->split ? few_span<true>() : few_span<false>();
        return;
    }
    if (bm == 256) p->cols = 256;
    p->stream = q8 && bm == 256;
    p->span = p->stream ? p->cols : linear_span(len, p->cols, p->tiles.tiles, N);
    p->stages = bm >= 128 ? 2 : bm == 64 || p->cols == 64 ? 3 : p->tiles.tiles * ((N + p->span - 1) / p->span) >= 2048 ? 2 : 3;
    p->listed = linear_listed(p->tiles, M, (N + p->span - 1) / p->span);
    p->workspace_bytes = p->listed ? p->tiles.workspace_bytes : 0;
}

hipError_t linear_tiles_launch(const LinearPlan& p, const LinearArgs& a, void* workspace, hipStream_t stream) {
    FfnArgs f = {};
    f.offsets = a.offsets;
    f.M = a.M;
    return ffn_tiles_launch(p.tiles, f, workspace, stream);
}

hipError_t linear_launch(const LinearPlan& p, const LinearArgs& a, void* workspace, hipStream_t stream) {
    if (p.listed) {
        const hipError_t e = linear_tiles_launch(p, a, workspace, stream);
        if (e != hipSuccess) return e;
    }
    char* ws = static_cast<char*>(workspace);
    if (p.stream) return linear_stream_launch(p, a, ws, stream);
    if (a.q8)
        forward<true>(p, a, ws, stream);
    else
        forward<false>(p, a, ws, stream);
    return hipGetLastError();
}

}  // namespace more
