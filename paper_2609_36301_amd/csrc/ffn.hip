// The experts' gated feed-forward block for gfx950: for every entry p = t k + j of a selection with
// expert e = idx[t][j],
//   A_p = silu(x_t Wg_e^T) * (x_t Wu_e^T)      [s]
//   y_p = gate_p * (A_p W2_e^T)                [h]
// with W1t[e] = [Wg_e; Wu_e] and W2t[e] = W2_e.  The entries are taken in the order of Sort + Count, so
// the rows of an expert are neighbours; they are cut into tiles of at most `bm` rows of one expert.
//
// Kernels of one call:
//   ffn_tiles   lists the tiles
//   ffn_up      both projections, the activation and the product of one tile and 64 hidden units:
//               A (bf16, sorted order) into the workspace
//   ffn_down    A W2^T times the gate, to the entry's row of y
// With few rows per expert (a decode step) ffn_few_up and ffn_few_down do the same without tiles.
// Numerics: both contractions take bf16 operands with fp32 accumulation; A is rounded to bf16 once (the
// matrix cores' operand type), or to two bf16 addends where few values are (FfnPlan::planes); the activation and
// the gate are applied in fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "ffn.h"
#include "ffn_device.h"
#include "ffn_up.h"

namespace more {

// ------------------------------------------------------------------------------ tiles
// A workgroup lists the tiles of 1024 experts, one per thread; up to kTileAlone experts it counts the tiles
// of all earlier experts itself (one launch), beyond it adds their workgroups' counts, which
// ffn_tile_sums_kernel has made (counting 2^20 experts' offsets in every workgroup would be 2^29 reads).
// The last workgroup adds the tiles of the dropped entries.
// Offsets that Sort + Count cannot have written are cut to [0, n], tiles past the list's end are not written
// and counts are 64 bits wide (offsets that go up and down can ask for n / bm tiles per expert), so that no
// call reads or writes outside its buffers.
constexpr int kTileThreads = 1024;
constexpr int32_t kTileAlone = 1 << 16;

__device__ __forceinline__ int32_t ffn_cut(int32_t v, int32_t n) { return v < 0 ? 0 : v > n ? n : v; }

// The tiles of expert e, from its offsets.
__device__ __forceinline__ int32_t ffn_tile_count(const int32_t* offsets, int32_t e, int32_t n, int32_t log_bm) {
    const int32_t len = ffn_cut(offsets[e + 1], n) - ffn_cut(offsets[e], n);
    return len > 0 ? (len + (1 << log_bm) - 1) >> log_bm : 0;
}

__global__ __launch_bounds__(kTileThreads) void ffn_tile_sums_kernel(const int32_t* __restrict__ offsets, int32_t M,
                                                                     int32_t n, int32_t log_bm,
                                                                     int64_t* __restrict__ sums) {
    __shared__ int64_t part[kTileThreads / 64];
    const int32_t e = (int32_t)blockIdx.x * kTileThreads + threadIdx.x;
    int64_t v = e < M ? ffn_tile_count(offsets, e, n, log_bm) : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < kTileThreads / 64; ++w) v += part[w];
    sums[blockIdx.x] = v;
}

__global__ __launch_bounds__(kTileThreads) void ffn_tiles_kernel(const int32_t* __restrict__ offsets, int32_t M,
                                                                 int32_t n, int32_t log_bm, int64_t bound,
                                                                 const int64_t* __restrict__ sums,
                                                                 int32_t* __restrict__ list) {
    FfnTile* tiles = reinterpret_cast<FfnTile*>(reinterpret_cast<char*>(list) + kFfnTileHeader);
    __shared__ int64_t part[2][kTileThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t bm1 = (1 << log_bm) - 1;
    const int32_t e0 = (int32_t)blockIdx.x * kTileThreads, e = e0 + tid;
    const int32_t valid = ffn_cut(offsets[M], n);
    const int32_t begin = ffn_cut(offsets[min(e, M)], n);
    const int32_t len = max(ffn_cut(offsets[min(e + 1, M)], n) - begin, 0);
    int64_t before = 0;
#pragma unroll 8
    for (int32_t q = tid; q < (sums ? (int32_t)blockIdx.x : e0); q += kTileThreads)
        before += sums ? sums[q] : (int64_t)ffn_tile_count(offsets, q, n, log_bm);
    // inclusive scan of the threads' tiles over the workgroup, and the sum of `before`
    const int32_t mine = (len + bm1) >> log_bm;
    int64_t scan = mine, sum = before;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(scan, d, 64);
        scan += lane >= d ? o : 0;
        sum += __shfl_xor(sum, d, 64);
    }
    if (lane == 63) part[0][wave] = scan;
    if (lane == 0) part[1][wave] = sum;
    __syncthreads();
    int64_t base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kTileThreads / 64; ++w) {
        total += part[0][w] + part[1][w];
        base += part[1][w] + (w < wave ? part[0][w] : 0);
    }
    const int64_t at = base + scan - mine;
    if (mine <= 16)
        for (int32_t r = 0; r < len && at + (r >> log_bm) < bound; r += bm1 + 1)
            tiles[at + (r >> log_bm)] = FfnTile{e, begin + r, min(len - r, bm1 + 1), 0};
    // experts with more tiles: the wave's lanes write them together
    for (uint64_t left = __ballot(mine > 16); left; left &= left - 1) {
        const int l = __builtin_ctzll(left);
        const int32_t len1 = __builtin_amdgcn_readlane(len, l), begin1 = __builtin_amdgcn_readlane(begin, l);
        const int32_t mine1 = (len1 + bm1) >> log_bm;
        const int64_t at1 = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int32_t)(at >> 32), l) << 32 |
                                      (uint32_t)__builtin_amdgcn_readlane((int32_t)at, l));
        for (int32_t q = lane; q < mine1 && at1 + q < bound; q += 64) {
            const int32_t r = q << log_bm;
            tiles[at1 + q] = FfnTile{e - lane + l, begin1 + r, min(len1 - r, bm1 + 1), 0};
        }
    }
    if (blockIdx.x == gridDim.x - 1) {
        const int32_t extra = (n - valid + bm1) >> log_bm;
        for (int32_t r = tid; r < extra; r += kTileThreads)
            if (total + r < bound) {
                const int32_t row = valid + (r << log_bm);
                tiles[total + r] = FfnTile{-1, row, min(n - row, bm1 + 1), 0};
            }
        // the count, the count without the dropped entries' tiles, and counters that a reader of the list may use
        if (tid == 0) list[0] = (int32_t)std::min<int64_t>(total + extra, bound);
        if (tid == 1) list[1] = (int32_t)std::min<int64_t>(total, bound);
        if (tid >= 8 && tid < 16) list[tid] = 0;
    }
}

// ------------------------------------------------------------------------------ down
// A workgroup computes y of one tile and `hspan` columns in steps of kCols: the rows of W2t are the M
// side, the tile's rows of A the N side.  The pipeline runs over (column step, contraction step) pairs,
// so that the short contraction of small experts (one step up to s = 64) does not drain it.  Bound like
// ffn_up: 4096 experts of h = 512, s = 64 with 32 rows 100 us, 4.2 TB/s (a third of it y); 32 experts of
// h = 2048, s = 1024 with 1024 rows 225 us, 611 TFLOP/s (256 x 256 tiles, half as many rounds over the chip
// as ffn_up, and the rest of the last one idle).  y is stored 8 bytes a lane, 32 bytes of a row, and L2 joins
// the lines (stored by way of LDS in whole lines it was slower here).
// STAGES: of tiles of 32 rows two leave room for four workgroups to a CU instead of two, so two are taken from
// eight workgroups per CU on, else three (us, two : three, 16904 workgroups, 1800 experts of h = 4096, s = 64 with
// one row 148 : 165; 2608, h = 1024, s = 128 14 : 18; 1328, h = 4096, s = 128 55 : 47).
template <int BM, int STAGES>
struct DownShape {
    static constexpr int kWaves = BM == 256 ? 8 : 4;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr bool kOnce = BM == 32;               // an expert has one tile, mostly
    static constexpr int kCols = BM == 256 ? 256 : 128;   // columns of a step
    static constexpr int kWavesM = BM >= 64 ? 2 : 4;
    static constexpr int kM = kCols / kWavesM / 16;
    static constexpr int kN = BM / (kWaves / kWavesM) / 16;
    static constexpr int kStages = STAGES;
    static constexpr int kRowsAt = kCols * 128;
    static constexpr int kStageBytes = kRowsAt + BM * 128;
    static constexpr int kLoads = (kCols + BM) / kWaves / 8;
};

constexpr int down_threads(int bm) { return bm == 256 ? 512 : 256; }
template <int BM, int STAGES>
__global__ __launch_bounds__(down_threads(BM), 2) void ffn_down_kernel(FfnArgs a, const void* __restrict__ list,
                                                               const uint16_t* __restrict__ hidden, int32_t hspan,
                                                               uint16_t* __restrict__ y) {
    using S = DownShape<BM, STAGES>;
    static_assert(S::kThreads == down_threads(BM), "");
    __shared__ __attribute__((aligned(1024))) char smem_raw[S::kStages * S::kStageBytes];
    LdsChar* smem = (LdsChar*)smem_raw;
    const FfnTile* tiles = ffn_tile_list(list);
    const int32_t s = a.s, h = a.h;
    const int32_t n = a.T * a.k;
    const int32_t spans = (h + hspan - 1) / hspan;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int wm = wave % S::kWavesM, wn = wave / S::kWavesM;
    const int64_t total = (int64_t)*static_cast<const int32_t*>(list) * spans;
    ffn_for_each(total, [&](int64_t item) {
        const FfnTile tile = tiles[item / spans];
        const int32_t h0 = (int32_t)(item % spans) * hspan, h1 = min(h, h0 + hspan);
        if (tile.expert < 0) {  // dropped entries: zero rows
            const int32_t pieces = (h1 - h0) / 8;
            for (int32_t i = threadIdx.x; i < tile.rows * pieces; i += S::kThreads) {
                const uint32_t p = a.sorted[tile.row0 + i / pieces];
                if (p < (uint32_t)n)
                    *reinterpret_cast<u32x4*>(y + (int64_t)p * h + h0 + 8 * (i % pieces)) = u32x4{0u, 0u, 0u, 0u};
            }
            return;
        }
        const uint16_t* W = a.W2t + (int64_t)tile.expert * h * s;
        RowTileLoader<S::kCols, S::kWaves, S::kOnce> weights;
        RowTileLoader<BM, S::kWaves> rows;
        rows.init([&](int i) { return hidden + (int64_t)(tile.row0 + min(i, tile.rows - 1)) * s; });
        uint32_t place[S::kN];
        float gate[S::kN];
#pragma unroll
        for (int j = 0; j < S::kN; ++j) {
            const int32_t row = 16 * (wn * S::kN + j) + (lane & 15);
            place[j] = row < tile.rows ? (uint32_t)a.sorted[tile.row0 + row] : 0xFFFFFFFFu;
            gate[j] = a.gate && place[j] < (uint32_t)n ? a.gate[place[j]] : 1.0f;
        }
        f32x4 acc[S::kM][S::kN];
#pragma unroll
        for (int i = 0; i < S::kM; ++i)
#pragma unroll
            for (int j = 0; j < S::kN; ++j) acc[i][j] = zero_f32x4();
        const int32_t ksteps = (s + kFfnBK - 1) / kFfnBK, kall = ksteps * a.planes;
        const int32_t hsteps = (h1 - h0 + S::kCols - 1) / S::kCols;
        // (column step, contraction step) of the next load and of the next compute
        int32_t lh = h0, lk = 0, ch = h0, ck = 0;
        using G = FfnGroups<S::kM, BM == 256 ? 4 : 2>;
        using M = FfnFragments<G::kSize>;
        using N = FfnFragments<S::kN>;
        ffn_pipeline<S::kStages, S::kLoads, G::kGroups, BM == 256, M, N>(
            kall * hsteps, 16 * wn * S::kN < tile.rows,
            [&](int, int slot) {
                if (lk == 0) weights.init([&](int i) { return W + (int64_t)min(lh + i, h - 1) * s; });
                const int32_t k0 = (lk < ksteps ? lk : lk - ksteps) * kFfnBK;
                weights.load(smem + slot * S::kStageBytes, k0, s);
            },
            [&](int, int slot) {
                const int32_t k0 = (lk < ksteps ? lk : lk - ksteps) * kFfnBK;
                rows.load(smem + slot * S::kStageBytes + S::kRowsAt, k0, s, lk < ksteps ? 0 : (int64_t)n * s);
                if (++lk == kall) {
                    lk = 0;
                    lh += S::kCols;
                }
            },
            ffn_work(
                [&](int slot, int kk, int group, M& m) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < S::kM)
                            m.v[i] = row_fragment(smem + slot * S::kStageBytes, 16 * (wm * S::kM + G::tile(group, i)), kk);
                },
                [&](int slot, int kk, N& f) {
#pragma unroll
                    for (int j = 0; j < S::kN; ++j)
                        f.v[j] = row_fragment(smem + slot * S::kStageBytes + S::kRowsAt, 16 * (wn * S::kN + j), kk);
                },
                [&](int group, const M& m, const N& f) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        if (G::tile(group, i) < S::kM)
#pragma unroll
                            for (int j = 0; j < S::kN; ++j) {
                                f32x4& c = acc[G::tile(group, i)][j];
                                c = mfma_16x16x32(m.v[i], f.v[j], c);
                            }
                },
                [&] {
                    if (++ck < kall) return;
#pragma unroll
                    for (int j = 0; j < S::kN; ++j) {
#pragma unroll
                        for (int i = 0; i < S::kM; ++i) {
                            const int32_t c = ch + 16 * (wm * S::kM + i) + 4 * (lane >> 4);
                            const f32x4 v = acc[i][j] * gate[j];
                            if (place[j] < (uint32_t)n && c < h1)
                                *reinterpret_cast<uint2*>(y + (int64_t)place[j] * h + c) =
                                    pack_bf16x4(v[0], v[1], v[2], v[3]);
                            acc[i][j] = zero_f32x4();
                        }
                    }
                    ck = 0;
                    ch += S::kCols;
                }));
    });
}

// ------------------------------------------------------------------------------ few rows per expert
// Where experts have one to a few rows, each of their weights is used for one product with up to 16
// rows, and the weights' way from memory is all that counts: they go straight into the registers of the
// 16x16x32 MFMA (16 weight rows against 16 tokens), with no LDS, no tile list and no barrier on the way.
// Workgroups are laid over the sorted entries; the one whose entry is the first, 17th, ... of its expert
// takes that and the next 15 entries, the others end at once.  One token, 8 experts of h = 2048, s = 64: 7.5 us
// up and 4.1 us down, most of it the three dependent reads (sorted, idx, weights) and the launch.
constexpr int kFewWaves = 8;
constexpr int kFewUnits = 16;    // hidden units of an up workgroup
constexpr int kFewCols = 32;     // columns of y per wave of a down workgroup

// Waves take pieces of 64 contraction values in turn and their sums are added in wave order.  (These kernels
// always carry A as two planes.)
__global__ __launch_bounds__(64 * kFewWaves) void ffn_few_up_kernel(FfnArgs a, uint16_t* __restrict__ hidden) {
    constexpr int kAhead = 4;  // pieces in flight per wave
    __shared__ f32x4 part[kFewWaves][2][64];
    const int32_t s = a.s, h = a.h, n = a.T * a.k;
    const int32_t groups = (s + kFewUnits - 1) / kFewUnits;
    const int wave = ffn_wave(), lane = ffn_lane();
    for (int64_t item = blockIdx.x; item < (int64_t)n * groups; item += gridDim.x) {
        const int32_t i = (int32_t)(item / groups), s0 = (int32_t)(item % groups) * kFewUnits;
        const FewRows f = few_rows(a.sorted, a.idx, a.offsets, a.M, n, i);
        const int32_t e = f.expert, rows = f.rows;
        if (rows == 0 || e < 0) continue;
        const int32_t at = 8 * (lane >> 4);
        const uint16_t* wg = a.W1t + ((int64_t)e * 2 * s + min(s0 + (lane & 15), s - 1)) * h + at;
        const uint16_t* wu = wg + (int64_t)s * h;
        // (the columns of lanes past the rows are not stored)
        const uint16_t* x = a.x + (int64_t)(f.p < (uint32_t)n ? f.p / (uint32_t)a.k : 0) * h + at;
        f32x4 g = zero_f32x4(), u = zero_f32x4();
        for (int32_t k0 = 64 * wave; k0 < h; k0 += 64 * kFewWaves * kAhead) {
            bf16x8 fg[kAhead][2], fu[kAhead][2], fx[kAhead][2];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int32_t k = k0 + 64 * kFewWaves * q + 32 * c;
                    const bool in = k + at < h;
                    fg[q][c] = few_load(wg + k, in);
                    fu[q][c] = few_load(wu + k, in);
                    fx[q][c] = few_load(x + k, in);
                }
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    g = mfma_16x16x32(fg[q][c], fx[q][c], g);
                    u = mfma_16x16x32(fu[q][c], fx[q][c], u);
                }
        }
        __syncthreads();  // the item before has been read
        part[wave][0][lane] = g;
        part[wave][1][lane] = u;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) {
                g += part[w][0][lane];
                u += part[w][1][lane];
            }
            const int32_t c = s0 + 4 * (lane >> 4);
            if ((lane & 15) < rows && c < s) {
                float v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = g[q] * ffn_sigmoid(g[q]) * u[q];
                uint16_t* out = hidden + (int64_t)(i + (lane & 15)) * s + c;
                *reinterpret_cast<uint2*>(out) = pack_bf16x4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint2*>(out + (int64_t)n * s) = pack_bf16_rest(v[0], v[1], v[2], v[3]);
            }
        }
    }
}

// A wave computes 32 columns (two groups of weight rows).  SPLIT: the waves share their 32 columns and take
// pieces of 32 contraction values in turn, their sums added in wave order; else each has columns of its
// own.  AHEAD pieces are in flight per wave.
template <bool SPLIT, int AHEAD>
__global__ __launch_bounds__(64 * kFewWaves) void ffn_few_down_kernel(FfnArgs a, const uint16_t* __restrict__ hidden,
                                                                   uint16_t* __restrict__ y) {
    constexpr int kSpan = SPLIT ? kFewCols : kFewWaves * kFewCols;
    constexpr int kStep = SPLIT ? 32 * kFewWaves : 32;  // from a wave's piece to its next
    __shared__ f32x4 part[SPLIT ? kFewWaves : 1][2][64];
    const int32_t s = a.s, h = a.h, n = a.T * a.k;
    const int32_t spans = (h + kSpan - 1) / kSpan;
    const int wave = ffn_wave(), lane = ffn_lane();
    for (int64_t item = blockIdx.x; item < (int64_t)n * spans; item += gridDim.x) {
        const int32_t i = (int32_t)(item / spans);
        const int32_t c0 = (int32_t)(item % spans) * kSpan + (SPLIT ? 0 : wave * kFewCols);
        if (c0 >= h) continue;  // (SPLIT: never)
        const FewRows f = few_rows(a.sorted, a.idx, a.offsets, a.M, n, i);
        const int32_t e = f.expert, rows = f.rows;
        if (rows == 0) continue;
        const uint32_t p = f.p;
        const bool mine = (lane & 15) < rows && p < (uint32_t)n;
        if (e < 0) {  // a dropped entry: zeros
            if (mine && (!SPLIT || wave == 0) && c0 + 8 * (lane >> 4) < h)
                *reinterpret_cast<u32x4*>(y + (int64_t)p * h + c0 + 8 * (lane >> 4)) = u32x4{0u, 0u, 0u, 0u};
            continue;
        }
        const int32_t at = 8 * (lane >> 4);
        const uint16_t* w[2];
#pragma unroll
        for (int r = 0; r < 2; ++r)
            w[r] = a.W2t + ((int64_t)e * h + min(c0 + 16 * r + (lane & 15), h - 1)) * s + at;
        const uint16_t* hid = hidden + (int64_t)(i + min(lane & 15, rows - 1)) * s + at;
        const float gate = a.gate && mine ? a.gate[p] : 1.0f;
        f32x4 acc[2] = {zero_f32x4(), zero_f32x4()};
        for (int32_t k0 = SPLIT ? 32 * wave : 0; k0 < s; k0 += kStep * AHEAD) {
            bf16x8 fw[2][AHEAD], fh[2][AHEAD];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                const int32_t k = k0 + kStep * q;
                const bool in = k + at < s;
                fh[0][q] = few_load(hid + k, in);
                fh[1][q] = few_load(hid + (int64_t)n * s + k, in);
#pragma unroll
                for (int r = 0; r < 2; ++r) fw[r][q] = few_load(w[r] + k, in);
            }
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    acc[r] = mfma_16x16x32(fw[r][q], fh[0][q], acc[r]);
                    acc[r] = mfma_16x16x32(fw[r][q], fh[1][q], acc[r]);
                }
        }
        if constexpr (SPLIT) {
            __syncthreads();  // the item before has been read
            part[wave][0][lane] = acc[0];
            part[wave][1][lane] = acc[1];
            __syncthreads();
            if (wave > 0) continue;
#pragma unroll
            for (int v = 1; v < kFewWaves; ++v) {
                acc[0] += part[v][0][lane];
                acc[1] += part[v][1][lane];
            }
        }
        if (!mine) continue;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int32_t c = c0 + 16 * r + 4 * (lane >> 4);
            const f32x4 v = acc[r] * gate;
            if (c < h) *reinterpret_cast<uint2*>(y + (int64_t)p * h + c) = pack_bf16x4(v[0], v[1], v[2], v[3]);
        }
    }
}

// ------------------------------------------------------------------------------ host
namespace {

size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }
constexpr int64_t kMaxBlocks = 1 << 19;

// a multiple of 8 workgroups, at most one per item
unsigned grid_of(int64_t items) {
    return (unsigned)(std::min<int64_t>((items + 7) / 8, kMaxBlocks / 8) * 8);
}

unsigned few_grid(int64_t items) { return (unsigned)std::min<int64_t>(items, 1 << 22); }

// Rows of a tile: 32 where experts have less than 24 rows (then mostly one tile, whose weights are not read
// again; us, 32 : 64 rows, 4096 experts of h = 512, s = 64 with 12 rows 164 : 185, with 24 185 : 205, with 32
// 222 : 215; 64 experts of h = 1024, s = 256 with 24 rows 32 : 27), else what costs least by ffn_cost.  Large
// tiles need less from the caches, small ones fill the chip: us for 64 : 128 : 256 rows,
//   32 experts of h = 2048, s = 1024, 48 rows 99 : 107 : 120, 384 rows 295 : 242 : 189, 1024 rows - : 535 : 473
//   64 experts of h = 1024, s = 512, 192 rows 81 : 73 : 66, 256 rows 101 : 92 : 109 (the 256-row tiles take one and
//   a half rounds), 1024 rows - : 310 : 276
//   a dense block of h = 2048, s = 1024, 1024 rows 36 : 47 : 82, 4096 rows 78 : 65 : 87, 8192 rows 148 : 124 : 98
// Over 196 shapes (1 to 4096 experts, 12 to 16384 rows each) the choice is 0.9% off the best on geometric
// mean and 21% at most; one by the mean number of rows alone was 11% off, and 2.6 times at most.
int32_t tile_rows(int64_t n, int32_t h, int32_t s, int32_t M) {
    if (n / std::max<int64_t>(1, std::min<int64_t>(n, M)) < 24) return 32;
    int32_t best = 64;
    int64_t least = INT64_MAX;
    for (int32_t bm = 64; bm <= 256; bm *= 2) {
        const int64_t tiles2 = ffn_expected_tiles2(n, M, bm);
        const int32_t units = bm == 256 ? UpShape<256>::kUnits : UpShape<128>::kUnits;
        const int32_t cols = bm == 256 ? DownShape<256, 2>::kCols : DownShape<128, 2>::kCols;
        const int64_t cost = ffn_cost(tiles2 * ((s + units - 1) / units) / 2, (h + kFfnBK - 1) / kFfnBK, bm) +
                             ffn_cost(tiles2 * ((h + cols - 1) / cols) / 2, (s + kFfnBK - 1) / kFfnBK, bm);
        if (cost < least) {
            least = cost;
            best = bm;
        }
    }
    return best;
}

template <int BM, int STAGES>
hipError_t forward(const FfnPlan& p, const FfnArgs& a, uint16_t* y, char* ws, hipStream_t stream) {
    uint16_t* hidden = reinterpret_cast<uint16_t*>(ws + p.off_hidden);
    using U = UpShape<BM>;
    using D = DownShape<BM, STAGES>;
    ffn_up_kernel<BM, false><<<grid_of(p.tiles * ((a.s + U::kUnits - 1) / U::kUnits)), U::kThreads, 0, stream>>>(
        a, ws + p.off_tiles, hidden, UpBackward{});
    ffn_down_kernel<BM, STAGES><<<grid_of(p.tiles * ((a.h + p.span - 1) / p.span)), D::kThreads, 0, stream>>>(
        a, ws + p.off_tiles, hidden, p.span, y);
    return hipGetLastError();
}

}  // namespace

int64_t ffn_expected_tiles2(int64_t n, int32_t M, int32_t bm) {
    const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(n, M));
    const double mean = (double)n / (double)groups, sd = M == 1 ? 0.0 : std::sqrt(mean);
    const int64_t lo = (int64_t)std::ceil(std::max(mean - sd, 1.0) / bm), hi = (int64_t)std::ceil((mean + sd) / bm);
    return groups * (lo + hi);
}

void ffn_tiles_plan(int64_t n, int32_t M, int32_t bm, FfnPlan* p) {
    *p = FfnPlan{};
    p->n = n;
    p->bm = bm;
    p->tiles = n / bm + std::min<int64_t>(M, n) + 1;
    p->off_tiles = 0;
    p->off_sums = align256(kFfnTileHeader + (size_t)p->tiles * sizeof(FfnTile));
    p->sums = M > kTileAlone ? (M + kTileThreads - 1) / kTileThreads : 0;
    p->workspace_bytes = p->off_sums + align256((size_t)p->sums * sizeof(int64_t));
}

// Upper bound on the workgroups along the entries that have work in the kernels without tiles.
static int64_t few_starts(const FfnPlan& p, int32_t M) {
    return std::min<int64_t>(p.n, std::min<int64_t>(p.n, M) + p.n / kFewRows);
}

// Whether the kernels without tiles are taken: while the weights that they read (once for every 16 rows) are
// few bytes and few workgroups end at once.  They save a launch and the latency of the stages, but stream at
// 4 TB/s where the tiled kernels reach 6: 16 MB even out the launch, and 40 KB every column and hidden unit that
// the stages run over.  us, without tiles : with, one row per expert: h = 2048, s = 64, 8 entries 10.8 : 20.8, 128
// entries 24 : 34, 512 entries 98 : 73; h = 1024, s = 512, 16 entries 16 : 19, 32 entries 30 : 22; h = 4096,
// s = 1024, 4 entries 27 : 43, 16 entries 78 : 61; a dense block of s = 1024, h = 2048, 32 rows 18 : 29, 128
// rows 52 : 40; s = 8, h = 3408, 1430 entries (20020 workgroups) 54 : 46.
static bool few(const FfnPlan& p, int32_t h, int32_t s, int32_t M) {
    const int64_t groups =
        std::max((s + kFewUnits - 1) / kFewUnits, (h + kFewWaves * kFewCols - 1) / (kFewWaves * kFewCols));
    return few_starts(p, M) * 6 * h * s <= ((int64_t)16 << 20) + (int64_t)40960 * (h + s) && p.n * groups <= 4096;
}

// Whether a workgroup of ffn_few_down shares columns: while the workgroups that have the whole contraction
// per wave would be few against its length.  us, sharing : not, h = 1024, s = 4096, 1 row 17 : 77; h = 4096,
// s = 1024, 4 entries 27 : 40, 16 entries 78.5 : 81; s = 256, 4 entries 17.0 : 18.6, 16 entries 31.5 : 24.5.
static bool few_split(const FfnPlan& p, int32_t h, int32_t s, int32_t M) {
    return 4 * few_starts(p, M) * ((h + kFewWaves * kFewCols - 1) / (kFewWaves * kFewCols)) <= s;
}

void ffn_make_plan(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends, FfnPlan* p) {
    ffn_tiles_plan(T * k, M, tile_rows(T * k, h, s, M), p);
    p->few = few(*p, h, s, M);
    if (p->few) {
        p->split = few_split(*p, h, s, M);
        p->span = p->split ? kFewCols : kFewWaves * kFewCols;
    } else {
        p->span = ffn_span(s, p->bm == 256 ? DownShape<256, 2>::kCols : DownShape<128, 2>::kCols, p->tiles, h);
        p->stages = p->bm >= 128 ? 2 : p->bm == 64 ? 3 : p->tiles * ((h + p->span - 1) / p->span) >= 2048 ? 2 : 3;
    }
    p->planes = addends == 2 || p->few || p->n * s <= kFfnTwoPlanes ? 2 : 1;
    p->off_hidden = p->workspace_bytes;
    p->workspace_bytes += align256((size_t)p->n * s * 2 * p->planes);
}

hipError_t ffn_tiles_launch(const FfnPlan& p, const FfnArgs& a, void* workspace, hipStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    const unsigned blocks = (unsigned)(((int64_t)a.M + kTileThreads - 1) / kTileThreads);
    const int32_t log_bm = __builtin_ctz(p.bm);
    int64_t* sums = p.sums ? reinterpret_cast<int64_t*>(ws + p.off_sums) : nullptr;
    if (sums) ffn_tile_sums_kernel<<<blocks, kTileThreads, 0, stream>>>(a.offsets, a.M, (int32_t)p.n, log_bm, sums);
    ffn_tiles_kernel<<<blocks, kTileThreads, 0, stream>>>(a.offsets, a.M, (int32_t)p.n, log_bm, p.tiles, sums,
                                                          reinterpret_cast<int32_t*>(ws + p.off_tiles));
    return hipGetLastError();
}

hipError_t ffn_launch(const FfnPlan& p, FfnArgs a, uint16_t* y, void* workspace, hipStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    a.planes = p.planes;
    if (p.few) {
        uint16_t* hidden = reinterpret_cast<uint16_t*>(ws + p.off_hidden);
        ffn_few_up_kernel<<<few_grid(p.n * ((a.s + kFewUnits - 1) / kFewUnits)), 64 * kFewWaves, 0, stream>>>(a, hidden);
        const unsigned blocks = few_grid(p.n * ((a.h + p.span - 1) / p.span));
        if (p.split)
            ffn_few_down_kernel<true, 4><<<blocks, 64 * kFewWaves, 0, stream>>>(a, hidden, y);
        else
            ffn_few_down_kernel<false, 2><<<blocks, 64 * kFewWaves, 0, stream>>>(a, hidden, y);
        return hipGetLastError();
    }
    hipError_t e = ffn_tiles_launch(p, a, ws, stream);
    if (e != hipSuccess) return e;
    switch (p.bm) {
        case 256: return forward<256, 2>(p, a, y, ws, stream);
        case 128: return forward<128, 2>(p, a, y, ws, stream);
        case 64: return forward<64, 3>(p, a, y, ws, stream);
        default: return p.stages == 2 ? forward<32, 2>(p, a, y, ws, stream) : forward<32, 3>(p, a, y, ws, stream);
    }
}

}  // namespace more
