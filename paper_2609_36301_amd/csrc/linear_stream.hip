// The experts' linear maps in 8-bit integers on tiles of 256 rows and 256 columns (gfx950): one workgroup to a CU, whose
// pipeline runs on from tile to tile.
//
// A tile of 256 x 256 fills a CU's LDS, so nothing else there hides what a tile costs beside its stages: the chain of
// reads from the tile list to the first operands, the drained pipeline, the stores of 128 KB.  Here the loads of the next
// tile's first stages are issued in the present one's last stages, and what they need to know is read ahead of that by
// the first wave, a step per stage and straight to LDS: the number of the next tile (from a counter of the workgroup's
// XCD: neighbouring tiles share an L2, and tiles with few rows take less time), its descriptor, its entries, their
// factors.  The tiles' order does not change any result.
// 32 experts of K = 1024, N = 2048 with 1024 rows 104 us, 1.3 PFLOP/s (a workgroup per tile 145); one of 4096 x 4096 with
// 16384 rows 244 us, 2.3 PFLOP/s, bound by LDS and the stages' loads.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ffn_device.h"
#include "linear.h"
#include "linear_device.h"

namespace more {

namespace {

constexpr int kTile = 256;     // rows and columns of a tile
constexpr int kStreamWaves = 8;
constexpr int kStreamThreads = 64 * kStreamWaves;
constexpr int kStageBytes = 2 * kTile * 128;

// A tile as it is known ahead: its place in the work (-1: none), its descriptor, its entries and their factors.
struct StreamTile {
    FfnTile tile;
    int32_t item, pad[11];
    uint32_t entry[kTile];
    float x_scale[kTile], gate[kTile], w_scale[kTile];
};

// LDS of a workgroup: two stages, and the tiles that are multiplied, loaded and read ahead.
struct StreamLds {
    char stage[2][kStageBytes];
    StreamTile ahead[3];
    char lines[kStreamWaves][kLinesScratch];
};
typedef __attribute__((address_space(3))) StreamLds LdsStream;
typedef __attribute__((address_space(3))) StreamTile LdsTile;
typedef __attribute__((address_space(3))) f32x4 LdsF32x4;

// Direct-to-LDS load of 4 bytes per lane.
__device__ __forceinline__ void dma4(const void* g, LdsChar* lds) { __builtin_amdgcn_global_load_lds(g, lds, 4, 0, 0); }

// The pipeline's steps as in ffn_steps, with two stages and an end that is not known ahead: more() tells after a step's
// products are under way whether another stage has been loaded.
template <int GROUPS, typename M, typename N, typename T, typename F, typename G, typename E, typename W>
__device__ __forceinline__ void stream_steps(T turn, F first, G second, E more, W w) {
    constexpr int kParts = 2 * GROUPS;
    M m[2];
    N n[2];
    w.read_n(0, 0, n[0]);
    w.read_m(0, 0, 0, m[0]);
    int slot = 0;
    for (bool begun = false;; begun = true) {
        bool another = false;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            const int then = part + 1;
            if (then < kParts) {
                if (then == GROUPS) w.read_n(slot, 1, n[1]);
                w.read_m(slot, then / GROUPS, then % GROUPS, m[then & 1]);
            } else {
                another = more();
                if (another) {
                    turn();
                    w.read_n(slot ^ 1, 0, n[0]);
                    w.read_m(slot ^ 1, 0, 0, m[0]);
                    first(slot);
                }
            }
            if (part == 0 && begun) second(slot ^ 1);
            w.multiply(part % GROUPS, m[part & 1], n[part / GROUPS]);
        }
        w.done();
        if (!another) return;
        slot ^= 1;
    }
}

__global__ __launch_bounds__(kStreamThreads, 2) void linear_stream_kernel(LinearArgs a, int32_t* __restrict__ list) {
    using Type = LinearType<true>;
    constexpr int kWavesM = 2, kM = kTile / kWavesM / 16, kN = kTile / (kStreamWaves / kWavesM) / 16;
    __shared__ __attribute__((aligned(1024))) char smem_raw[sizeof(StreamLds)];
    LdsStream* lds = (LdsStream*)(LdsChar*)smem_raw;
    const int32_t n = a.T * a.k, len = a.len, cols = a.N;
    const int32_t spans = (cols + kTile - 1) / kTile, ksteps = (len + kFfnBK - 1) / kFfnBK;
    const int wave = ffn_wave(), lane = ffn_lane();
    const int wm = wave % kWavesM, wn = wave / kWavesM;
    LdsChar* lines = (LdsChar*)lds->lines[wave];
    const FfnTile* tiles = ffn_tile_list(list);
    // this XCD's share of the work: items [base, base + count)
    const int64_t total = (int64_t)list[1] * spans, share = (total + 7) / 8;
    const int xcd = blockIdx.x & 7;
    const int64_t base = xcd * share;
    const int32_t count = (int32_t)max((int64_t)0, min(share, total - base));
    int32_t* counter = list + 8 + xcd;

    auto stage = [&](int slot) { return (LdsChar*)lds->stage[slot]; };
    // the steps of reading a tile ahead (by the first wave)
    auto read_tile = [&](LdsTile* t, int32_t q) {  // q: place in the share
        const bool in = q < count;
        if (lane == 0) t->item = in ? q : -1;
        if (in && lane < 4)
            dma4(reinterpret_cast<const int32_t*>(tiles + (base + q) / spans) + lane, (LdsChar*)&t->tile);
    };
    auto read_entries = [&](LdsTile* t) {
        const int32_t row0 = t->tile.row0, last = t->tile.rows - 1;
#pragma unroll
        for (int i = 0; i < kTile / 64; ++i)
            dma4(a.sorted + row0 + min(64 * i + lane, last), (LdsChar*)(t->entry + 64 * i));
    };
    auto read_factors = [&](LdsTile* t) {
#pragma unroll
        for (int i = 0; i < kTile / 64; ++i) {
            const uint32_t p = min(t->entry[64 * i + lane], (uint32_t)n - 1u);
            dma4(a.x_scale + p / (uint32_t)a.k, (LdsChar*)(t->x_scale + 64 * i));
            if (a.gate) dma4(a.gate + p, (LdsChar*)(t->gate + 64 * i));
            const int32_t c = (int32_t)((base + t->item) % spans) * kTile + 64 * i + lane;
            dma4(a.w_scale + (int64_t)t->tile.expert * cols + min(c, cols - 1), (LdsChar*)(t->w_scale + 64 * i));
        }
    };

    // the loads' side: the tile, its rows and columns of W, the next contraction step, the tile's steps so far
    RowTileLoader<kTile, kStreamWaves> rows, weights;
    int load_at = 0, lk = 0;
    int32_t ticket = 0;
    auto begin_loads = [&] {
        LdsTile* t = lds->ahead + load_at;
        const int32_t c0 = (int32_t)((base + t->item) % spans) * kTile;
        const uint16_t* W = a.W + (int64_t)t->tile.expert * len * cols;
        rows.init([&](int i) {
            const uint32_t p = t->entry[i];
            return a.x + (int64_t)(p < (uint32_t)n ? p / (uint32_t)a.k : 0) * len;
        });
        weights.init([&](int i) { return W + (int64_t)min(c0 + i, cols - 1) * len; });
    };
    bool loading = count > (int32_t)(blockIdx.x >> 3);
    int pending = 0;  // stages loaded and not yet multiplied
    auto first = [&](int slot) {
        if (!loading) return;
        if (lk == 0 && pending > 0) begin_loads();
        weights.load(stage(slot), lk * kFfnBK, len);
    };
    auto second = [&](int slot) {
        if (!loading) return;
        rows.load(stage(slot) + kTile * 128, lk * kFfnBK, len);
        ++pending;
        const int next_at = load_at == 2 ? 0 : load_at + 1;
        if (wave == 0) {
            LdsTile* t = lds->ahead + next_at;
            if (lk == 0) {
                if (lane == 0) ticket = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            } else if (lk == 1) {
                read_tile(t, __builtin_amdgcn_readfirstlane(ticket) + (int32_t)(gridDim.x >> 3));
            } else if (lk == 2) {
                if (t->item >= 0) read_entries(t);
            } else if (lk == 3) {
                if (t->item >= 0) read_factors(t);
            }
        }
        if (++lk == ksteps) {  // (at least five steps: the next tile is known by now)
            lk = 0;
            load_at = next_at;
            loading = __builtin_amdgcn_readfirstlane(lds->ahead[next_at].item) >= 0;
        }
    };

    if (loading) {
        // the first tile, step by step
        LdsTile* t = lds->ahead;
        if (wave == 0) read_tile(t, (int32_t)(blockIdx.x >> 3));
        ffn_barrier<0>();
        if (wave == 0) read_entries(t);
        ffn_barrier<0>();
        if (wave == 0) read_factors(t);
        begin_loads();
        first(0);
        second(0);
        first(1);
        second(1);
        ffn_barrier<0>();

        typename Type::Acc acc[kM][kN];
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j) acc[i][j] = Type::zero();
        // the products' side: the tile, the next contraction step, whether the wave has wanted rows
        int at = 0, ck = 0;
        bool live = 16 * wn * kN < __builtin_amdgcn_readfirstlane(t->tile.rows);
        using G = FfnGroups<kM, 4>;
        using MF = FfnFragments<G::kSize>;
        using NF = FfnFragments<kN>;
        stream_steps<4, MF, NF>(
            [&] { ffn_barrier<0>(); }, first, second, [&] { return pending > 1; },
            ffn_work(
                [&](int slot, int kk, int group, MF& m) {
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
                        m.v[i] = row_fragment(stage(slot), 16 * (wm * kM + G::tile(group, i)), kk);
                },
                [&](int slot, int kk, NF& f) {
#pragma unroll
                    for (int j = 0; j < kN; ++j)
                        f.v[j] = row_fragment(stage(slot) + kTile * 128, 16 * (wn * kN + j), kk);
                },
                [&](int group, const MF& m, const NF& f) {
                    if (!live) return;
#pragma unroll
                    for (int i = 0; i < G::kSize; ++i)
#pragma unroll
                        for (int j = 0; j < kN; ++j) {
                            auto& c = acc[G::tile(group, i)][j];
                            c = Type::multiply(m.v[i], f.v[j], c);
                        }
                },
                [&] {
                    --pending;
                    if (++ck < ksteps) return;
                    LdsTile* t = lds->ahead + at;
                    const int32_t in_tile = 16 * wm * kM + 4 * (lane >> 4);
                    const int32_t c0 = (int32_t)((base + t->item) % spans) * kTile + in_tile;
#pragma unroll
                    for (int j = 0; j < kN; ++j) {
                        const int32_t row0 = 16 * (wn * kN + j), row = row0 + (lane & 15);
                        const float factor = a.gate ? t->x_scale[row] * t->gate[row] : t->x_scale[row];
                        auto value = [&](int i) {
                            const f32x4 ws = *reinterpret_cast<LdsF32x4*>(t->w_scale + in_tile + 16 * i);
                            f32x4 v;
#pragma unroll
                            for (int q = 0; q < 4; ++q) v[q] = (float)acc[i][j][q] * ws[q] * factor;
                            return v;
                        };
                        auto store = [&](auto wide) {
                            using L = Lines<decltype(wide)::value>;
                            using Out = typename L::Element;
#pragma unroll
                            for (int i0 = 0; i0 < kM; i0 += L::kTiles) {
#pragma unroll
                                for (int i = 0; i < L::kTiles; ++i) L::place(lines, i, value(i0 + i));
                                const int32_t c = c0 - 4 * (lane >> 4) + 16 * i0;
                                L::store(lines, cols - c, a.whole, [&](int r) -> Out* {
                                    const uint32_t e = t->entry[row0 + r];
                                    return row0 + r < t->tile.rows && e < (uint32_t)n
                                               ? static_cast<Out*>(a.y) + (int64_t)e * cols + c : nullptr;
                                });
                            }
                        };
                        if (a.wide) store(std::true_type{});
                        else store(std::false_type{});
#pragma unroll
                        for (int i = 0; i < kM; ++i) acc[i][j] = Type::zero();
                    }
                    ck = 0;
                    at = at == 2 ? 0 : at + 1;
                    live = 16 * wn * kN < __builtin_amdgcn_readfirstlane(lds->ahead[at].tile.rows);
                }));
    }
    const int32_t valid = min(max(a.offsets[a.M], 0), n);
    for (int32_t i = valid + (int32_t)blockIdx.x; i < n; i += (int32_t)gridDim.x) {
        const uint32_t p = a.sorted[i];
        if (p >= (uint32_t)n) continue;
        for (int32_t c = 8 * (int32_t)threadIdx.x; c < cols; c += 8 * kStreamThreads) {
            linear_zero(a, p, c);
        }
    }
}

}  // namespace

hipError_t linear_stream_launch(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream) {
    const int64_t items = p.tiles.tiles * ((a.N + kTile - 1) / kTile);
    const unsigned blocks = (unsigned)(std::min<int64_t>((items + 7) / 8, 256 / 8) * 8);
    linear_stream_kernel<<<blocks, kStreamThreads, 0, stream>>>(a, reinterpret_cast<int32_t*>(ws + p.tiles.off_tiles));
    return hipGetLastError();
}

}  // namespace more
