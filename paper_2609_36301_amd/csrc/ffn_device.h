// Device helpers of the experts' feed-forward kernels (gfx950): the tile list, LDS tiles filled by
// direct-to-LDS loads, their fragments for the 16x16x32 bf16 MFMA, and the work loop.
//
// A workgroup has four or eight waves.  An operand tile is one of two kinds, 128 bytes of K per row or column:
//   row tile     ROWS x 64: row m or n holds 64 consecutive values of the contraction axis
//   column tile  64 x COLS: row kappa holds consecutive values of the other axis; its fragments are read
//                with the transposing 8-byte LDS read (ds_read_b64_tr_b16)
// A direct-to-LDS load writes lane l's 16 bytes at 16 l, so the layout is permuted at the source: the
// 16-byte piece (row tile) or 32-byte piece (column tile) that lies at a place is XORed with bits of the
// row, which spreads the 16 rows that a fragment read touches over all banks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"

namespace more {

constexpr int kFfnBK = 64;  // contraction values per stage

// A tile: rows [row0, row0 + rows) of the sorted entries, all of expert `expert` (-1: dropped entries).
struct FfnTile {
    int32_t expert, row0, rows, pad;
};
// The tile list: a count, then (256 bytes on) the tiles.
constexpr size_t kFfnTileHeader = 256;
__device__ __forceinline__ const FfnTile* ffn_tile_list(const void* tiles) {
    return reinterpret_cast<const FfnTile*>(static_cast<const char*>(tiles) + kFfnTileHeader);
}

// Source of the pieces that lie outside a matrix (zero, never written).
static __device__ __attribute__((aligned(16))) uint16_t ffn_zeros[64];

typedef __attribute__((address_space(3))) char LdsChar;
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// s_waitcnt immediate: at most n vector memory operations outstanding, all LDS operations done.
__host__ __device__ constexpr int ffn_wait_imm(int n) {
    return (n & 15) | ((n >> 4) << 14) | (7 << 4);
}
// Direct-to-LDS load of 16 bytes per lane: lane l of the wave writes lds + 16 l (lds wave-uniform).
// ONCE marks data that no other workgroup wants (nontemporal).
template <bool ONCE = false>
__device__ __forceinline__ void ffn_dma16(const uint16_t* g, LdsChar* lds) {
    __builtin_amdgcn_global_load_lds(g, lds, 16, 0, ONCE ? 2 : 0);
}
// Workgroup barrier that leaves at most VM of the wave's own vector memory operations outstanding.
template <int VM>
__device__ __forceinline__ void ffn_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(ffn_wait_imm(VM));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ int ffn_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ int ffn_lane() { return threadIdx.x & 63; }

// How a tile's 16-byte pieces get to LDS: straight (load: direct-to-LDS loads), or by way of registers
// (fetch, then put).  The compiler lets a transposing LDS read wait for every direct-to-LDS load before it, so
// the kernels that read column tiles take the second way (but for col_fragments2).
template <int LOADS>
struct Staged {
    u32x4 v[LOADS];
};

// Fills a row tile.  Lane l of a load takes row l / 8 of eight and the piece (l % 8) ^ (l / 8) of its
// 128 bytes; a wave fills ROWS / WAVES rows.
template <int ROWS, int WAVES, bool ONCE = false>
struct RowTileLoader {
    static constexpr int kPerWave = ROWS / WAVES;
    static constexpr int kLoads = kPerWave / 8;
    static constexpr int kBytes = ROWS * 128;
    const uint16_t* p[kLoads];
    int piece;

    // row_of(i): the first element of tile row i (any readable row where row i is not wanted)
    template <typename F>
    __device__ __forceinline__ void init(F row_of) {
        const int l = ffn_lane(), w = ffn_wave();
        piece = ((l & 7) ^ (l >> 3)) * 8;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) p[i] = row_of(w * kPerWave + 8 * i + (l >> 3)) + piece;
    }
    // contraction values [k0, k0 + 64) of K (a multiple of 8); past K: zeros.  `plane`: elements from the
    // rows to those meant
    template <typename F>
    __device__ __forceinline__ void each(int k0, int K, int64_t plane, F f) const {
        if (k0 + kFfnBK <= K) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) f(i, p[i] + (plane + k0));
        } else {
            const bool in = k0 + piece < K;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) f(i, in ? p[i] + (plane + k0) : ffn_zeros);
        }
    }
    __device__ __forceinline__ void load(LdsChar* lds, int k0, int K, int64_t plane = 0) const {
        LdsChar* at = lds + ffn_wave() * kPerWave * 128;
        each(k0, K, plane, [&](int i, const uint16_t* g) { ffn_dma16<ONCE>(g, at + i * 1024); });
    }
    using Stage = Staged<kLoads>;
    __device__ __forceinline__ void fetch(Stage& s, int k0, int K, int64_t plane = 0) const {
        each(k0, K, plane, [&](int i, const uint16_t* g) { s.v[i] = *reinterpret_cast<const u32x4*>(g); });
    }
    __device__ __forceinline__ void put(LdsChar* lds, const Stage& s) const {
        LdsChar* at = lds + ffn_wave() * kPerWave * 128 + ffn_lane() * 16;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(at + i * 1024) = s.v[i];
    }
};
// Fragment of 16 rows and contraction values 32 kk .. 32 kk + 31: lane l gets row l % 16, values
// 8 (l / 16) .. + 7.
__device__ __forceinline__ bf16x8 row_fragment(const LdsChar* lds, int row0, int kk) {
    const int l = ffn_lane();
    const int row = row0 + (l & 15);
    const int piece = (4 * kk + (l >> 4)) ^ (row & 7);
    return __builtin_bit_cast(
        bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(lds + row * 128 + piece * 16));
}

// A column tile lies in panels of 64 columns (64 rows of 128 bytes, 8 KiB).  The 32-byte piece of row
// kappa that holds columns 16 q .. 16 q + 15 of its panel lies at q ^ column_swizzle(kappa): a
// transposing read takes rows 0-3, 8-11, 16-19 and 24-27 (or four on) of 32, and these then meet every
// 32 bytes of the 256-byte bank row twice.  (Panels, not rows of the whole tile: a fragment's address is
// then one of four per lane plus a constant.)
constexpr int kFfnPanel = 64 * 128;
__device__ __forceinline__ int column_swizzle(int kappa) { return ((kappa >> 1) & 1) | (((kappa >> 3) & 1) << 1); }

// Fills a column tile: a load takes eight rows of a panel, a wave the same rows of every panel.
template <int COLS, int WAVES>
struct ColTileLoader {
    static constexpr int kPanels = COLS / 64;
    static constexpr int kGroups = 8 / WAVES;             // groups of eight rows per wave
    static constexpr int kLoads = kPanels * kGroups;      // per wave
    static constexpr int kBytes = COLS * 128;
    int col[kGroups];   // first column in the panel of the lane's piece

    // the lane's row in the wave's i-th group
    __device__ __forceinline__ int row(int i) const { return 8 * (ffn_wave() + WAVES * i) + (ffn_lane() >> 3); }
    __device__ __forceinline__ void init() {
        const int c = ffn_lane() & 7;  // 16-byte place in the row
#pragma unroll
        for (int i = 0; i < kGroups; ++i) col[i] = 16 * ((c >> 1) ^ column_swizzle(row(i))) + 8 * (c & 1);
    }
    // row_of(i): the address of column 0 of the lane's row in group i, or NULL (zeros); columns from
    // `cols` on (a multiple of 8) are zeros
    using Stage = Staged<kLoads>;
    template <typename F>
    __device__ __forceinline__ void fetch(Stage& s, int cols, F row_of) const {
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            const uint16_t* r = row_of(i);
#pragma unroll
            for (int q = 0; q < kPanels; ++q) {
                const int c = 64 * q + col[i];
                s.v[i * kPanels + q] = *reinterpret_cast<const u32x4*>(r && c < cols ? r + c : ffn_zeros);
            }
        }
    }
    template <typename F>
    __device__ __forceinline__ void load(LdsChar* lds, int cols, F row_of) const {
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            const uint16_t* r = row_of(i);
            LdsChar* at = lds + (ffn_wave() + WAVES * i) * 1024;
#pragma unroll
            for (int q = 0; q < kPanels; ++q) {
                const int c = 64 * q + col[i];
                ffn_dma16(r && c < cols ? r + c : ffn_zeros, at + q * kFfnPanel);
            }
        }
    }
    __device__ __forceinline__ void put(LdsChar* lds, const Stage& s) const {
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            LdsChar* at = lds + (ffn_wave() + WAVES * i) * 1024 + ffn_lane() * 16;
#pragma unroll
            for (int q = 0; q < kPanels; ++q)
                *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(at + q * kFfnPanel) = s.v[i * kPanels + q];
        }
    }
};
// Fragment of columns col0 .. col0 + 15 (col0 a multiple of 16) and rows 32 kk .. 32 kk + 31: lane l
// gets column l % 16, rows 8 (l / 16) .. + 7.
__device__ __forceinline__ bf16x8 col_fragment(LdsChar* lds, int col0, int kk) {
    const int l = ffn_lane();
    const int kappa = 8 * (l >> 4) + ((l & 15) >> 2);
    LdsChar* a = lds + kappa * 128 + ((((col0 >> 4) & 3) ^ column_swizzle(kappa)) << 5) + ((l & 3) << 3) +
                 (col0 >> 6) * kFfnPanel + kk * 32 * 128;
    // rows kappa + 4 have the same swizzle
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4*>(a));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        reinterpret_cast<__attribute__((address_space(3))) s16x4*>(a + 4 * 128));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The fragments of two neighbouring column tiles (col0 .. col0 + 31), read and waited for in one block: the
// compiler lets the builtin's reads wait for all direct-to-LDS loads in flight, so tiles filled by those are read
// this way.  (256 x 256 tiles with one operand a column tile: 5% faster than by way of registers; with both, as in
// the weight gradients, 14% slower.)
__device__ __forceinline__ void col_fragments2(LdsChar* lds, int col0, int kk, bf16x8& f0, bf16x8& f1) {
    const int l = ffn_lane();
    const int kappa = 8 * (l >> 4) + ((l & 15) >> 2);
    LdsChar* row = lds + kappa * 128 + ((l & 3) << 3) + (col0 >> 6) * kFfnPanel + kk * 32 * 128;
    const int q = (col0 >> 4) & 3, swizzle = column_swizzle(kappa);
    const uint32_t a0 = (uint32_t)(uintptr_t)(row + ((q ^ swizzle) << 5));
    const uint32_t a1 = (uint32_t)(uintptr_t)(row + (((q + 1) ^ swizzle) << 5));
    s16x4 lo0, hi0, lo1, hi1;
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4\n\t"
        "ds_read_b64_tr_b16 %1, %4 offset:512\n\t"
        "ds_read_b64_tr_b16 %2, %5\n\t"
        "ds_read_b64_tr_b16 %3, %5 offset:512\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(lo0), "=&v"(hi0), "=&v"(lo1), "=&v"(hi1)
        : "v"(a0), "v"(a1)
        : "memory");
    f0 = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo0, hi0, 0, 1, 2, 3, 4, 5, 6, 7));
    f1 = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo1, hi1, 0, 1, 2, 3, 4, 5, 6, 7));
}

// four fp32 -> four bf16 (round to nearest even)
__device__ __forceinline__ uint2 pack_bf16x4(float a, float b, float c, float d) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint2, bf16x4{(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d});
}

// What bf16 leaves of v (0 where the rounded value is not finite: it stands alone then).
__device__ __forceinline__ float bf16_rest(float v) {
    const float hi = (float)(__bf16)v;
    return __builtin_fabsf(hi) < __builtin_huge_valf() ? v - hi : 0.0f;
}
__device__ __forceinline__ uint2 pack_bf16_rest(float a, float b, float c, float d) {
    return pack_bf16x4(bf16_rest(a), bf16_rest(b), bf16_rest(c), bf16_rest(d));
}

// Stores of 16 rows of 128 bytes each (64 bf16 columns) from accumulator tiles, by way of a wave's own
// 2304 bytes of LDS: an accumulator tile holds 4 columns of a row per lane, and storing those straight, 32
// bytes of a row at a time, takes longer than whole lines (the first weight gradient of 4096 experts with
// s = 64, h = 512: 204 us against 148).  place_bf16 puts column tile i into place, then flush_rows reads
// 16 bytes per lane and stores each row to row_of(row) (NULL: nothing), `left` bytes of it (a multiple of
// 16) at most.  A wave's LDS accesses are in order, so there is no barrier.
constexpr int kFfnScratch = 16 * 144;
__device__ __forceinline__ void place_bf16(LdsChar* scratch, int i, f32x4 v) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const int l = ffn_lane();
    const uint2 b = pack_bf16x4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<__attribute__((address_space(3))) u32x2*>(scratch + (l & 15) * 144 + i * 32 + (l >> 4) * 8) =
        u32x2{b.x, b.y};
}
// ONCE marks rows that this call does not read again (nontemporal).
template <bool ONCE = false, typename F>
__device__ __forceinline__ void flush_rows(LdsChar* scratch, int left, F row_of) {
    const int l = ffn_lane(), at = (l & 7) * 16;
#pragma unroll
    for (int r = 0; r < 16; r += 8) {
        const int row = r + (l >> 3);
        char* p = reinterpret_cast<char*>(row_of(row));
        const u32x4 v = *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(scratch + row * 144 + at);
        if (!p || at >= left) continue;
        if constexpr (ONCE)
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p + at));
        else
            *reinterpret_cast<u32x4*>(p + at) = v;
    }
}

// Work items [0, total) over the grid (a multiple of 8 workgroups): workgroups are dealt to the 8 XCDs
// in turn, so item q of XCD d is d ceil(total / 8) + q and neighbouring items share an L2.
template <typename F>
__device__ __forceinline__ void ffn_for_each(int64_t total, F body) {
    const int64_t chunk = (total + 7) / 8;
    const int64_t base = (int64_t)(blockIdx.x & 7) * chunk;
    for (int64_t q = blockIdx.x >> 3; q < chunk; q += gridDim.x >> 3) {
        if (base + q >= total) break;
        body(base + q);
    }
}

// The products of `steps` stages of an LDS ring of `stages`.  A stage's product runs in parts: for each
// half kk of its contraction values, the M-side fragments in GROUPS groups against the N-side fragments.
// `w` gives read_m(slot, kk, group, m) and read_n(slot, kk, n), which fill fragments of types M and N,
// multiply(group, m, n), and done(), which follows the last product of a step.  The fragments of a part
// are read while the part before is multiplied, across steps too, so that the LDS works while the matrix
// cores do.  turn(step, slot) stands before the last part of every step but the last: there the
// next stage has to become readable, and the present one has been read and can be filled again.  first(step, slot)
// stands ahead of the last part's product and second(step, slot) ahead of the next step's first, for loads in two
// halves: issued at once they hold all waves up while the matrix cores run dry (32 experts of h = 2048, s = 1024
// with 1024 rows, up 317 us against 340, in the backward pass 358 against 442).
template <int GROUPS, typename M, typename N, typename T, typename F, typename G, typename W>
__device__ __forceinline__ void ffn_steps(int steps, int stages, T turn, F first, G second, W w) {
    constexpr int kParts = 2 * GROUPS;
    M m[2];
    N n[2];
    w.read_n(0, 0, n[0]);
    w.read_m(0, 0, 0, m[0]);
    int slot = 0, before = 0;
    for (int step = 0; step < steps; ++step) {
        const int next = slot + 1 == stages ? 0 : slot + 1;
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            const int then = part + 1;
            if (then < kParts) {
                if (then == GROUPS) w.read_n(slot, 1, n[1]);
                w.read_m(slot, then / GROUPS, then % GROUPS, m[then & 1]);
            } else if (step + 1 < steps) {
                turn(step, slot);
                w.read_n(next, 0, n[0]);
                w.read_m(next, 0, 0, m[0]);
                first(step, slot);
            }
            if (part == 0 && step > 0) second(step - 1, before);
            w.multiply(part % GROUPS, m[part & 1], n[part / GROUPS]);
        }
        w.done();
        before = slot;
        slot = next;
    }
}
// The same for a wave that has no wanted rows: it only loads.
template <typename T, typename F, typename G>
__device__ __forceinline__ void ffn_loads_only(int steps, int stages, T turn, F first, G second) {
    int slot = 0;
    for (int step = 0; step + 1 < steps; ++step) {
        turn(step, slot);
        first(step, slot);
        second(step, slot);
        slot = slot + 1 == stages ? 0 : slot + 1;
    }
}

// The pipeline with direct-to-LDS loads: load1(slot, step) and load2(slot, step) issue LOADS of them per wave
// together, STAGES stages ahead.  A wave's own vector memory operations complete in the order in which they were
// issued, so the next stage's loads are known to have landed while those of later stages are outstanding.
// SPLIT: the two halves apart (tiles of 256 rows, with one workgroup to a CU; with more, others multiply meanwhile).
template <int STAGES, int LOADS, int GROUPS, bool SPLIT, typename M, typename N, typename L1, typename L2, typename W>
__device__ __forceinline__ void ffn_pipeline(int steps, bool live, L1 load1, L2 load2, W w) {
    ffn_barrier<0>();  // the previous work item's reads are over
#pragma unroll
    for (int i = 0; i < STAGES; ++i)
        if (i < steps) {
            load1(i, i);
            load2(i, i);
        }
    if (steps >= STAGES) {
        ffn_barrier<(STAGES - 1) * LOADS>();
    } else {
        ffn_barrier<0>();
    }
    auto turn = [&](int step, int slot) {
        if (step + STAGES <= steps) {
            ffn_barrier<(STAGES - 2) * LOADS>();
        } else {
            ffn_barrier<0>();
        }
        if (!SPLIT && step + STAGES < steps) {
            load1(step + STAGES, slot);
            load2(step + STAGES, slot);
        }
    };
    auto first = [&](int step, int slot) {
        if (SPLIT && step + STAGES < steps) load1(step + STAGES, slot);
    };
    auto second = [&](int step, int slot) {
        if (SPLIT && step + STAGES < steps) load2(step + STAGES, slot);
    };
    if (live)
        ffn_steps<GROUPS, M, N>(steps, STAGES, turn, first, second, w);
    else
        ffn_loads_only(steps, STAGES, turn, first, second);
}

// A stage of both operands on its way through registers.
template <typename A, typename B>
struct StagePair {
    typename A::Stage a;
    typename B::Stage b;
};

// The pipeline by way of registers, two stages in LDS: fetch(step, s) reads a stage into registers,
// put(slot, s) writes it to LDS a step later, and another step later it is multiplied.  (Both at the turn: in
// halves as above the products were 10% slower.)
template <typename S, int GROUPS, typename M, typename N, typename F, typename P, typename W>
__device__ __forceinline__ void ffn_pipeline_staged(int steps, bool live, F fetch, P put, W w) {
    S s;
    ffn_barrier<63>();  // the previous work item's reads are over
    fetch(0, s);
    if (steps > 1) {
        S s1;
        fetch(1, s1);
        put(0, s);
        put(1, s1);
    } else {
        put(0, s);
    }
    if (steps > 2) fetch(2, s);
    ffn_barrier<63>();
    auto turn = [&](int step, int slot) {
        ffn_barrier<63>();
        if (step + 2 < steps) put(slot, s);
        if (step + 3 < steps) fetch(step + 3, s);
    };
    auto none = [](int, int) {};
    if (live)
        ffn_steps<GROUPS, M, N>(steps, 2, turn, none, none, w);
    else
        ffn_loads_only(steps, 2, turn, none, none);
}

// The four functions of a pipeline as one argument.
template <typename RM, typename RN, typename P, typename D>
struct FfnWork {
    RM read_m;
    RN read_n;
    P multiply;
    D done;
};
template <typename RM, typename RN, typename P, typename D>
__device__ __forceinline__ FfnWork<RM, RN, P, D> ffn_work(RM rm, RN rn, P p, D d) {
    return FfnWork<RM, RN, P, D>{rm, rn, p, d};
}
template <int COUNT>
struct FfnFragments {
    bf16x8 v[COUNT];
};
// TILES M-side tiles in GROUPS groups (the last ones may be short).
template <int TILES, int GROUPS = 2>
struct FfnGroups {
    static constexpr int kGroups = GROUPS;
    static constexpr int kSize = (TILES + GROUPS - 1) / GROUPS;
    __device__ static constexpr int tile(int group, int i) { return group * kSize + i; }
};

__device__ __forceinline__ f32x4 zero_f32x4() { return f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }

// 1 / (1 + e^-v): v_exp_f32 and v_rcp_f32 (1 ulp each); e^-v = inf gives 0.
__device__ __forceinline__ float ffn_sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * v));
}

}  // namespace more
