// Device helpers of the experts' linear maps (gfx950): the two operand types, and how results are stored.
#pragma once

#include <type_traits>

#include "ffn_device.h"
#include "linear.h"

namespace more {

// The two types share everything but the matrix instruction: a 16-byte fragment holds eight bf16 or sixteen
// int8 values of a row, and both operands take the same ones.
template <bool I8>
struct LinearType {
    using Acc = f32x4;
    static __device__ __forceinline__ Acc zero() { return zero_f32x4(); }
    static __device__ __forceinline__ Acc multiply(bf16x8 a, bf16x8 b, Acc c) { return mfma_16x16x32(a, b, c); }
};
template <>
struct LinearType<true> {
    using Acc = i32x4;
    static __device__ __forceinline__ Acc zero() { return i32x4{0, 0, 0, 0}; }
    static __device__ __forceinline__ Acc multiply(bf16x8 a, bf16x8 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};

// Work items (tile, span) over the grid, for workgroups of THREADS threads: body(tile, span), a span by its number.  The tiles
// come from the list (ffn_for_each), or (OWN, a workgroup for every item) each workgroup counts them up to its own, in the
// list's order.  Offsets that Sort + Count cannot have written are cut as for the list: to [0, n], and there are `bound`
// tiles at most (few, so that the counts of kLinearOwn experts fit 32 bits whatever the offsets are).  `lds` holds the
// counts ahead of the body.
template <int BM, int THREADS, bool OWN, typename F>
__device__ __forceinline__ void linear_for_each(const LinearArgs& a, const void* __restrict__ list, int32_t bound,
                                                int32_t spans, LdsChar* lds, F body) {
    if constexpr (!OWN) {
        ffn_for_each((int64_t)*static_cast<const int32_t*>(list) * spans, [&](int64_t item) {
            const FfnTile tile = ffn_tile_list(list)[item / spans];
            body(tile, (int32_t)(item % spans));
        });
    } else {
        typedef __attribute__((address_space(3))) int32_t LdsInt;
        constexpr int kEach = kLinearOwn / THREADS, kWaves = THREADS / 64;
        const int lane = ffn_lane(), wave = ffn_wave();
        LdsInt* part = (LdsInt*)lds;
        LdsInt* found = part + kWaves;
        // a thread's experts from e0 on: where they begin, their tiles; the tiles before them and of all experts
        const int32_t n = a.T * a.k, e0 = (int32_t)threadIdx.x * kEach;
        auto offset = [&](int32_t e) { return min(max(a.offsets[min(e, a.M)], 0), n); };
        int32_t begin[kEach + 1];
        const int32_t valid = offset(a.M);
#pragma unroll
        for (int i = 0; i <= kEach; ++i) begin[i] = offset(e0 + i);
        auto count = [&](int i) { return (max(begin[i + 1] - begin[i], 0) + BM - 1) / BM; };
        int32_t mine = 0, sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) mine += count(i);
        int32_t first = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int32_t o = __shfl_up(first, d, 64);
            first += lane >= d ? o : 0;
        }
        if (lane == 63) part[wave] = first;
        first -= mine;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            first += w < wave ? part[w] : 0;
            sum += part[w];
        }
        const int32_t tiles = __builtin_amdgcn_readfirstlane(min(sum + (n - valid + BM - 1) / BM, bound));
        const int32_t total = tiles * spans, chunk = (total + 7) / 8;
        const int32_t q = (int32_t)(blockIdx.x >> 3), item = (int32_t)(blockIdx.x & 7) * chunk + q;
        if (q >= chunk || item >= total) return;
        const int32_t at = item / spans;
        if (at >= sum) {  // of the dropped entries
            if (threadIdx.x == 0) {
                const int32_t row = valid + (at - sum) * BM;
                found[0] = -1, found[1] = row, found[2] = min(n - row, BM);
            }
        } else if (at >= first && at < first + mine) {
            int32_t left = at - first;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (left >= 0 && left < count(i)) {
                    const int32_t row = begin[i] + left * BM;
                    found[0] = e0 + i, found[1] = row, found[2] = min(begin[i + 1] - row, BM);
                }
                left -= count(i);
            }
        }
        __syncthreads();
        FfnTile tile;
        tile.expert = __builtin_amdgcn_readfirstlane(found[0]);
        tile.row0 = __builtin_amdgcn_readfirstlane(found[1]);
        tile.rows = __builtin_amdgcn_readfirstlane(found[2]);
        __syncthreads();  // the body may write its LDS
        body(tile, item % spans);
    }
}

// The factor of entry p's row, and four columns of an accumulator as they are stored.
template <bool I8>
__device__ __forceinline__ float linear_row_scale(const LinearArgs& a, uint32_t p, int32_t n) {
    if constexpr (!I8) return 1.0f;
    if (p >= (uint32_t)n) return 0.0f;
    const float s = a.x_scale[p / (uint32_t)a.k];
    return a.gate ? s * a.gate[p] : s;
}
__device__ __forceinline__ void linear_put(void* out, bool wide, int64_t at, f32x4 v) {
    if (wide)
        *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = v;
    else
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = pack_bf16x4(v[0], v[1], v[2], v[3]);
}
// The factors of the lane's four of 16 columns from c on (columns past the last are not stored).
template <bool I8>
__device__ __forceinline__ f32x4 linear_w_scale(const float* w_scale, int32_t c, int32_t N) {
    if constexpr (!I8) return zero_f32x4();
    return *reinterpret_cast<const f32x4*>(w_scale + min(c + 4 * (ffn_lane() >> 4), N - 4));
}
template <bool I8>
__device__ __forceinline__ f32x4 linear_value(typename LinearType<I8>::Acc acc, float row_scale, f32x4 w_scale) {
    if constexpr (!I8) return acc;
    f32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = (float)acc[q] * w_scale[q] * row_scale;
    return v;
}
// Two neighbouring accumulators in bf16, exchanged among the lanes of a row so that a lane holds eight of its 32 columns,
// the ones from 8 (l / 16) on: stored 16 bytes a lane, a row's 64 bytes are whole (8 bytes a lane, as the
// accumulators lie, they are written in two halves, twice as many requests to L2).
__device__ __forceinline__ u32x4 linear_pair(f32x4 a, f32x4 b) {
    const uint2 x = pack_bf16x4(a[0], a[1], a[2], a[3]), y = pack_bf16x4(b[0], b[1], b[2], b[3]);
    auto r = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false);
    r = __builtin_amdgcn_permlane16_swap(r[0], r[1], false, false);
    auto s = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
    s = __builtin_amdgcn_permlane16_swap(s[0], s[1], false, false);
    return u32x4{(uint32_t)r[0], (uint32_t)s[0], (uint32_t)r[1], (uint32_t)s[1]};
}
// Whole lines: 16 rows of 128 bytes (64 columns of bf16, 32 of fp32) by way of a wave's own 2 KiB of LDS, from where a
// store takes eight rows.  The 16-byte pieces of a row are XORed with the row's number, which spreads them over the banks.
// A wave's LDS accesses are in order, so there is no barrier.  Nontemporal whole lines reach memory without being read
// first: the gradients of 4096 experts, N = 512, K = 64, 32 rows 65 us, plain lines 98, nontemporal halves of lines 84.  Rows
// that split lines are stored plainly, so that L2 joins the parts of different workgroups (us, nontemporal : plain,
// 65536 rows, K = 128, N = 2040 182 : 122, but N = 2048 78 : 119; dx of K = 1808, N = 24, 34656 rows 67 : 38), but for dW,
// whose rows lie one after the other and make lines together (K = 528, N = 128, 4096 experts 175 : 266).
constexpr int kLinesScratch = 16 * 128;
template <bool WIDE>
struct Lines {
    static constexpr int kTiles = WIDE ? 2 : 4;  // accumulators of 16 columns to a line
    using Element = typename std::conditional<WIDE, float, uint16_t>::type;
    // accumulator i of the line
    static __device__ __forceinline__ void place(LdsChar* scratch, int i, f32x4 v) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const int l = ffn_lane(), row = l & 15, g = l >> 4;
        if constexpr (WIDE) {
            *reinterpret_cast<__attribute__((address_space(3))) f32x4*>(scratch + row * 128 + (((4 * i + g) ^ (row & 7)) << 4)) = v;
        } else {
            const uint2 b = pack_bf16x4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<__attribute__((address_space(3))) u32x2*>(
                scratch + row * 128 + (((2 * i + (g >> 1)) ^ (row & 7)) << 4) + ((g & 1) << 3)) = u32x2{b.x, b.y};
        }
    }
    // row_of(r): where row r goes (NULL: nowhere); `left` elements of it at most (whole pieces); `whole` as in LinearArgs
    template <typename F>
    static __device__ __forceinline__ void store(LdsChar* scratch, int left, bool whole, F row_of) {
        const int l = ffn_lane(), piece = l & 7;
#pragma unroll
        for (int r = 0; r < 16; r += 8) {
            const int row = r + (l >> 3);
            char* p = reinterpret_cast<char*>(row_of(row));
            const u32x4 v =
                *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(scratch + row * 128 + ((piece ^ (row & 7)) << 4));
            u32x4* to = reinterpret_cast<u32x4*>(p + 16 * piece);
            const bool in = p && piece * (16 / (int)sizeof(Element)) < left;
            if (whole) {
                if (in) __builtin_nontemporal_store(v, to);
                asm volatile("; whole lines");  // (else the compiler makes one plain store of both)
            } else {
                if (in) *to = v;
            }
        }
    }
};

// Zeros to columns c .. c + 7 of entry p's row.
__device__ __forceinline__ void linear_zero(const LinearArgs& a, uint32_t p, int32_t c) {
    const int64_t at = (int64_t)p * a.N + c;
    const u32x4 z = {0u, 0u, 0u, 0u};
    if (a.wide) {
        u32x4* y = reinterpret_cast<u32x4*>(static_cast<float*>(a.y) + at);
        y[0] = z;
        y[1] = z;
    } else {
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + at) = z;
    }
}

}  // namespace more
