// Device helpers of the distillation loss (gfx950): elements of a row, and what a row's group of threads shares.
#pragma once

#include <type_traits>

#include "device_common.h"

namespace more {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
__device__ __forceinline__ float minus_inf() { return -__builtin_huge_valf(); }

// A 16-byte piece of a row: eight bf16 or four fp32 values.
template <bool WIDE>
struct Piece {
    static constexpr int kCount = WIDE ? 4 : 8;
    static constexpr uint32_t kNone = WIDE ? 0xFF800000u : 0xFF80FF80u;  // -infinity
    using Element = typename std::conditional<WIDE, float, uint16_t>::type;
    static __device__ __forceinline__ float value(const u32x4& v, int i) {
        const uint32_t w = v[WIDE ? i : i / 2];  // (a copy: the bit cast of a vector's element took element 0)
        return __builtin_bit_cast(float, WIDE ? w : i % 2 ? w & 0xFFFF0000u : w << 16);
    }
    static __device__ __forceinline__ float value(Element e) {
        if constexpr (WIDE) return e;
        else return bf16_bits_to_f32(e);
    }
    static __device__ __forceinline__ Element element(float f) {
        if constexpr (WIDE) return f;
        else return __builtin_bit_cast(uint16_t, (__bf16)f);
    }
    static __device__ __forceinline__ u32x4 pack(const float (&f)[kCount]) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (WIDE) v[i] = __builtin_bit_cast(uint32_t, f[i]);
            else v[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)f[2 * i], (__bf16)f[2 * i + 1]});
        }
        return v;
    }
};

template <int THREADS>
__device__ __forceinline__ void group_sync() {
    if constexpr (THREADS == 64) {
        wave_lds_sync();
    } else {
        __syncthreads();
    }
}

// Over the wave's lanes, by moves that stay in the vector unit.
template <typename F>
__device__ __forceinline__ float wave_reduce(float v, F f) {
    v = f(v, lane_xor<1>(v));
    v = f(v, lane_xor<2>(v));
    v = f(v, lane_xor<4>(v));
    v = f(v, lane_xor<8>(v));
    float a, b;
    lane_pair16(v, a, b);
    v = f(a, b);
    lane_pair32(v, a, b);
    return f(a, b);
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
    return wave_reduce(v, [](float a, float b) { return a + b; });
}

}  // namespace more
