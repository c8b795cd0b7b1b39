// Distillation from a teacher's top logits for gfx950.  With row t's student logits z [V], its teacher's entries
// (id_j, v_j), j < k, the temperature tau, and e_j = exp((v_j - max v) / tau) over the valid entries,
//   q_j = e_j / sum e,   m = max z,   Z = sum_e exp((z_e - m) / tau),   P_e = exp((z_e - m) / tau) / Z
//   loss = tau^2 sum_j q_j (ln q_j - ln P_(id_j))
//        = tau^2 (ln Z - ln sum e + sum_j q_j ((v_j - max v) - (z_(id_j) - m)) / tau)
//   d loss / dz_e = tau (P_e - sum_(j: id_j = e) q_j)
// An entry is valid if its id lies in [0, V) and its value is not -infinity; a row without valid entries has loss 0
// and gradient 0.
//
// Memory-bound: a row's logits are read once and stay in registers between maximum, sum and gradient, so that the loss
// with its gradient is one read and one write.  A group of threads takes a row, R pieces of 16 bytes to a thread; rows
// that do not fit are read again instead.  Rows start at any element: pieces are aligned in memory, the first and the
// last piece of a row are taken by elements, so nothing outside the row is touched.
// The teacher's entries lie in LDS; after its stores a thread goes through them and stores the gradients of those
// in its own pieces over the first ones (same lane, same address: in order).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "distill.h"
#include "device_common.h"

namespace more {

namespace {

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
    // piece u of a row that begins `off` elements into piece 0
    static __device__ __forceinline__ u32x4 load(const Element* row, int32_t off, int32_t V, int32_t u) {
        const int32_t e0 = u * kCount - off;
        if (e0 >= 0 && e0 + kCount <= V) return *reinterpret_cast<const u32x4*>(row + e0);
        u32x4 v = {kNone, kNone, kNone, kNone};
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            if (e0 + i < 0 || e0 + i >= V) continue;
            if constexpr (WIDE) {
                v[i] = __builtin_bit_cast(uint32_t, row[e0 + i]);
            } else {
                const uint32_t b = row[e0 + i];
                v[i / 2] = i % 2 ? (v[i / 2] & 0xFFFFu) | b << 16 : (v[i / 2] & 0xFFFF0000u) | b;
            }
        }
        return v;
    }
};

struct Stats {
    float m, s;  // the maximum, and the sum of exp2((z - m) c)
};

template <int THREADS>
__device__ __forceinline__ void group_sync() {
    if constexpr (THREADS == 64) {
        wave_lds_sync();
    } else {
        __syncthreads();
    }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// The value of every thread's v over a row's group (waves in order).
template <int THREADS, bool MAX>
__device__ __forceinline__ float group_reduce(float v, float* part) {
    v = MAX ? wave_max(v) : wave_sum(v);
    if constexpr (THREADS == 64) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = MAX ? fmaxf(v, part[w]) : v + part[w];
    return v;
}

// RESIDENT: the row's pieces (R per thread) stay in registers; else they are read again (R at a time).
template <bool WIDE, int THREADS, int R, bool RESIDENT>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void distill_kernel(DistillArgs a) {
    using P = Piece<WIDE>;
    using Element = typename P::Element;
    constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;  // rows of a workgroup
    constexpr int kCount = P::kCount;
    extern __shared__ float dynamic[];  // per row: q (or 0), z and id of the teacher's entries
    __shared__ float part_max[16], part_sum[16], total[kRows];
    const int group = threadIdx.x / THREADS, tid = threadIdx.x % THREADS;
    float* q_of = dynamic + (int64_t)group * 3 * a.k;
    float* z_of = q_of + a.k;
    int32_t* id_of = reinterpret_cast<int32_t*>(z_of + a.k);
    const float c = kLog2e / a.tau;
    for (int64_t row = (int64_t)blockIdx.x * kRows + group; row < a.T; row += (int64_t)gridDim.x * kRows) {
        const Element* z = static_cast<const Element*>(a.logits) + row * a.ld;
        const int32_t off = (int32_t)((reinterpret_cast<uintptr_t>(z) & 15) / sizeof(Element));
        const int32_t pieces = (int32_t)(((int64_t)off + a.V + kCount - 1) / kCount);
        u32x4 v[R];
        if constexpr (RESIDENT) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int32_t u = tid + r * THREADS;
                v[r] = u32x4{P::kNone, P::kNone, P::kNone, P::kNone};
                if (u < pieces) v[r] = P::load(z, off, a.V, u);
            }
        }
        // the teacher, by the group's first wave
        float top = minus_inf(), sum_q = 0.0f;
        if (tid < 64) {
            for (int32_t j = tid; j < a.k; j += 64) {
                const int32_t id = a.ids[row * a.k + j];
                const float t = a.values[row * a.k + j];
                const bool valid = (uint32_t)id < (uint32_t)a.V && t != minus_inf();
                id_of[j] = valid ? id : -1;
                q_of[j] = t;
                z_of[j] = valid ? P::value(z[id]) : 0.0f;
                if (valid) top = fmaxf(top, t);
            }
            top = wave_max(top);
            bool any = false;
            for (int32_t j = tid; j < a.k; j += 64) {
                const bool valid = id_of[j] >= 0;
                const float e = valid ? __builtin_amdgcn_exp2f((q_of[j] - top) * c) : 0.0f;
                sum_q += e;
                any |= valid;
            }
            sum_q = wave_sum(sum_q);
            if (__ballot(any) == 0) sum_q = 0.0f;
            if (tid == 0) total[group] = __ballot(any) == 0 ? 0.0f : sum_q;
        }
        // maximum and sum of the row
        Stats st;
        if (a.m_in) {
            st = Stats{a.m_in[row], a.Z_in[row]};
        } else if constexpr (RESIDENT) {
            float m = minus_inf();
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < kCount; ++i) m = fmaxf(m, P::value(v[r], i));
            st.m = group_reduce<THREADS, true>(m, part_max);
            float s = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < kCount; ++i) s += __builtin_amdgcn_exp2f((P::value(v[r], i) - st.m) * c);
            st.s = group_reduce<THREADS, false>(s, part_sum);
        } else {
            // a running maximum and sum per thread
            float m = minus_inf(), s = 0.0f;
            for (int32_t u0 = tid; u0 < pieces; u0 += R * THREADS) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int32_t u = u0 + r * THREADS;
                    v[r] = u32x4{P::kNone, P::kNone, P::kNone, P::kNone};
                    if (u < pieces) v[r] = P::load(z, off, a.V, u);
                }
                float to = m;
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < kCount; ++i) to = fmaxf(to, P::value(v[r], i));
                const float base = to == minus_inf() ? 0.0f : to;  // (nothing but -infinity so far)
                s *= __builtin_amdgcn_exp2f((m - base) * c);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < kCount; ++i) s += __builtin_amdgcn_exp2f((P::value(v[r], i) - base) * c);
                m = to;
            }
            st.m = group_reduce<THREADS, true>(m, part_max);
            st.s = group_reduce<THREADS, false>(m == st.m ? s : s * __builtin_amdgcn_exp2f((m - st.m) * c), part_sum);
        }
        group_sync<THREADS>();  // the teacher's entries and their sum are there
        const float U = total[group];
        const bool some = U != 0.0f;  // (NaN values make U NaN)
        if (tid < 64) {
            float dot = 0.0f;
            for (int32_t j = tid; j < a.k; j += 64) {
                const bool valid = id_of[j] >= 0;
                const float d = q_of[j] - top;
                const float q = valid ? __builtin_amdgcn_exp2f(d * c) / U : 0.0f;
                // (an entry whose q is zero has no share, whatever the student says)
                if (q != 0.0f) dot += q * (d - (z_of[j] - st.m));
                q_of[j] = q;
            }
            dot = wave_sum(dot);
            if (tid == 0) {
                if (a.loss)
                    a.loss[row] = some ? a.tau * a.tau *
                                             ((__builtin_amdgcn_logf(st.s) - __builtin_amdgcn_logf(U)) * kLn2 + dot / a.tau)
                                       : 0.0f;
                if (a.m) a.m[row] = st.m;
                if (a.Z) a.Z[row] = st.s;
            }
        }
        if (a.dlogits) {
            Element* dz = static_cast<Element*>(a.dlogits) + row * a.ldd;
            const float g = a.tau * (a.weight ? a.weight[row] : 1.0f), gp = g / st.s;
            // the stores' pieces are the loads' (they need not be aligned in dlogits)
            const bool vector = ((reinterpret_cast<uintptr_t>(dz) & 15) / sizeof(Element)) == (uintptr_t)off;
            auto store = [&](int32_t u, const u32x4& w) {
                const int32_t e0 = u * kCount - off;
                float f[kCount];
#pragma unroll
                for (int i = 0; i < kCount; ++i)
                    f[i] = some ? gp * __builtin_amdgcn_exp2f((P::value(w, i) - st.m) * c) : 0.0f;
                if (vector && e0 >= 0 && e0 + kCount <= a.V) {
                    *reinterpret_cast<u32x4*>(dz + e0) = P::pack(f);
                } else {
#pragma unroll
                    for (int i = 0; i < kCount; ++i)
                        if (e0 + i >= 0 && e0 + i < a.V) dz[e0 + i] = P::element(f[i]);
                }
            };
            if constexpr (RESIDENT) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int32_t u = tid + r * THREADS;
                    if (u < pieces) store(u, v[r]);
                }
            } else {
                for (int32_t u0 = tid; u0 < pieces; u0 += R * THREADS) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int32_t u = u0 + r * THREADS;
                        if (u < pieces) v[r] = P::load(z, off, a.V, u);
                    }
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int32_t u = u0 + r * THREADS;
                        if (u < pieces) store(u, v[r]);
                    }
                }
            }
            group_sync<THREADS>();  // q is there
            if (some) {
                for (int32_t j = 0; j < a.k; ++j) {
                    const int32_t id = id_of[j];
                    if (id < 0 || (id + off) / kCount % THREADS != tid) continue;
                    float q = 0.0f;  // (an id may occur more than once)
                    for (int32_t i = 0; i < a.k; ++i) q += id_of[i] == id ? q_of[i] : 0.0f;
                    dz[id] = P::element(gp * __builtin_amdgcn_exp2f((z_of[j] - st.m) * c) - g * q);
                }
            }
        }
        group_sync<THREADS>();  // LDS may be written again
    }
}

template <bool WIDE, int THREADS, int R, bool RESIDENT = true>
void launch(const DistillArgs& a, hipStream_t stream) {
    const int rows = THREADS < 256 ? 256 / THREADS : 1, threads = THREADS < 256 ? 256 : THREADS;
    const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)a.T + rows - 1) / rows, 1 << 20);
    distill_kernel<WIDE, THREADS, R, RESIDENT><<<blocks, threads, (size_t)rows * 3 * a.k * sizeof(float), stream>>>(a);
}

template <bool WIDE>
void launch(const DistillArgs& a, hipStream_t stream) {
    const int32_t count = Piece<WIDE>::kCount;
    const int64_t pieces = ((int64_t)a.V + 2 * count - 2) / count;  // of a row that begins at the worst place
    if (pieces <= 64)
        launch<WIDE, 64, 1>(a, stream);
    else if (pieces <= 128)
        launch<WIDE, 64, 2>(a, stream);
    else if (pieces <= 256)
        launch<WIDE, 64, 4>(a, stream);
    else if (pieces <= 1024)
        launch<WIDE, 256, 4>(a, stream);
    else if (pieces <= 2048)
        launch<WIDE, 256, 8>(a, stream);
    else if (pieces <= 4096)
        launch<WIDE, 512, 8>(a, stream);
    else if (pieces <= 8192)
        launch<WIDE, 1024, 8>(a, stream);
    else if (pieces <= 16384)
        launch<WIDE, 1024, 16>(a, stream);
    else
        launch<WIDE, 1024, 4, false>(a, stream);
}

}  // namespace

hipError_t distill_launch(const DistillArgs& a, hipStream_t stream) {
    if (a.wide)
        launch<true>(a, stream);
    else
        launch<false>(a, stream);
    return hipGetLastError();
}

}  // namespace more
