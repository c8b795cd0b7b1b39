// Distillation (distill.hip) for gfx950 where a teacher's entries may cover most classes or all, V <= 2 k.
//
// There P and Q come close as the temperature grows: the loss is tau^2 times what is left of ln Z - ln U and a sum of like
// size, the gradient tau (P - Q), and fp32 leaves the error tau^2 2^-24 of a loss that stays the same (V = k = 64, tau = 256:
// 0.732 for 0.744).  (With V > 2 k the entries have at most about half of a flat P, and nothing cancels.)  So all is made of
// what stays small.  With x = d / tau, write
//   e^x = n(x) + r(x),   n = 1 and r = e^x - 1 (its series) where |x| <= 1/2, else n = 0 and r = e^x
//   Z = Nz + A,  U = Nu + B      (of the classes, with d = z - m; of the valid entries, with d = v - max v)
// where Nz and Nu are whole numbers.  For a class with e^x = n + r and the sums n' + r' of its entries,
//   Z U (P - Q) = (n Nu - n' Nz) + n B - n' A + r U - r' Z
// in which whole parts cancel exactly and the others are as small as x.  The loss is a sum of terms that are not negative, and
// of the classes without an entry less those that have more than one:
//   loss = tau^2 (sum_j (q_j ln(q_j / P_j) - q_j + P_j) + sum_e (1 - count_e) P_e)
// with P_j phi(q_j / P_j - 1) for the first where n = 1 for both, phi(s) = (1 + s) ln(1 + s) - s = s^2/2 - s^3/6 + ...
//
// A row's classes and its entries lie in LDS, and each r is made once.  Bound by instructions: 16384 rows of 128 fp32, k = 64,
// loss and gradient 15.3 us (distill_kernel 17.0), the loss alone 13.1 (9.9), the gradient alone 11.6 (15.2); 4096 of 1024,
// k = 1024, both 30 (340: there repeated ids are looked for among all pairs, here the counts tell).  A wave takes a row
// of up to 512 classes (16384 of 300 bf16, k = 200, loss alone, 64 threads : 256 27 : 47).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "distill.h"
#include "distill_device.h"

namespace more {

namespace {

struct Parts {
    float whole, rest;
    __device__ __forceinline__ float sum() const { return whole + rest; }
};
// of e^(d / tau), c = log2(e) / tau; NaN stays NaN
__device__ __forceinline__ Parts parts(float d, float inv, float c) {
    const float x = d * inv;
    if (!(__builtin_fabsf(x) <= 0.5f)) return Parts{0.0f, __builtin_amdgcn_exp2f(d * c)};
    float p = 1.0f / 40320;  // x + x^2 (1/2! + x/3! + ... + x^6/8!): the next term is below 2^-26 of the first
    p = __builtin_fmaf(p, x, 1.0f / 5040);
    p = __builtin_fmaf(p, x, 1.0f / 720);
    p = __builtin_fmaf(p, x, 1.0f / 120);
    p = __builtin_fmaf(p, x, 1.0f / 24);
    p = __builtin_fmaf(p, x, 1.0f / 6);
    p = __builtin_fmaf(p, x, 0.5f);
    return Parts{1.0f, __builtin_fmaf(x * x, p, x)};
}
// phi(s) / s^2 for |s| <= 1/8: 1/2 - s/6 + s^2/12 - ... + s^6/56 - s^7/72, the terms (-s)^i / ((i + 1) (i + 2))
__device__ __forceinline__ float phi_of_square(float s) {
    float p = -1.0f / 72;
    p = __builtin_fmaf(p, s, 1.0f / 56);
    p = __builtin_fmaf(p, s, -1.0f / 42);
    p = __builtin_fmaf(p, s, 1.0f / 30);
    p = __builtin_fmaf(p, s, -1.0f / 20);
    p = __builtin_fmaf(p, s, 1.0f / 12);
    p = __builtin_fmaf(p, s, -1.0f / 6);
    return __builtin_fmaf(p, s, 0.5f);
}

// The sums of COUNT values over a row's threads (waves in order).
template <int THREADS, int COUNT>
__device__ __forceinline__ void sums(float (&v)[COUNT], float (*part)[4]) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = wave_sum(v[i]);
    if constexpr (THREADS == 64) return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < COUNT; ++i) part[i][threadIdx.x >> 6] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = (part[i][0] + part[i][1]) + (part[i][2] + part[i][3]);
}

template <bool WIDE, int THREADS>
__global__ __launch_bounds__(256) void distill_cover_kernel(DistillArgs a) {
    using P = Piece<WIDE>;
    using Element = typename P::Element;
    constexpr int kRows = 256 / THREADS;  // rows of a workgroup
    extern __shared__ __attribute__((aligned(16))) float dynamic[];
    __shared__ float part_first[3][4], part_sums[4][4], part_loss[3][4];
    const int group = kRows == 1 ? 0 : threadIdx.x / THREADS, tid = kRows == 1 ? threadIdx.x : threadIdx.x % THREADS;
    const int32_t V = a.V, k = a.k;
    // of the classes: z, then the rest; the gradient; the number of entries, and kNear where the whole part is one
    // of the entries: v, then the rest; the id (-1: not valid) and kNear
    constexpr int32_t kNear = 1 << 16;
    static_assert(2 * kDistillMaxTeacher < kNear, "ids and counts");
    float* r_of = dynamic + group * (3 * V + 2 * k);
    float* g_of = r_of + V;
    float* v_of = g_of + V;
    int32_t* id_of = reinterpret_cast<int32_t*>(v_of + k);
    int32_t* count_of = id_of + k;
    auto stored = [&](float rest, int32_t flags) { return Parts{flags & kNear ? 1.0f : 0.0f, rest}; };
    const float c = kLog2e / a.tau, inv = 1.0f / a.tau;

    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.T; first += (int64_t)gridDim.x * kRows) {
        const int64_t row = first + group;
        if (kRows > 1 && row >= a.T) break;
        const Element* z = static_cast<const Element*>(a.logits) + row * a.ld;
        float m = minus_inf(), top = minus_inf();
        bool some = false;
        for (int32_t e = tid; e < V; e += THREADS) {
            const float v = P::value(z[e]);
            r_of[e] = v;
            m = fmaxf(m, v);
        }
        for (int32_t j = tid; j < k; j += THREADS) {
            const int32_t id = a.ids[row * k + j];
            const float v = a.values[row * k + j];
            const bool valid = (uint32_t)id < (uint32_t)V && v != minus_inf();
            id_of[j] = valid ? id : -1;
            v_of[j] = v;
            if (valid) top = fmaxf(top, v), some = true;
        }
        m = wave_max(m);
        top = wave_max(top);
        some = __any(some);
        if constexpr (THREADS == 256) {
            if ((tid & 63) == 0) {
                part_first[0][tid >> 6] = m;
                part_first[1][tid >> 6] = top;
                part_first[2][tid >> 6] = some ? 1.0f : 0.0f;
            }
        }
        if constexpr (THREADS == 256) {
            __syncthreads();
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                m = fmaxf(m, part_first[0][w]);
                top = fmaxf(top, part_first[1][w]);
                some |= part_first[2][w] != 0.0f;
            }
        }
        if (a.m_in) m = a.m_in[row];
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // Nz, A, Nu, B
        for (int32_t e = tid; e < V; e += THREADS) {
            const Parts p = parts(r_of[e] - m, inv, c);
            r_of[e] = p.rest;
            sum[0] += p.whole;
            sum[1] += p.rest;
            count_of[e] = p.whole != 0.0f ? kNear : 0;
        }
        group_sync<THREADS>();  // the counts can be added to
        for (int32_t j = tid; j < k; j += THREADS) {
            const int32_t id = id_of[j];
            if (id < 0) continue;
            const Parts p = parts(v_of[j] - top, inv, c);
            v_of[j] = p.rest;
            if (p.whole != 0.0f) id_of[j] = id | kNear;
            sum[2] += p.whole;
            sum[3] += p.rest;
            atomicAdd(count_of + id, 1);  // (whole numbers: their order does not matter)
        }
        sums<THREADS, 4>(sum, part_sums);
        group_sync<THREADS>();  // rests and counts are there
        const float Nz = sum[0], Nu = sum[2], B = sum[3], U = Nu + B;
        float A = sum[1], Z = Nz + A;
        if (a.Z_in) {  // (the same Z, unless it was summed otherwise)
            A += a.Z_in[row] - Z;
            Z = a.Z_in[row];
        }
        const float inv_Z = 1.0f / Z, inv_U = 1.0f / U;
        if (!a.m_in) {
            // classes without entries less those with more than one: in whole parts and rests; then the entries' terms
            float loss[3] = {0.0f, 0.0f, 0.0f};
            if (a.loss && some) {
                for (int32_t e = tid; e < V; e += THREADS) {
                    const int32_t count = count_of[e];
                    const float left = (float)(1 - (count & (kNear - 1)));
                    if (left == 0.0f) continue;
                    loss[0] += count & kNear ? left : 0.0f;
                    loss[1] += left * r_of[e];
                }
                const float lnZ = __builtin_amdgcn_logf(Z) * kLn2, lnU = __builtin_amdgcn_logf(U) * kLn2;
                for (int32_t j = tid; j < k; j += THREADS) {
                    if (id_of[j] < 0) continue;
                    const int32_t id = id_of[j] & (kNear - 1);
                    const Parts p = stored(r_of[id], count_of[id]), q = stored(v_of[j], id_of[j]);
                    const float Pj = p.sum() * inv_Z;
                    if (p.whole * q.whole != 0.0f) {
                        const float D = (Nu - Nz) + (B - A) + p.rest * U - q.rest * Z;
                        const float s = -D * inv_U * __builtin_amdgcn_rcpf(p.sum());
                        if (__builtin_fabsf(s) <= 0.125f) {
                            const float ts = a.tau * s;  // (s^2 alone might underflow)
                            loss[2] += Pj * ts * ts * phi_of_square(s);
                        } else {
                            const float ratio = 1.0f + s;
                            loss[2] += a.tau * a.tau * Pj * (ratio * (__builtin_amdgcn_logf(ratio) * kLn2) - s);
                        }
                    } else {
                        const float Qj = q.sum() * inv_U;
                        loss[2] += a.tau * a.tau * (Pj - Qj);
                        // (an entry whose q is zero has no share, whatever the student says)
                        if (Qj != 0.0f)
                            loss[2] += a.tau * Qj * (a.tau * (lnZ - lnU) +
                                                     ((a.values[row * k + j] - top) - (P::value(z[id]) - m)));
                    }
                }
            }
            sums<THREADS, 3>(loss, part_loss);
            if (tid == 0) {
                if (a.loss) a.loss[row] = some ? loss[2] + a.tau * a.tau * ((loss[0] + loss[1]) * inv_Z) : 0.0f;
                if (a.m) a.m[row] = m;
                if (a.Z) a.Z[row] = Z;
            }
        }
        if (a.dlogits) {
            Element* dz = static_cast<Element*>(a.dlogits) + row * a.ldd;
            const float g = a.tau * (a.weight ? a.weight[row] : 1.0f), of_P = g * inv_Z, of_D = of_P * inv_U;
            if (some) {
                for (int32_t j = tid; j < k; j += THREADS) {
                    if (id_of[j] < 0) continue;
                    const int32_t id = id_of[j] & (kNear - 1), count = count_of[id];
                    const Parts p = stored(r_of[id], count);
                    Parts q = stored(v_of[j], id_of[j]);
                    if ((count & (kNear - 1)) > 1) {  // of all entries of the class (each of them finds the same)
                        q = {0.0f, 0.0f};
                        for (int32_t i = 0; i < k; ++i) {
                            if (id_of[i] < 0 || (id_of[i] & (kNear - 1)) != id) continue;
                            q.whole += id_of[i] & kNear ? 1.0f : 0.0f;
                            q.rest += v_of[i];
                        }
                    }
                    const float D = (p.whole * Nu - q.whole * Nz) + (p.whole * B - q.whole * A) + (p.rest * U - q.rest * Z);
                    g_of[id] = of_D * D;
                }
                group_sync<THREADS>();  // the entries' gradients are there
            }
            for (int32_t e = tid; e < V; e += THREADS) {
                float v = 0.0f;
                if (some) v = count_of[e] & (kNear - 1) ? g_of[e] : of_P * stored(r_of[e], count_of[e]).sum();
                dz[e] = P::element(v);
            }
        }
        group_sync<THREADS>();  // LDS may be written again
    }
}

template <bool WIDE, int THREADS>
void launch(const DistillArgs& a, hipStream_t stream) {
    const int rows = 256 / THREADS;
    const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)a.T + rows - 1) / rows, 1 << 20);
    const size_t lds = (size_t)rows * (3 * a.V + 2 * a.k) * sizeof(float);
    distill_cover_kernel<WIDE, THREADS><<<blocks, 256, lds, stream>>>(a);
}

template <bool WIDE>
void launch(const DistillArgs& a, hipStream_t stream) {
    if (a.V <= 512 && a.k <= 512)  // (40 KiB of LDS at most)
        launch<WIDE, 64>(a, stream);
    else
        launch<WIDE, 256>(a, stream);
}

}  // namespace

hipError_t distill_cover_launch(const DistillArgs& a, hipStream_t stream) {
    if (a.wide)
        launch<true>(a, stream);
    else
        launch<false>(a, stream);
    return hipGetLastError();
}

}  // namespace more
