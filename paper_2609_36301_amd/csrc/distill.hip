// Distillation from a teacher's top logits for gfx950.  With row t's student logits z [V], its teacher's entries
// (id_j, v_j), j < k, the temperature tau, and e_j = exp((v_j - max v) / tau) over the valid entries,
//   q_j = e_j / sum e,   m = max z,   Z = sum_e exp((z_e - m) / tau),   P_e = exp((z_e - m) / tau) / Z
//   loss = tau^2 sum_j q_j (ln q_j - ln P_(id_j))
//        = tau^2 (ln Z - ln sum e + sum_j q_j ((v_j - max v) - (z_(id_j) - m)) / tau)
//   d loss / dz_e = tau (P_e - sum_(j: id_j = e) q_j)
// An entry is valid if its id lies in [0, V) and its value is not -infinity; a row without valid entries has loss 0
// and gradient 0.  (V > 2 k: with more entries P and Q may nearly cancel, see distill_cover.hip.)
//
// Memory-bound: a row's logits are read once and stay in registers between maximum, sum and gradient, so that the loss
// with its gradient is one read and one write: 8192 rows of 32001 bf16 187 us, 5.6 TB/s; 16384 of 4096 fp32 154 us in two
// calls, 5.2 TB/s; 37 of 1001 4.9 us in a graph.  A group of threads takes a row, R pieces of 16 bytes to a thread; rows
// that do not fit are read again instead.  Rows start at any element: the pieces are those that lie at multiples of 16
// bytes, and each of the few elements before and behind them is some thread's own, so nothing outside the row is touched.
// The teacher's entries lie in LDS; a wave waits for its stores, then its lanes store the gradients of those entries that
// lie in its own pieces over the first ones (us, one entry after the other by the lane that holds it, without a wait : so,
// 13370 rows of 194 fp32, k = 28 22.8 : 13.4; 16384 of 4096, k = 64 120 : 103, k = 8 93.9 : 95.6).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "distill.h"
#include "distill_device.h"

namespace more {

namespace {

// What keeps a row of bf16 in as many registers as it has bytes: its pieces are unpacked again where they are used next,
// and one after the other (unpacked all at once, 8192 rows of 32001 take 812 us).
__device__ __forceinline__ void one_by_one() { __builtin_amdgcn_sched_barrier(0); }
template <int R>
__device__ __forceinline__ void keep_packed(u32x4 (&v)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) asm volatile("" : "+v"(v[r]));
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

// hi + low += v, of which only the lower part is rounded.
__device__ __forceinline__ void join(float& hi, float& low, float v) {
#pragma clang fp contract(off)
    const float sum = hi + v, of_v = sum - hi;
    low += (hi - (sum - of_v)) + (v - of_v);
    hi = sum;
}

// RESIDENT: the row's pieces (R per thread) stay in registers; else they are read again (R at a time).  ONCE: nontemporal
// loads and stores.
template <bool WIDE, int THREADS, int R, bool RESIDENT, bool ONCE>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void distill_kernel(DistillArgs a) {
    using P = Piece<WIDE>;
    using Element = typename P::Element;
    using Bits = typename std::conditional<WIDE, uint32_t, uint16_t>::type;
    constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;  // rows of a workgroup
    constexpr int kCount = P::kCount;
    extern __shared__ __attribute__((aligned(16))) float dynamic[];
    __shared__ float part_max[16], part_sum[16], total[kRows];
    const int group = kRows == 1 ? 0 : threadIdx.x / THREADS;
    // the teacher's entries: q (first v), id, z, and the sum of q over the entries of their class
    const int32_t k4 = (a.k + 3) & ~3;
    float* q_of = dynamic + (int64_t)group * 4 * k4;
    int32_t* id_of = reinterpret_cast<int32_t*>(q_of + k4);
    float* z_of = q_of + 2 * k4;
    float* sum_of = q_of + 3 * k4;
    const float c = kLog2e / a.tau;

    // What a thread has of a row: pieces, an element before or behind them, one of the first 64 teacher's entries.
    struct Mine {
        u32x4 v[R];
        float own, value;
        int32_t id;
    };
    struct Place {
        const Element* z;
        int32_t head, pieces, edge;  // elements before the pieces; the thread's own element (V or more: none)
    };
    auto place = [&](int64_t row, int tid) {
        Place at;
        at.z = static_cast<const Element*>(a.logits) + row * a.ld;
        const int32_t off = (int32_t)((reinterpret_cast<uintptr_t>(at.z) & 15) / sizeof(Element));
        at.head = off ? min(kCount - off, a.V) : 0;
        at.pieces = (a.V - at.head) / kCount;
        at.edge = tid < at.head ? tid : tid < 2 * kCount ? tid + at.pieces * kCount : a.V;
        return at;
    };
    auto load = [&](Mine& x, const Place& at, int32_t u0) {
        const u32x4* p = reinterpret_cast<const u32x4*>(at.z + at.head);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int32_t u = u0 + r * THREADS;
            x.v[r] = u32x4{P::kNone, P::kNone, P::kNone, P::kNone};
            if (u >= at.pieces) continue;
            if constexpr (ONCE) x.v[r] = __builtin_nontemporal_load(p + (uint32_t)u);
            else x.v[r] = p[(uint32_t)u];
        }
    };
    auto fetch = [&](Mine& x, const Place& at, int64_t row, int tid) {
        x.id = -1;
        x.value = x.own = minus_inf();
        if (tid < 64 && tid < a.k) {
            x.id = a.ids[row * a.k + tid];
            x.value = a.values[row * a.k + tid];
        }
        if (at.edge < a.V) x.own = P::value(at.z[at.edge]);
        if constexpr (RESIDENT) load(x, at, tid);
    };

    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.T; first += (int64_t)gridDim.x * kRows) {
        const int64_t row = first + group;
        if (kRows > 1 && row >= a.T) break;
        int tid = kRows == 1 ? threadIdx.x : threadIdx.x % THREADS;
        asm volatile("" : "+v"(tid));  // (places are computed again for each row, not kept in registers)
        const Place at = place(row, tid);
        Mine x;
        fetch(x, at, row, tid);
        // the teacher, by the group's first wave
        float top = minus_inf();
        if (tid < 64) {
            float z0 = 0.0f;
            const bool valid0 = (uint32_t)x.id < (uint32_t)a.V && x.value != minus_inf();
            if (valid0) z0 = P::value(at.z[x.id]);
            for (int32_t j = tid; j < k4; j += 64) {
                const bool first64 = j < 64;
                const int32_t id = first64 ? x.id : j < a.k ? a.ids[row * a.k + j] : -1;
                const float t = first64 ? x.value : j < a.k ? a.values[row * a.k + j] : minus_inf();
                const bool valid = first64 ? valid0 : (uint32_t)id < (uint32_t)a.V && t != minus_inf();
                id_of[j] = valid ? id : -1;
                q_of[j] = t;
                z_of[j] = first64 ? z0 : valid ? P::value(at.z[id]) : 0.0f;
                if (valid) top = fmaxf(top, t);
            }
            top = wave_max(top);
            float sum = 0.0f;
            bool any = false;
            for (int32_t j = tid; j < a.k; j += 64) {
                const bool valid = id_of[j] >= 0;
                sum += valid ? __builtin_amdgcn_exp2f((q_of[j] - top) * c) : 0.0f;
                any |= valid;
            }
            sum = wave_sum(sum);
            const bool none = __ballot(any) == 0;
            if (tid == 0) total[group] = none ? 0.0f : sum;
        }
        // maximum m and sum Z of the row
        float m = x.own, Z;
        if (a.m_in) {
            m = a.m_in[row];
            Z = a.Z_in[row];
        } else if constexpr (RESIDENT) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int i = 0; i < kCount; ++i) m = fmaxf(m, P::value(x.v[r], i));
                one_by_one();
            }
            m = group_reduce<THREADS, true>(m, part_max);
            keep_packed(x.v);
            Z = __builtin_amdgcn_exp2f((x.own - m) * c);
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int i = 0; i < kCount; ++i) Z += __builtin_amdgcn_exp2f((P::value(x.v[r], i) - m) * c);
                one_by_one();
            }
            Z = group_reduce<THREADS, false>(Z, part_sum);
            keep_packed(x.v);
        } else {
            // A running maximum and sum per thread: R pieces are summed apart and then join a sum of two floats (one after
            // the other, the roundings of V / THREADS terms add up: 1.9e-4 of Z on 2^26 ascending fp32 logits).  Its exponents count from
            // `base`, which follows the maximum in steps of 2^8: a step rounds the sum, so that there are few.
            float base = m, low = 0.0f;
            Z = m == minus_inf() ? 0.0f : m == m ? 1.0f : m;
            for (int32_t u0 = tid; u0 < at.pieces; u0 += R * THREADS) {
                load(x, at, u0);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < kCount; ++i) m = fmaxf(m, P::value(x.v[r], i));
                const bool move = (m - base) * c > 8.0f;  // (infinite where there was nothing but -infinity)
                const float f = move ? __builtin_amdgcn_exp2f((base - m) * c) : 1.0f;
                Z *= f;
                low *= f;
                base = move ? m : base;
                const float from = base == minus_inf() ? 0.0f : base;
                float part = 0.0f;
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < kCount; ++i) part += __builtin_amdgcn_exp2f((P::value(x.v[r], i) - from) * c);
                join(Z, low, part);
            }
            m = group_reduce<THREADS, true>(m, part_max);
            Z = group_reduce<THREADS, false>((Z + low) * __builtin_amdgcn_exp2f((base - m) * c), part_sum);
        }
        group_sync<THREADS>();  // the teacher's entries and their sum are there
        const float U = total[group];
        const bool some = U != 0.0f;  // (NaN values make U NaN)
        if (tid < 64) {
            float dot = 0.0f;
            for (int32_t j = tid; j < a.k; j += 64) {
                const float d = q_of[j] - top;
                const float q = id_of[j] >= 0 ? __builtin_amdgcn_exp2f(d * c) / U : 0.0f;
                // (an entry whose q is zero has no share, whatever the student says)
                if (q != 0.0f) dot += q * (d - (z_of[j] - m));
                q_of[j] = q;
            }
            dot = wave_sum(dot);
            if (tid == 0) {
                if (a.loss)
                    a.loss[row] = some ? a.tau * a.tau *
                                             ((__builtin_amdgcn_logf(Z) - __builtin_amdgcn_logf(U)) * kLn2 + dot / a.tau)
                                       : 0.0f;
                if (a.m) a.m[row] = m;
                if (a.Z) a.Z[row] = Z;
            }
        }
        if (a.dlogits) {
            // an id may occur more than once: its entries' q together (by all waves where there are many; those of the
            // first 64 by the wave that made them)
            if (a.k > 64) group_sync<THREADS>();
            else wave_lds_sync();
            for (int32_t j = tid; j < a.k; j += THREADS) {
                const int32_t id = id_of[j];
                float q = 0.0f;
                for (int32_t i = 0; i < k4; i += 4) {
                    const i32x4 ids = *reinterpret_cast<const i32x4*>(id_of + i);
                    const f32x4 qs = *reinterpret_cast<const f32x4*>(q_of + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) q += ids[e] == id ? qs[e] : 0.0f;
                }
                sum_of[j] = q;
            }
            Element* dz = static_cast<Element*>(a.dlogits) + row * a.ldd;
            const float g = a.tau * (a.weight ? a.weight[row] : 1.0f), gp = g / Z;
            // (the pieces of z need not lie at multiples of 16 bytes of dlogits)
            u32x4* to = reinterpret_cast<u32x4*>(dz + at.head);
            const bool vector = (reinterpret_cast<uintptr_t>(to) & 15) == 0;
            auto put = [&](int32_t u, const u32x4& w) {
                if (vector) {
                    if constexpr (ONCE) __builtin_nontemporal_store(w, to + (uint32_t)u);
                    else to[(uint32_t)u] = w;
                } else {
#pragma unroll
                    for (int i = 0; i < kCount; ++i) {
                        const uint32_t b = w[WIDE ? i : i / 2];
                        dz[at.head + u * kCount + i] = __builtin_bit_cast(Element, (Bits)(WIDE || i % 2 == 0 ? b : b >> 16));
                    }
                }
            };
            auto gradient = [&](const u32x4& w) {
                float f[kCount];
#pragma unroll
                for (int i = 0; i < kCount; ++i) f[i] = gp * __builtin_amdgcn_exp2f((P::value(w, i) - m) * c);
                return P::pack(f);
            };
            if (!some) {  // no teacher: zeros
                for (int32_t u = tid; u < at.pieces; u += THREADS) put(u, u32x4{0u, 0u, 0u, 0u});
            } else if constexpr (RESIDENT) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int32_t u = tid + r * THREADS;
                    if (u < at.pieces) put(u, gradient(x.v[r]));
                    one_by_one();
                }
            } else {
                for (int32_t u0 = tid; u0 < at.pieces; u0 += R * THREADS) {
                    load(x, at, u0);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const int32_t u = u0 + r * THREADS;
                        if (u < at.pieces) put(u, gradient(x.v[r]));
                    }
                }
            }
            if (at.edge < a.V) dz[at.edge] = P::element(some ? gp * __builtin_amdgcn_exp2f((x.own - m) * c) : 0.0f);
            group_sync<THREADS>();  // the sums are there
            if (some) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the wave's pieces have been written
                for (int32_t j = tid & 63; j < a.k; j += 64) {
                    const int32_t id = id_of[j], in = id - at.head, end = at.pieces * kCount;
                    // the thread whose piece or own element it is
                    const int32_t owner = in < 0 ? id : in < end ? (int32_t)((uint32_t)in / kCount % THREADS) : id - end;
                    if (id >= 0 && owner >> 6 == tid >> 6)
                        dz[id] = P::element(gp * __builtin_amdgcn_exp2f((z_of[j] - m) * c) - g * sum_of[j]);
                }
            }
        }
        group_sync<THREADS>();  // LDS may be written again
    }
}

template <bool WIDE, int THREADS, int R, bool RESIDENT = true, bool LONG = true>
void launch(const DistillArgs& a, hipStream_t stream) {
    const int rows = THREADS < 256 ? 256 / THREADS : 1, threads = THREADS < 256 ? 256 : THREADS;
    const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)a.T + rows - 1) / rows, 1 << 20);
    const size_t lds = (size_t)rows * 4 * ((a.k + 3) & ~3) * sizeof(float);
    // Long rows of logits beyond the last-level cache's 256 MB pass by it (us, plain : nontemporal, 8192 rows of 32001
    // bf16 203 : 191, of 16384 fp32 213 : 199; short rows are slower by it, 32768 of 512 fp32 36 : 43).
    const bool once = LONG && (int64_t)a.T * a.V * (WIDE ? 4 : 2) > (int64_t)256 << 20;
    if (once)
        distill_kernel<WIDE, THREADS, R, RESIDENT, LONG><<<blocks, threads, lds, stream>>>(a);
    else
        distill_kernel<WIDE, THREADS, R, RESIDENT, false><<<blocks, threads, lds, stream>>>(a);
}

// Threads and pieces by the row's length: as few threads as leave a thread up to 8 pieces (more workgroups to a CU, that
// compute while others wait), then up to 16 (us, 8192 rows of 32001 bf16, 512 threads : 1024 191 : 300; 4096 of 65536
// 221 : 241; 16384 of 4096, 64 threads : 256 54 : 67).  A call that reads its rows once, for the loss alone or with known
// statistics, need not keep them (us, kept : not, 4096 rows of 65536 bf16, loss 91 : 81, gradient 195 : 186; 2048 of
// 131072, loss 122 : 91; with both 219 : 274).
template <bool WIDE>
void launch(const DistillArgs& a, hipStream_t stream) {
    const int32_t pieces = a.V / Piece<WIDE>::kCount;
    const bool few = a.k <= 256;  // (four rows' entries in LDS)
    if (few && pieces <= 64)
        launch<WIDE, 64, 1, true, false>(a, stream);
    else if (few && pieces <= 128)
        launch<WIDE, 64, 2, true, false>(a, stream);
    else if (few && pieces <= 256)
        launch<WIDE, 64, 4, true, false>(a, stream);
    else if (few && pieces <= 512)
        launch<WIDE, 64, 8, true, false>(a, stream);
    else if (pieces <= 1024)
        launch<WIDE, 256, 4>(a, stream);
    else if (pieces <= 2048)
        launch<WIDE, 256, 8>(a, stream);
    else if (pieces <= 4096)
        launch<WIDE, 512, 8>(a, stream);
    else if (!a.dlogits || a.m_in)
        launch<WIDE, 512, 8, false>(a, stream);
    else if (pieces <= 8192)
        launch<WIDE, 512, 16>(a, stream);
    else if (pieces <= 16384)
        launch<WIDE, 1024, 16>(a, stream);
    else
        launch<WIDE, 1024, 4, false>(a, stream);
}

}  // namespace

hipError_t distill_launch(const DistillArgs& a, hipStream_t stream) {
    if (a.V <= 2 * a.k) return distill_cover_launch(a, stream);
    if (a.wide)
        launch<true>(a, stream);
    else
        launch<false>(a, stream);
    return hipGetLastError();
}

}  // namespace more
