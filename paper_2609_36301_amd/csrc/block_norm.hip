// The end of one block and the norm before the next, in one pass, for gfx950.  Per token t:
//   u   = sum_j y[t][j]                        (the block's output: k slot rows, e.g. of k experts)
//   n   = u / rms(u), or u                     rms(v) = sqrt(mean(v^2) + eps)
//   r'  = alpha r + gate[t] (w_after n)        (gate and residual scale)
//   xn  = w_before r' / rms(r')
// and its backward pass: with q = w_before dxn, D the gradient of r' and p = gate D w_after,
//   D    = dr_out + (q - n' mean(q n')) / rms(r')   with n' = r' / rms(r')
//   dr   = alpha D
//   du   = (p - n mean(p n)) / rms(u)   (or p)
//   dw_before = sum_t dxn n',  dw_after = sum_t gate D n,  dgate = sum_c D w_after n
// All sums are fp32; xn is normalised from the unrounded r'.  (1 / rms is never raised to its third power, which
// leaves fp32 for rows of zeros with a small eps and for rows of large values.)
//
// Bound by memory: every row is read once and kept in registers, W waves to a row (a wave for short
// rows), eight columns of 16 (bf16) or 32 bytes per lane and chunk, CH chunks per lane.  Measured: forward, 32768
// tokens of h = 2048, k = 8, fp32 residual 316 us, 5.9 TB/s; 128 tokens of h = 4096, k = 16 6.9 us, 3 TB/s (with
// four waves, two chunks and four of the k rows in flight 15.1 us: the bytes in flight count there); backward, 16381 tokens of
// h = 2032, fp32 residual, gate and the router's addend 137 us, 5.3 TB/s, and 7 us for the weights' partial rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "device_common.h"
#include "layer.h"

namespace more {

namespace {

// A workgroup holds four rows of one wave each, or one row of W waves.
constexpr int norm_threads(int W) { return W == 1 ? 256 : 64 * W; }
constexpr int norm_rows(int W) { return W == 1 ? 4 : 1; }

struct V8 {
    float v[8];
};

__device__ __forceinline__ V8 unpack8(u32x4 b) {
    V8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o.v[2 * i] = __builtin_bit_cast(float, b[i] << 16);
        o.v[2 * i + 1] = __builtin_bit_cast(float, b[i] & 0xFFFF0000u);
    }
    return o;
}
__device__ __forceinline__ V8 load8(const uint16_t* p) { return unpack8(*reinterpret_cast<const u32x4*>(p)); }
__device__ __forceinline__ V8 load8(const float* p) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
    return V8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ void store8(uint16_t* p, const V8& x) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)x.v[i];
    *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, o);
}
__device__ __forceinline__ void store8(float* p, const V8& x) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{x.v[4], x.v[5], x.v[6], x.v[7]};
}
template <bool WIDE>
__device__ __forceinline__ V8 load_resid(const void* p, int64_t at) {
    return WIDE ? load8(static_cast<const float*>(p) + at) : load8(static_cast<const uint16_t*>(p) + at);
}
template <bool WIDE>
__device__ __forceinline__ void store_resid(void* p, int64_t at, const V8& x) {
    if constexpr (WIDE)
        store8(static_cast<float*>(p) + at, x);
    else
        store8(static_cast<uint16_t*>(p) + at, x);
}

// Sums of a row's waves (the W waves of a workgroup's row; every lane gets them).  `red` is shared
// memory of N W floats that no other sum of the same row step uses.
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* red) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] += lane_xor<1>(v[i]);
        v[i] += lane_xor<2>(v[i]);
        v[i] += lane_xor<4>(v[i]);
        v[i] += lane_xor<8>(v[i]);
        float a, b;
        lane_pair16(v[i], a, b);
        v[i] = a + b;
        v[i] = sum_pair32(v[i]);
    }
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[i * W + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = red[i * W];
#pragma unroll
            for (int w = 1; w < W; ++w) v[i] += red[i * W + w];
        }
    }
}

}  // namespace

// ------------------------------------------------------------------------------ forward
template <int W, int CH, bool WIDE>
__global__ __launch_bounds__(norm_threads(W)) void block_norm_kernel(NormArgs a) {
    constexpr int kRows = norm_rows(W);  // rows per workgroup
    __shared__ float red[2][W];
    const int lane = threadIdx.x & (64 * W - 1);
    const int64_t t = (int64_t)blockIdx.x * kRows + (W == 1 ? threadIdx.x >> 6 : 0);
    if (t >= a.T) return;  // W > 1: uniform over the workgroup
    const int32_t h = a.h;
    const float inv_h = 1.0f / (float)h;
    V8 r[CH], u[CH];
    bool in[CH];
    int32_t c[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        c[i] = 8 * (lane + 64 * W * i);
        in[i] = c[i] < h;
        u[i] = V8{};
        r[i] = V8{};
        if (in[i]) r[i] = load_resid<WIDE>(a.r, t * h + c[i]);
    }
    if (a.k > 0) {
        const uint16_t* y = a.y + t * a.k * h;
        constexpr int kAhead = 8;  // rows in flight, added in order
        for (int32_t j = 0; j < a.k; j += kAhead) {
            u32x4 v[kAhead][CH];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    v[q][i] = u32x4{0u, 0u, 0u, 0u};
                    if (in[i] && j + q < a.k)
                        v[q][i] = __builtin_nontemporal_load(
                            reinterpret_cast<const u32x4*>(y + (int64_t)(j + q) * h + c[i]));  // not read again
                }
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const V8 x = unpack8(v[q][i]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[i].v[e] += x.v[e];
                }
        }
        float scale = a.gate ? a.gate[t] : 1.0f;
        if (a.norm_after) {
            float ss[1] = {0.0f};
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) ss[0] = __builtin_fmaf(u[i].v[e], u[i].v[e], ss[0]);
            row_sums<W, 1>(ss, red[0]);
            scale *= rsqrtf(__builtin_fmaf(ss[0], inv_h, a.eps));
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (!in[i]) continue;
            if (a.u) store8(a.u + t * h + c[i], u[i]);
            V8 w;
            if (a.w_after) w = load8(a.w_after + c[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float b = a.w_after ? u[i].v[e] * scale * w.v[e] : u[i].v[e] * scale;
                r[i].v[e] = __builtin_fmaf(a.alpha, r[i].v[e], b);
            }
            store_resid<WIDE>(a.r_out, t * h + c[i], r[i]);
        }
    }
    if (!a.xn) return;
    float ss[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss[0] = __builtin_fmaf(r[i].v[e], r[i].v[e], ss[0]);
    row_sums<W, 1>(ss, red[1]);
    const float rs = rsqrtf(__builtin_fmaf(ss[0], inv_h, a.eps));
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (!in[i]) continue;
        const V8 w = load8(a.w_before + c[i]);
        V8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = r[i].v[e] * rs * w.v[e];
        store8(a.xn + t * h + c[i], o);
    }
}

// ------------------------------------------------------------------------------ backward
// A workgroup takes every gridDim-th group of rows; a lane keeps the columns it owns, so the weights'
// gradients are summed in its registers over the workgroup's rows and written as one partial row per
// workgroup: parts [workgroup][2][h] (dw_after, dw_before).
template <int W, int CH, bool WIDE>
__global__ __launch_bounds__(norm_threads(W)) void block_norm_backward_kernel(NormArgs a, float* __restrict__ parts) {
    constexpr int kRows = norm_rows(W);
    __shared__ float red[2][3 * W];
    __shared__ float fold[W == 1 ? 2 * 4 * 512 * CH : 1];
    const int lane = threadIdx.x & (64 * W - 1);
    const int32_t h = a.h;
    const float inv_h = 1.0f / (float)h;
    const bool block = a.ub != nullptr;
    const bool before = a.dxn || a.dxn32;
    V8 wa[CH], wb[CH], dwa[CH], dwb[CH];
    bool in[CH];
    int32_t c[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        c[i] = 8 * (lane + 64 * W * i);
        in[i] = c[i] < h;
        dwa[i] = dwb[i] = wb[i] = V8{};
#pragma unroll
        for (int e = 0; e < 8; ++e) wa[i].v[e] = 1.0f;
        if (in[i] && a.w_after) wa[i] = load8(a.w_after + c[i]);
        if (in[i] && a.w_before) wb[i] = load8(a.w_before + c[i]);
    }
    for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < a.T; t0 += (int64_t)gridDim.x * kRows) {
        const int64_t t = t0 + (W == 1 ? threadIdx.x >> 6 : 0);
        if (t >= a.T) continue;  // W > 1: never
        V8 r[CH], u[CH], D[CH], dn[CH];
        float s1[3] = {0.0f, 0.0f, 0.0f};  // sum r^2, sum q r, sum u^2
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            r[i] = u[i] = D[i] = dn[i] = V8{};
            if (!in[i]) continue;
            const int64_t at = t * h + c[i];
            r[i] = load_resid<WIDE>(a.r, at);
            if (block) u[i] = load8(a.ub + at);
            if (a.dr_out) D[i] = load_resid<WIDE>(a.dr_out, at);
            if (a.dxn) dn[i] = load8(a.dxn + at);
            if (a.dxn32) {
                const V8 x = load8(a.dxn32 + at);
#pragma unroll
                for (int e = 0; e < 8; ++e) dn[i].v[e] += x.v[e];
            }
        }
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s1[0] = __builtin_fmaf(r[i].v[e], r[i].v[e], s1[0]);
                s1[1] = __builtin_fmaf(dn[i].v[e] * wb[i].v[e], r[i].v[e], s1[1]);
                s1[2] = __builtin_fmaf(u[i].v[e], u[i].v[e], s1[2]);
            }
        row_sums<W, 3>(s1, red[0]);
        if (before) {
            const float rs = rsqrtf(__builtin_fmaf(s1[0], inv_h, a.eps));
            const float m = rs * (s1[1] * inv_h);
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float n = r[i].v[e] * rs;
                    dwb[i].v[e] = __builtin_fmaf(dn[i].v[e], n, dwb[i].v[e]);
                    D[i].v[e] += rs * (dn[i].v[e] * wb[i].v[e] - n * m);
                }
        }
        const float alpha = block ? a.alpha : 1.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (!in[i]) continue;
            V8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o.v[e] = alpha * D[i].v[e];
            store_resid<WIDE>(a.dr, t * h + c[i], o);
        }
        if (block) {
            const float gate = a.gate ? a.gate[t] : 1.0f;
            const float ru = a.norm_after ? rsqrtf(__builtin_fmaf(s1[2], inv_h, a.eps)) : 1.0f;
            float s2[1] = {0.0f};  // sum D w_after u
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s2[0] = __builtin_fmaf(D[i].v[e] * wa[i].v[e], u[i].v[e], s2[0]);
                    dwa[i].v[e] = __builtin_fmaf(gate * D[i].v[e], u[i].v[e] * ru, dwa[i].v[e]);
                }
            row_sums<W, 1>(s2, red[1]);
            const float m = a.norm_after ? ru * (s2[0] * inv_h) : 0.0f;
            if (a.dgate && lane == 0) a.dgate[t] = s2[0] * ru;
            const float p = gate * ru;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                if (!in[i]) continue;
                V8 o;
#pragma unroll
                for (int e = 0; e < 8; ++e) o.v[e] = p * (D[i].v[e] * wa[i].v[e] - u[i].v[e] * ru * m);
                store8(a.du + t * h + c[i], o);
            }
        }
        // red[0] is written again only after the second sum's barrier; without a block there is none
        if (W > 1 && !block) __syncthreads();
    }
    float* out = parts + (int64_t)blockIdx.x * 2 * h;
    if constexpr (W == 1) {  // the four waves' rows are added in order
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            store8(fold + (wave * 2 + 0) * 512 * CH + c[i], dwa[i]);
            store8(fold + (wave * 2 + 1) * 512 * CH + c[i], dwb[i]);
        }
        __syncthreads();
        for (int32_t i = threadIdx.x; i < 2 * h; i += norm_threads(W)) {
            const int32_t which = i / h, col = i - which * h;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v += fold[(w * 2 + which) * 512 * CH + col];
            out[i] = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (!in[i]) continue;
            store8(out + c[i], dwa[i]);
            store8(out + h + c[i], dwb[i]);
        }
    }
}

// The partial rows added in a fixed order: 16 columns per workgroup, 16 threads to a column, each adding
// every sixteenth row.
__global__ __launch_bounds__(256) void block_norm_dw_kernel(const float* __restrict__ parts, int32_t rows, int32_t h,
                                                         float* __restrict__ dw_after,
                                                         float* __restrict__ dw_before) {
    __shared__ float red[16][17];
    const int col = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int32_t c = (int32_t)blockIdx.x * 16 + col;  // of 2h (a multiple of 16)
    float v = 0.0f;
#pragma unroll 8
    for (int32_t i = group; i < rows; i += 16) v += parts[(int64_t)i * 2 * h + c];
    red[group][col] = v;
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int g = 1; g < 16; ++g) v += red[g][col];
    float* out = c < h ? dw_after : dw_before;
    if (out) out[c < h ? c : c - h] = v;
}

// ------------------------------------------------------------------------------ host
namespace {

// Workgroups of the backward pass: a partial row of weight gradients each.
int32_t backward_blocks(int64_t T, int32_t h) {
    const int64_t rows = h <= 1024 ? (T + 3) / 4 : T;
    return (int32_t)std::min<int64_t>(rows, 1024);
}

// In launches of at most 2^22 workgroups (a launch may not have 2^32 threads along an axis).
template <int W, int CH>
hipError_t forward(NormArgs a, hipStream_t stream) {
    constexpr int64_t kMaxRows = (int64_t)norm_rows(W) << 22;
    const int64_t T = a.T, resid = a.wide ? 4 : 2;
    for (int64_t t = 0; t < T; t += kMaxRows) {
        a.T = (int32_t)std::min(T - t, kMaxRows);
        const unsigned blocks = (unsigned)((a.T + norm_rows(W) - 1) / norm_rows(W));
        if (a.wide)
            block_norm_kernel<W, CH, true><<<blocks, norm_threads(W), 0, stream>>>(a);
        else
            block_norm_kernel<W, CH, false><<<blocks, norm_threads(W), 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int64_t step = a.T * (int64_t)a.h;
        a.r = static_cast<const char*>(a.r) + step * resid;
        if (a.r_out) a.r_out = static_cast<char*>(a.r_out) + step * resid;
        if (a.y) a.y += step * a.k;
        if (a.u) a.u += step;
        if (a.xn) a.xn += step;
        if (a.gate) a.gate += a.T;
    }
    return hipSuccess;
}

template <int W, int CH>
hipError_t backward(const NormArgs& a, float* parts, int32_t blocks, hipStream_t stream) {
    if (a.wide)
        block_norm_backward_kernel<W, CH, true><<<blocks, norm_threads(W), 0, stream>>>(a, parts);
    else
        block_norm_backward_kernel<W, CH, false><<<blocks, norm_threads(W), 0, stream>>>(a, parts);
    return hipGetLastError();
}

}  // namespace

hipError_t block_norm_launch(const NormArgs& a, hipStream_t stream) {
    if (a.h <= 512) return forward<1, 1>(a, stream);
    if (a.h <= 1024) return forward<1, 2>(a, stream);
    if (a.h <= 2048) return forward<4, 1>(a, stream);
    if (a.h <= 4096) return forward<8, 1>(a, stream);
    return forward<8, 2>(a, stream);
}

size_t block_norm_backward_workspace(int64_t T, int32_t h) {
    return (size_t)backward_blocks(T, h) * 2 * h * sizeof(float);
}

hipError_t block_norm_backward_launch(const NormArgs& a, void* workspace, hipStream_t stream) {
    float* parts = static_cast<float*>(workspace);
    const int32_t blocks = backward_blocks(a.T, a.h);
    hipError_t e = hipSuccess;
    if (blocks > 0) {
        if (a.h <= 512) e = backward<1, 1>(a, parts, blocks, stream);
        else if (a.h <= 1024) e = backward<1, 2>(a, parts, blocks, stream);
        else if (a.h <= 2048) e = backward<4, 1>(a, parts, blocks, stream);
        else if (a.h <= 4096) e = backward<8, 1>(a, parts, blocks, stream);
        else e = backward<8, 2>(a, parts, blocks, stream);
        if (e != hipSuccess) return e;
    }
    if (!a.dw_after && !a.dw_before) return e;
    block_norm_dw_kernel<<<(unsigned)(2 * a.h / 16), 256, 0, stream>>>(parts, blocks, a.h, a.dw_after, a.dw_before);
    return hipGetLastError();
}

}  // namespace more
