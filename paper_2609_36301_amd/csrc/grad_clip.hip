// The 2-norm of many gradients together and their scaling to a largest norm, for gfx950:
//   N = sqrt(sum over all tensors and elements of g^2),  c = min(1, max_norm / (N + eps)),  out = c g.
// Two kernels per kClipBatch tensors.  grad_sumsq adds squares in fp64 (no overflow: the largest fp32
// squared is 1e77; fp64 keeps pace with memory here) in a fixed order, one partial per workgroup;
// grad_scale adds the partials, every workgroup for itself, and scales.  Bound by memory: two reads of
// the gradients and a write; in place a factor of one writes nothing.  538 MB of gradients: 138 us for the
// squares (3.9 TB/s) and 270 us for the scaling (4.0 TB/s; with an ordinary second read and ordinary stores,
// and uneven shares, the call took 466 us); 1.6 MB: 4.4 and 5.4 us, each a launch and the latency of its reads.
// Many tensors are bound by the launches, two for every kClipBatch: 1000 of 4096 elements 197 us, 10000 2.4 ms; every
// scaling workgroup adds the partials of all batches, which shows from there on (30000 tensors 8.8 ms).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "device_common.h"
#include "layer.h"

namespace more {

namespace {

constexpr int kClipThreads = 256;
constexpr int64_t kClipBlocks = 2048;  // workgroups (and partials) per batch at most

// The tensor of a work item.
__device__ __forceinline__ int clip_tensor(const ClipBatch& b, int64_t item) {
    int lo = 0, hi = b.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (b.first[mid] <= item) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double clip_wave_sum(double v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

__device__ __forceinline__ double clip_block_sum(double v, double* red) {
    v = clip_wave_sum(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < kClipThreads / 64; ++w) v += red[w];
    return v;
}

__device__ __forceinline__ double square(float v) { return (double)v * (double)v; }

}  // namespace

__global__ __launch_bounds__(kClipThreads) void grad_sumsq_kernel(ClipBatch b, double* __restrict__ parts) {
    __shared__ double red[kClipThreads / 64];
    double sum = 0.0;
    for (int64_t item = blockIdx.x; item < b.first[b.n]; item += gridDim.x) {
        const int i = clip_tensor(b, item);
        const int64_t at = (item - b.first[i]) * b.chunk;
        const int32_t len = (int32_t)min((int64_t)b.chunk, b.numel[i] - at);
        const int32_t vec = b.vec[i] ? (b.bits[i] == 32 ? len / 4 : len / 8) : 0;
        if (b.bits[i] == 32) {
            const float* g = static_cast<const float*>(b.in[i]) + at;
#pragma unroll 8
            for (int32_t q = threadIdx.x; q < vec; q += kClipThreads) {
                const f32x4 v = reinterpret_cast<const f32x4*>(g)[q];
                sum += (square(v[0]) + square(v[1])) + (square(v[2]) + square(v[3]));
            }
            for (int32_t q = 4 * vec + threadIdx.x; q < len; q += kClipThreads) sum += square(g[q]);
        } else {
            const uint16_t* g = static_cast<const uint16_t*>(b.in[i]) + at;
#pragma unroll 8
            for (int32_t q = threadIdx.x; q < vec; q += kClipThreads) {
                const u32x4 v = reinterpret_cast<const u32x4*>(g)[q];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum += square(__builtin_bit_cast(float, v[e] << 16)) +
                           square(__builtin_bit_cast(float, v[e] & 0xFFFF0000u));
            }
            for (int32_t q = 8 * vec + threadIdx.x; q < len; q += kClipThreads) sum += square(bf16_bits_to_f32(g[q]));
        }
    }
    sum = clip_block_sum(sum, red);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kClipThreads) void grad_scale_kernel(ClipBatch b, const double* __restrict__ parts,
                                                               int32_t nparts, float max_norm, float eps,
                                                               float* __restrict__ norm) {
    __shared__ double red[kClipThreads / 64];
    double sum = 0.0;
#pragma unroll 8
    for (int32_t i = threadIdx.x; i < nparts; i += kClipThreads) sum += parts[i];
    const double n = sqrt(clip_block_sum(sum, red));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    double cd = (double)max_norm / (n + (double)eps);
    if (cd > 1.0) cd = 1.0;  // a NaN stays one
    const float c = (float)cd;
    for (int64_t item = blockIdx.x; item < b.first[b.n]; item += gridDim.x) {
        const int i = clip_tensor(b, item);
        if (c == 1.0f && b.in[i] == b.out[i]) continue;
        const int64_t at = (item - b.first[i]) * b.chunk;
        const int32_t len = (int32_t)min((int64_t)b.chunk, b.numel[i] - at);
        const int32_t vec = b.vec[i] ? (b.bits[i] == 32 ? len / 4 : len / 8) : 0;
        if (b.bits[i] == 32) {
            const float* g = static_cast<const float*>(b.in[i]) + at;
            float* o = static_cast<float*>(b.out[i]) + at;
#pragma unroll 8
            for (int32_t q = threadIdx.x; q < vec; q += kClipThreads)
                __builtin_nontemporal_store(__builtin_nontemporal_load(reinterpret_cast<const f32x4*>(g) + q) * c,
                                            reinterpret_cast<f32x4*>(o) + q);
            for (int32_t q = 4 * vec + threadIdx.x; q < len; q += kClipThreads) o[q] = g[q] * c;
        } else {
            const uint16_t* g = static_cast<const uint16_t*>(b.in[i]) + at;
            uint16_t* o = static_cast<uint16_t*>(b.out[i]) + at;
#pragma unroll 8
            for (int32_t q = threadIdx.x; q < vec; q += kClipThreads) {
                const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(g) + q);
                bf16x8 r;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    r[2 * e] = (__bf16)(__builtin_bit_cast(float, v[e] << 16) * c);
                    r[2 * e + 1] = (__bf16)(__builtin_bit_cast(float, v[e] & 0xFFFF0000u) * c);
                }
                __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<u32x4*>(o) + q);
            }
            for (int32_t q = 8 * vec + threadIdx.x; q < len; q += kClipThreads)
                o[q] = __builtin_bit_cast(uint16_t, (__bf16)(bf16_bits_to_f32(g[q]) * c));
        }
    }
}

// ------------------------------------------------------------------------------ host
namespace {

// Elements per work item: so many that kClipBlocks workgroups have about one item each, within 2048 (a
// 16-byte bf16 load per thread: small sets fill more of the chip) and 16384 (eight such loads in flight; 538 MB
// take 138 us for the squares and 269 for the scaling, with 8192 197 and 260; 512 workgroups 141 and 346, 1024 to
// 4096 the same as 2048).
int32_t clip_chunk(const int64_t* numel, int32_t n) {
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) total += numel[i];
    return (int32_t)std::min<int64_t>(16384, std::max<int64_t>(1, total / (2048 * kClipBlocks)) * 2048);
}

int64_t batch_items(const int64_t* numel, int32_t first, int32_t count, int32_t chunk) {
    int64_t items = 0;
    for (int32_t i = 0; i < count; ++i) items += (numel[first + i] + chunk - 1) / chunk;
    return items;
}

// At most kClipBlocks workgroups with the same number of items each (but for the last ones).
int64_t batch_blocks(int64_t items) {
    const int64_t rounds = std::max<int64_t>(1, (items + kClipBlocks - 1) / kClipBlocks);
    return std::max<int64_t>(1, (items + rounds - 1) / rounds);
}

}  // namespace

size_t grad_clip_workspace(const int64_t* numel, int32_t n) {
    int64_t parts = 0;
    const int32_t chunk = clip_chunk(numel, n);
    for (int32_t first = 0; first == 0 || first < n; first += kClipBatch)
        parts += batch_blocks(batch_items(numel, first, std::min(kClipBatch, n - first), chunk));
    return (size_t)parts * sizeof(double);
}

hipError_t grad_clip_launch(const void* const* in, void* const* out, const int64_t* numel, const int32_t* bits, int32_t n,
                            float max_norm, float eps, float* norm, void* workspace, hipStream_t stream) {
    double* parts = static_cast<double*>(workspace);
    int64_t nparts = 0;
    const int32_t chunk = clip_chunk(numel, n);
    for (int pass = 0; pass < 2; ++pass) {
        int64_t at = 0;
        for (int32_t first = 0; first == 0 || first < n; first += kClipBatch) {
            ClipBatch b = {};
            b.n = std::min(kClipBatch, n - first);
            b.chunk = chunk;
            for (int32_t i = 0; i < b.n; ++i) {
                b.in[i] = in[first + i];
                b.out[i] = out[first + i];
                b.numel[i] = numel[first + i];
                b.bits[i] = (uint8_t)bits[first + i];
                b.vec[i] = ((reinterpret_cast<uintptr_t>(b.in[i]) | reinterpret_cast<uintptr_t>(b.out[i])) & 15) == 0;
                b.first[i + 1] = b.first[i] + (b.numel[i] + chunk - 1) / chunk;
            }
            const unsigned blocks = (unsigned)batch_blocks(b.first[b.n]);
            if (pass == 0)
                grad_sumsq_kernel<<<blocks, kClipThreads, 0, stream>>>(b, parts + at);
            else
                grad_scale_kernel<<<blocks, kClipThreads, 0, stream>>>(b, parts, (int32_t)nparts, max_norm, eps,
                                                                       first == 0 ? norm : nullptr);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            at += blocks;
        }
        nparts = at;
    }
    return hipSuccess;
}

}  // namespace more
