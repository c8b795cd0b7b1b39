// Launch entry points of the layer's ends (block_norm.hip) and of the gradient clipping (grad_clip.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace more {

// Longest row of the norms: eight waves with two chunks of eight columns per lane.
constexpr int32_t kNormMaxH = 8192;

struct NormArgs {
    const void* r;          // forward: residual in; backward: r_out of the forward pass
    int32_t wide;           // the residual is fp32 (else bf16)
    const uint16_t* y;      // [T][k][h] (k = 0: none)
    int32_t T, h, k;
    const float* w_after;   // [h] or NULL (ones)
    const float* w_before;  // [h] or NULL (no norm before the next block)
    const float* gate;      // [T] or NULL (ones)
    float alpha, eps;
    int32_t norm_after;
    // forward outputs
    void* r_out;
    uint16_t* u;            // or NULL
    uint16_t* xn;
    // backward
    const uint16_t* ub;     // u of the forward pass, or NULL (no block)
    const void* dr_out;     // or NULL (zero)
    const uint16_t* dxn;    // or NULL
    const float* dxn32;     // or NULL
    void* dr;
    uint16_t* du;
    float *dw_after, *dw_before, *dgate;  // each or NULL
};

hipError_t block_norm_launch(const NormArgs& a, hipStream_t stream);
size_t block_norm_backward_workspace(int64_t T, int32_t h);
hipError_t block_norm_backward_launch(const NormArgs& a, void* workspace, hipStream_t stream);

// Tensors of one launch: the descriptors travel in the kernel's arguments.
constexpr int kClipBatch = 48;
struct ClipBatch {
    const void* in[kClipBatch];
    void* out[kClipBatch];
    int64_t numel[kClipBatch];
    int64_t first[kClipBatch + 1];  // first work item of each tensor
    uint8_t bits[kClipBatch];
    uint8_t vec[kClipBatch];        // in and out are 16-byte aligned
    int32_t n;
    int32_t chunk;                  // elements per work item
};
size_t grad_clip_workspace(const int64_t* numel, int32_t n);
hipError_t grad_clip_launch(const void* const* in, void* const* out, const int64_t* numel, const int32_t* bits, int32_t n,
                            float max_norm, float eps, float* norm, void* workspace, hipStream_t stream);

}  // namespace more
