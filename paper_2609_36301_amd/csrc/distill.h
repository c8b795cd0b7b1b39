// Launch entry points of the distillation loss (distill.hip, distill_cover.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace more {

constexpr int32_t kDistillMaxTeacher = 1024;

struct DistillArgs {
    const void* logits;   // [T] rows of V values, `ld` apart; fp32 (wide) or bf16
    int32_t T, V, k, wide;
    int64_t ld, ldd;
    const int32_t* ids;   // [T][k]
    const float* values;  // [T][k]
    const float* weight;  // [T] or NULL (ones)
    float tau;
    const float *m_in, *Z_in;  // [T]: the statistics are known (backward), or NULL
    float *loss, *m, *Z;       // [T], each or NULL
    void* dlogits;             // [T] rows of V values, `ldd` apart, of the logits' type, or NULL; may be logits
};

hipError_t distill_launch(const DistillArgs& a, hipStream_t stream);

// The same for V <= 2 k (distill_cover.hip).
hipError_t distill_cover_launch(const DistillArgs& a, hipStream_t stream);

}  // namespace more
