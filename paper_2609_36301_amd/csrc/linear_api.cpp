// C ABI of the experts' linear maps, the quantisation of rows and the distillation loss: argument validation and
// launch (more.h).  Every check runs on the host before anything is enqueued, so an error status means the stream was
// not touched.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "more.h"
#include "distill.h"
#include "linear.h"

namespace {

constexpr int64_t kMaxRows = 0x7FFFFFFF;
constexpr int64_t kMaxEntries = kMaxRows - 0xFFFF;  // (the kernels add a tile's rows to an entry in 32 bits)
constexpr int32_t kMaxM = 1 << 30;
constexpr int32_t kMaxWidth = 65536;

static_assert(MORE_TEACHER_K_MAX == more::kDistillMaxTeacher, "the header's limit is the kernels'");

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

more_status from_hip(hipError_t e) { return e == hipSuccess ? MORE_OK : MORE_ERR_HIP; }

more_status check_linear(int64_t T, int32_t K, int32_t N, int32_t M, int32_t k, int32_t step) {
    if (T < 0 || K <= 0 || N <= 0 || M <= 0 || k < 1) return MORE_ERR_INVALID_ARG;
    if (K % step != 0 || N % 8 != 0 || K > kMaxWidth || N > MORE_LINEAR_N_MAX || k > MORE_K_MAX || M >= kMaxM ||
        T > kMaxEntries || T * (int64_t)k > kMaxEntries)
        return MORE_ERR_UNSUPPORTED;
    return MORE_OK;
}

// The part of a forward call that both types share.
more_status forward(more::LinearArgs a, int64_t T, int32_t y_bits, void* workspace, size_t workspace_bytes,
                    void* stream) {
    if (!a.W || !a.offsets || (T != 0 && (!a.x || !a.idx || !a.sorted || !a.y)) || (y_bits != 16 && y_bits != 32))
        return MORE_ERR_INVALID_ARG;
    if (!aligned(a.x, 16) || !aligned(a.W, 16) || !aligned(a.y, 16) || !aligned(a.idx, 4) || !aligned(a.offsets, 4) ||
        !aligned(a.sorted, 4) || !aligned(workspace, 256))
        return MORE_ERR_INVALID_ARG;
    const int32_t per = a.q8 ? 2 : 1;
    const more_status st = check_linear(T, a.len * per, a.N, a.M, a.k, 8 * per);
    if (st != MORE_OK) return st;
    if (T == 0) return MORE_OK;
    more::LinearPlan p;
    more::linear_make_plan(T, a.len, a.N, a.M, a.k, a.q8, &p);
    if (p.workspace_bytes != 0 && (!workspace || workspace_bytes < p.workspace_bytes)) return MORE_ERR_WORKSPACE;
    a.T = (int32_t)T;
    a.wide = y_bits == 32;
    a.whole = more::linear_whole(a.y, a.N * (int64_t)(y_bits / 8));
    return from_hip(more::linear_launch(p, a, workspace, static_cast<hipStream_t>(stream)));
}

more::LinearArgs linear_args(const void* x, const void* W, int32_t K, int32_t N, int32_t M, int32_t k,
                             const int32_t* idx, const int32_t* offsets, const int32_t* sorted, bool q8) {
    more::LinearArgs a = {};
    a.x = static_cast<const uint16_t*>(x);
    a.W = static_cast<const uint16_t*>(W);
    a.len = q8 ? K / 2 : K;
    a.N = N;
    a.M = M;
    a.k = k;
    a.idx = idx;
    a.offsets = offsets;
    a.sorted = sorted;
    a.q8 = q8;
    return a;
}

more_status workspace_size(int64_t T, int32_t K, int32_t N, int32_t M, int32_t k, bool q8, size_t* bytes) {
    if (!bytes) return MORE_ERR_INVALID_ARG;
    const more_status st = check_linear(T, K, N, M, k, q8 ? 16 : 8);
    if (st != MORE_OK) return st;
    more::LinearPlan p;
    more::linear_make_plan(T, q8 ? K / 2 : K, N, M, k, q8, &p);
    *bytes = T == 0 ? 0 : p.workspace_bytes;
    return MORE_OK;
}

more_status check_distill(const void* logits, int32_t bits, int64_t T, int32_t V, int64_t ld, const int32_t* ids,
                          const float* values, int32_t k, float tau, const void* dlogits, int64_t ldd) {
    if (T < 0 || V < 1 || k < 1 || (bits != 16 && bits != 32) || !isfinite(tau) || tau <= 0.0f || ld < V ||
        (dlogits && ldd < V) || (T != 0 && (!logits || !ids || !values)))
        return MORE_ERR_INVALID_ARG;
    if (!aligned(logits, bits / 8) || !aligned(dlogits, bits / 8) || !aligned(ids, 4) || !aligned(values, 4) ||
        (dlogits && dlogits == logits && ldd != ld))
        return MORE_ERR_INVALID_ARG;
    constexpr int64_t kMaxStride = (int64_t)1 << 40;
    // (beyond these tau^2 and log2(e) / tau leave fp32)
    if (tau < 0x1p-40f || tau > 0x1p40f) return MORE_ERR_UNSUPPORTED;
    if (V > 1 << 30 || k > MORE_TEACHER_K_MAX || T > kMaxRows || ld > kMaxStride || (dlogits && ldd > kMaxStride))
        return MORE_ERR_UNSUPPORTED;
    return MORE_OK;
}

more::DistillArgs distill_args(const void* logits, int32_t bits, int64_t T, int32_t V, int64_t ld, const int32_t* ids,
                               const float* values, int32_t k, float tau, const float* weight, void* dlogits,
                               int64_t ldd) {
    more::DistillArgs a = {};
    a.logits = logits;
    a.wide = bits == 32;
    a.T = (int32_t)T;
    a.V = V;
    a.k = k;
    a.ld = ld;
    a.ldd = ldd;
    a.ids = ids;
    a.values = values;
    a.weight = weight;
    a.tau = tau;
    a.dlogits = dlogits;
    return a;
}

}  // namespace

extern "C" {

more_status more_expert_linear_workspace_size(int64_t T, int32_t K, int32_t N, int32_t M, int32_t k, size_t* bytes) {
    return workspace_size(T, K, N, M, k, false, bytes);
}

more_status more_expert_linear_q8_workspace_size(int64_t T, int32_t K, int32_t N, int32_t M, int32_t k,
                                                 size_t* bytes) {
    return workspace_size(T, K, N, M, k, true, bytes);
}

more_status more_expert_linear(const uint16_t* x, const uint16_t* Wt, int64_t T, int32_t K, int32_t N, int32_t M,
                               int32_t k, const int32_t* idx, const int32_t* offsets, const int32_t* sorted, void* y,
                               int32_t y_bits, void* workspace, size_t workspace_bytes, void* stream) {
    more::LinearArgs a = linear_args(x, Wt, K, N, M, k, idx, offsets, sorted, false);
    a.y = y;
    return forward(a, T, y_bits, workspace, workspace_bytes, stream);
}

more_status more_expert_linear_q8(const int8_t* q, const float* q_scale, const int8_t* Wq, const float* w_scale,
                                  int64_t T, int32_t K, int32_t N, int32_t M, int32_t k, const int32_t* idx,
                                  const int32_t* offsets, const int32_t* sorted, const float* gate, void* y,
                                  int32_t y_bits, void* workspace, size_t workspace_bytes, void* stream) {
    if (!w_scale || (T != 0 && !q_scale) || !aligned(w_scale, 16) || !aligned(q_scale, 4) || !aligned(gate, 4))
        return MORE_ERR_INVALID_ARG;
    if (K > 0 && K % 16 != 0) return MORE_ERR_UNSUPPORTED;
    more::LinearArgs a = linear_args(q, Wq, K, N, M, k, idx, offsets, sorted, true);
    a.x_scale = q_scale;
    a.w_scale = w_scale;
    a.gate = gate;
    a.y = y;
    return forward(a, T, y_bits, workspace, workspace_bytes, stream);
}

more_status more_expert_linear_backward_workspace_size(int64_t T, int32_t K, int32_t N, int32_t M, int32_t k,
                                                       size_t* bytes) {
    if (!bytes) return MORE_ERR_INVALID_ARG;
    const more_status st = check_linear(T, K, N, M, k, 8);
    if (st != MORE_OK) return st;
    more::LinearPlan p;
    more::linear_backward_make_plan(T, K, N, M, k, &p);
    *bytes = T == 0 ? 0 : p.workspace_bytes;
    return MORE_OK;
}

more_status more_expert_linear_backward(const uint16_t* x, const uint16_t* Wt, int64_t T, int32_t K, int32_t N,
                                        int32_t M, int32_t k, const int32_t* idx, const int32_t* offsets,
                                        const int32_t* sorted, const uint16_t* dy, uint16_t* dx, uint16_t* dWt,
                                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!Wt || !offsets || (T != 0 && (!x || !idx || !sorted || !dy || (!dx && !dWt)))) return MORE_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(Wt, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(dWt, 16) ||
        !aligned(idx, 4) || !aligned(offsets, 4) || !aligned(sorted, 4) || !aligned(workspace, 256))
        return MORE_ERR_INVALID_ARG;
    const more_status st = check_linear(T, K, N, M, k, 8);
    if (st != MORE_OK) return st;
    more::LinearPlan p;
    more::linear_backward_make_plan(T, K, N, M, k, &p);
    if (T != 0 && p.workspace_bytes != 0 && (!workspace || workspace_bytes < p.workspace_bytes))
        return MORE_ERR_WORKSPACE;
    more::LinearArgs a = linear_args(x, Wt, K, N, M, k, idx, offsets, sorted, false);
    a.T = (int32_t)T;
    a.dy = dy;
    a.dx = dx;
    a.dW = dWt;
    return from_hip(more::linear_backward_launch(p, a, workspace, static_cast<hipStream_t>(stream)));
}

more_status more_expert_linear_plan(int64_t T, int32_t K, int32_t N, int32_t M, int32_t k, int32_t kind,
                                    more_linear_plan* plan) {
    if (!plan || kind < 0 || kind > 2) return MORE_ERR_INVALID_ARG;
    const more_status st = check_linear(T, K, N, M, k, kind == 2 ? 16 : 8);
    if (st != MORE_OK) return st;
    more::LinearPlan p;
    *plan = {};
    if (kind == 1) {
        more::linear_backward_make_plan(T, K, N, M, k, &p);
        plan->stages = 2;
        plan->dw_rows = p.dw_rows;
        plan->dw_cols = p.dw_cols;
        plan->dw_runs = p.dw_parts;
        plan->dw_span = p.dw_span;
    } else {
        more::linear_make_plan(T, kind == 2 ? K / 2 : K, N, M, k, kind == 2, &p);
        plan->stages = p.stages;
    }
    plan->tile_rows = p.few ? 0 : p.tiles.bm;
    plan->cols = p.few ? p.span : p.cols;
    plan->span = p.span;
    plan->listed = p.listed;
    return MORE_OK;
}

more_status more_quantize_rows(const uint16_t* x, int64_t T, int32_t width, int32_t gated, int8_t* q, float* scale,
                               void* stream) {
    if (T < 0 || width <= 0 || (T != 0 && (!x || !q || !scale))) return MORE_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 4)) return MORE_ERR_INVALID_ARG;
    if (width % 16 != 0 || width > kMaxWidth || T > kMaxRows) return MORE_ERR_UNSUPPORTED;
    if (T == 0) return MORE_OK;
    return from_hip(more::quantize_rows_launch(x, T, width, gated != 0, q, scale, static_cast<hipStream_t>(stream)));
}

more_status more_distill(const void* logits, int32_t bits, int64_t T, int32_t V, int64_t ld, const int32_t* teacher_idx,
                         const float* teacher_val, int32_t k, float tau, const float* weight, float* loss, float* m,
                         float* Z, void* dlogits, int64_t ld_dlogits, void* stream) {
    if (T != 0 && !loss && !m && !Z && !dlogits) return MORE_ERR_INVALID_ARG;
    if (!aligned(weight, 4) || !aligned(loss, 4) || !aligned(m, 4) || !aligned(Z, 4)) return MORE_ERR_INVALID_ARG;
    const more_status st =
        check_distill(logits, bits, T, V, ld, teacher_idx, teacher_val, k, tau, dlogits, ld_dlogits);
    if (st != MORE_OK || T == 0) return st;
    more::DistillArgs a =
        distill_args(logits, bits, T, V, ld, teacher_idx, teacher_val, k, tau, weight, dlogits, ld_dlogits);
    a.loss = loss;
    a.m = m;
    a.Z = Z;
    return from_hip(more::distill_launch(a, static_cast<hipStream_t>(stream)));
}

more_status more_distill_backward(const void* logits, int32_t bits, int64_t T, int32_t V, int64_t ld, const float* m,
                                  const float* Z, const int32_t* teacher_idx, const float* teacher_val, int32_t k,
                                  float tau, const float* dloss, void* dlogits, int64_t ld_dlogits, void* stream) {
    if (T != 0 && (!m || !Z || !dloss || !dlogits)) return MORE_ERR_INVALID_ARG;
    if (!aligned(dloss, 4) || !aligned(m, 4) || !aligned(Z, 4)) return MORE_ERR_INVALID_ARG;
    const more_status st =
        check_distill(logits, bits, T, V, ld, teacher_idx, teacher_val, k, tau, dlogits, ld_dlogits);
    if (st != MORE_OK || T == 0) return st;
    more::DistillArgs a =
        distill_args(logits, bits, T, V, ld, teacher_idx, teacher_val, k, tau, dloss, dlogits, ld_dlogits);
    a.m_in = m;
    a.Z_in = Z;
    return from_hip(more::distill_launch(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
