// C ABI of the layer around the router: argument validation and launch (more.h).  Every check runs on
// the host before anything is enqueued, so an error status means the stream was not touched.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "more.h"
#include "ffn.h"
#include "layer.h"

namespace {

constexpr int64_t kMaxEntries = 0x7FFFFFFF;
constexpr int64_t kMaxFfnEntries = kMaxEntries - 0xFFFF;  // (the kernels add a tile's rows to an entry in 32 bits)
constexpr int32_t kMaxM = 1 << 30;
constexpr int32_t kMaxWidth = 65536;

static_assert(MORE_NORM_H_MAX == more::kNormMaxH, "the header's limit is the kernels'");

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

more_status from_hip(hipError_t e) { return e == hipSuccess ? MORE_OK : MORE_ERR_HIP; }

more_status check_ffn(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends) {
    if (T < 0 || h <= 0 || s <= 0 || M <= 0 || k < 1 || (addends != 0 && addends != 2)) return MORE_ERR_INVALID_ARG;
    if (h % 16 != 0 || s % 8 != 0 || h > kMaxWidth || s > kMaxWidth || k > MORE_K_MAX || M >= kMaxM ||
        T > kMaxFfnEntries || T * (int64_t)k > kMaxFfnEntries)
        return MORE_ERR_UNSUPPORTED;
    return MORE_OK;
}

more_status check_norm(int64_t T, int32_t h, int32_t resid_bits, float alpha, float eps) {
    if (T < 0 || h <= 0 || (resid_bits != 16 && resid_bits != 32) || !isfinite(alpha) || !isfinite(eps) ||
        eps <= 0.0f)
        return MORE_ERR_INVALID_ARG;
    if (h % 16 != 0 || h > MORE_NORM_H_MAX || T > kMaxEntries) return MORE_ERR_UNSUPPORTED;
    return MORE_OK;
}

more::FfnArgs ffn_args(const uint16_t* x, const uint16_t* W1t, const uint16_t* W2t, int64_t T, int32_t h,
                       int32_t s, int32_t M, int32_t k, const int32_t* idx, const int32_t* offsets,
                       const int32_t* sorted, const float* gate) {
    more::FfnArgs a = {};
    a.x = x;
    a.W1t = W1t;
    a.W2t = W2t;
    a.T = (int32_t)T;
    a.h = h;
    a.s = s;
    a.M = M;
    a.k = k;
    a.idx = idx;
    a.offsets = offsets;
    a.sorted = sorted;
    a.gate = gate;
    return a;
}

}  // namespace

extern "C" {

more_status more_expert_ffn_workspace_size_ex(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends,
                                              size_t* bytes) {
    if (!bytes) return MORE_ERR_INVALID_ARG;
    more_status st = check_ffn(T, h, s, M, k, addends);
    if (st != MORE_OK) return st;
    more::FfnPlan p;
    more::ffn_make_plan(T, h, s, M, k, addends, &p);
    *bytes = T == 0 ? 0 : p.workspace_bytes;
    return MORE_OK;
}

more_status more_expert_ffn_workspace_size(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, size_t* bytes) {
    return more_expert_ffn_workspace_size_ex(T, h, s, M, k, 0, bytes);
}

more_status more_expert_ffn_ex(const uint16_t* x, const uint16_t* W1t, const uint16_t* W2t, int64_t T, int32_t h,
                               int32_t s, int32_t M, int32_t k, int32_t addends, const int32_t* idx,
                               const int32_t* offsets, const int32_t* sorted, const float* gate, uint16_t* y,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (!W1t || !W2t || !offsets || (T != 0 && (!x || !idx || !sorted || !y))) return MORE_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(W1t, 16) || !aligned(W2t, 16) || !aligned(y, 16) || !aligned(idx, 4) ||
        !aligned(offsets, 4) || !aligned(sorted, 4) || !aligned(gate, 4) || !aligned(workspace, 256))
        return MORE_ERR_INVALID_ARG;
    more_status st = check_ffn(T, h, s, M, k, addends);
    if (st != MORE_OK) return st;
    if (T == 0) return MORE_OK;
    more::FfnPlan p;
    more::ffn_make_plan(T, h, s, M, k, addends, &p);
    if (!workspace || workspace_bytes < p.workspace_bytes) return MORE_ERR_WORKSPACE;
    return from_hip(more::ffn_launch(p, ffn_args(x, W1t, W2t, T, h, s, M, k, idx, offsets, sorted, gate), y, workspace,
                                     static_cast<hipStream_t>(stream)));
}

more_status more_expert_ffn(const uint16_t* x, const uint16_t* W1t, const uint16_t* W2t, int64_t T, int32_t h,
                            int32_t s, int32_t M, int32_t k, const int32_t* idx, const int32_t* offsets,
                            const int32_t* sorted, const float* gate, uint16_t* y, void* workspace,
                            size_t workspace_bytes, void* stream) {
    return more_expert_ffn_ex(x, W1t, W2t, T, h, s, M, k, 0, idx, offsets, sorted, gate, y, workspace, workspace_bytes,
                              stream);
}

more_status more_expert_ffn_plan(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends,
                                 int32_t backward, more_expert_plan* plan) {
    if (!plan) return MORE_ERR_INVALID_ARG;
    more_status st = check_ffn(T, h, s, M, k, addends);
    if (st != MORE_OK) return st;
    more::FfnPlan p;
    *plan = {};
    if (backward) {
        more::ffn_backward_make_plan(T, h, s, M, k, addends, &p);
        plan->tile_rows = p.bm;
        plan->stages = 2;
        plan->dw_tile = p.dw_tile;
        plan->dw_runs = p.dw_parts;
        plan->dw1_span = p.dw1_span;
        plan->dw2_span = p.dw2_span;
    } else {
        more::ffn_make_plan(T, h, s, M, k, addends, &p);
        plan->tile_rows = p.few ? 0 : p.bm;
        plan->stages = p.stages;
    }
    plan->addends = p.planes;
    plan->span = p.span;
    return MORE_OK;
}

more_status more_expert_ffn_backward_workspace_size_ex(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k,
                                                       int32_t addends, size_t* bytes) {
    if (!bytes) return MORE_ERR_INVALID_ARG;
    more_status st = check_ffn(T, h, s, M, k, addends);
    if (st != MORE_OK) return st;
    more::FfnPlan p;
    more::ffn_backward_make_plan(T, h, s, M, k, addends, &p);
    *bytes = T == 0 ? 0 : p.workspace_bytes;
    return MORE_OK;
}

more_status more_expert_ffn_backward_workspace_size(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k,
                                                    size_t* bytes) {
    return more_expert_ffn_backward_workspace_size_ex(T, h, s, M, k, 0, bytes);
}

more_status more_expert_ffn_backward_ex(const uint16_t* x, const uint16_t* W1t, const uint16_t* W2t, int64_t T,
                                        int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends, const int32_t* idx,
                                        const int32_t* offsets, const int32_t* sorted, const float* gate,
                                        const uint16_t* du, uint16_t* dx, uint16_t* dW1t, uint16_t* dW2t, float* dgate,
                                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!W1t || !W2t || !offsets || !dW1t || !dW2t || (T != 0 && (!x || !idx || !sorted || !du || !dx)) ||
        (dgate && !gate))
        return MORE_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(W1t, 16) || !aligned(W2t, 16) || !aligned(du, 16) || !aligned(dx, 16) ||
        !aligned(dW1t, 16) || !aligned(dW2t, 16) || !aligned(idx, 4) || !aligned(offsets, 4) || !aligned(sorted, 4) ||
        !aligned(gate, 4) || !aligned(dgate, 4) || !aligned(workspace, 256))
        return MORE_ERR_INVALID_ARG;
    more_status st = check_ffn(T, h, s, M, k, addends);
    if (st != MORE_OK) return st;
    more::FfnPlan p;
    more::ffn_backward_make_plan(T, h, s, M, k, addends, &p);
    if (T != 0 && (!workspace || workspace_bytes < p.workspace_bytes)) return MORE_ERR_WORKSPACE;
    more::FfnArgs a = ffn_args(x, W1t, W2t, T, h, s, M, k, idx, offsets, sorted, gate);
    a.du = du;
    a.dx = dx;
    a.dW1t = dW1t;
    a.dW2t = dW2t;
    a.dgate = dgate;
    return from_hip(more::ffn_backward_launch(p, a, workspace, static_cast<hipStream_t>(stream)));
}

more_status more_expert_ffn_backward(const uint16_t* x, const uint16_t* W1t, const uint16_t* W2t, int64_t T, int32_t h,
                                     int32_t s, int32_t M, int32_t k, const int32_t* idx, const int32_t* offsets,
                                     const int32_t* sorted, const float* gate, const uint16_t* du, uint16_t* dx,
                                     uint16_t* dW1t, uint16_t* dW2t, float* dgate, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    return more_expert_ffn_backward_ex(x, W1t, W2t, T, h, s, M, k, 0, idx, offsets, sorted, gate, du, dx, dW1t, dW2t,
                                       dgate, workspace, workspace_bytes, stream);
}

more_status more_block_norm(const void* r, int32_t resid_bits, const uint16_t* y, int64_t T, int32_t h, int32_t k,
                            const float* w_after, const float* w_before, const float* gate, float alpha, float eps,
                            int32_t norm_after, void* r_out, uint16_t* u, uint16_t* xn, void* stream) {
    if (k < 0 || (k == 0 && (y || w_after || gate || r_out || u || !w_before))) return MORE_ERR_INVALID_ARG;
    // the token-sized buffers of an empty batch may be NULL (an empty tensor has no storage)
    if (T != 0 && (!r || (k > 0 && (!y || !r_out)) || (xn == nullptr) != (w_before == nullptr)))
        return MORE_ERR_INVALID_ARG;
    if (!aligned(r, 16) || !aligned(y, 16) || !aligned(w_after, 16) || !aligned(w_before, 16) || !aligned(gate, 4) ||
        !aligned(r_out, 16) || !aligned(u, 16) || !aligned(xn, 16))
        return MORE_ERR_INVALID_ARG;
    more_status st = check_norm(T, h, resid_bits, alpha, eps);
    if (st != MORE_OK) return st;
    if (k > 65536 || T * (int64_t)k > kMaxEntries) return MORE_ERR_UNSUPPORTED;
    if (T == 0) return MORE_OK;
    more::NormArgs a = {};
    a.r = r;
    a.wide = resid_bits == 32;
    a.y = y;
    a.T = (int32_t)T;
    a.h = h;
    a.k = k;
    a.w_after = w_after;
    a.w_before = w_before;
    a.gate = gate;
    a.alpha = alpha;
    a.eps = eps;
    a.norm_after = norm_after != 0;
    a.r_out = r_out;
    a.u = u;
    a.xn = xn;
    return from_hip(more::block_norm_launch(a, static_cast<hipStream_t>(stream)));
}

more_status more_block_norm_backward_workspace_size(int64_t T, int32_t h, size_t* bytes) {
    if (!bytes) return MORE_ERR_INVALID_ARG;
    more_status st = check_norm(T, h, 16, 1.0f, 1.0f);
    if (st != MORE_OK) return st;
    *bytes = more::block_norm_backward_workspace(T, h);
    return MORE_OK;
}

more_status more_block_norm_backward(const uint16_t* u, const void* r_out, int32_t resid_bits, const void* dr_out,
                                     const uint16_t* dxn, const float* dxn32, int64_t T, int32_t h,
                                     const float* w_after, const float* w_before, const float* gate, float alpha,
                                     float eps, int32_t norm_after, void* dr, uint16_t* du, float* dw_after,
                                     float* dw_before, float* dgate, void* workspace, size_t workspace_bytes,
                                     void* stream) {
    if ((dw_before && !w_before) || (dgate && !gate)) return MORE_ERR_INVALID_ARG;
    if (T != 0) {
        if (!r_out || !dr || (!dr_out && !dxn && !dxn32) || (w_before != nullptr) != (dxn || dxn32) ||
            (u ? !du : (w_after || gate || du || dw_after)))
            return MORE_ERR_INVALID_ARG;
    }
    if (!aligned(u, 16) || !aligned(r_out, 16) || !aligned(dr_out, 16) || !aligned(dxn, 16) || !aligned(dxn32, 16) ||
        !aligned(w_after, 16) || !aligned(w_before, 16) || !aligned(gate, 4) || !aligned(dr, 16) || !aligned(du, 16) ||
        !aligned(dw_after, 4) || !aligned(dw_before, 4) || !aligned(dgate, 4) || !aligned(workspace, 16))
        return MORE_ERR_INVALID_ARG;
    more_status st = check_norm(T, h, resid_bits, alpha, eps);
    if (st != MORE_OK) return st;
    if (T != 0 && (!workspace || workspace_bytes < more::block_norm_backward_workspace(T, h)))
        return MORE_ERR_WORKSPACE;
    more::NormArgs a = {};
    a.r = r_out;
    a.wide = resid_bits == 32;
    a.T = (int32_t)T;
    a.h = h;
    a.w_after = w_after;
    a.w_before = w_before;
    a.gate = gate;
    a.alpha = alpha;
    a.eps = eps;
    a.norm_after = norm_after != 0;
    a.ub = u;
    a.dr_out = dr_out;
    a.dxn = dxn;
    a.dxn32 = dxn32;
    a.dr = dr;
    a.du = du;
    a.dw_after = dw_after;
    a.dw_before = dw_before;
    a.dgate = dgate;
    return from_hip(more::block_norm_backward_launch(a, workspace, static_cast<hipStream_t>(stream)));
}

more_status more_grad_clip_workspace_size(const int64_t* numel, int32_t n, size_t* bytes) {
    if (!bytes || n < 0 || (n > 0 && !numel)) return MORE_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] < 0) return MORE_ERR_INVALID_ARG;
        if (numel[i] > (int64_t)1 << 40) return MORE_ERR_UNSUPPORTED;
    }
    *bytes = more::grad_clip_workspace(numel, n);
    return MORE_OK;
}

more_status more_grad_clip(const void* const* in, void* const* out, const int64_t* numel, const int32_t* bits,
                           int32_t n, float max_norm, float eps, float* norm, void* workspace, size_t workspace_bytes,
                           void* stream) {
    size_t need = 0;
    more_status st = more_grad_clip_workspace_size(numel, n, &need);
    if (st != MORE_OK) return st;
    if ((n > 0 && (!in || !out || !bits)) || !isfinite(max_norm) || max_norm < 0.0f || !isfinite(eps) || eps <= 0.0f ||
        !aligned(norm, 4) || !aligned(workspace, 16))
        return MORE_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n; ++i) {
        if (bits[i] != 16 && bits[i] != 32) return MORE_ERR_INVALID_ARG;
        if (numel[i] > 0 && (!in[i] || !out[i] || !aligned(in[i], bits[i] / 8) || !aligned(out[i], bits[i] / 8)))
            return MORE_ERR_INVALID_ARG;
    }
    if (!workspace || workspace_bytes < need) return MORE_ERR_WORKSPACE;
    return from_hip(more::grad_clip_launch(in, out, numel, bits, n, max_norm, eps, norm, workspace,
                                           static_cast<hipStream_t>(stream)));
}

}  // extern "C"
