"""MoRE low-rank mixture-of-experts router for AMD Instinct MI355X (gfx950).

The compute lives in libmore.so (HIP kernels behind the C ABI declared in include/more.h).
This package holds the library, its build script (`python -m paper_2609_36301_amd.build`),
ctypes bindings with torch tensors (`router`; `layer` for the experts, norms and gradient clipping
around it; `linear` for the experts' linear maps in bf16 and 8-bit integers; `distill` for learning from a
teacher's top logits), and the seeded input generator (`inputs`).

    from paper_2609_36301_amd import route_lowrank
    out = route_lowrank(x, R1t, R2t, k)      # out.idx [T][k] int32, out.gate [T][k] fp32
    tr = route_lowrank_train(x, R1t, R2t, k) # + tr.m, tr.Z [T], tr.psum [M] fp32
    gr = route_lowrank_backward(x, R1t, R2t, tr.idx, dtop, pbar, tr.m, tr.Z)  # gr.dx, gr.dR1t, gr.dR2t
    y = expert_ffn(x, W1t, W2t, out.idx, *dispatch_sort(out.idx, M), out.gate)  # [T k][h] bf16
    y = expert_linear(x, Wt, out.idx, *dispatch_sort(out.idx, M))                # [T k][N] bf16
    end = block_norm(r, y, w_after=w1, w_before=w2)                             # end.r, end.xn
"""
__all__ = ["route_lowrank", "route_lowrank_train", "route_fullrank", "route_fullrank_fused",
           "expert_histogram",
           "dispatch_sort", "LowrankRouter", "LowrankTrainRouter", "lowrank_workspace_size",
           "lowrank_train_workspace_size", "route_lowrank_backward", "LowrankBackward",
           "lowrank_backward_workspace_size", "Gradients", "lowrank_plan", "lowrank_route",
           "fullrank_workspace_size", "Routing", "TrainRouting"]
_LAYER = ["expert_ffn", "expert_ffn_backward", "ExpertFFN", "ExpertFFNBackward", "ExpertGradients",
          "expert_ffn_workspace_size", "expert_ffn_backward_workspace_size", "expert_ffn_plan", "block_norm",
          "block_norm_backward", "BlockNorm", "BlockNormBackward", "BlockEnd", "BlockEndGradients",
          "block_norm_backward_workspace_size", "clip_gradients", "GradClipper"]
_LINEAR = ["expert_linear", "expert_linear_backward", "expert_linear_q8", "quantize_rows", "ExpertLinear",
           "ExpertLinearBackward", "ExpertLinearQ8", "QuantizeRows", "QuantizedRows", "LinearGradients",
           "expert_linear_workspace_size", "expert_linear_backward_workspace_size",
           "expert_linear_q8_workspace_size", "expert_linear_plan"]
_DISTILL = ["distill_loss", "distill_backward", "Distill", "DistillBackward", "Distillation"]
__all__ += _LAYER + _LINEAR + _DISTILL


def __getattr__(name):
    if name in _LAYER:
        from . import layer
        return getattr(layer, name)
    if name in _LINEAR:
        from . import linear
        return getattr(linear, name)
    if name in _DISTILL:
        from . import distill
        return getattr(distill, name)
    if name in __all__:
        from . import router
        return getattr(router, name)
    raise AttributeError(name)
