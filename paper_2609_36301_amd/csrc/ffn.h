// Plans and launch entry points of the experts' gated feed-forward block (ffn.hip, ffn_backward.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace more {

struct FfnArgs {
    const uint16_t* x;       // [T][h]
    const uint16_t* W1t;     // [M][2s][h], gate rows then up rows
    const uint16_t* W2t;     // [M][h][s]
    int32_t T, h, s, M, k;
    const int32_t* idx;      // [T][k]
    const int32_t* offsets;  // [M + 1]
    const int32_t* sorted;   // [T k]
    const float* gate;       // [T][k] or NULL (all ones)
    // backward
    const uint16_t* du;      // [T][h]
    uint16_t* dx;            // [T][h]
    uint16_t* dW1t;          // [M][2s][h]
    uint16_t* dW2t;          // [M][h][s]
    float* dgate;            // [T][k] or NULL
    int32_t planes;          // of what the kernels hand on in bf16 (FfnPlan::planes)
};

struct FfnPlan {
    int64_t n;        // T k entries
    int32_t bm;       // rows of a tile (all of one expert)
    int32_t few;      // (forward) the kernels without tiles
    int32_t split;    // (forward, without tiles) the waves of a down workgroup share columns
    int32_t stages;   // (forward, tiles) of the down kernel's ring
    int32_t span;     // columns of y (backward: of the shares of dx) that a workgroup takes
    int32_t da0_span; // (backward, tiles of 256 rows) columns of dA0 that a workgroup takes
    // The hidden units (and, backward, the gradients of the pre-activations) go from kernel to kernel in bf16,
    // the matrix cores' operand type: one rounding each (planes = 1), which sits in all its products and makes the
    // results' error 1.41 times that of their own rounding, on average over many; or a sum of two bf16
    // (planes = 2; [planes][n][s] and [planes][n][2s]), which leaves the results' own rounding alone and doubles
    // the operations of the products that read them.  Two where the caller asks for them, in the kernels without
    // tiles, and for n s <= 2^15, where the errors of few roundings do not average out (at 512 values the factor
    // scatters by 10%) and two cost a few us.  us, one : two, forward and backward: 600 experts of h = 2048, s = 64
    // with one row 58 : 68 and 205 : 232; a dense block of h = 4096, s = 128, 300 rows 41 : 43 and 110 : 119; and
    // far above, 4096 experts of h = 512, s = 64 with 32 rows 226 : 248 and 660 : 784; 32 experts of h = 2048,
    // s = 1024 with 1024 rows 473 : 594 and 1435 : 2498 (on tiles of 128 rows).
    int32_t planes;
    int64_t tiles;    // bound on the number of tiles
    int32_t sums;     // workgroups that count tiles ahead of the list (0: none)
    int32_t dw_tile;  // rows and columns of a tile of the weight gradients (128 or 256)
    int32_t dw_parts; // parts of an expert's entries whose weight gradients are summed apart
    int32_t dw1_span, dw2_span;  // of h that a workgroup of dW1t and of dW2t takes
    size_t off_tiles, off_sums, off_hidden, off_dgu, off_da0, off_dxs, off_dgp, off_dwp;
    size_t workspace_bytes;
};

// addends: 2 for two planes at every size, 0 for the rule beside FfnPlan::planes
void ffn_make_plan(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends, FfnPlan* p);
void ffn_backward_make_plan(int64_t T, int32_t h, int32_t s, int32_t M, int32_t k, int32_t addends, FfnPlan* p);
hipError_t ffn_launch(const FfnPlan& p, FfnArgs a, uint16_t* y, void* workspace, hipStream_t stream);
hipError_t ffn_backward_launch(const FfnPlan& p, FfnArgs a, void* workspace, hipStream_t stream);

// Columns that a workgroup takes, in steps of `step`, of a product whose contraction is `len` long: a
// single step where the contraction alone fills the pipeline (eight stages), or where the groups of rows are
// too few to fill the chip four times over with more; else up to 512.  us, forward and backward, single step :
// up to 512 (experts chosen evenly, as for all rules here; with popularities that fall off as in a trained router
// the first shape takes 226 + 660): 4096 experts of h = 512, s = 64, 32 rows 256 + 680 : 215 + 621; 128 experts of h = 2048, s = 320,
// 256 rows 276 + 886 : 264 + 844; 200 experts of h = 528, s = 72, 9 rows 24 + 61 : 26 + 74.
inline int32_t ffn_span(int32_t len, int32_t step, int64_t groups, int32_t cols) {
    return len > 512 || groups * ((cols + 511) / 512) < 1024 ? step : 512;
}

// What `items` workgroups with tiles of `bm` rows cost that run `steps` stages each: the rounds in which they
// fill the chip (two of up to 128 rows to a CU, one of 256) times the stages times the time of a stage.  The
// stages' times were fitted to 196 measured shapes: against one of 128-row tiles, two to a CU, 0.8 with one to
// a CU, 0.75 with 64 rows (half the work) and 1.6 with 256 (four times the work, one to a CU).
inline int64_t ffn_cost(int64_t items, int64_t steps, int32_t bm) {
    const int64_t slots = bm == 256 ? 256 : 512;
    const int64_t stage = bm == 256 ? 32 : bm == 128 ? (items <= 256 ? 16 : 20) : 15;
    return (items + slots - 1) / slots * steps * stage;
}
constexpr int64_t kFfnTwoPlanes = 1 << 15;

// Twice the expected number of tiles of n entries over M experts whose rows scatter by their mean's root.
int64_t ffn_expected_tiles2(int64_t n, int32_t M, int32_t bm);

// The part of a plan that concerns the tile list.
void ffn_tiles_plan(int64_t n, int32_t M, int32_t bm, FfnPlan* p);

// Lists the tiles (shared by both directions).
hipError_t ffn_tiles_launch(const FfnPlan& p, const FfnArgs& a, void* workspace, hipStream_t stream);

}  // namespace more
