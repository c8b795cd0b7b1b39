// Plans and launch entry points of the experts' linear maps (linear.hip, linear_backward.hip) and of the
// quantisation of rows (quantize.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ffn.h"

namespace more {

// Rows of x and W are `len` words of 16 bits long: bf16 values, or pairs of int8 (q8).
struct LinearArgs {
    const uint16_t* x;       // [T][len]
    const uint16_t* W;       // [M][N][len]
    int32_t T, len, N, M, k;
    const int32_t* idx;      // [T][k]
    const int32_t* offsets;  // [M + 1]
    const int32_t* sorted;   // [T k]
    int32_t q8, wide;        // int8 operands; y in fp32
    int32_t whole;           // rows of the result (y; dx or its shares) are whole lines of 128 bytes
    const float* x_scale;    // (q8) [T]
    const float* w_scale;    // (q8) [M][N]
    const float* gate;       // (q8) [T][k] or NULL
    void* y;                 // [T k][N]
    // backward (bf16)
    const uint16_t* dy;      // [T k][N]
    uint16_t* dx;            // [T][len]
    uint16_t* dW;            // [M][N][len]
};

struct LinearPlan {
    FfnPlan tiles;    // the tile list: n, bm, tiles, sums and their places
    int32_t listed;   // the tiles are listed by a launch of their own
    int32_t few;      // (forward) the kernels without tiles
    int32_t split;    // (forward, without tiles) the waves of a workgroup share its columns
    int32_t cols;     // columns of a step
    int32_t stages;   // (forward, tiles) of the LDS ring
    int32_t span;     // columns that a workgroup takes
    int32_t stream;   // (q8, tiles of 256 rows) the pipeline runs on from tile to tile
    int32_t both;              // (backward) one launch makes both gradients
    int32_t dw_rows, dw_cols;  // rows and columns of a tile of dW
    int32_t dw_by_rows;        // a workgroup's tiles lie along N, not K
    int32_t dw_parts;          // runs of an expert's entries that are summed apart
    int32_t dw_span;           // of that side that a workgroup takes
    size_t off_shares, off_parts;
    size_t workspace_bytes;
};

// Whether rows of `bytes` bytes from p on are whole lines.
inline int32_t linear_whole(const void* p, int64_t bytes) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)bytes) & 127) == 0;
}

void linear_make_plan(int64_t T, int32_t len, int32_t N, int32_t M, int32_t k, bool q8, LinearPlan* p);
void linear_backward_make_plan(int64_t T, int32_t len, int32_t N, int32_t M, int32_t k, LinearPlan* p);
hipError_t linear_launch(const LinearPlan& p, const LinearArgs& a, void* workspace, hipStream_t stream);
hipError_t linear_backward_launch(const LinearPlan& p, LinearArgs a, void* workspace, hipStream_t stream);

// The product in 8-bit integers on tiles of 256 rows and 256 columns whose contraction has at least kStreamSteps
// stages (linear_stream.hip), after the tile list.
constexpr int32_t kStreamSteps = 5;
hipError_t linear_stream_launch(const LinearPlan& p, const LinearArgs& a, char* ws, hipStream_t stream);

// Columns (rows of dW) that a workgroup takes, in steps of `step`, of a product whose contraction is `len` long over `groups`
// groups of rows.
int32_t linear_span(int64_t len, int32_t step, int64_t groups, int32_t side);

// Whether the tiles of a plan are listed by a launch of their own; else each workgroup finds its tile from the offsets, of
// at most kLinearOwn experts.
constexpr int32_t kLinearOwn = 1024;
bool linear_listed(const FfnPlan& tiles, int32_t M, int64_t spans);

// Lists the tiles of a plan.
hipError_t linear_tiles_launch(const LinearPlan& p, const LinearArgs& a, void* workspace, hipStream_t stream);

// Rows of a tile (32 to 256) of a product of n entries over M experts, `cols` columns (in steps of `cols_of`, of 256 with
// tiles of 256 rows) and `steps` stages.
// (kProductSplit: a map whose stages of a row touch two lines)
enum LinearProduct { kProductMap, kProductSplit, kProductDx, kProductQ8 };
int32_t linear_tile_rows(int64_t n, int32_t M, int32_t cols, int32_t cols_of, int64_t steps, LinearProduct product);

// q [T][width] int8 and scale [T] of the rows of x: bf16 [T][width], or (gated) [T][2 width].
hipError_t quantize_rows_launch(const uint16_t* x, int64_t T, int32_t width, bool gated, int8_t* q, float* scale,
                                hipStream_t stream);

}  // namespace more
