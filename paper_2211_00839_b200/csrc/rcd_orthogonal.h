// What the translation units of rcd_orthogonalize share.
#pragma once

#include "rcd_elem.cuh"
#include "rcd_linear.h"

namespace rcd {

constexpr int kUp = 10;                    // X, A and B are held times 2^kUp
constexpr int kMostSteps = 64;

// All steps in one launch (rcd_orthogonal_fused.cu).
struct FusedParams {
    __half *x0, *x1, *a, *b;               // [batch][rows][cols] twice, [batch][side][side] twice; whole 64s
    const float *factor;                   // [batch], of the first step
    float *parts;                          // sums of pieces: [tile][piece][128][64]
    uint32_t *counters;                    // kFusedCounters zeros
    __nv_bfloat16 *o;
    int64_t ldO, stepO;
    int32_t rowsO, colsO;                  // of the output
    int32_t rows, cols, side, batch, steps;
    bool tall;
    int32_t splits[3];                     // pieces of the k axis of a step's products
    int32_t *status;
    float coefficients[3 * kMostSteps];
};
constexpr int kFusedTile = 128 * 64 * 4;
constexpr int kFusedTileCounters = 256, kFusedCounters = 1 + 3 * kFusedTileCounters;
struct FusedPlan { bool use; int32_t grid, splits[3]; size_t parts; };
FusedPlan fused_plan(const rcd_ctx *ctx, int64_t batch, int64_t rows, int64_t cols);
rcd_status launch_fused(rcd_ctx *ctx, const FusedParams &p, const FusedPlan &plan, cudaStream_t st);

}  // namespace rcd
