// What the translation units of rcd_orthogonalize share.
#pragma once

#include "rcd_elem.cuh"
#include "rcd_linear.h"

namespace rcd {

constexpr int kUp = 10;                    // X, A and B are held times 2^kUp
constexpr int kMostSteps = 64;

// All steps in one launch (rcd_orthogonal_fused.cu): the phases of a step.
struct FusedPhase {
    int32_t M, N, slabs, team, per;        // team: CTAs that share a tile, 1, 2 or 4; per: slabs of a piece
    int32_t stepA, stepB;                  // rows of an operand from matrix to matrix
    int32_t tilesN, tiles;                 // of a matrix
    bool acrossA, acrossB, symmetric;
};
constexpr int kFusedUnits = 8;             // tiles per CTA and phase at most
struct FusedPlan { bool possible; int32_t grid, cluster; double stepUs; FusedPhase phases[3]; };        // stepUs: an estimate
struct FusedParams {
    __half *x0, *x1, *a, *b;               // [batch][rows][cols] twice, [batch][side][side] twice; whole 64s
    const __half *low;                     // what x0 lacks of an fp32 G, times 2^kLowUp, or null
    const float *factor;                   // [batch], of the first step
    uint32_t *counter;                     // zero
    __nv_bfloat16 *o;
    int64_t ldO, stepO;
    int32_t rowsO, colsO;                  // of the output
    int32_t rows, cols, side, batch, steps, cluster;
    bool tall;
    FusedPhase phases[3];
    int32_t *status;
    float coefficients[3 * kMostSteps];
};
FusedPlan fused_plan(rcd_ctx *ctx, int64_t batch, int64_t rows, int64_t cols, bool tall);
rcd_status launch_fused(rcd_ctx *ctx, const FusedParams &p, const FusedPlan &plan, cudaStream_t st);

// A cluster per matrix (rcd_orthogonal_cluster.cu): of how many CTAs, 0 where it does not take the size; no workspace.
int cluster_for(rcd_ctx *ctx, int64_t rows, int64_t cols);
rcd_status launch_cluster(rcd_ctx *ctx, const rcd_orthogonalize_args &a, int cluster, cudaStream_t st);

}  // namespace rcd
