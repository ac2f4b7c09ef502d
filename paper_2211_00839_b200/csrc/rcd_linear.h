// What the translation units of rcd_linear and rcd_linear_backward share.
#pragma once

#include <type_traits>

#include "rcd_elem.cuh"

namespace rcd {

#define RCD_TRY(call) do { const rcd_status rs__ = (call); if (rs__ != RCD_OK) return rs__; } while (0)

// What is done with an accumulator on its way out: z = acc [* xs[m] * ws[n]] + bias[n], y = act(z) + residual.
struct Epilogue {
    const float *xs, *ws, *bias;
    const void *residual;
    void *y, *z;
    int64_t ldr, ldy, ldz;
    rcd_elem type;                         // of y, residual and z
    int32_t act;
};

// C[m][n] = sum over k of A(m, k) B(n, k).  An operand has its k elements next to each other (rows lie `ld` apart), or, with
// `across`, its m or n elements (and steps of k are `ld` apart).
struct Operand { const void *p; int64_t ld; bool across; };
struct Product {
    rcd_elem type;
    int64_t M, N, K;
    Operand a, b;
    Epilogue out;
};

size_t product_workspace(rcd_ctx *ctx, const Product &p);
rcd_status launch_product(rcd_ctx *ctx, const Product &p, void *workspace, cudaStream_t st);

// The product of few rows (rcd_linear_few.cu; no workspace), and whether it takes one.
bool few_rows(const Product &p);
rcd_status launch_few_rows(rcd_ctx *ctx, const Product &p, cudaStream_t st);

// out[c] = sum over the rows of partial[rows][d], in a fixed order
rcd_status launch_column_sums(rcd_ctx *ctx, const float *partial, int64_t rows, int64_t d, float *out, cudaStream_t st);

// Counters of a call's launches, and the word that rcd_sync_status asks for.
inline void begin_operator(rcd_ctx *ctx)
{
    ctx->kernelLaunches = 0;
    ctx->tcLaunches = 0;
    ctx->statusDev = ctx->statusOwn + kOperatorStatus;
}

rcd_status check_rows(rcd_ctx *ctx, const char *name, const void *p, int64_t rows, int64_t ld, int64_t len, rcd_elem type);

}  // namespace rcd
