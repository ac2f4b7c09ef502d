// What the translation units of rcd_linear and rcd_linear_backward share.
#pragma once

#include <type_traits>

#include "rcd_elem.cuh"

namespace rcd {

#define RCD_TRY(call) do { const rcd_status rs__ = (call); if (rs__ != RCD_OK) return rs__; } while (0)

// How a product ends.  kPlain: rcd_linear's epilogue, or partial sums as they are.  kLoss: every row's logits of a tile to a
// reference and a sum of exponentials; nothing else leaves the SM.  kLogitGrads: logits to their gradients (kOneTile: where a tile has all classes, Product::oneTile).  kScaled: alpha times the product
// plus beta times the residual, symmetric ones from their lower half; a batch of matrices.  kScaledLow: the same (Product says kScaled) where the residual has a second part: a kernel
// of its own, since those instructions in all of kScaled's cost every product 0.5 us (8 updates of 1024 x 2048 454 -> 467 us).
enum Form { kPlain, kLoss, kLogitGrads, kScaled, kScaledLow, kOneTile };

// What is done with an accumulator on its way out: z = acc [* xs[m] * ws[n]] + bias[n], y = act(z) + residual.
struct Epilogue {
    const float *xs, *ws, *bias;
    const void *residual;
    void *y, *z;
    int64_t ldr, ldy, ldz;
    rcd_elem type;                         // of y, residual and z
    int32_t act;
};

// The head whose logits a product makes (rcd_head.cu).
struct Head {
    const int32_t *labels;                 // [rows]
    int32_t classes, firstClass;           // of all pieces; the class that column 0 is
    float2 *parts;                         // out [2 tile columns][rows]: reference and sum of exponentials of half a tile's columns
    float *picked;                         // out [rows]: the label's logit
    float *loss, *lseOut;                  // out [rows] (lseOut may be null), in place of parts and picked: where one tile takes all classes
    const float *lse, *dloss, *dlse;       // [rows]; null: ones, zeros
    const float *up;                       // a power of two that the gradients are multiplied by; null: 1
    float *sums;                           // out [32-row groups][n], or null: columns of the gradients, not multiplied by it
};
// alpha * factor^alphaPower times the product plus beta * factor^betaPower times the residual; powers from 0 to 2.
struct Scaling {
    float alpha, beta;
    const float *factor;                   // one for every matrix of the batch, or null: 1
    int32_t alphaPower, betaPower;
    rcd_elem residualType;
    const void *low;                       // fp16, laid out as the residual, or null: what that lacks, times 2^kLowUp
};
constexpr int kLowUp = 11;                 // (half a step of fp16 at most of the residual's entries: as large as they are, then)

// C[m][n] = sum over k of A(m, k) B(n, k).  An operand has its k elements next to each other (rows lie `ld` apart), or, with
// `across`, its m or n elements (and steps of k are `ld` apart).
struct Operand { const void *p; int64_t ld; bool across; };
struct Product {
    rcd_elem type;
    int64_t M, N, K;
    Operand a, b;
    Epilogue out;
    Form form;                             // kPlain where nothing is said
    Head head;
    Scaling scaling;
    bool oneTile;                          // kLogitGrads: the N columns are all classes and go into one tile
    bool symmetric;                        // kScaled: the output is, and M is N; both halves of it are written
    int64_t batch;                         // kScaled: matrices (0: one), whose rows lie below one another, in every argument this many apart:
    int64_t aStep, bStep, yStep, rStep;
};
struct KernelChoice { const void *kernel; int bit; };          // bit: of rcd_ctx::productReady
KernelChoice head_kernel(Form form, bool oneTile, int wide, bool pair);
KernelChoice scaled_kernel(int order, int wide, bool pair, bool low);
constexpr int kPlainKernels = 20, kHeadKernels = 8, kScaledKernels = 18, kScaledLowKernels = 8;    // (and 4 of kOneTile)

size_t product_workspace(rcd_ctx *ctx, const Product &p);
int64_t product_tile_columns(rcd_ctx *ctx, const Product &p);          // kLoss: of what parts holds
rcd_status launch_product(rcd_ctx *ctx, const Product &p, void *workspace, cudaStream_t st);

// The product of few rows (rcd_linear_few.cu; no workspace), and whether it takes one.
bool few_rows(const Product &p);
rcd_status launch_few_rows(rcd_ctx *ctx, const Product &p, cudaStream_t st);

double product_cycles(rcd_ctx *ctx, const Product &p);                 // the estimate that the choice of tiles goes by

// Rows of any start and distance to rows that start on 16 bytes.
bool rows_mappable(const void *p, int64_t ld, int64_t eb);
rcd_status launch_pack(rcd_ctx *ctx, const void *from, int64_t ld, int64_t rows, int64_t len, int64_t eb, void *to, int64_t ldTo, cudaStream_t st);

// A launch that may overtake the end of the kernel before it in its stream; the kernel begins with after_the_one_before().
template <typename... Args>
rcd_status launch_early(rcd_ctx *ctx, void (*kernel)(Args...), dim3 grid, unsigned threads, cudaStream_t st, typename std::common_type<Args>::type... args)
{
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
    config.stream = st;
    config.attrs = &early;
    config.numAttrs = 1;
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaLaunchKernelEx(&config, kernel, args...));
    return RCD_OK;
}
#ifdef __CUDACC__
// Before a kernel's first access to memory: the one before it has ended; and the next one may come up, as far as it does not touch memory.
__device__ __forceinline__ void after_the_one_before()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
#endif

// out[c] = sum over the rows of partial[rows][d], in a fixed order
rcd_status launch_column_sums(rcd_ctx *ctx, const float *partial, int64_t rows, int64_t d, float *out, cudaStream_t st);

// Counters of a call's launches, and the word that rcd_sync_status asks for.
inline void begin_operator(rcd_ctx *ctx)
{
    ctx->kernelLaunches = 0;
    ctx->tcLaunches = 0;
    ctx->statusDev = ctx->statusOwn + kOperatorStatus;
}

// Checks of arguments.  An area: a rectangle of memory that a call reads or writes.
struct Area { const void *p; int64_t rows, ld, len, bytes; };
bool areas_meet(const Area &a, const Area &b);
rcd_status check_apart(rcd_ctx *ctx, const Area *out, int outs, const Area *in, int ins);
rcd_status check_sizes(rcd_ctx *ctx, int64_t rows, int64_t n, int64_t k);
rcd_status check_floats(rcd_ctx *ctx, const char *name, const float *p);
rcd_status check_workspace(rcd_ctx *ctx, const void *ws, size_t have, size_t need);
rcd_status check_rows(rcd_ctx *ctx, const char *name, const void *p, int64_t rows, int64_t ld, int64_t len, rcd_elem type);

}  // namespace rcd
