// A weight gradient with its singular values brought near one by Newton-Schulz products (rcd_orthogonalize).
//
//   X = G / (|G| + eps);  steps times:  A = X X^T,  B = b A + c A A,  X = a X + B X         (X^T X and X B where G is taller than wide)
//
// The products run on the tensor cores in fp16 with sums in fp32, and X, A and B stand between them as fp16 times 2^10: entries of X are at most 1.2
// or so and some 1 / sqrt(cols) mostly, which is well inside the type's normal range then, and 11 bits are kept where bf16 would keep 8 (each
// rounding grows by up to a per step where X is small: 1.1e-3 of the result's norm in fp16 for 1024 x 1024 normal values, 8.9e-3 in bf16; rounding the result
// itself to bf16 takes 1.7e-3).  X's roundings in the sum a X are what counts, and the earliest most, where a few strong directions make the entries and the weak ones grow: so the first
// step adds G itself, an fp32 one as two fp16 (one direction a hundred times as strong as the noise: 2.1e-2 -> 5e-3; 8 of 1024 x 2048: 474 -> 491 us), while A and the product B X take its
// first part alone.  G is brought into range by a power of two alone, so that a 16-bit G is held exactly; what is left of its norm, a factor between 1 and 2, goes into the
// first step's products as a number that their epilogue reads.  A and B are symmetric: tiles on and below the diagonal are computed and
// stored both ways.
//
// Three forms: a side of at most 128 in a cluster per matrix (rcd_orthogonal_cluster.cu); all steps in one launch (rcd_orthogonal_fused.cu), where the time goes into the
// steps' waiting for one another; launches of their own with tiles of up to 256 x 256 on pairs of SMs, where it goes into the products (4096 x 4096: 1.15 ms, 1.19 PFLOP/s of
// what has to be computed, 72 % of cuBLAS's rate in bursts).
#include "rcd_orthogonal.h"
#include "rcd_product.cuh"

namespace rcd {

// (what has a second part is the last product of an update's step: X times a square or the other way, with an output of 16 bits)
KernelChoice scaled_kernel(int order, int wide, bool pair, bool low)
{
    constexpr int bit = kPlainKernels + kHeadKernels, lowBit = bit + kScaledKernels;
    if (!low) return product_choice_by_order<kScaled>(order, wide, pair, bit);
    if (order == 0) return wide ? product_choice<kScaledLow, false, false, false, 64>(pair, lowBit) : product_choice<kScaledLow, false, false, false, 0>(pair, lowBit + 2);
    return wide ? product_choice<kScaledLow, false, false, true, 64>(pair, lowBit + 4) : product_choice<kScaledLow, false, false, true, 0>(pair, lowBit + 6);
}

namespace {

constexpr int kMostParts = 256;            // sums of squares per matrix

struct Gradient { const void *p; int64_t ld, step; int32_t rows, cols; };

// kVec neighbours of a row, as 16-byte accesses take them; 1 where rows do not start on 16 bytes.
template <typename T, int kVec>
__global__ void __launch_bounds__(256) squares_kernel(Gradient g, double *__restrict__ parts)
{
    after_the_one_before();
    __shared__ double sh[8];
    const T *p = (const T *)g.p + blockIdx.y * g.step;
    const int64_t perRow = (g.cols + kVec - 1) / kVec, total = perRow * g.rows;
    double s = 0.0;                        // (64 bits: squares of fp32's or bf16's range)
#pragma unroll 4
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / perRow, c = (i - r * perRow) * kVec;
        float v[kVec];
        if (c + kVec <= g.cols) load_pack<kVec>(v, p + r * g.ld + c);
        else {
#pragma unroll
            for (int j = 0; j < kVec; ++j) v[j] = c + j < g.cols ? to_float(p[r * g.ld + c + j]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j) s += (double)v[j] * (double)v[j];
    }
    s = warp_sum(s);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) s += sh[i];
        parts[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
    }
}

// G times the power of two that brings |G| + eps to 2^(kUp - 1) .. 2^kUp, and the factor that is left of 2^kUp / (|G| + eps); zeros up to whole 64 rows and columns.  Of an
// fp32 G also what fp16 leaves of it.
template <typename T, int kVec>
__global__ void __launch_bounds__(256) bring_up_kernel(Gradient g, const double *__restrict__ parts, int32_t count, float eps, __half *__restrict__ x, __half *__restrict__ low, int32_t rowsX, int32_t colsX,
                                                       float *__restrict__ factor, uint32_t *__restrict__ counter)
{
    after_the_one_before();
    __shared__ float scales[2];
    if (threadIdx.x < 32) {
        double s = 0.0;
        for (int i = threadIdx.x; i < count; i += 32) s += parts[(int64_t)blockIdx.y * count + i];
        s = warp_sum(s);
        if (threadIdx.x == 0) {
            const double norm = sqrt(s) + (double)eps;
            int e = 0;
            double f = norm == 0.0 ? 0.0 : NAN;                        // (of nothing: zeros; a G that is not finite: NaN)
            if (norm > 0.0 && norm < (double)INFINITY) {
                e = kUp - 1 - ilogb(norm);
                f = ldexp(1.0, kUp) / ldexp(norm, e);
            }
            scales[0] = ldexpf(1.0f, e / 2);                           // (2^e alone may be out of fp32's range)
            scales[1] = ldexpf(1.0f, e - e / 2);
            if (blockIdx.x == 0) factor[blockIdx.y] = (float)f;
        }
    }
    __syncthreads();
    if (counter && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *counter = 0;
    const float up0 = scales[0], up1 = scales[1];
    const T *p = (const T *)g.p + blockIdx.y * g.step;
    __half *to = x + (int64_t)blockIdx.y * rowsX * colsX;
    const int64_t perRow = colsX / 8, total = perRow * rowsX;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / perRow, c = (i - r * perRow) * 8;
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (r < g.rows) {
            const T *from = p + r * g.ld + c;
            if (kVec > 1 && c + 8 <= g.cols) load_pack<8>(v, from);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = c + j < g.cols ? to_float(from[j]) : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = v[j] * up0 * up1;
        store_pack<8>(to + r * colsX + c, v);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (v[j] - __half2float(__float2half_rn(v[j]))) * (float)(1 << kLowUp);
            store_pack<8>(low + (int64_t)blockIdx.y * rowsX * colsX + r * colsX + c, v);
        }
    }
}

// X to the output where its matrices lie in a way that the last product cannot write.
__global__ void __launch_bounds__(256) bring_out_kernel(const __half *__restrict__ x, int32_t rowsX, int32_t colsX, __nv_bfloat16 *__restrict__ o, int64_t ld, int64_t step, int32_t rows, int32_t cols)
{
    after_the_one_before();
    const int64_t total = (int64_t)rows * cols;
    x += (int64_t)blockIdx.y * rowsX * colsX;
    o += blockIdx.y * step;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / cols, c = i - r * cols;
        o[r * ld + c] = __float2bfloat16_rn(__half2float(x[r * colsX + c]) * (1.0f / (1 << kUp)));
    }
}

rcd_status check(rcd_ctx *ctx, const rcd_orthogonalize_args &a)
{
    constexpr int64_t most = 1 << 16;
    if (!elem_is_float(a.type)) return fail(ctx, RCD_ERR_INVALID_ARG, "g must be bf16, fp16 or fp32, got type %d", (int)a.type);
    if (a.batch < 0 || a.rows < 0 || a.cols < 0) return fail(ctx, RCD_ERR_INVALID_ARG, "batch=%lld, rows=%lld or cols=%lld is negative", (long long)a.batch, (long long)a.rows, (long long)a.cols);
    if (a.batch >= most || a.rows > most || a.cols > most) return fail(ctx, RCD_ERR_UNSUPPORTED, "batch=%lld, rows=%lld, cols=%lld: 65535 matrices of 65536 x 65536 at most", (long long)a.batch, (long long)a.rows, (long long)a.cols);
    if (a.steps < 1 || a.steps > kMostSteps) return fail(ctx, RCD_ERR_INVALID_ARG, "steps=%d must be from 1 to 64", (int)a.steps);
    if (!a.coefficients_host) return fail(ctx, RCD_ERR_INVALID_ARG, "coefficients is null");
    for (int i = 0; i < 3 * a.steps; ++i)
        if (!(fabsf(a.coefficients_host[i]) <= 1e4f)) return fail(ctx, RCD_ERR_INVALID_ARG, "coefficient %d is not within 1e4", i);
    if (!(a.eps >= 0.0f) || a.eps > 3e38f) return fail(ctx, RCD_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (a.batch == 0 || a.rows == 0 || a.cols == 0) return RCD_OK;
    RCD_TRY(check_rows(ctx, "g", a.g_dev, a.rows, a.ld_g, a.cols, a.type));
    RCD_TRY(check_rows(ctx, "o", a.o_dev, a.rows, a.ld_o, a.cols, RCD_ELEM_BF16));
    auto span = [&](int64_t ld) { return (a.rows - 1) * ld + a.cols; };
    if (a.batch > 1 && (a.step_g < span(a.ld_g) || a.step_o < span(a.ld_o) || a.step_g > (1LL << 40) || a.step_o > (1LL << 40)))
        return fail(ctx, RCD_ERR_INVALID_ARG, "matrices lie %lld and %lld elements apart and are %lld and %lld long", (long long)a.step_g, (long long)a.step_o, (long long)span(a.ld_g), (long long)span(a.ld_o));
    const int64_t large = (std::max(a.rows, a.cols) + 63) / 64 * 64;
    if (a.batch * large > 0x7fffffffLL) return fail(ctx, RCD_ERR_UNSUPPORTED, "batch=%lld: more than 2^31 rows", (long long)a.batch);
    return RCD_OK;
}

struct Layout {
    bool tall;
    int64_t rows, cols, side;              // of X, A and B, whole 64s
    int32_t parts;
    FusedPlan fused;
    bool inOne;                            // all steps in one launch
    size_t x[2], low, a, b, squares, factor, counter, product, bytes;
};
// Step i's products; (first of them, second, third).
struct Step { Product gram, poly, x; };
Step step_of(const rcd_orthogonalize_args &a, const Layout &l, unsigned char *ws, int i, bool direct)
{
    Step s{};
    const float down = 1.0f / (1 << kUp);
    const float *c = a.coefficients_host + 3 * i;
    void *from = ws + l.x[i & 1], *to = ws + l.x[(i + 1) & 1], *gram = ws + l.a, *poly = ws + l.b;
    const float *factor = i == 0 ? (const float *)(ws + l.factor) : nullptr;
    for (Product *p : {&s.gram, &s.poly, &s.x}) {
        p->type = RCD_ELEM_F16;
        p->form = kScaled;
        p->batch = a.batch;
        p->out.type = RCD_ELEM_F16;
        p->scaling.residualType = RCD_ELEM_F16;
    }
    s.gram.M = s.gram.N = l.side;
    s.gram.K = l.tall ? l.rows : l.cols;
    s.gram.a = s.gram.b = {from, l.cols, l.tall};
    s.gram.aStep = s.gram.bStep = l.rows;
    s.gram.yStep = l.side;
    s.gram.symmetric = true;
    s.gram.out.y = gram;
    s.gram.out.ldy = l.side;
    s.gram.scaling.alpha = down;
    s.gram.scaling.factor = factor;
    s.gram.scaling.alphaPower = 2;

    s.poly.M = s.poly.N = s.poly.K = l.side;
    s.poly.a = s.poly.b = {gram, l.side, false};
    s.poly.aStep = s.poly.bStep = s.poly.yStep = s.poly.rStep = l.side;
    s.poly.symmetric = true;
    s.poly.out.residual = gram;
    s.poly.out.ldr = l.side;
    s.poly.out.y = poly;
    s.poly.out.ldy = l.side;
    s.poly.scaling.alpha = c[2] * down;
    s.poly.scaling.beta = c[1];

    s.x.M = l.rows;
    s.x.N = l.cols;
    s.x.K = l.side;
    const Operand x = {from, l.cols, !l.tall}, b = {poly, l.side, false};
    s.x.a = l.tall ? x : b;
    s.x.b = l.tall ? b : x;
    s.x.aStep = l.tall ? l.rows : l.side;
    s.x.bStep = l.tall ? l.side : l.rows;
    s.x.yStep = s.x.rStep = l.rows;
    s.x.out.residual = from;
    s.x.out.ldr = l.cols;
    s.x.out.y = to;
    s.x.out.ldy = l.cols;
    s.x.scaling.alpha = down;
    s.x.scaling.beta = c[0];
    s.x.scaling.factor = factor;
    s.x.scaling.alphaPower = s.x.scaling.betaPower = 1;
    s.x.scaling.low = i == 0 && a.type == RCD_ELEM_F32 ? ws + l.low : nullptr;
    if (direct) {
        s.x.M = a.rows;
        s.x.N = a.cols;
        s.x.yStep = a.batch > 1 ? a.step_o / a.ld_o : a.rows;
        s.x.out.type = RCD_ELEM_BF16;
        s.x.out.y = a.o_dev;
        s.x.out.ldy = a.ld_o;
        s.x.scaling.alpha *= down;
        s.x.scaling.beta *= down;
    }
    return s;
}
// Whether the last product writes the output itself: its matrices lie whole rows apart, and pieces of 32 rows end where a matrix does.
bool direct_output(const rcd_orthogonalize_args &a) { return a.batch == 1 || (a.step_o % a.ld_o == 0 && a.rows % 32 == 0 && a.batch * (a.step_o / a.ld_o) < 0x7fffffffLL); }

Layout layout_of(rcd_ctx *ctx, const rcd_orthogonalize_args &a)
{
    Layout l{};
    l.tall = a.rows > a.cols;
    l.rows = (a.rows + 63) / 64 * 64;
    l.cols = (a.cols + 63) / 64 * 64;
    l.side = std::min(l.rows, l.cols);
    // (16 elements a thread at least, two CTAs per SM over the batch at most)
    l.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>({kMostParts, (a.rows * a.cols + 4095) / 4096, std::max<int64_t>(1, 2 * ctx->smCount / a.batch)}));
    size_t at = 0;
    auto place = [&](size_t bytes) { const size_t here = at; at += align_up(bytes); return here; };
    for (size_t &x : l.x) x = place((size_t)(a.batch * l.rows * l.cols) * 2);
    l.low = place(a.type == RCD_ELEM_F32 ? (size_t)(a.batch * l.rows * l.cols) * 2 : 0);
    l.a = place((size_t)(a.batch * l.side * l.side) * 2);
    l.b = place((size_t)(a.batch * l.side * l.side) * 2);
    l.squares = place((size_t)(a.batch * l.parts) * 8);
    l.factor = place((size_t)a.batch * 4);
    l.fused = fused_plan(ctx, a.batch, l.rows, l.cols, l.tall);
    if (l.fused.possible) {
        // Launches of their own take 4.3 us each besides the products.  (Both measured: 512 x 512 103 us in one launch, 133 in 17; 1024 x 2048 189 and 204; 1536 x 1536
        // 304 and 228.)
        const Step s = step_of(a, l, nullptr, 0, false);
        double us = 0.0;
        for (const Product *p : {&s.gram, &s.poly, &s.x}) us += 4.3 + product_cycles(ctx, *p) / 1900.0;
        l.inOne = l.fused.stepUs < us;
    }
    l.counter = place(l.inOne ? 4 : 0);
    l.product = l.bytes = at;
    if (l.inOne) return l;
    size_t most = 0;
    for (const bool direct : {false, true}) {
        const Step s = step_of(a, l, nullptr, 0, direct && direct_output(a));
        for (const Product *p : {&s.gram, &s.poly, &s.x}) most = std::max(most, product_workspace(ctx, *p));
    }
    l.bytes = at + align_up(most);
    return l;
}

}  // namespace

}  // namespace rcd

using namespace rcd;

extern "C" rcd_status rcd_orthogonalize_workspace_bytes(rcd_ctx *ctx, const rcd_orthogonalize_args *args, size_t *bytes_out)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    if (!args || !bytes_out) return fail(ctx, RCD_ERR_INVALID_ARG, "args or output is null");
    RCD_TRY(check(ctx, *args));
    *bytes_out = args->batch == 0 || args->rows == 0 || args->cols == 0 || cluster_for(ctx, args->rows, args->cols) ? 0 : layout_of(ctx, *args).bytes;
    return RCD_OK;
}

extern "C" rcd_status rcd_orthogonalize(rcd_ctx *ctx, const rcd_orthogonalize_args *args, void *workspace_dev, size_t workspace_bytes, void *cuda_stream)
{
    size_t need = 0;
    RCD_TRY(rcd_orthogonalize_workspace_bytes(ctx, args, &need));
    const rcd_orthogonalize_args &a = *args;
    begin_operator(ctx);
    if (a.batch == 0 || a.rows == 0 || a.cols == 0) return RCD_OK;
    RCD_TRY(check_workspace(ctx, workspace_dev, workspace_bytes, need));
    const int64_t eb = elem_bytes(a.type);
    // (two views of a batch: its matrices, one for each step; and, where they lie whole rows apart, its rows and those between them.  Either may show that nothing is shared.)
    auto matrices = [&](const void *p, int64_t ld, int64_t step, int64_t bytes) { return Area{p, a.batch, step, (a.rows - 1) * ld + a.cols, bytes}; };
    auto rows = [&](const void *p, int64_t ld, int64_t step, int64_t bytes) {
        if (a.batch > 1 && step % ld) return matrices(p, ld, step, bytes);
        return Area{p, (a.batch > 1 ? (a.batch - 1) * (step / ld) : 0) + a.rows, ld, a.cols, bytes};
    };
    const Area o = matrices(a.o_dev, a.ld_o, a.step_o, 2), g0 = matrices(a.g_dev, a.ld_g, a.step_g, eb);
    const Area out[] = {{need ? workspace_dev : nullptr, 1, (int64_t)need, (int64_t)need, 1}};
    const Area in[] = {o, g0};
    RCD_TRY(check_apart(ctx, out, 1, in, 2));
    if (areas_meet(o, g0)) {
        const Area outRows[] = {rows(a.o_dev, a.ld_o, a.step_o, 2)}, inRows[] = {rows(a.g_dev, a.ld_g, a.step_g, eb)};
        RCD_TRY(check_apart(ctx, outRows, 1, inRows, 1));
    }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    RCD_CUDA(ctx, cudaSetDevice(ctx->device));
    if (const int cluster = cluster_for(ctx, a.rows, a.cols)) return launch_cluster(ctx, a, cluster, st);
    unsigned char *ws = (unsigned char *)workspace_dev;
    const Layout l = layout_of(ctx, a);
    const Gradient g{a.g_dev, a.ld_g, a.batch > 1 ? a.step_g : 0, (int32_t)a.rows, (int32_t)a.cols};
    const bool aligned = rows_aligned(a.g_dev, a.ld_g, eb, 16) && (a.batch == 1 || a.step_g * eb % 16 == 0);
    auto bring_up = [&](auto t, auto vec) -> rcd_status {
        using T = decltype(t);
        constexpr int kVec = decltype(vec)::value;
        RCD_TRY(launch_early(ctx, squares_kernel<T, kVec>, dim3((unsigned)l.parts, (unsigned)a.batch), 256, st, g, (double *)(ws + l.squares)));
        const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>((l.rows * l.cols / 8 + 255) / 256, 8 * ctx->smCount / a.batch));
        return launch_early(ctx, bring_up_kernel<T, kVec>, dim3(grid, (unsigned)a.batch), 256, st, g, (const double *)(ws + l.squares), l.parts, a.eps, (__half *)(ws + l.x[0]), (__half *)(ws + l.low), (int32_t)l.rows,
                            (int32_t)l.cols, (float *)(ws + l.factor), l.inOne ? (uint32_t *)(ws + l.counter) : nullptr);
    };
    auto by_type = [&](auto t) {
        return aligned ? bring_up(t, std::integral_constant<int, 16 / sizeof(t)>()) : bring_up(t, std::integral_constant<int, 1>());
    };
    RCD_TRY(a.type == RCD_ELEM_BF16 ? by_type(__nv_bfloat16()) : a.type == RCD_ELEM_F16 ? by_type(__half()) : by_type(0.0f));
    if (l.inOne) {
        FusedParams p{};
        p.x0 = (__half *)(ws + l.x[0]);
        p.x1 = (__half *)(ws + l.x[1]);
        p.low = a.type == RCD_ELEM_F32 ? (const __half *)(ws + l.low) : nullptr;
        p.a = (__half *)(ws + l.a);
        p.b = (__half *)(ws + l.b);
        p.factor = (const float *)(ws + l.factor);
        p.counter = (uint32_t *)(ws + l.counter);
        p.o = (__nv_bfloat16 *)a.o_dev;
        p.ldO = a.ld_o;
        p.stepO = a.batch > 1 ? a.step_o : 0;
        p.rowsO = (int32_t)a.rows; p.colsO = (int32_t)a.cols;
        p.rows = (int32_t)l.rows; p.cols = (int32_t)l.cols; p.side = (int32_t)l.side;
        p.batch = (int32_t)a.batch;
        p.steps = a.steps;
        p.cluster = l.fused.cluster;
        p.tall = l.tall;
        for (int k = 0; k < 3; ++k) p.phases[k] = l.fused.phases[k];
        p.status = ctx->statusOwn + kOperatorStatus;
        for (int i = 0; i < 3 * a.steps; ++i) p.coefficients[i] = a.coefficients_host[i];
        return launch_fused(ctx, p, l.fused, st);
    }
    const bool direct = direct_output(a);
    for (int i = 0; i < a.steps; ++i) {
        const Step s = step_of(a, l, ws, i, direct && i == a.steps - 1);
        for (const Product *p : {&s.gram, &s.poly, &s.x}) RCD_TRY(launch_product(ctx, *p, ws + l.product, st));
    }
    if (!direct) {
        const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>((a.rows * a.cols + 1023) / 1024, 8 * ctx->smCount / a.batch));
        return launch_early(ctx, bring_out_kernel, dim3(grid, (unsigned)a.batch), 256, st, (const __half *)(ws + l.x[a.steps & 1]), (int32_t)l.rows, (int32_t)l.cols, (__nv_bfloat16 *)a.o_dev, a.ld_o,
                            a.step_o, (int32_t)a.rows, (int32_t)a.cols);
    }
    return RCD_OK;
}
