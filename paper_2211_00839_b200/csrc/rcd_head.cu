// Softmax cross entropy of a head's logits without the logits in memory (rcd_linear_cross_entropy), and its gradients.
//
//   z = x w^T + b,  lse[r] = log(sum over v of exp(z[r][v])),  loss[r] = lse[r] - z[r][label]
//   dz = (dloss + dlse) exp(z - lse) - dloss [v = label],  dx = dz w,  dw = dz^T x,  db = sum over rows of dz
//
// Forward: the product's epilogue keeps, for every row, a reference and the sum of exp(z - reference) over half a tile's columns (8 bytes in place of
// 4 x 128), and a second kernel joins them.  Backward: for a piece of the classes at a time the logits are made again, and leave the SM as dz in
// the products' type, as a tensor-core operand has to be; then the piece's share of dx and its rows of dw.  dx of several pieces adds up in fp32.
#include "rcd_product.cuh"

namespace rcd {

KernelChoice head_kernel(Form form, bool oneTile, int wide, bool pair)
{
    constexpr int oneBit = kPlainKernels + kHeadKernels + kScaledKernels + kScaledLowKernels;
    if (oneTile) return wide ? product_choice<kOneTile, false, false, false, 64>(pair, oneBit) : product_choice<kOneTile, false, false, false, 0>(pair, oneBit + 2);
    if (form == kLoss) return wide ? product_choice<kLoss, false, false, false, 32>(pair, kPlainKernels + 2) : product_choice<kLoss, false, false, false, 0>(pair, kPlainKernels);
    return wide ? product_choice<kLogitGrads, false, false, false, 64>(pair, kPlainKernels + 6) : product_choice<kLogitGrads, false, false, false, 0>(pair, kPlainKernels + 4);
}

namespace {

// Joins a row's parts: kRowsPer rows per CTA, whose other threads share the parts out; neighbours meet by shuffles (one row) or in shared memory.
template <int kRowsPer>
__global__ void __launch_bounds__(1024) join_loss_kernel(const float2 *__restrict__ parts, int64_t count, int64_t rows, const float *__restrict__ picked,
                                                         const int32_t *__restrict__ labels, int32_t classes, float *__restrict__ loss, float *__restrict__ lse, int32_t *status)
{
    after_the_one_before();
    __shared__ SumOfExp sh[32][kRowsPer];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int64_t row = (int64_t)blockIdx.x * kRowsPer + (kRowsPer == 32 ? lane : 0), first = kRowsPer == 32 ? warp : threadIdx.x, step = kRowsPer == 32 ? warps : blockDim.x;
    SumOfExp s = no_terms();
    if (row < rows) {
#pragma unroll 8
        for (int64_t i = first; i < count; i += step) {
            const float2 x = parts[i * rows + row];
            join_terms(s, {x.x, x.y});
        }
    }
    if constexpr (kRowsPer == 1) {
#pragma unroll
        for (int o = 16; o; o >>= 1) join_terms(s, {__shfl_xor_sync(0xffffffffu, s.top, o), __shfl_xor_sync(0xffffffffu, s.sum, o)});
        if (lane == 0) sh[warp][0] = s;
    } else {
        sh[warp][lane] = s;
    }
    __syncthreads();
    if (warp || row >= rows || (kRowsPer == 1 && lane)) return;
    for (int i = 1; i < warps; ++i) join_terms(s, sh[i][kRowsPer == 32 ? lane : 0]);
    finish_loss(s, labels[row], classes, picked[row], loss + row, lse ? lse + row : nullptr, status);
}

// fp16: a power of two that brings the largest gradient of a logit to 2^13..2^14, so that those 2^-38 of it are still held (p is small almost
// everywhere, and a mean's dloss is 1 / rows); up[1] takes it out of the products again.  dloss counts where a row's gradients take it, and what is not
// finite does not: other rows keep their digits beside it.
__global__ void __launch_bounds__(1024) choose_up_kernel(const float *__restrict__ dloss, const float *__restrict__ dlse, const int32_t *__restrict__ labels, int32_t classes, int64_t rows,
                                                         float *__restrict__ up)
{
    after_the_one_before();
    __shared__ float sh[32];
    float most = 0.0f;
    for (int64_t r = threadIdx.x; r < rows; r += 1024) {
        const int32_t label = labels[r];
        const float g = label < 0 || label >= classes ? 0.0f : dloss ? fabsf(dloss[r]) : 1.0f, size = g + (dlse ? fabsf(dlse[r]) : 0.0f);
        if (size < INFINITY) most = fmaxf(most, size);
    }
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = most;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 32; ++i) most = fmaxf(most, sh[i]);
    int e = 0;
    if (most > 0.0f) e = 13 - ilogbf(most);
    e = max(-100, min(100, e));
    up[0] = ldexpf(1.0f, e);
    up[1] = ldexpf(1.0f, -e);
}

// The sum of the pieces' shares to dx's type.
template <typename T>
__global__ void __launch_bounds__(256) round_rows_kernel(const float *__restrict__ from, int64_t ld, int64_t rows, int64_t len, T *__restrict__ to, int64_t ldTo)
{
    after_the_one_before();
    const int64_t perRow = (len + 3) / 4;
    const bool whole = ((uintptr_t)to) % (4 * sizeof(T)) == 0 && ldTo % 4 == 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * perRow; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / perRow, c = (i - r * perRow) * 4;
        float v[4];
        load_pack<4>(v, from + r * ld + c);
        if (whole && c + 4 <= len) store_pack<4>(to + r * ldTo + c, v);
        else
            for (int j = 0; j < 4 && c + j < len; ++j) to[r * ldTo + c + j] = from_float<T>(v[j]);
    }
}

constexpr int64_t kMostTiles = 1LL << 28;

rcd_status check_head(rcd_ctx *ctx, int64_t rows, int64_t n, int64_t k, rcd_elem type)
{
    if (type != RCD_ELEM_BF16 && type != RCD_ELEM_F16) return fail(ctx, RCD_ERR_INVALID_ARG, "x and w must be bf16 or fp16, got type %d", (int)type);
    RCD_TRY(check_sizes(ctx, rows, n, k));
    if (n <= 0) return fail(ctx, RCD_ERR_INVALID_ARG, "n=%lld: there is no class", (long long)n);
    if ((rows + 127) / 128 * ((n + 63) / 64) > kMostTiles) return fail(ctx, RCD_ERR_UNSUPPORTED, "rows=%lld, n=%lld: more than 2^28 tiles", (long long)rows, (long long)n);
    return RCD_OK;
}
rcd_status check_labels(rcd_ctx *ctx, const int32_t *labels)
{
    if (!labels) return fail(ctx, RCD_ERR_INVALID_ARG, "labels is null");
    if (((uintptr_t)labels) % 4) return fail(ctx, RCD_ERR_INVALID_ARG, "labels is not aligned to its type");
    return RCD_OK;
}
rcd_status check_forward(rcd_ctx *ctx, const rcd_cross_entropy_args &a)
{
    RCD_TRY(check_head(ctx, a.rows, a.n, a.k, a.type));
    if (a.rows == 0) return RCD_OK;
    RCD_TRY(check_rows(ctx, "x", a.x_dev, a.rows, a.ldx, a.k, a.type));
    RCD_TRY(check_rows(ctx, "w", a.w_dev, a.n, a.ldw, a.k, a.type));
    RCD_TRY(check_labels(ctx, a.labels_dev));
    if (!a.loss_dev) return fail(ctx, RCD_ERR_INVALID_ARG, "loss is null");
    RCD_TRY(check_floats(ctx, "bias", a.bias_dev_or_null));
    RCD_TRY(check_floats(ctx, "loss", a.loss_dev));
    return check_floats(ctx, "lse", a.lse_dev_or_null);
}

Product logits(int64_t rows, int64_t n, int64_t k, rcd_elem type, const void *x, int64_t ldx, const void *w, int64_t ldw, const float *bias, Form form)
{
    Product p{};
    p.type = type;
    p.M = rows; p.N = n; p.K = k;
    p.a = {x, ldx, false};
    p.b = {w, ldw, false};
    p.out.bias = bias;
    p.out.type = form == kLoss ? RCD_ELEM_F32 : type;
    p.form = form;
    return p;
}

struct ForwardPlan {
    Product p;
    int64_t parts;
    size_t picked, product, bytes;         // parts lie first
};
ForwardPlan forward_plan(rcd_ctx *ctx, const rcd_cross_entropy_args &a, unsigned char *ws)
{
    ForwardPlan f{};
    f.p = logits(a.rows, a.n, a.k, a.type, a.x_dev, a.ldx, a.w_dev, a.ldw, a.bias_dev_or_null, kLoss);
    f.parts = 2 * product_tile_columns(ctx, f.p);
    f.p.head.labels = a.labels_dev;
    f.p.head.classes = (int32_t)a.n;
    if (f.parts == 2) {                    // one tile takes all classes
        f.p.head.loss = a.loss_dev;
        f.p.head.lseOut = a.lse_dev_or_null;
        f.bytes = align_up(product_workspace(ctx, f.p));
        return f;
    }
    f.picked = align_up((size_t)(f.parts * a.rows) * sizeof(float2));
    f.product = f.picked + align_up((size_t)a.rows * 4);
    f.bytes = f.product + align_up(product_workspace(ctx, f.p));
    f.p.head.parts = (float2 *)ws;
    f.p.head.picked = (float *)(ws + f.picked);
    return f;
}

rcd_status check_back(rcd_ctx *ctx, const rcd_cross_entropy_back_args &a)
{
    RCD_TRY(check_head(ctx, a.rows, a.n, a.k, a.type));
    if (a.piece < 0) return fail(ctx, RCD_ERR_INVALID_ARG, "piece=%lld is negative", (long long)a.piece);
    if (a.dw_dev_or_null && a.dw_type != a.type && a.dw_type != RCD_ELEM_F32) return fail(ctx, RCD_ERR_INVALID_ARG, "dw must have the type of x or be fp32, got type %d", (int)a.dw_type);
    RCD_TRY(check_floats(ctx, "dbias", a.dbias_dev_or_null));
    if (a.dw_dev_or_null) RCD_TRY(check_rows(ctx, "dw", a.dw_dev_or_null, a.n, a.ld_dw, a.k, a.dw_type));
    if (a.rows == 0) return RCD_OK;
    RCD_TRY(check_rows(ctx, "x", a.x_dev, a.rows, a.ldx, a.k, a.type));
    RCD_TRY(check_rows(ctx, "w", a.w_dev, a.n, a.ldw, a.k, a.type));
    if (a.dx_dev_or_null) RCD_TRY(check_rows(ctx, "dx", a.dx_dev_or_null, a.rows, a.ld_dx, a.k, a.type));
    RCD_TRY(check_labels(ctx, a.labels_dev));
    if (!a.lse_dev) return fail(ctx, RCD_ERR_INVALID_ARG, "lse is null");
    RCD_TRY(check_floats(ctx, "lse", a.lse_dev));
    RCD_TRY(check_floats(ctx, "bias", a.bias_dev_or_null));
    RCD_TRY(check_floats(ctx, "dloss", a.dloss_dev_or_null));
    return check_floats(ctx, "dlse", a.dlse_dev_or_null);
}

// Classes whose dz is in memory at once: 512 MB of it where the caller does not say.  (Fewer and larger pieces: dx's sum goes through memory once a piece.  8192 x 4096 over 32 768 classes: 4.3 to 5.0 ms in one piece, 5.3
// in four; over 131 072 19.7 to 20.5 in one, in four and in eight.)
constexpr int64_t kPieceBytes = 512LL << 20;
int64_t piece_of(const rcd_cross_entropy_back_args &a)
{
    const int64_t piece = a.piece ? a.piece : std::max<int64_t>(kPieceBytes / (2 * a.rows), 256);
    return piece >= a.n ? a.n : std::max<int64_t>(piece / 64 * 64, 64);      // (dz's rows of whole 128 bytes)
}

// Classes that a tile may have all of.  (dx and dw are far from showing what is gained.  Calls get from 13 % shorter, since the chunks are longer, to 9 % longer, where small tiles would fill more SMs:
// 128 x 8192 over 250 classes 82 -> 71 us, 5000 x 512 over 256 34 -> 37.)
constexpr int kMostOneTile = 256;

// Where the parts of a backward pass's workspace lie, and the products of the piece of classes from `first` on.
struct BackPlan {
    int64_t piece, pieces, ldDz, ldSum;
    bool sumDx;                            // dx of several pieces: in fp32
    bool sumRows;                          // dbias: over groups of 32 rows, where there are several
    bool packX, packW;                     // copies whose rows start on 16 bytes, which all products read
    int64_t ldPacked;
    size_t dz, sum, sums, up, x, w, product, bytes;
    Product z, dx, dw;
};
BackPlan back_plan(rcd_ctx *ctx, const rcd_cross_entropy_back_args &a, unsigned char *ws, int64_t first)
{
    BackPlan b{};
    const int64_t eb = elem_bytes(a.type);
    b.piece = piece_of(a);
    b.pieces = (a.n + b.piece - 1) / b.piece;
    const int64_t n = std::min(b.piece, a.n - first);
    b.ldDz = (b.piece + 63) / 64 * 64;
    b.ldSum = (a.k + 3) / 4 * 4;
    b.sumDx = a.dx_dev_or_null && b.pieces > 1;
    b.sumRows = a.dbias_dev_or_null && a.rows > 32;
    size_t at = 0;
    auto place = [&](bool wanted, size_t bytes) { const size_t here = at; if (wanted) at += align_up(bytes); return here; };
    b.dz = place(true, (size_t)(a.rows * b.ldDz) * 2);
    b.sum = place(b.sumDx, (size_t)(a.rows * b.ldSum) * 4);
    b.sums = place(b.sumRows, (size_t)((a.rows + 31) / 32 * b.piece) * 4);
    b.up = place(a.type == RCD_ELEM_F16, 8);
    b.packX = !rows_mappable(a.x_dev, a.ldx, eb);
    b.packW = !rows_mappable(a.w_dev, a.ldw, eb);
    b.ldPacked = (a.k + 7) / 8 * 8;
    b.x = place(b.packX, (size_t)(a.rows * b.ldPacked) * 2);
    b.w = place(b.packW, (size_t)(b.piece * b.ldPacked) * 2);
    b.product = at;
    const float *up = a.type == RCD_ELEM_F16 ? (const float *)(ws + b.up) : nullptr;
    const void *x = b.packX ? ws + b.x : a.x_dev, *w = b.packW ? ws + b.w : (const unsigned char *)a.w_dev + first * a.ldw * eb;
    const int64_t ldx = b.packX ? b.ldPacked : a.ldx, ldw = b.packW ? b.ldPacked : a.ldw;
    b.z = logits(a.rows, n, a.k, a.type, x, ldx, w, ldw, a.bias_dev_or_null ? a.bias_dev_or_null + first : nullptr, kLogitGrads);
    b.z.oneTile = a.dbias_dev_or_null && a.n <= kMostOneTile && b.pieces == 1;
    b.z.out.y = ws + b.dz;
    b.z.out.ldy = b.ldDz;
    b.z.head.labels = a.labels_dev;
    b.z.head.classes = (int32_t)a.n;
    b.z.head.firstClass = (int32_t)first;
    b.z.head.lse = a.lse_dev;
    b.z.head.dloss = a.dloss_dev_or_null;
    b.z.head.dlse = a.dlse_dev_or_null;
    b.z.head.up = up;
    b.z.head.sums = b.sumRows ? (float *)(ws + b.sums) : a.dbias_dev_or_null ? a.dbias_dev_or_null + first : nullptr;
    // (fp16: the power of two is taken out again)
    b.dx.type = b.dw.type = a.type;
    b.dx.form = b.dw.form = up ? kScaled : kPlain;
    b.dx.M = a.rows; b.dx.N = a.k; b.dx.K = n;
    b.dx.a = {ws + b.dz, b.ldDz, false};
    b.dx.b = {w, ldw, true};
    b.dx.out.type = b.sumDx ? RCD_ELEM_F32 : a.type;
    b.dx.out.y = b.sumDx ? (void *)(ws + b.sum) : a.dx_dev_or_null;
    b.dx.out.ldy = b.sumDx ? b.ldSum : a.ld_dx;
    if (b.sumDx && first > 0) {
        b.dx.out.residual = b.dx.out.y;
        b.dx.out.ldr = b.ldSum;
    }
    b.dw.M = n; b.dw.N = a.k; b.dw.K = a.rows;
    b.dw.a = {ws + b.dz, b.ldDz, true};
    b.dw.b = {x, ldx, true};
    b.dw.out.type = a.dw_type;
    b.dw.out.y = a.dw_dev_or_null ? (unsigned char *)a.dw_dev_or_null + first * a.ld_dw * elem_bytes(a.dw_type) : nullptr;
    b.dw.out.ldy = a.ld_dw;
    b.dx.scaling = {1.0f, 1.0f, up ? up + 1 : nullptr, 1, 0, b.dx.out.type, nullptr};
    b.dw.scaling = {1.0f, 0.0f, up ? up + 1 : nullptr, 1, 0, b.dw.out.type, nullptr};
    size_t most = product_workspace(ctx, b.z);
    if (a.dx_dev_or_null) most = std::max(most, product_workspace(ctx, b.dx));
    if (a.dw_dev_or_null) most = std::max(most, product_workspace(ctx, b.dw));
    b.bytes = b.product + align_up(most);
    return b;
}
// (the last piece is smaller and may be gone about otherwise)
size_t back_workspace(rcd_ctx *ctx, const rcd_cross_entropy_back_args &a)
{
    const BackPlan b = back_plan(ctx, a, nullptr, 0);
    return b.pieces == 1 ? b.bytes : std::max(b.bytes, back_plan(ctx, a, nullptr, (b.pieces - 1) * b.piece).bytes);
}

}  // namespace

}  // namespace rcd

using namespace rcd;

extern "C" rcd_status rcd_linear_cross_entropy_workspace_bytes(rcd_ctx *ctx, const rcd_cross_entropy_args *args, size_t *bytes_out)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    if (!args || !bytes_out) return fail(ctx, RCD_ERR_INVALID_ARG, "args or output is null");
    RCD_TRY(check_forward(ctx, *args));
    *bytes_out = args->rows == 0 ? 0 : forward_plan(ctx, *args, nullptr).bytes;
    return RCD_OK;
}

extern "C" rcd_status rcd_linear_cross_entropy(rcd_ctx *ctx, const rcd_cross_entropy_args *args, void *workspace_dev, size_t workspace_bytes, void *cuda_stream)
{
    size_t need = 0;
    RCD_TRY(rcd_linear_cross_entropy_workspace_bytes(ctx, args, &need));
    const rcd_cross_entropy_args &a = *args;
    begin_operator(ctx);
    if (a.rows == 0) return RCD_OK;
    RCD_TRY(check_workspace(ctx, workspace_dev, workspace_bytes, need));
    const int64_t eb = elem_bytes(a.type);
    const Area out[] = {{a.loss_dev, 1, a.rows, a.rows, 4}, {a.lse_dev_or_null, 1, a.rows, a.rows, 4}, {need ? workspace_dev : nullptr, 1, (int64_t)need, (int64_t)need, 1}};
    const Area in[] = {{a.x_dev, a.rows, a.ldx, a.k, eb}, {a.w_dev, a.n, a.ldw, a.k, eb}, {a.bias_dev_or_null, 1, a.n, a.n, 4}, {a.labels_dev, 1, a.rows, a.rows, 4}};
    RCD_TRY(check_apart(ctx, out, 3, in, 4));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    RCD_CUDA(ctx, cudaSetDevice(ctx->device));
    unsigned char *ws = (unsigned char *)workspace_dev;
    const ForwardPlan f = forward_plan(ctx, a, ws);
    RCD_TRY(launch_product(ctx, f.p, ws + f.product, st));
    if (f.p.head.loss) return RCD_OK;
    // (few rows: a CTA each, whose threads lie along the parts; 32 rows per CTA take 6 us for one row of 286 parts)
    const bool few = a.rows <= 2 * ctx->smCount;
    const unsigned threads = 32 * (unsigned)std::min<int64_t>(few ? (f.parts + 31) / 32 : f.parts, 32);
    return launch_early(ctx, few ? join_loss_kernel<1> : join_loss_kernel<32>, dim3((unsigned)(few ? a.rows : (a.rows + 31) / 32)), threads, st, f.p.head.parts, f.parts, a.rows,
                        f.p.head.picked, a.labels_dev, (int32_t)a.n, a.loss_dev, a.lse_dev_or_null, ctx->statusOwn + kOperatorStatus);
}

extern "C" rcd_status rcd_linear_cross_entropy_backward_workspace_bytes(rcd_ctx *ctx, const rcd_cross_entropy_back_args *args, size_t *bytes_out)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    if (!args || !bytes_out) return fail(ctx, RCD_ERR_INVALID_ARG, "args or output is null");
    RCD_TRY(check_back(ctx, *args));
    *bytes_out = args->rows == 0 ? 0 : back_workspace(ctx, *args);
    return RCD_OK;
}

extern "C" rcd_status rcd_linear_cross_entropy_backward(rcd_ctx *ctx, const rcd_cross_entropy_back_args *args, void *workspace_dev, size_t workspace_bytes, void *cuda_stream)
{
    size_t need = 0;
    RCD_TRY(rcd_linear_cross_entropy_backward_workspace_bytes(ctx, args, &need));
    const rcd_cross_entropy_back_args &a = *args;
    RCD_TRY(check_workspace(ctx, workspace_dev, workspace_bytes, need));
    const int64_t eb = elem_bytes(a.type), wb = a.dw_dev_or_null ? elem_bytes(a.dw_type) : 1;
    const Area out[] = {{a.dx_dev_or_null, a.rows, a.ld_dx, a.k, eb}, {a.dw_dev_or_null, a.n, a.ld_dw, a.k, wb}, {a.dbias_dev_or_null, 1, a.n, a.n, 4},
                        {need ? workspace_dev : nullptr, 1, (int64_t)need, (int64_t)need, 1}};
    const Area in[] = {{a.x_dev, a.rows, a.ldx, a.k, eb}, {a.w_dev, a.n, a.ldw, a.k, eb}, {a.bias_dev_or_null, 1, a.n, a.n, 4}, {a.labels_dev, 1, a.rows, a.rows, 4},
                       {a.lse_dev, 1, a.rows, a.rows, 4}, {a.dloss_dev_or_null, 1, a.rows, a.rows, 4}, {a.dlse_dev_or_null, 1, a.rows, a.rows, 4}};
    RCD_TRY(check_apart(ctx, out, 4, in, 7));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    RCD_CUDA(ctx, cudaSetDevice(ctx->device));
    begin_operator(ctx);
    if (a.rows == 0) {                     // sums over nothing
        if (a.dw_dev_or_null) RCD_CUDA(ctx, cudaMemset2DAsync(a.dw_dev_or_null, (size_t)(a.ld_dw * wb), 0, (size_t)(a.k * wb), (size_t)a.n, st));
        if (a.dbias_dev_or_null) RCD_CUDA(ctx, cudaMemsetAsync(a.dbias_dev_or_null, 0, (size_t)a.n * 4, st));
        return RCD_OK;
    }
    if (!a.dx_dev_or_null && !a.dw_dev_or_null && !a.dbias_dev_or_null) return RCD_OK;
    unsigned char *ws = (unsigned char *)workspace_dev;
    BackPlan b = back_plan(ctx, a, ws, 0);
    if (a.type == RCD_ELEM_F16) {
        RCD_TRY(launch_early(ctx, choose_up_kernel, dim3(1), 1024, st, a.dloss_dev_or_null, a.dlse_dev_or_null, a.labels_dev, (int32_t)a.n, a.rows,
                             (float *)(ws + b.up)));
    }
    if (b.packX) RCD_TRY(launch_pack(ctx, a.x_dev, a.ldx, a.rows, a.k, eb, ws + b.x, b.ldPacked, st));
    for (int64_t i = 0; i < b.pieces; ++i) {
        if (i) b = back_plan(ctx, a, ws, i * b.piece);
        if (b.packW) RCD_TRY(launch_pack(ctx, (const unsigned char *)a.w_dev + i * b.piece * a.ldw * eb, a.ldw, b.z.N, a.k, eb, ws + b.w, b.ldPacked, st));
        RCD_TRY(launch_product(ctx, b.z, ws + b.product, st));
        if (b.sumRows) RCD_TRY(launch_column_sums(ctx, b.z.head.sums, (a.rows + 31) / 32, b.z.N, a.dbias_dev_or_null + i * b.piece, st));
        if (a.dx_dev_or_null) RCD_TRY(launch_product(ctx, b.dx, ws + b.product, st));
        if (a.dw_dev_or_null) RCD_TRY(launch_product(ctx, b.dw, ws + b.product, st));
    }
    if (b.sumDx) {
        const unsigned grid = (unsigned)std::min<int64_t>((a.rows * ((a.k + 3) / 4) + 255) / 256, (int64_t)ctx->smCount * 16);
        return a.type == RCD_ELEM_BF16 ? launch_early(ctx, round_rows_kernel<__nv_bfloat16>, dim3(grid), 256, st, (const float *)(ws + b.sum), b.ldSum, a.rows, a.k, (__nv_bfloat16 *)a.dx_dev_or_null, a.ld_dx)
                                       : launch_early(ctx, round_rows_kernel<__half>, dim3(grid), 256, st, (const float *)(ws + b.sum), b.ldSum, a.rows, a.k, (__half *)a.dx_dev_or_null, a.ld_dx);
    }
    return RCD_OK;
}
