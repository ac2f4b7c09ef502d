// Matrix product with bias, activation and residual in its epilogue (rcd_linear) and its gradients: argument checks, the order of
// the launches, and the pass that takes dy through the activation's derivative.  (The products: rcd_linear_tc.cu.)
//
//   z = x w^T [* sx[row] * sw[column]] + b,  y = act(z) + r
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum over rows of dz
#include "rcd_act.cuh"
#include "rcd_linear.h"

namespace rcd {

namespace {

// dz = dy * act'(z), rounded to the products' type, and the sums of its columns over this CTA's rows.  Bound by memory: 16-byte accesses
// where rows allow it, 32 threads along a row, 8 rows at a time; a thread's sums meet those of the other seven in shared memory.
constexpr int kSlopeRows = 32;
template <typename T, int VEC>
__global__ void __launch_bounds__(256) slope_kernel(const T *__restrict__ dy, int64_t ldDy, const T *__restrict__ z, int64_t ldZ, int64_t rows, int64_t n, int act,
                                                    T *__restrict__ dz, int64_t ldDz, float *__restrict__ partial)
{
    __shared__ float sh[8][32 * VEC + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col0 = (int64_t)blockIdx.x * 32 * VEC, col = col0 + lane * VEC;
    const int64_t chunks = (rows + kSlopeRows - 1) / kSlopeRows;
    for (int64_t chunk = blockIdx.y; chunk < chunks; chunk += gridDim.y) {
        float s[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[i] = 0.0f;
        if (col < n) {
            // (a thread's four rows are all asked for before the first is worked on)
            constexpr int kMine = kSlopeRows / 8;
            Pack<T, VEC> g[kMine], x[kMine];
            const int64_t row0 = chunk * kSlopeRows + warp;
#pragma unroll
            for (int k = 0; k < kMine; ++k)
                if (row0 + 8 * k < rows) {
                    g[k] = *reinterpret_cast<const Pack<T, VEC> *>(dy + (row0 + 8 * k) * ldDy + col);
                    if (z) x[k] = *reinterpret_cast<const Pack<T, VEC> *>(z + (row0 + 8 * k) * ldZ + col);
                }
#pragma unroll
            for (int k = 0; k < kMine; ++k)
                if (row0 + 8 * k < rows) {
                    float d[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) d[i] = to_float(g[k].v[i]);
                    if (z) {
                        float o[VEC];
#pragma unroll
                        for (int i = 0; i < VEC; ++i) o[i] = to_float(x[k].v[i]);
                        slopes<VEC>(d, o, act);
                    }
                    if (dz) store_pack<VEC>(dz + (row0 + 8 * k) * ldDz + col, d);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) s[i] += d[i];
                }
        }
        if (partial) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) sh[warp][lane * VEC + i] = s[i];
            __syncthreads();
            for (int c = threadIdx.x; c < 32 * VEC && col0 + c < n; c += 256) {
                float o = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) o += sh[k][c];
                partial[chunk * n + col0 + c] = o;
            }
            __syncthreads();
        }
    }
}

// out[c] = sum over the rows of partial, in a fixed order: 32 columns per CTA, 32 warps take every 32nd row.
__global__ void __launch_bounds__(1024) column_sums_kernel(const float *__restrict__ partial, int32_t rows, int64_t d, float *__restrict__ out)
{
    after_the_one_before();
    __shared__ float sh[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < d)
        for (int r = warp; r < rows; r += 32) s += partial[(int64_t)r * d + col];
    sh[warp][lane] = s;
    __syncthreads();
    s = warp_sum(sh[lane][warp]);
    if (lane == 0 && (int64_t)blockIdx.x * 32 + warp < d) out[(int64_t)blockIdx.x * 32 + warp] = s;
}

rcd_status check_act(rcd_ctx *ctx, rcd_activation act)
{
    if (act < RCD_ACT_NONE || act > RCD_ACT_SILU) return fail(ctx, RCD_ERR_INVALID_ARG, "unknown activation %d", (int)act);
    return RCD_OK;
}

rcd_status check_linear(rcd_ctx *ctx, const rcd_linear_args &a)
{
    if (a.type != RCD_ELEM_I8 && a.type != RCD_ELEM_BF16 && a.type != RCD_ELEM_F16) return fail(ctx, RCD_ERR_INVALID_ARG, "x and w must be int8, bf16 or fp16, got type %d", (int)a.type);
    if (!elem_is_float(a.y_type)) return fail(ctx, RCD_ERR_INVALID_ARG, "y must be bf16, fp16 or fp32, got type %d", (int)a.y_type);
    RCD_TRY(check_sizes(ctx, a.rows, a.n, a.k));
    RCD_TRY(check_act(ctx, a.activation));
    if (a.type == RCD_ELEM_I8 && 16384LL * a.k > 0x7fffffffLL) return fail(ctx, RCD_ERR_UNSUPPORTED, "k=%lld: an int8 dot product could overflow int32", (long long)a.k);
    if (a.type != RCD_ELEM_I8 && (a.x_scales_dev_or_null || a.w_scales_dev_or_null)) return fail(ctx, RCD_ERR_INVALID_ARG, "scales are for int8 products");
    if (a.rows == 0 || a.n == 0) return RCD_OK;
    RCD_TRY(check_rows(ctx, "x", a.x_dev, a.rows, a.ldx, a.k, a.type));
    RCD_TRY(check_rows(ctx, "w", a.w_dev, a.n, a.ldw, a.k, a.type));
    RCD_TRY(check_rows(ctx, "y", a.y_dev, a.rows, a.ldy, a.n, a.y_type));
    RCD_TRY(check_rows(ctx, "residual", a.residual_dev_or_null, 0, a.ld_residual, a.n, a.y_type));
    RCD_TRY(check_rows(ctx, "preact", a.preact_dev_or_null, 0, a.ld_preact, a.n, a.y_type));
    RCD_TRY(check_floats(ctx, "x_scales", a.x_scales_dev_or_null));
    RCD_TRY(check_floats(ctx, "w_scales", a.w_scales_dev_or_null));
    return check_floats(ctx, "bias", a.bias_dev_or_null);
}
Product linear_product(const rcd_linear_args &a)
{
    Product p{};
    p.type = a.type;
    p.M = a.rows; p.N = a.n; p.K = a.k;
    p.a = {a.x_dev, a.ldx, false};
    p.b = {a.w_dev, a.ldw, false};
    p.out = {a.x_scales_dev_or_null, a.w_scales_dev_or_null, a.bias_dev_or_null, a.residual_dev_or_null, a.y_dev, a.preact_dev_or_null,
             a.ld_residual, a.ldy, a.ld_preact, a.y_type, (int32_t)a.activation};
    return p;
}

rcd_status check_back(rcd_ctx *ctx, const rcd_linear_back_args &a)
{
    if (a.type != RCD_ELEM_BF16 && a.type != RCD_ELEM_F16) return fail(ctx, RCD_ERR_INVALID_ARG, "type must be bf16 or fp16, got %d", (int)a.type);
    RCD_TRY(check_sizes(ctx, a.rows, a.n, a.k));
    RCD_TRY(check_act(ctx, a.activation));
    if (a.dw_dev_or_null && a.dw_type != a.type && a.dw_type != RCD_ELEM_F32) return fail(ctx, RCD_ERR_INVALID_ARG, "dw must have the type of x or be fp32, got type %d", (int)a.dw_type);
    RCD_TRY(check_floats(ctx, "dbias", a.dbias_dev_or_null));
    if (a.dw_dev_or_null) RCD_TRY(check_rows(ctx, "dw", a.dw_dev_or_null, a.n, a.ld_dw, a.k, a.dw_type));
    if (a.dx_dev_or_null && a.rows > 0) RCD_TRY(check_rows(ctx, "dx", a.dx_dev_or_null, a.rows, a.ld_dx, a.k, a.type));
    if (a.rows == 0 || a.n == 0) return RCD_OK;
    RCD_TRY(check_rows(ctx, "dy", a.dy_dev, a.rows, a.ld_dy, a.n, a.type));
    if (a.dw_dev_or_null) RCD_TRY(check_rows(ctx, "x", a.x_dev, a.rows, a.ldx, a.k, a.type));
    if (a.dx_dev_or_null) RCD_TRY(check_rows(ctx, "w", a.w_dev, a.n, a.ldw, a.k, a.type));
    if (a.activation != RCD_ACT_NONE) RCD_TRY(check_rows(ctx, "preact", a.preact_dev_or_null, a.rows, a.ld_preact, a.n, a.type));
    else if (a.preact_dev_or_null) return fail(ctx, RCD_ERR_INVALID_ARG, "preact is given, but there is no activation");
    return RCD_OK;
}

// The launches of a backward pass, and where their parts of the workspace lie.
struct BackPlan {
    bool slope, sums;                      // dz is written; the columns are summed
    int64_t ldDz, chunks;
    size_t dz, partial, dxWork, dwWork, bytes;
    Product dx, dw;
};
BackPlan back_plan(rcd_ctx *ctx, const rcd_linear_back_args &a, unsigned char *base)
{
    BackPlan b{};
    b.slope = a.activation != RCD_ACT_NONE && (a.dx_dev_or_null || a.dw_dev_or_null);
    b.sums = a.dbias_dev_or_null != nullptr;
    b.ldDz = (a.n + 7) / 8 * 8;
    b.chunks = (a.rows + kSlopeRows - 1) / kSlopeRows;
    b.dz = 0;
    b.partial = align_up(b.slope ? (size_t)(a.rows * b.ldDz) * 2 : 0);
    const size_t work = b.partial + align_up(b.sums ? (size_t)(b.chunks * a.n) * 4 : 0);
    const Operand dzRows = b.slope ? Operand{base + b.dz, b.ldDz, false} : Operand{a.dy_dev, a.ld_dy, false};
    b.dx.type = b.dw.type = a.type;
    b.dx.M = a.rows; b.dx.N = a.k; b.dx.K = a.n;
    b.dx.a = dzRows;
    b.dx.b = {a.w_dev, a.ldw, true};
    b.dx.out.y = a.dx_dev_or_null; b.dx.out.ldy = a.ld_dx; b.dx.out.type = a.type;
    b.dw.M = a.n; b.dw.N = a.k; b.dw.K = a.rows;
    b.dw.a = {dzRows.p, dzRows.ld, true};
    b.dw.b = {a.x_dev, a.ldx, true};
    b.dw.out.y = a.dw_dev_or_null; b.dw.out.ldy = a.ld_dw; b.dw.out.type = a.dw_type;
    b.dxWork = b.dwWork = work;            // (one product after the other: the same memory)
    size_t most = 0;
    if (a.dx_dev_or_null) most = std::max(most, product_workspace(ctx, b.dx));
    if (a.dw_dev_or_null) most = std::max(most, product_workspace(ctx, b.dw));
    b.bytes = work + align_up(most);
    return b;
}

}  // namespace

rcd_status check_sizes(rcd_ctx *ctx, int64_t rows, int64_t n, int64_t k)
{
    constexpr int64_t most = 1LL << 30;
    if (rows < 0 || rows > most || n < 0 || n > most) return fail(ctx, RCD_ERR_INVALID_ARG, "rows=%lld or n=%lld out of range", (long long)rows, (long long)n);
    if (k <= 0 || k > most) return fail(ctx, RCD_ERR_INVALID_ARG, "k=%lld must be from 1 to 2^30", (long long)k);
    return RCD_OK;
}
rcd_status check_floats(rcd_ctx *ctx, const char *name, const float *p)
{
    if (((uintptr_t)p) % 4) return fail(ctx, RCD_ERR_INVALID_ARG, "%s is not aligned to its type", name);
    return RCD_OK;
}

bool areas_meet(const Area &a, const Area &b) { return ranges_meet(a.p, a.rows, a.ld, a.len, a.bytes, b.p, b.rows, b.ld, b.len, b.bytes); }
rcd_status check_apart(rcd_ctx *ctx, const Area *out, int outs, const Area *in, int ins)
{
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < ins; ++j)
            if (areas_meet(out[i], in[j])) return fail(ctx, RCD_ERR_INVALID_ARG, "an output or the workspace overlaps another argument");
        for (int j = 0; j < i; ++j)
            if (areas_meet(out[i], out[j])) return fail(ctx, RCD_ERR_INVALID_ARG, "an output or the workspace overlaps another argument");
    }
    return RCD_OK;
}
rcd_status check_workspace(rcd_ctx *ctx, const void *ws, size_t have, size_t need)
{
    if (need == 0) return RCD_OK;
    if (!ws || have < need) return fail(ctx, RCD_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu needed", ws ? have : 0, need);
    if (((uintptr_t)ws) % kAlign) return fail(ctx, RCD_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    return RCD_OK;
}

rcd_status check_rows(rcd_ctx *ctx, const char *name, const void *p, int64_t rows, int64_t ld, int64_t len, rcd_elem type)
{
    if (rows > 0 && !p) return fail(ctx, RCD_ERR_INVALID_ARG, "%s is null", name);
    if (!p) return RCD_OK;
    if (ld < len || ld > (1LL << 40)) return fail(ctx, RCD_ERR_INVALID_ARG, "%s: rows lie %lld elements apart and are %lld long", name, (long long)ld, (long long)len);
    if (((uintptr_t)p) % elem_bytes(type)) return fail(ctx, RCD_ERR_INVALID_ARG, "%s is not aligned to its type", name);
    return RCD_OK;
}

rcd_status launch_column_sums(rcd_ctx *ctx, const float *partial, int64_t rows, int64_t d, float *out, cudaStream_t st)
{
    return launch_early(ctx, column_sums_kernel, dim3((unsigned)((d + 31) / 32)), 1024, st, partial, (int32_t)rows, d, out);
}

}  // namespace rcd

using namespace rcd;

extern "C" rcd_status rcd_linear_workspace_bytes(rcd_ctx *ctx, const rcd_linear_args *args, size_t *bytes_out)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    if (!args || !bytes_out) return fail(ctx, RCD_ERR_INVALID_ARG, "args or output is null");
    RCD_TRY(check_linear(ctx, *args));
    *bytes_out = args->rows == 0 || args->n == 0 ? 0 : product_workspace(ctx, linear_product(*args));
    return RCD_OK;
}

extern "C" rcd_status rcd_linear(rcd_ctx *ctx, const rcd_linear_args *args, void *workspace_dev, size_t workspace_bytes, void *cuda_stream)
{
    size_t need = 0;
    RCD_TRY(rcd_linear_workspace_bytes(ctx, args, &need));
    const rcd_linear_args &a = *args;
    begin_operator(ctx);
    if (a.rows == 0 || a.n == 0) return RCD_OK;
    RCD_TRY(check_workspace(ctx, workspace_dev, workspace_bytes, need));
    const int64_t eb = elem_bytes(a.type), yb = elem_bytes(a.y_type);
    const Area out[] = {{a.y_dev, a.rows, a.ldy, a.n, yb}, {a.preact_dev_or_null, a.rows, a.ld_preact, a.n, yb}, {need ? workspace_dev : nullptr, 1, (int64_t)need, (int64_t)need, 1}};
    const Area in[] = {{a.x_dev, a.rows, a.ldx, a.k, eb}, {a.w_dev, a.n, a.ldw, a.k, eb}, {a.residual_dev_or_null, a.rows, a.ld_residual, a.n, yb},
                       {a.bias_dev_or_null, 1, a.n, a.n, 4}, {a.x_scales_dev_or_null, 1, a.rows, a.rows, 4}, {a.w_scales_dev_or_null, 1, a.n, a.n, 4}};
    RCD_TRY(check_apart(ctx, out, 3, in, 6));
    RCD_CUDA(ctx, cudaSetDevice(ctx->device));
    return launch_product(ctx, linear_product(a), workspace_dev, (cudaStream_t)cuda_stream);
}

extern "C" rcd_status rcd_linear_backward_workspace_bytes(rcd_ctx *ctx, const rcd_linear_back_args *args, size_t *bytes_out)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    if (!args || !bytes_out) return fail(ctx, RCD_ERR_INVALID_ARG, "args or output is null");
    RCD_TRY(check_back(ctx, *args));
    *bytes_out = args->rows == 0 || args->n == 0 ? 0 : back_plan(ctx, *args, nullptr).bytes;
    return RCD_OK;
}

extern "C" rcd_status rcd_linear_backward(rcd_ctx *ctx, const rcd_linear_back_args *args, void *workspace_dev, size_t workspace_bytes,
                                          void *cuda_stream)
{
    size_t need = 0;
    RCD_TRY(rcd_linear_backward_workspace_bytes(ctx, args, &need));
    const rcd_linear_back_args &a = *args;
    RCD_TRY(check_workspace(ctx, workspace_dev, workspace_bytes, need));
    const int64_t eb = elem_bytes(a.type), wb = a.dw_dev_or_null ? elem_bytes(a.dw_type) : 1;
    const Area out[] = {{a.dx_dev_or_null, a.rows, a.ld_dx, a.k, eb}, {a.dw_dev_or_null, a.n, a.ld_dw, a.k, wb}, {a.dbias_dev_or_null, 1, a.n, a.n, 4},
                        {need ? workspace_dev : nullptr, 1, (int64_t)need, (int64_t)need, 1}};
    const Area in[] = {{a.dy_dev, a.rows, a.ld_dy, a.n, eb}, {a.preact_dev_or_null, a.rows, a.ld_preact, a.n, eb},
                       {a.dw_dev_or_null ? a.x_dev : nullptr, a.rows, a.ldx, a.k, eb}, {a.dx_dev_or_null ? a.w_dev : nullptr, a.n, a.ldw, a.k, eb}};
    RCD_TRY(check_apart(ctx, out, 4, in, 4));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    RCD_CUDA(ctx, cudaSetDevice(ctx->device));
    begin_operator(ctx);
    if (a.rows == 0 || a.n == 0) {         // sums over nothing
        if (a.n > 0 && a.dw_dev_or_null) RCD_CUDA(ctx, cudaMemset2DAsync(a.dw_dev_or_null, (size_t)(a.ld_dw * wb), 0, (size_t)(a.k * wb), (size_t)a.n, st));
        if (a.n > 0 && a.dbias_dev_or_null) RCD_CUDA(ctx, cudaMemsetAsync(a.dbias_dev_or_null, 0, (size_t)a.n * 4, st));
        if (a.rows > 0 && a.dx_dev_or_null) RCD_CUDA(ctx, cudaMemset2DAsync(a.dx_dev_or_null, (size_t)(a.ld_dx * eb), 0, (size_t)(a.k * eb), (size_t)a.rows, st));
        return RCD_OK;
    }
    unsigned char *ws = (unsigned char *)workspace_dev;
    const BackPlan b = back_plan(ctx, a, ws);
    if (b.slope || b.sums) {
        float *partial = b.sums ? (float *)(ws + b.partial) : nullptr;
        const int64_t per = rows_aligned(a.dy_dev, a.ld_dy, eb, 16) && rows_aligned(a.preact_dev_or_null, a.ld_preact, eb, 16) && a.n % 8 == 0 ? 256 : 32;
        const dim3 grid((unsigned)((a.n + per - 1) / per), (unsigned)std::min<int64_t>(b.chunks, 65535));
        auto run = [&](auto t) {
            using T = decltype(t);
            auto *kernel = per == 256 ? slope_kernel<T, 8> : slope_kernel<T, 1>;
            kernel<<<grid, 256, 0, st>>>((const T *)a.dy_dev, a.ld_dy, (const T *)a.preact_dev_or_null, a.ld_preact, a.rows, a.n, (int)a.activation,
                                                  b.slope ? (T *)(ws + b.dz) : nullptr, b.ldDz, partial);
        };
        if (a.type == RCD_ELEM_BF16) run(__nv_bfloat16());
        else run(__half());
        ctx->kernelLaunches++;
        RCD_CUDA(ctx, cudaGetLastError());
        if (b.sums) RCD_TRY(launch_column_sums(ctx, partial, b.chunks, a.n, a.dbias_dev_or_null, st));
    }
    if (a.dx_dev_or_null) RCD_TRY(launch_product(ctx, b.dx, ws + b.dxWork, st));
    if (a.dw_dev_or_null) RCD_TRY(launch_product(ctx, b.dw, ws + b.dwWork, st));
    return RCD_OK;
}
