// Root-mean-square norm of rows, with the residual's addition and output in 16, 32 or 8 bits, and its gradients.
//
//   h = x + r,  t = h w,  rstd = 1 / sqrt(mean(h^2) + eps),  y = t rstd      (rcd.h states the 8-bit forms)
//   g = dy w,   dx = rstd (g - h rstd^2 mean(g h)) + dsum,   dw = sum over rows of dy h rstd
//
// Both are bound by memory: every input is read once and every output written once.  A row belongs to a group of 32 to 512
// threads that keep it in registers (up to 32 elements each) from its load to its store; what the group has to agree on (a sum and a
// maximum; two sums) is one reduction by shuffles, and above a warp one exchange in shared memory.
#include "rcd_norm.cuh"

namespace rcd {

namespace {

constexpr int kRowThreads = 512;           // at most: 128 registers each
constexpr int kMostWidth = 16384;          // that many threads with 32 elements each

// A thread's part of a row's sum of squares and of its largest |t|; h becomes t = h w.
// One scale: the sum in 64 bits, whose rounding to rstd's 32 no order of summation changes (a value next to a border
// between two integers falls on the same side every time).
template <int VEC, int NV>
__device__ __forceinline__ void row_sums(const NormParams &p, float (&h)[NV][VEC], int tid, int G, double &sum, float &a)
{
    if (p.normalize) {
        if (p.invScale > 0.0f) {
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += (double)h[c][i] * (double)h[c][i];
        } else {
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[i & 3] = fmaf(h[c][i], h[c][i], s[i & 3]);
            sum = (double)((s[0] + s[1]) + (s[2] + s[3]));
        }
    }
    if (p.w) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
            if (col < p.d) {
                float w[VEC];
                load_typed<VEC>(w, p.w, col, p.wType);
#pragma unroll
                for (int i = 0; i < VEC; ++i) h[c][i] *= w[i];
            }
        }
    }
    if (p.yType == RCD_ELEM_I8 && p.invScale == 0.0f) {
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) a = max_nan(a, fabsf(h[c][i]));
    }
}
// t, the row's sum of squares and its largest |t| -> the row's output.
template <typename T, int VEC, int NV>
__device__ __forceinline__ void finish_row(const NormParams &p, float (&h)[NV][VEC], int64_t row, int tid, int G, double sum, float a)
{
    const bool rowScale = p.yType == RCD_ELEM_I8 && p.invScale == 0.0f;
    float rstd;
    if (p.invScale > 0.0f) rstd = rstd_of(sum, p);
    else rstd = rstd_of((float)sum, p);
    bool raised = false;
    const float inv = rowScale ? row_scale(a, rstd, tid == 0 ? p.scales + row : nullptr, &raised) : p.invScale;
    if (raised) {
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) h[c][i] *= kRaise;
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * G + tid) * VEC;
        if (col >= p.d) continue;
        if (p.yType == RCD_ELEM_I8) {
            Pack<int8_t, VEC> q;
#pragma unroll
            for (int i = 0; i < VEC; ++i) q.v[i] = to_int8<true>(rowScale ? h[c][i] * inv : (h[c][i] * rstd) * inv);
            *reinterpret_cast<Pack<int8_t, VEC> *>((int8_t *)p.y + row * p.ldy + col) = q;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) h[c][i] *= rstd;
            store_typed<VEC>(p.y, row * p.ldy + col, p.yType, h[c]);
        }
    }
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(kRowThreads) rms_norm_kernel(const __grid_constant__ NormParams p)
{
    __shared__ double shSum[32];
    __shared__ float shMax[32];
    const int G = p.group, tid = threadIdx.x & (G - 1), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / G) + threadIdx.x / G;
    const bool mine = row < p.rows;
    float h[NV][VEC];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * G + tid) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[c][i] = 0.0f;
        if (mine && col < p.d) {
            load_pack<VEC>(h[c], (const T *)p.x + row * p.ldx + col);
            if (p.r) {
                float r[VEC];
                load_pack<VEC>(r, (const T *)p.r + row * p.ldr + col);
#pragma unroll
                for (int i = 0; i < VEC; ++i) h[c][i] += r[i];
            }
            if (p.sum) store_pack<VEC>((T *)p.sum + row * p.lds + col, h[c]);
        }
    }
    double sum64 = 0.0;
    float a = 0.0f;
    row_sums<VEC, NV>(p, h, tid, G, sum64, a);
    sum64 = warp_sum(sum64);
    a = warp_max_nan(a);
    if (G > 32) {
        if (lane == 0) { shSum[warp] = sum64; shMax[warp] = a; }
        __syncthreads();
        const int first = (threadIdx.x / G) * (G / 32);
        sum64 = 0.0;
        a = 0.0f;
        for (int k = 0; k < G / 32; ++k) { sum64 += shSum[first + k]; a = max_nan(a, shMax[first + k]); }
    }
    if (mine) finish_row<T, VEC, NV>(p, h, row, tid, G, sum64, a);
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(kRowThreads) rms_norm_back_kernel(const __grid_constant__ NormBackParams p)
{
    __shared__ float2 sh[2][32];
    const int G = p.group, tid = threadIdx.x & (G - 1), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int perCta = blockDim.x / G, group = threadIdx.x / G;
    float dw[NV][VEC], w[NV][VEC];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * G + tid) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) { dw[c][i] = 0.0f; w[c][i] = 1.0f; }
        if (p.w && col < p.d) load_typed<VEC>(w[c], p.w, col, p.wType);
    }
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * perCta; row0 < p.rows; row0 += (int64_t)gridDim.x * perCta, turn ^= 1) {
        const int64_t row = row0 + group;
        const bool mine = row < p.rows;
        Pack<T, VEC> dy[NV], h[NV];                          // (as they are: half the registers of fp32)
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
            if (mine && col < p.d) {
                dy[c] = *reinterpret_cast<const Pack<T, VEC> *>((const T *)p.dy + row * p.ldDy + col);
                h[c] = *reinterpret_cast<const Pack<T, VEC> *>((const T *)p.h + row * p.ldH + col);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) { dy[c].v[i] = from_float<T>(0.0f); h[c].v[i] = from_float<T>(0.0f); }
            }
        }
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float x = to_float(h[c].v[i]);
                s.x = fmaf(x, x, s.x);
                s.y = fmaf(to_float(dy[c].v[i]) * w[c][i], x, s.y);
            }
        s.x = warp_sum(s.x);
        s.y = warp_sum(s.y);
        if (G > 32) {
            if (lane == 0) sh[turn][warp] = s;               // (two buffers: one barrier per row)
            __syncthreads();
            s = make_float2(0.0f, 0.0f);
            for (int k = 0; k < G / 32; ++k) { const float2 o = sh[turn][group * (G / 32) + k]; s.x += o.x; s.y += o.y; }
        }
        if (!mine) continue;
        const float v = s.x / (float)p.d + p.eps;
        const float rstd = v > 0.0f ? 1.0f / sqrtf(v) : v == 0.0f ? 0.0f : v;
        const float back = rstd * (rstd * (s.y / (float)p.d));       // (rstd^2 alone leaves fp32 where rstd does not)
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
            if (col >= p.d) continue;
            float dx[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float x = to_float(h[c].v[i]), y = to_float(dy[c].v[i]);
                dx[i] = rstd * (y * w[c][i] - x * back);
                dw[c][i] = fmaf(y, x * rstd, dw[c][i]);
            }
            if (p.dsum) {
                float o[VEC];
                load_pack<VEC>(o, (const T *)p.dsum + row * p.ldDsum + col);
#pragma unroll
                for (int i = 0; i < VEC; ++i) dx[i] += o[i];
            }
            store_pack<VEC>((T *)p.dx + row * p.ldDx + col, dx);
        }
    }
    if (p.partial) {
        float *to = p.partial + ((int64_t)blockIdx.x * perCta + group) * p.d;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (col + i < p.d) to[col + i] = dw[c][i];
        }
    }
}

// Threads per row and accesses per thread (a power of two of them): few rows get as many threads as the row has pieces, since then only
// latency counts; many rows four accesses per thread, which leaves fewer exchanges.
struct RowShape { int group, nv; };
RowShape row_shape(int64_t rows, int64_t d, int vec, int mostNv, int manyNv, int smCount)
{
    const int64_t pieces = (d + vec - 1) / vec;
    const int least = pow2_at_least((pieces + mostNv - 1) / mostNv);
    int group = std::min(kRowThreads, pow2_at_least(pieces));
    if (rows > 8 * smCount) group = std::min(group, pow2_at_least((pieces + manyNv - 1) / manyNv));
    RowShape s;
    s.group = std::max(group, least);
    s.nv = 1;
    while ((int64_t)s.nv * s.group < pieces) s.nv *= 2;
    return s;
}

rcd_status check_norm_sizes(rcd_ctx *ctx, int64_t rows, int64_t d, float eps)
{
    if (rows < 0 || rows > 0x7fffffffLL) return fail(ctx, RCD_ERR_INVALID_ARG, "rows=%lld out of range", (long long)rows);
    if (d <= 0) return fail(ctx, RCD_ERR_INVALID_ARG, "d=%lld must be positive", (long long)d);
    if (d > kMostWidth) return fail(ctx, RCD_ERR_UNSUPPORTED, "d=%lld: rows of at most %d elements are supported", (long long)d, kMostWidth);
    if (!(eps >= 0.0f) || !(eps < INFINITY)) return fail(ctx, RCD_ERR_INVALID_ARG, "eps must be finite and not negative");
    return RCD_OK;
}

template <typename T, int VEC, int NV>
void launch_norm(const NormParams &p, int threads, cudaStream_t st)
{
    const int perCta = threads / p.group;
    rms_norm_kernel<T, VEC, NV><<<(unsigned)((p.rows + perCta - 1) / perCta), threads, 0, st>>>(p);
}
// (no call needs more accesses: 512 threads with 32 elements each hold the widest row)
template <typename T, int VEC>
void launch_norm_nv(const NormParams &p, int nv, int threads, cudaStream_t st)
{
    if constexpr (VEC == 1) {
        if (nv <= 4) launch_norm<T, VEC, 4>(p, threads, st);
        else if (nv <= 16) launch_norm<T, VEC, 16>(p, threads, st);
        else launch_norm<T, VEC, 32>(p, threads, st);
    } else {
        if (nv == 1) launch_norm<T, VEC, 1>(p, threads, st);
        else if (nv == 2) launch_norm<T, VEC, 2>(p, threads, st);
        else if (nv == 4) launch_norm<T, VEC, 4>(p, threads, st);
        else if constexpr (VEC == 4) launch_norm<T, VEC, 8>(p, threads, st);
    }
}
template <typename T>
void launch_norm_type(NormParams &p, bool vectors, int smCount, cudaStream_t st)
{
    constexpr int VEC = 16 / sizeof(T);
    const RowShape s = vectors ? row_shape(p.rows, p.d, VEC, 32 / VEC, 4, smCount) : row_shape(p.rows, p.d, 1, 32, 32, smCount);
    p.group = s.group;
    const int threads = std::max(256, s.group);
    if (vectors) launch_norm_nv<T, VEC>(p, s.nv, threads, st);
    else launch_norm_nv<T, 1>(p, s.nv, threads, st);
}

rcd_status norm_rows(rcd_ctx *ctx, const rcd_norm_args &a, bool normalize, cudaStream_t st)
{
    if (!elem_is_float(a.x_type)) return fail(ctx, RCD_ERR_INVALID_ARG, "x must be bf16, fp16 or fp32, got type %d", (int)a.x_type);
    if (!elem_is_float(a.y_type) && a.y_type != RCD_ELEM_I8) return fail(ctx, RCD_ERR_INVALID_ARG, "unknown type %d of y", (int)a.y_type);
    if (a.weight_dev_or_null && !elem_is_float(a.weight_type)) return fail(ctx, RCD_ERR_INVALID_ARG, "unknown type %d of the weight", (int)a.weight_type);
    RCD_TRY(check_norm_sizes(ctx, a.rows, a.d, a.eps));
    const bool i8 = a.y_type == RCD_ELEM_I8;
    if (!i8 && (a.scales_dev_or_null || a.scale != 0.0f)) return fail(ctx, RCD_ERR_INVALID_ARG, "scales are for int8 output");
    if (i8 && a.scale != 0.0f) {
        if (!(a.scale > 0.0f) || !(a.scale < INFINITY) || !(1.0f / a.scale < INFINITY)) return fail(ctx, RCD_ERR_INVALID_ARG, "scale must be 0, or positive with a finite reciprocal");
        if (a.scales_dev_or_null) return fail(ctx, RCD_ERR_INVALID_ARG, "one scale for all rows, or one for each: not both");
    }
    if (i8 && a.scale == 0.0f && !a.scales_dev_or_null && a.rows > 0) return fail(ctx, RCD_ERR_INVALID_ARG, "scales is null");
    if (((uintptr_t)a.scales_dev_or_null) % 4) return fail(ctx, RCD_ERR_INVALID_ARG, "scales are not aligned to their type");
    RCD_TRY(check_rows(ctx, "x", a.x_dev, a.rows, a.ldx, a.d, a.x_type));
    RCD_TRY(check_rows(ctx, "y", a.y_dev, a.rows, a.ldy, a.d, a.y_type));
    RCD_TRY(check_rows(ctx, "residual", a.residual_dev_or_null, 0, a.ld_residual, a.d, a.x_type));
    RCD_TRY(check_rows(ctx, "sum", a.sum_dev_or_null, 0, a.ld_sum, a.d, a.x_type));
    if (a.weight_dev_or_null) RCD_TRY(check_rows(ctx, "weight", a.weight_dev_or_null, 1, a.d, a.d, a.weight_type));
    const int64_t xb = elem_bytes(a.x_type), yb = elem_bytes(a.y_type);
    auto meets = [&](const void *out, int64_t rows, int64_t ld, int64_t len, int64_t bytes, bool isSum) {
        if (ranges_meet(out, rows, ld, len, bytes, a.x_dev, a.rows, a.ldx, a.d, xb) && !(isSum && out == a.x_dev && ld == a.ldx)) return true;
        if (ranges_meet(out, rows, ld, len, bytes, a.residual_dev_or_null, a.rows, a.ld_residual, a.d, xb) && !(isSum && out == a.residual_dev_or_null && ld == a.ld_residual)) return true;
        return ranges_meet(out, rows, ld, len, bytes, a.weight_dev_or_null, 1, a.d, a.d, a.weight_dev_or_null ? elem_bytes(a.weight_type) : 1);
    };
    if (meets(a.y_dev, a.rows, a.ldy, a.d, yb, false) || meets(a.sum_dev_or_null, a.rows, a.ld_sum, a.d, xb, true) ||
        meets(a.scales_dev_or_null, 1, a.rows, a.rows, 4, false) ||
        ranges_meet(a.y_dev, a.rows, a.ldy, a.d, yb, a.sum_dev_or_null, a.rows, a.ld_sum, a.d, xb) ||
        ranges_meet(a.y_dev, a.rows, a.ldy, a.d, yb, a.scales_dev_or_null, 1, a.rows, a.rows, 4) ||
        ranges_meet(a.sum_dev_or_null, a.rows, a.ld_sum, a.d, xb, a.scales_dev_or_null, 1, a.rows, a.rows, 4))
        return fail(ctx, RCD_ERR_INVALID_ARG, "an output overlaps another argument");
    begin_operator(ctx);
    if (a.rows == 0) return RCD_OK;

    RCD_CUDA(ctx, cudaSetDevice(ctx->device));
    NormParams p{};
    p.rows = a.rows;
    p.d = (int32_t)a.d;
    p.x = a.x_dev; p.r = a.residual_dev_or_null; p.w = a.weight_dev_or_null;
    p.ldx = a.ldx; p.ldr = a.ld_residual; p.lds = a.ld_sum; p.ldy = a.ldy;
    p.wType = a.weight_type; p.yType = a.y_type;
    p.eps = a.eps;
    p.invScale = i8 && a.scale > 0.0f ? 1.0f / a.scale : 0.0f;
    p.normalize = normalize;
    p.sum = a.sum_dev_or_null; p.y = a.y_dev; p.scales = a.scales_dev_or_null;
    p.status = ctx->statusOwn + kOperatorStatus;
    const int64_t vec = 16 / xb;
    const bool vectors = a.d % vec == 0 && rows_aligned(p.x, p.ldx, xb, 16) && rows_aligned(p.r, p.ldr, xb, 16) && rows_aligned(p.sum, p.lds, xb, 16) &&
                         rows_aligned(p.y, p.ldy, yb, std::min<int64_t>(16, vec * yb)) &&
                         rows_aligned(p.w, 0, 1, p.w ? std::min<int64_t>(16, vec * elem_bytes(a.weight_type)) : 1);
    const Ring ring = vectors ? ring_shape(a.d, xb, a.residual_dev_or_null ? 2 : 1, false) : Ring{};
    if (vectors && ring_pays(a.rows, a.d, false)) {
        RCD_TRY(launch_norm_ring(ctx, p, a.x_type, ring, st));
    }
    else if (a.x_type == RCD_ELEM_BF16) launch_norm_type<__nv_bfloat16>(p, vectors, ctx->smCount, st);
    else if (a.x_type == RCD_ELEM_F16) launch_norm_type<__half>(p, vectors, ctx->smCount, st);
    else launch_norm_type<float>(p, vectors, ctx->smCount, st);
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return RCD_OK;
}

// The backward pass runs as many CTAs as fit the SMs at once, each with its share of the rows.
struct BackShape { RowShape s; int threads, ctas; bool vectors, useRing; Ring ring; int64_t partialRows; };
BackShape back_shape(const rcd_ctx *ctx, const rcd_norm_back_args &a)
{
    BackShape b{};
    const int64_t eb = elem_bytes(a.type), vec = 16 / eb;
    b.vectors = a.d % vec == 0 && rows_aligned(a.dy_dev, a.ld_dy, eb, 16) && rows_aligned(a.h_dev, a.ld_h, eb, 16) && rows_aligned(a.dsum_dev_or_null, a.ld_dsum, eb, 16) &&
                rows_aligned(a.dx_dev, a.ld_dx, eb, 16) &&
                rows_aligned(a.weight_dev_or_null, 0, 1, a.weight_dev_or_null ? std::min<int64_t>(16, vec * elem_bytes(a.weight_type)) : 1);
    if (b.vectors) {
        b.ring = ring_shape(a.d, eb, a.dsum_dev_or_null ? 3 : 2, true);
        // (weights of the rows' type or fp32)
        b.useRing = ring_pays(a.rows, a.d, true) && (!a.weight_dev_or_null || a.weight_type == a.type || a.weight_type == RCD_ELEM_F32);
        if (b.useRing) {
            b.partialRows = ring_ctas(ctx, a.rows, b.ring);
            return b;
        }
    }
    b.s = b.vectors ? row_shape(a.rows, a.d, (int)vec, (int)(32 / vec), 1, ctx->smCount) : row_shape(a.rows, a.d, 1, 32, 8, ctx->smCount);
    b.threads = std::max(256, b.s.group);
    const int perCta = b.threads / b.s.group;
    b.ctas = (int)std::min<int64_t>((a.rows + perCta - 1) / perCta, (int64_t)ctx->smCount * (1024 / b.threads));
    b.partialRows = (int64_t)b.ctas * perCta;
    return b;
}

template <typename T, int VEC, int NV>
void launch_back(const NormBackParams &p, const BackShape &b, cudaStream_t st) { rms_norm_back_kernel<T, VEC, NV><<<b.ctas, b.threads, 0, st>>>(p); }
template <typename T>
void launch_back_type(const NormBackParams &p, const BackShape &b, cudaStream_t st)
{
    constexpr int VEC = 16 / sizeof(T);
    const int nv = b.s.nv;
    if (b.vectors) {
        if (nv == 1) launch_back<T, VEC, 1>(p, b, st);
        else if (nv == 2) launch_back<T, VEC, 2>(p, b, st);
        else if (nv == 4) launch_back<T, VEC, 4>(p, b, st);
        else if constexpr (VEC == 4) launch_back<T, VEC, 8>(p, b, st);
    } else {
        if (nv <= 4) launch_back<T, 1, 4>(p, b, st);
        else if (nv <= 8) launch_back<T, 1, 8>(p, b, st);
        else launch_back<T, 1, 32>(p, b, st);
    }
}

rcd_status check_norm_back(rcd_ctx *ctx, const rcd_norm_back_args &a)
{
    if (!elem_is_float(a.type)) return fail(ctx, RCD_ERR_INVALID_ARG, "type must be bf16, fp16 or fp32, got %d", (int)a.type);
    if (a.weight_dev_or_null && !elem_is_float(a.weight_type)) return fail(ctx, RCD_ERR_INVALID_ARG, "unknown type %d of the weight", (int)a.weight_type);
    RCD_TRY(check_norm_sizes(ctx, a.rows, a.d, a.eps));
    RCD_TRY(check_rows(ctx, "dy", a.dy_dev, a.rows, a.ld_dy, a.d, a.type));
    RCD_TRY(check_rows(ctx, "h", a.h_dev, a.rows, a.ld_h, a.d, a.type));
    RCD_TRY(check_rows(ctx, "dsum", a.dsum_dev_or_null, 0, a.ld_dsum, a.d, a.type));
    RCD_TRY(check_rows(ctx, "dx", a.dx_dev, a.rows, a.ld_dx, a.d, a.type));
    if (a.weight_dev_or_null) RCD_TRY(check_rows(ctx, "weight", a.weight_dev_or_null, 1, a.d, a.d, a.weight_type));
    if (((uintptr_t)a.dweight_dev_or_null) % 4) return fail(ctx, RCD_ERR_INVALID_ARG, "dweight is not aligned to its type");
    return RCD_OK;
}

}  // namespace

}  // namespace rcd

using namespace rcd;

extern "C" rcd_status rcd_rms_norm(rcd_ctx *ctx, const rcd_norm_args *args, void *cuda_stream)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    if (!args) return fail(ctx, RCD_ERR_INVALID_ARG, "args is null");
    return norm_rows(ctx, *args, true, (cudaStream_t)cuda_stream);
}

extern "C" rcd_status rcd_quantize_rows(rcd_ctx *ctx, const void *x_dev, rcd_elem x_type, int64_t rows, int64_t d, int64_t ldx,
                                        int8_t *q_dev, int64_t ldq, float *scales_dev, void *cuda_stream)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    rcd_norm_args a{};
    a.rows = rows; a.d = d;
    a.x_type = x_type; a.x_dev = x_dev; a.ldx = ldx;
    a.y_type = RCD_ELEM_I8; a.y_dev = q_dev; a.ldy = ldq;
    a.scales_dev_or_null = scales_dev;
    return norm_rows(ctx, a, false, (cudaStream_t)cuda_stream);
}

extern "C" rcd_status rcd_rms_norm_backward_workspace_bytes(rcd_ctx *ctx, const rcd_norm_back_args *args, size_t *bytes_out)
{
    if (!ctx) return RCD_ERR_INVALID_ARG;
    if (!args || !bytes_out) return fail(ctx, RCD_ERR_INVALID_ARG, "args or output is null");
    RCD_TRY(check_norm_back(ctx, *args));
    *bytes_out = args->dweight_dev_or_null && args->rows > 0 ? align_up((size_t)back_shape(ctx, *args).partialRows * (size_t)args->d * sizeof(float)) : 0;
    return RCD_OK;
}

extern "C" rcd_status rcd_rms_norm_backward(rcd_ctx *ctx, const rcd_norm_back_args *args, void *workspace_dev, size_t workspace_bytes,
                                            void *cuda_stream)
{
    size_t need = 0;
    RCD_TRY(rcd_rms_norm_backward_workspace_bytes(ctx, args, &need));
    const rcd_norm_back_args &a = *args;
    if (workspace_bytes < need || (need && !workspace_dev)) return fail(ctx, RCD_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu needed", workspace_dev ? workspace_bytes : 0, need);
    if (need && ((uintptr_t)workspace_dev) % kAlign) return fail(ctx, RCD_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const int64_t eb = elem_bytes(a.type);
    const void *const out[3] = {a.dx_dev, a.dweight_dev_or_null, need ? workspace_dev : nullptr};
    const int64_t outRows[3] = {a.rows, 1, 1}, outLd[3] = {a.ld_dx, a.d, (int64_t)need}, outLen[3] = {a.d, a.d, (int64_t)need}, outBytes[3] = {eb, 4, 1};
    for (int k = 0; k < 3; ++k) {
        bool meets = ranges_meet(out[k], outRows[k], outLd[k], outLen[k], outBytes[k], a.dy_dev, a.rows, a.ld_dy, a.d, eb) ||
                     ranges_meet(out[k], outRows[k], outLd[k], outLen[k], outBytes[k], a.h_dev, a.rows, a.ld_h, a.d, eb) ||
                     ranges_meet(out[k], outRows[k], outLd[k], outLen[k], outBytes[k], a.dsum_dev_or_null, a.rows, a.ld_dsum, a.d, eb) ||
                     ranges_meet(out[k], outRows[k], outLd[k], outLen[k], outBytes[k], a.weight_dev_or_null, 1, a.d, a.d, a.weight_dev_or_null ? elem_bytes(a.weight_type) : 1);
        for (int j = 0; j < k; ++j) meets = meets || ranges_meet(out[k], outRows[k], outLd[k], outLen[k], outBytes[k], out[j], outRows[j], outLd[j], outLen[j], outBytes[j]);
        if (meets) return fail(ctx, RCD_ERR_INVALID_ARG, "an output or the workspace overlaps another argument");
    }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    RCD_CUDA(ctx, cudaSetDevice(ctx->device));
    begin_operator(ctx);
    if (a.rows == 0) {
        if (a.dweight_dev_or_null) RCD_CUDA(ctx, cudaMemsetAsync(a.dweight_dev_or_null, 0, (size_t)a.d * sizeof(float), st));
        return RCD_OK;
    }
    const BackShape b = back_shape(ctx, a);
    NormBackParams p{};
    p.rows = a.rows; p.d = (int32_t)a.d; p.group = b.s.group;
    p.dy = a.dy_dev; p.h = a.h_dev; p.w = a.weight_dev_or_null; p.dsum = a.dsum_dev_or_null;
    p.ldDy = a.ld_dy; p.ldH = a.ld_h; p.ldDsum = a.ld_dsum; p.ldDx = a.ld_dx;
    p.wType = a.weight_type;
    p.eps = a.eps;
    p.dx = a.dx_dev;
    p.partial = a.dweight_dev_or_null ? (float *)workspace_dev : nullptr;
    p.status = ctx->statusOwn + kOperatorStatus;
    if (b.useRing) {
        RCD_TRY(launch_norm_back_ring(ctx, p, a.type, b.ring, st));
    }
    else if (a.type == RCD_ELEM_BF16) launch_back_type<__nv_bfloat16>(p, b, st);
    else if (a.type == RCD_ELEM_F16) launch_back_type<__half>(p, b, st);
    else launch_back_type<float>(p, b, st);
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return p.partial ? launch_column_sums(ctx, p.partial, b.partialRows, a.d, a.dweight_dev_or_null, st) : RCD_OK;
}
