// Matrix product of few rows (rcd_linear up to 32): every weight is read for at most 32 rows, so the weights' way from memory is the
// bound (2048 x 2048 bf16: 1.3 us), and before it a call's launches.  One launch, no tensor maps and no workspace.
//
// A CTA takes 16 rows of the weights, its 8 or 16 warps share the k axis in pieces of 64 bytes per row.  A thread loads 16 bytes of two weight
// rows and of one row in eight of x straight into the fragments of mma.sync (m16n8k16, int8 m16n8k32): both operands hold the same k in the same place,
// and the order of k is the same for both, so that no fragment needs to be put together through shared memory.  (The fifth-generation tensor
// cores want their operands in shared memory and an accumulator of 128 rows; nothing of their rate is needed here.)  The warps' sums meet in shared
// memory, fp32 ones after every 512 k in a register of their own, since the tensor cores cut sums off (see rcd_linear_tc.cu).
#include "rcd_act.cuh"
#include "rcd_linear.h"

namespace rcd {

namespace {

constexpr int kFewRows = 32;
constexpr int kTileW = 16;                              // weight rows per CTA

struct FewParams {
    const void *x, *w;
    int64_t ldx, ldw;
    int32_t M, N, kBytes;
    Epilogue e;
};

template <typename T, bool kInt8>
__device__ __forceinline__ void mma_few(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (kInt8) {
        int32_t d[4] = {__float_as_int(c[0]), __float_as_int(c[1]), __float_as_int(c[2]), __float_as_int(c[3])};
        asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = __int_as_float(d[i]);
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    } else {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
}

// kBlocks: groups of eight rows of x.
template <typename T, int kBlocks>
__global__ void __launch_bounds__(512) few_rows_kernel(const __grid_constant__ FewParams p)
{
    constexpr bool kInt8 = sizeof(T) == 1;
    constexpr int kUnroll = kBlocks == 4 ? 2 : 4;       // pieces under way per warp
    extern __shared__ float sums[];                     // [warps][kBlocks * 8][kTileW]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, g = lane >> 2, t = lane & 3;
    const int n0 = blockIdx.x * kTileW;
    const unsigned char *const wA = (const unsigned char *)p.w + (int64_t)min(n0 + g, p.N - 1) * p.ldw * (int64_t)sizeof(T);
    const unsigned char *const wB = (const unsigned char *)p.w + (int64_t)min(n0 + g + 8, p.N - 1) * p.ldw * (int64_t)sizeof(T);
    const unsigned char *x[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) x[b] = (const unsigned char *)p.x + (int64_t)min(b * 8 + g, p.M - 1) * p.ldx * (int64_t)sizeof(T);    // (rows past the last: their sums go nowhere)
    float acc[kBlocks][4], total[kBlocks][4];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) { acc[b][i] = 0.0f; total[b][i] = 0.0f; }
    const int step = warps * 64;
    int since = 0;
    for (int k0 = warp * 64; k0 < p.kBytes; k0 += step * kUnroll) {
        uint4 a[kUnroll], c[kUnroll], v[kUnroll][kBlocks];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = k0 + u * step + t * 16;
            const uint4 zero = make_uint4(0, 0, 0, 0);
            const bool in = at < p.kBytes;
            a[u] = in ? __ldg((const uint4 *)(wA + at)) : zero;
            c[u] = in ? __ldg((const uint4 *)(wB + at)) : zero;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) v[u][b] = in ? __ldg((const uint4 *)(x[b] + at)) : zero;
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                mma_few<T, kInt8>(acc[b], a[u].x, c[u].x, a[u].y, c[u].y, v[u][b].x, v[u][b].y);
                mma_few<T, kInt8>(acc[b], a[u].z, c[u].z, a[u].w, c[u].w, v[u][b].z, v[u][b].w);
            }
        if constexpr (!kInt8) {
            since += kUnroll * 32;
            if (since >= 512) {
                since = 0;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) { total[b][i] += acc[b][i]; acc[b][i] = 0.0f; }
            }
        }
    }
    // a lane's sums: weight rows g and g + 8, rows 2 t and 2 t + 1 of x
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sums[(warp * kBlocks * 8 + b * 8 + 2 * t + (i & 1)) * kTileW + g + (i >> 1) * 8] = kInt8 ? acc[b][i] : total[b][i] + acc[b][i];
    __syncthreads();
    const Epilogue &e = p.e;
    for (int i = threadIdx.x; i < p.M * kTileW; i += blockDim.x) {
        const int m = i / kTileW, n = n0 + i % kTileW;
        if (n >= p.N) continue;
        float z[1];
        if constexpr (kInt8) {
            int32_t s = 0;
            for (int k = 0; k < warps; ++k) s += __float_as_int(sums[k * kBlocks * 8 * kTileW + i]);
            z[0] = (float)s;
            if (e.xs) z[0] *= e.xs[m];
            if (e.ws) z[0] *= e.ws[n];
        } else {
            float s = 0.0f;
            for (int k = 0; k < warps; ++k) s += sums[k * kBlocks * 8 * kTileW + i];
            z[0] = s;
        }
        if (e.bias) z[0] += e.bias[n];
        if (e.z) store_typed<1>(e.z, m * e.ldz + n, e.type, z);
        activate(z, e.act);
        if (e.residual) {
            float r[1];
            load_typed<1>(r, e.residual, m * e.ldr + n, e.type);
            z[0] += r[0];
        }
        store_typed<1>(e.y, m * e.ldy + n, e.type, z);
    }
}

template <typename T>
void launch_typed(const FewParams &p, int threads, cudaStream_t st)
{
    const unsigned grid = (unsigned)((p.N + kTileW - 1) / kTileW);
    const int blocks = p.M <= 8 ? 1 : p.M <= 16 ? 2 : 4;
    const size_t bytes = (size_t)(threads / 32) * blocks * 8 * kTileW * sizeof(float);          // at most 32 KB
    if (blocks == 1) few_rows_kernel<T, 1><<<grid, threads, bytes, st>>>(p);
    else if (blocks == 2) few_rows_kernel<T, 2><<<grid, threads, bytes, st>>>(p);
    else few_rows_kernel<T, 4><<<grid, threads, bytes, st>>>(p);
}

}  // namespace

// Up to 8 rows always, up to 16 where the weights are at most 64 MB, up to 32 at most 24 MB: x comes from L1 once per 16 weight rows, and
// beyond that its way is longer than the weights'.  us here : with the tiles of rcd_linear_tc.cu, weights of
//   2 MB (512 x 2048 bf16)   1 row 3.2 : 8.5     16 rows 3.7 : 8.6     32 rows 5.0 : 9.0
//   8 MB (2048 x 2048 bf16)        3.7 : 10.4            4.5 : 10.5            5.7 : 9.9
//   16 MB (4096 x 4096 int8)       4.3 : 12.8            7.1 : 11.7            9.7 : 14.6
//   32 MB (4096 x 4096 bf16)       10.6 : 19.1           14.1 : 17.4           18.4 : 17.3
//   64 MB (4096 x 8192 bf16)       17.2 : 23.3           23.2 : 23.0           30.6 : 23.1
//   128 MB (8192 x 8192 bf16)      30.6 : 35.6           40.7 : 35.8           50.7 : 33.9
bool few_rows(const Product &p)
{
    const int64_t eb = elem_bytes(p.type), weights = p.N * p.K * eb;
    return p.M <= kFewRows && (p.M <= 8 || weights <= (p.M <= 16 ? 64LL << 20 : 24LL << 20)) && !p.a.across && !p.b.across && p.K * eb % 16 == 0 &&
           p.K * eb < (1LL << 30) && rows_aligned(p.a.p, p.a.ld, eb, 16) && rows_aligned(p.b.p, p.b.ld, eb, 16);
}

rcd_status launch_few_rows(rcd_ctx *ctx, const Product &p, cudaStream_t st)
{
    FewParams q{};
    q.x = p.a.p; q.w = p.b.p;
    q.ldx = p.a.ld; q.ldw = p.b.ld;
    q.M = (int32_t)p.M; q.N = (int32_t)p.N;
    q.kBytes = (int32_t)(p.K * elem_bytes(p.type));
    q.e = p.out;
    // (twice the warps where there are at most two CTAs per SM and every warp still has a piece)
    const int threads = (p.N + kTileW - 1) / kTileW <= 2 * ctx->smCount && q.kBytes >= 1024 ? 512 : 256;
    if (p.type == RCD_ELEM_I8) launch_typed<int8_t>(q, threads, st);
    else if (p.type == RCD_ELEM_BF16) launch_typed<__nv_bfloat16>(q, threads, st);
    else launch_typed<__half>(q, threads, st);
    ctx->kernelLaunches++;
    RCD_CUDA(ctx, cudaGetLastError());
    return RCD_OK;
}

}  // namespace rcd
