// What the translation units of rcd_rms_norm and its gradients share.
#pragma once

#include <type_traits>

#include "rcd_linear.h"
#include "rcd_ring.h"
#include "rcd_tc.cuh"

namespace rcd {

struct NormParams {
    int64_t rows;
    int32_t d, group;                      // threads per row
    const void *x, *r, *w;
    int64_t ldx, ldr, lds, ldy;
    rcd_elem wType, yType;
    float eps, invScale;                   // invScale > 0: 8 bits on one scale
    bool normalize;
    void *sum, *y;
    float *scales;
    int32_t *status;
};

struct NormBackParams {
    int64_t rows;
    int32_t d, group;
    const void *dy, *h, *w, *dsum;
    int64_t ldDy, ldH, ldDsum, ldDx;
    rcd_elem wType;
    float eps;
    void *dx;
    float *partial;                        // [groups of the launch][d], or null
    int32_t *status;
};

inline int pow2_at_least(int64_t x)
{
    int g = 32;
    while (g < x) g *= 2;
    return g;
}

#ifdef __CUDACC__
__device__ __forceinline__ float warp_max_nan(float a)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    return a;
}
__device__ __forceinline__ float rstd_of(float sum, const NormParams &p)
{
    if (!p.normalize) return 1.0f;
    const float v = sum / (float)p.d + p.eps;
    return v > 0.0f ? 1.0f / sqrtf(v) : v == 0.0f ? 0.0f : v;
}
__device__ __forceinline__ float rstd_of(double sum, const NormParams &p)
{
    if (!p.normalize) return 1.0f;
    const double v = sum / (double)p.d + (double)p.eps;
    return v > 0.0 ? (float)(1.0 / sqrt(v)) : v == 0.0 ? 0.0f : (float)v;
}
// 127 / a, and the row's scale.  Where 127 / a would leave fp32 (a below 4e-37) it is that of the row times 2^64: the row is to be `raised` first.
constexpr float kRaise = 18446744073709551616.0f;
__device__ __forceinline__ float row_scale(float a, float rstd, float *scale, bool *raised)
{
    const bool fine = a < INFINITY;                            // (not so for a NaN)
    if (scale) *scale = fine ? rstd * a / 127.0f : NAN;
    *raised = a > 0.0f && a < 7.8886091e-31f;                  // 2^-100
    return fine && a > 0.0f ? 127.0f / (*raised ? a * kRaise : a) : 0.0f;
}
// To the nearest integer, halves to even; a NaN is 0.  (With a scale per row nothing is above 127.)
template <bool kCut>
__device__ __forceinline__ int8_t to_int8(float x)
{
    const int q = __float2int_rn(x);
    return (int8_t)(kCut ? max(-127, min(127, q)) : q);
}
// ---- many rows: every group of warps draws its rows through a ring of its own in shared memory ----
//
// With a row per CTA the loads stop while the row is reduced and stored, and CTAs come and go: 3.7 TB/s.  Here one CTA per SM stays;
// the first lane of a group (1 to 16 warps, up to 32 elements per lane) orders whole rows by bulk copies (cp.async.bulk, an mbarrier per
// slot) one to four rows ahead, so that some 150 KB per SM are always on their way.  A slot is ordered again as soon as its row lies in
// registers (forward) or has been gone through twice (backward).
constexpr int kRingWarps = 24;                     // (16: 132 us where 24 take 121, 50 000 x 2048 bf16 with residual to int8)
constexpr int kRingStages = 4;
constexpr int kRingBytes = 200 * 1024;
constexpr uint32_t kSpinLimit = 1u << 22;               // polls of ~64 ns: a quarter of a second

struct Ring { int warpsPerRow, groups, stages, slotBytes; };

struct RingShared {
    uint64_t bar[kRingWarps][kRingStages];
    float4 part[2][kRingWarps];
    int32_t abort;
};

// Bounded.  When it runs out the CTA goes on with what is there and says so in the status word: its groups stay in step (RingTurn: and
// order nothing more).
__device__ __forceinline__ bool ring_wait(uint64_t *bar, uint32_t parity, RingShared *sh, uint32_t limit = kSpinLimit)
{
    for (uint32_t spin = 0; spin < limit; ++spin) {
        if (mbar_test(bar, parity)) return true;
        if (spin > 64) {
            if (*(volatile int32_t *)&sh->abort) return false;
            __nanosleep(64);
        }
    }
    atomicExch(&sh->abort, 1);
    return false;
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(smem_addr(dst)), "l"(src), "r"(bytes), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void group_barrier(int group, int threads) { asm volatile("bar.sync %0, %1;" :: "r"(1 + group), "r"(threads) : "memory"); }

__device__ __forceinline__ void ring_begin(RingShared *sh, const Ring &ring)
{
    if (threadIdx.x == 0) {
        for (int g = 0; g < ring.groups; ++g)
            for (int k = 0; k < ring.stages; ++k) mbar_init(&sh->bar[g][k], 1);
        sh->abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
}
// After an expired wait: what was ordered lands before the CTA leaves.
__device__ __forceinline__ void ring_end(RingShared *sh, int32_t *status)
{
    __syncthreads();
    if (*(volatile int32_t *)&sh->abort) {
        let_copies_land();
        if (threadIdx.x == 0) atomicOr(status, kDevTimeout);
    }
}

#endif

// The ring's shape for rows of `streams` inputs of d elements: up to 32 elements per lane, as many warps as leave every group two slots.
inline Ring ring_shape(int64_t d, int64_t eb, int streams, bool sums)
{
    Ring g;
    const int64_t vec = 16 / eb, mostPerLane = 32 / vec;
    g.warpsPerRow = pow2_at_least((d / vec + mostPerLane - 1) / mostPerLane) / 32;
    g.slotBytes = (int)(((int64_t)streams * d * eb + 127) / 128 * 128);
    g.groups = std::max(1, kRingWarps / g.warpsPerRow);
    auto slots = [&]() { return kRingBytes / g.slotBytes / g.groups; };
    while (g.groups > 1 && (slots() < 2 || (sums && g.groups * d * 4 > kRingBytes))) --g.groups;     // (the groups' sums of columns take the ring's place at the end)
    g.stages = std::max(1, std::min(kRingStages, slots()));
    return g;
}
// Whether the ring is the faster form.  It takes 3.5 us more to set out than a row per CTA.  bf16, us, ring : row per CTA, rows of
//   512   forward with residual 9600 rows 9.8 : 7.0, 50 000 43.7 : 47   backward 600 9.3 : 8.5, 1200 9.8 : 10.8
//   2048  1200 6.8 : 6.1, 2400 8.8 : 9.8, 9600 24.5 : 40.7              600 11.4 : 11.9, 9600 35.3 : 41.6
//   4096  600 6.1 : 6.9, 1200 8.4 : 9.9                                 148 10.9 : 8.5, 296 11.1 : 11.9
//   16384 148 5.5 : 6.4, 600 17.2 : 23.2                                148 15.4 : 22.2
inline bool ring_pays(int64_t rows, int64_t d, bool back) { return rows * d >= (back ? 1LL << 20 : d >= 1024 ? 4LL << 20 : 12LL << 20); }

template <typename Kernel, typename Params>
rcd_status launch_ring(rcd_ctx *ctx, Kernel *kernel, const Params &p, const Ring &g, int ctas, size_t bytes, cudaStream_t st)
{
    RCD_CUDA(ctx, allow_shared(kernel, 220 * 1024));
    kernel<<<ctas, 32 * g.groups * g.warpsPerRow, bytes, st>>>(p, g);
    return RCD_OK;
}
inline int ring_ctas(const rcd_ctx *ctx, int64_t rows, const Ring &g) { return (int)std::min<int64_t>(ctx->smCount, (rows + g.groups - 1) / g.groups); }

// Accesses per lane and row, as the kernels are built for: 2 or 4 of 16-bit elements, 4 or 8 of fp32.
template <int VEC, typename Go>
rcd_status by_accesses(int64_t d, const Ring &g, Go go)
{
    constexpr int kFew = 16 / VEC, kMany = 32 / VEC;
    const int64_t per = (d / VEC + 32 * g.warpsPerRow - 1) / (32 * g.warpsPerRow);
    return per <= kFew ? go(std::integral_constant<int, kFew>()) : go(std::integral_constant<int, kMany>());
}

// The launches for many rows (rcd_norm_ring.cu, rcd_norm_ring_back.cu).
rcd_status launch_norm_ring(rcd_ctx *ctx, const NormParams &p, rcd_elem type, const Ring &g, cudaStream_t st);
rcd_status launch_norm_back_ring(rcd_ctx *ctx, const NormBackParams &p, rcd_elem type, const Ring &g, cudaStream_t st);

}  // namespace rcd
