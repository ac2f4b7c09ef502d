// Gradients of the root-mean-square norm of many rows: the kernel of rcd_norm.cuh's ring.
#include "rcd_norm.cuh"

namespace rcd {

namespace {

// Backward: the row is gone through twice, for the sums and for the gradients, from its slot.  What a lane adds up for dw stays in
// its registers; the groups of a CTA join theirs in the ring's memory at the end, one row of `partial` per CTA.
template <typename T, int NV, typename W, bool kWeight>
__global__ void __launch_bounds__(32 * kRingWarps, 1) rms_norm_back_ring_kernel(const __grid_constant__ NormBackParams p, const __grid_constant__ Ring ring)
{
    constexpr int VEC = 16 / sizeof(T), P = VEC / 2;
    [[maybe_unused]] const W *const weights = (const W *)p.w;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ RingShared sh;
    ring_begin(&sh, ring);
    const int lane = threadIdx.x & 31, gw = ring.warpsPerRow, G = 32 * gw;
    const int group = (threadIdx.x >> 5) / gw, inGroup = (threadIdx.x >> 5) % gw, tid = inGroup * 32 + lane;
    const int64_t first = (int64_t)group * gridDim.x + blockIdx.x, step = (int64_t)gridDim.x * ring.groups;
    const uint32_t rowBytes = (uint32_t)p.d * sizeof(T);
    unsigned char *const slots = smem + (size_t)group * ring.stages * ring.slotBytes;
    auto order = [&](int64_t row, int slot) {
        if (row >= p.rows) return;
        unsigned char *const at = slots + slot * ring.slotBytes;
        mbar_expect_tx(&sh.bar[group][slot], p.dsum ? 3 * rowBytes : 2 * rowBytes);
        bulk_load(at, (const T *)p.dy + row * p.ldDy, rowBytes, &sh.bar[group][slot]);
        bulk_load(at + rowBytes, (const T *)p.h + row * p.ldH, rowBytes, &sh.bar[group][slot]);
        if (p.dsum) bulk_load(at + 2 * rowBytes, (const T *)p.dsum + row * p.ldDsum, rowBytes, &sh.bar[group][slot]);
    };
    if (tid == 0)
        for (int k = 0; k < ring.stages; ++k) order(first + k * step, k);
    Two dw[NV][P];
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int i = 0; i < P; ++i) dw[c][i] = two(0.0f, 0.0f);
    RingTurn at;
    int turn = 0;
    for (int64_t row = first; row < p.rows; row += step, turn ^= 1) {
        at.waited(ring_wait(&sh.bar[group][at.slot], at.parity, &sh));
        const T *const dyRow = reinterpret_cast<const T *>(slots + at.slot * ring.slotBytes), *const hRow = dyRow + p.d, *const sumRow = hRow + p.d;
        Two hh = two(0.0f, 0.0f), gh = hh;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
            if (col < p.d) {
                Two g[P], h[P];
                load_twos<P>(g, dyRow + col);
                load_twos<P>(h, hRow + col);
                if constexpr (kWeight) {
                    Two w[P];
                    load_twos<P>(w, weights + col);
#pragma unroll
                    for (int i = 0; i < P; ++i) g[i] = mul2(g[i], w[i]);
                }
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    hh = fma2(h[i], h[i], hh);
                    gh = fma2(g[i], h[i], gh);
                }
            }
        }
        const float2 hs = parts(hh), gs = parts(gh);
        float2 s = make_float2(warp_sum(hs.x + hs.y), warp_sum(gs.x + gs.y));
        if (gw > 1) {
            if (lane == 0) sh.part[turn][threadIdx.x >> 5] = make_float4(s.x, s.y, 0.0f, 0.0f);
            group_barrier(group, G);
            s = make_float2(0.0f, 0.0f);
            for (int k = 0; k < gw; ++k) {
                const float4 o = sh.part[turn][group * gw + k];
                s.x += o.x;
                s.y += o.y;
            }
        }
        const float v = s.x / (float)p.d + p.eps;
        const float rstd = v > 0.0f ? 1.0f / sqrtf(v) : v == 0.0f ? 0.0f : v;
        const float back = rstd * (rstd * (s.y / (float)p.d));       // (rstd^2 alone leaves fp32 where rstd does not)
        const Two r2 = two(rstd, rstd), b2 = two(-back, -back);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
            if (col < p.d) {
                Two g[P], h[P];
                load_twos<P>(g, dyRow + col);
                load_twos<P>(h, hRow + col);
#pragma unroll
                for (int i = 0; i < P; ++i) dw[c][i] = fma2(g[i], mul2(h[i], r2), dw[c][i]);
                if constexpr (kWeight) {
                    Two w[P];
                    load_twos<P>(w, weights + col);
#pragma unroll
                    for (int i = 0; i < P; ++i) g[i] = mul2(g[i], w[i]);
                }
#pragma unroll
                for (int i = 0; i < P; ++i) g[i] = mul2(r2, fma2(h[i], b2, g[i]));
                if (p.dsum) {
                    Two o[P];
                    load_twos<P>(o, sumRow + col);
#pragma unroll
                    for (int i = 0; i < P; ++i) g[i] = add2(g[i], o[i]);
                }
                store_twos<P>((T *)p.dx + row * p.ldDx + col, g);
            }
        }
        if (gw == 1) __syncwarp();
        else group_barrier(group, G);
        if (tid == 0 && at.may_order()) order(row + ring.stages * step, at.slot);
        at.next(ring.stages);
    }
    ring_end(&sh, p.status);
    if (p.partial) {                                        // (every copy has landed and been read)
        float *const all = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
            if (col < p.d) store_twos<P>(all + (size_t)group * p.d + col, dw[c]);
        }
        __syncthreads();
        for (int col = threadIdx.x; col < p.d; col += blockDim.x) {
            float o = 0.0f;
            for (int g = 0; g < ring.groups; ++g) o += all[(size_t)g * p.d + col];
            p.partial[(int64_t)blockIdx.x * p.d + col] = o;
        }
    }
}

template <typename T>
rcd_status launch_typed(rcd_ctx *ctx, const NormBackParams &p, const Ring &g, cudaStream_t st)
{
    const int ctas = ring_ctas(ctx, p.rows, g);
    const size_t bytes = std::max((size_t)g.groups * g.stages * g.slotBytes, p.partial ? (size_t)g.groups * p.d * 4 : 0);
    return by_accesses<16 / (int)sizeof(T)>(p.d, g, [&](auto nv) {
        constexpr int NV = decltype(nv)::value;
        if (!p.w) return launch_ring(ctx, rms_norm_back_ring_kernel<T, NV, float, false>, p, g, ctas, bytes, st);
        if (p.wType == RCD_ELEM_F32) return launch_ring(ctx, rms_norm_back_ring_kernel<T, NV, float, true>, p, g, ctas, bytes, st);
        return launch_ring(ctx, rms_norm_back_ring_kernel<T, NV, T, true>, p, g, ctas, bytes, st);
    });
}

}  // namespace

rcd_status launch_norm_back_ring(rcd_ctx *ctx, const NormBackParams &p, rcd_elem type, const Ring &g, cudaStream_t st)
{
    return type == RCD_ELEM_BF16  ? launch_typed<__nv_bfloat16>(ctx, p, g, st)
           : type == RCD_ELEM_F16 ? launch_typed<__half>(ctx, p, g, st) : launch_typed<float>(ctx, p, g, st);
}

}  // namespace rcd
