// Root-mean-square norm of many rows: the kernel of rcd_norm.cuh's ring.
#include "rcd_norm.cuh"

namespace rcd {

namespace {

// The lane's pairs times the weights, if any.  (What is the same for the whole launch is asked once per row, not per element: at 17
// instructions an element this kernel was bound by their latency.)
template <int P, int NV, typename W>
__device__ __forceinline__ void times_weights(Two (&h)[NV][P], const W *w, int d, int tid, int G)
{
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * G + tid) * 2 * P;
        if (col < d) {
            Two o[P];
            load_twos<P>(o, w + col);
#pragma unroll
            for (int i = 0; i < P; ++i) h[c][i] = mul2(h[c][i], o[i]);
        }
    }
}
template <int P, int NV, typename Y>
__device__ __forceinline__ void store_row(const Two (&h)[NV][P], Y *y, int d, int tid, int G, float rstd)
{
    const Two r = two(rstd, rstd);
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * G + tid) * 2 * P;
        if (col < d) {
            Two o[P];
#pragma unroll
            for (int i = 0; i < P; ++i) o[i] = mul2(h[c][i], r);
            store_twos<P>(y + col, o);
        }
    }
}

enum { kOutFloat, kOutRowScale, kOutOneScale };
template <typename T, int NV, int kOut>
__global__ void __launch_bounds__(32 * kRingWarps, 1) rms_norm_ring_kernel(const __grid_constant__ NormParams p, const __grid_constant__ Ring ring)
{
    constexpr int VEC = 16 / sizeof(T), P = VEC / 2;
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
        mbar_expect_tx(&sh.bar[group][slot], p.r ? 2 * rowBytes : rowBytes);
        bulk_load(slots + slot * ring.slotBytes, (const T *)p.x + row * p.ldx, rowBytes, &sh.bar[group][slot]);
        if (p.r) bulk_load(slots + slot * ring.slotBytes + rowBytes, (const T *)p.r + row * p.ldr, rowBytes, &sh.bar[group][slot]);
    };
    if (tid == 0)
        for (int k = 0; k < ring.stages; ++k) order(first + k * step, k);
    RingTurn at;
    int turn = 0;
    for (int64_t row = first; row < p.rows; row += step, turn ^= 1) {
        at.waited(ring_wait(&sh.bar[group][at.slot], at.parity, &sh));
        const T *const x = reinterpret_cast<const T *>(slots + at.slot * ring.slotBytes);
        Two h[NV][P];
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * G + tid) * VEC;
            if (col < p.d) {
                load_twos<P>(h[c], x + col);
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i) h[c][i] = two(0.0f, 0.0f);
            }
        }
        if (p.r) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * G + tid) * VEC;
                if (col < p.d) {
                    Two o[P];
                    load_twos<P>(o, x + p.d + col);
#pragma unroll
                    for (int i = 0; i < P; ++i) h[c][i] = add2(h[c][i], o[i]);
                }
            }
        }
        if (gw == 1) {
            __syncwarp();
            if (tid == 0 && at.may_order()) order(row + ring.stages * step, at.slot);
        }
        if (p.sum) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * G + tid) * VEC;
                if (col < p.d) store_twos<P>((T *)p.sum + row * p.lds + col, h[c]);
            }
        }
        float sum = 0.0f, a = 0.0f;
        [[maybe_unused]] double sum64 = 0.0;
        if constexpr (kOut == kOutOneScale) {               // (in 64 bits: see row_sums)
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 f = parts(h[c][i]);
                    sum64 += (double)f.x * (double)f.x;
                    sum64 += (double)f.y * (double)f.y;
                }
        } else {
            Two s[2] = {two(0.0f, 0.0f), two(0.0f, 0.0f)};
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < P; ++i) s[i & 1] = fma2(h[c][i], h[c][i], s[i & 1]);
            const float2 f = parts(add2(s[0], s[1]));
            sum = f.x + f.y;
        }
        if (p.w) {
            if (p.wType == RCD_ELEM_F32) times_weights<P, NV>(h, (const float *)p.w, p.d, tid, G);
            else if (p.wType == RCD_ELEM_BF16) times_weights<P, NV>(h, (const __nv_bfloat16 *)p.w, p.d, tid, G);
            else times_weights<P, NV>(h, (const __half *)p.w, p.d, tid, G);
        }
        if constexpr (kOut == kOutRowScale) {
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 f = parts(h[c][i]);
                    a = max_nan(a, max_nan(fabsf(f.x), fabsf(f.y)));
                }
            a = warp_max_nan(a);
        }
        if constexpr (kOut == kOutOneScale) sum64 = warp_sum(sum64);
        else sum = warp_sum(sum);
        if (gw > 1) {
            if (lane == 0) {
                if constexpr (kOut == kOutOneScale) sh.part[turn][threadIdx.x >> 5] = make_float4(__int_as_float(__double2loint(sum64)), __int_as_float(__double2hiint(sum64)), 0.0f, 0.0f);
                else sh.part[turn][threadIdx.x >> 5] = make_float4(sum, a, 0.0f, 0.0f);
            }
            group_barrier(group, G);
            if (tid == 0 && at.may_order()) order(row + ring.stages * step, at.slot);
            sum = a = 0.0f;
            sum64 = 0.0;
            for (int k = 0; k < gw; ++k) {
                const float4 o = sh.part[turn][group * gw + k];
                if constexpr (kOut == kOutOneScale) {
                    sum64 += __hiloint2double(__float_as_int(o.y), __float_as_int(o.x));
                } else {
                    sum += o.x;
                    a = max_nan(a, o.y);
                }
            }
        }
        const float rstd = kOut == kOutOneScale ? rstd_of(sum64, p) : rstd_of(sum, p);
        if constexpr (kOut == kOutFloat) {
            if (p.yType == RCD_ELEM_F32) store_row<P, NV>(h, (float *)p.y + row * p.ldy, p.d, tid, G, rstd);
            else if (p.yType == RCD_ELEM_BF16) store_row<P, NV>(h, (__nv_bfloat16 *)p.y + row * p.ldy, p.d, tid, G, rstd);
            else store_row<P, NV>(h, (__half *)p.y + row * p.ldy, p.d, tid, G, rstd);
        } else {
            float inv = p.invScale;
            if constexpr (kOut == kOutRowScale) {
                bool raised;
                inv = row_scale(a, rstd, tid == 0 ? p.scales + row : nullptr, &raised);
                if (raised) {
#pragma unroll
                    for (int c = 0; c < NV; ++c)
#pragma unroll
                        for (int i = 0; i < P; ++i) h[c][i] = mul2(h[c][i], two(kRaise, kRaise));
                }
            }
            const Two by = kOut == kOutRowScale ? two(inv, inv) : two(rstd, rstd), then = two(inv, inv);
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * G + tid) * VEC;
                if (col < p.d) {
                    Pack<int8_t, VEC> q;
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        Two v = mul2(h[c][i], by);
                        if constexpr (kOut == kOutOneScale) v = mul2(v, then);
                        const float2 f = parts(v);
                        q.v[2 * i] = to_int8<kOut == kOutOneScale>(f.x);
                        q.v[2 * i + 1] = to_int8<kOut == kOutOneScale>(f.y);
                    }
                    *reinterpret_cast<Pack<int8_t, VEC> *>((int8_t *)p.y + row * p.ldy + col) = q;
                }
            }
        }
        at.next(ring.stages);
    }
    ring_end(&sh, p.status);
}

template <typename T>
rcd_status launch_typed(rcd_ctx *ctx, const NormParams &p, const Ring &g, cudaStream_t st)
{
    const int ctas = ring_ctas(ctx, p.rows, g);
    const size_t bytes = (size_t)g.groups * g.stages * g.slotBytes;
    return by_accesses<16 / (int)sizeof(T)>(p.d, g, [&](auto nv) {
        constexpr int NV = decltype(nv)::value;
        if (p.yType != RCD_ELEM_I8) return launch_ring(ctx, rms_norm_ring_kernel<T, NV, kOutFloat>, p, g, ctas, bytes, st);
        if (p.invScale == 0.0f) return launch_ring(ctx, rms_norm_ring_kernel<T, NV, kOutRowScale>, p, g, ctas, bytes, st);
        return launch_ring(ctx, rms_norm_ring_kernel<T, NV, kOutOneScale>, p, g, ctas, bytes, st);
    });
}
}  // namespace

rcd_status launch_norm_ring(rcd_ctx *ctx, const NormParams &p, rcd_elem type, const Ring &g, cudaStream_t st)
{
    return type == RCD_ELEM_BF16  ? launch_typed<__nv_bfloat16>(ctx, p, g, st)
           : type == RCD_ELEM_F16 ? launch_typed<__half>(ctx, p, g, st) : launch_typed<float>(ctx, p, g, st);
}

}  // namespace rcd
