// Elements of the operators between hidden states and features: loads that widen to fp32, stores that round once.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "rcd_internal.h"

namespace rcd {

inline int64_t elem_bytes(rcd_elem t) { return t == RCD_ELEM_I8 ? 1 : t == RCD_ELEM_F32 ? 4 : 2; }
inline bool elem_is_float(rcd_elem t) { return t == RCD_ELEM_BF16 || t == RCD_ELEM_F16 || t == RCD_ELEM_F32; }

// Whether two matrices (rows, elements from row to row, elements of a row, bytes of an element) share a byte; an output may not share one with
// another argument.  Matrices whose rows lie equally far apart, as column slices of one buffer do, are told apart by their columns;
// others by their first and last byte.
inline bool ranges_meet(const void *a, int64_t aRows, int64_t aLd, int64_t aLen, int64_t aBytes,
                        const void *b, int64_t bRows, int64_t bLd, int64_t bLen, int64_t bBytes)
{
    if (!a || !b || aRows <= 0 || bRows <= 0 || aLen <= 0 || bLen <= 0) return false;
    const int64_t la = aLen * aBytes, lb = bLen * bBytes;
    const uintptr_t a0 = (uintptr_t)a, a1 = a0 + (uintptr_t)((aRows - 1) * aLd * aBytes + la);
    const uintptr_t b0 = (uintptr_t)b, b1 = b0 + (uintptr_t)((bRows - 1) * bLd * bBytes + lb);
    if (a1 <= b0 || b1 <= a0) return false;
    const int64_t pitch = aRows > 1 ? aLd * aBytes : bLd * bBytes;          // (a single row lies as far from the next as one likes)
    if ((bRows > 1 && bLd * bBytes != pitch) || pitch < la || pitch < lb) return true;
    const int64_t column = a0 <= b0 ? (int64_t)(b0 - a0) % pitch : (pitch - (int64_t)(a0 - b0) % pitch) % pitch;     // of b's rows, from a's
    return column < la || column + lb > pitch;
}
// Whether every row of a matrix starts on `align` bytes (null: nothing to load).
inline bool rows_aligned(const void *p, int64_t ld, int64_t bytes, int64_t align)
{
    return !p || (((uintptr_t)p) % align == 0 && ld * bytes % align == 0);
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// VEC neighbouring elements, in as few accesses of up to 16 bytes as their size allows.
template <typename T, int VEC> struct alignas(sizeof(T) * VEC < 16 ? sizeof(T) * VEC : 16) Pack { T v[VEC]; };
template <int VEC, typename T>
__device__ __forceinline__ void load_pack(float (&out)[VEC], const T *p)
{
    const Pack<T, VEC> x = *reinterpret_cast<const Pack<T, VEC> *>(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[i] = to_float(x.v[i]);
}
template <int VEC, typename T>
__device__ __forceinline__ void store_pack(T *p, const float (&x)[VEC])
{
    Pack<T, VEC> o;
#pragma unroll
    for (int i = 0; i < VEC; ++i) o.v[i] = from_float<T>(x[i]);
    *reinterpret_cast<Pack<T, VEC> *>(p) = o;
}
template <int VEC>
__device__ __forceinline__ void load_typed(float (&out)[VEC], const void *p, int64_t i, rcd_elem type)
{
    if (type == RCD_ELEM_BF16) load_pack<VEC>(out, (const __nv_bfloat16 *)p + i);
    else if (type == RCD_ELEM_F16) load_pack<VEC>(out, (const __half *)p + i);
    else load_pack<VEC>(out, (const float *)p + i);
}
template <int VEC>
__device__ __forceinline__ void store_typed(void *p, int64_t i, rcd_elem type, const float (&x)[VEC])
{
    if (type == RCD_ELEM_BF16) store_pack<VEC>((__nv_bfloat16 *)p + i, x);
    else if (type == RCD_ELEM_F16) store_pack<VEC>((__half *)p + i, x);
    else store_pack<VEC>((float *)p + i, x);
}
// Two fp32 numbers in 64 bits: sm_100 adds, multiplies and fuses them in one instruction, each rounded as alone.
struct Two { unsigned long long v; };
__device__ __forceinline__ Two two(float lo, float hi)
{
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 parts(Two x)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x.v));
    return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) { Two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Two add2(Two a, Two b) { Two r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { Two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ Two widen(uint32_t x, __nv_bfloat16) { return two(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
__device__ __forceinline__ Two widen(uint32_t x, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&x));
    return two(f.x, f.y);
}
__device__ __forceinline__ uint32_t narrow(Two x, __nv_bfloat16)
{
    const float2 f = parts(x);
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&b);
}
__device__ __forceinline__ uint32_t narrow(Two x, __half)
{
    const float2 f = parts(x);
    const __half2 b = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&b);
}
// 2 P neighbouring elements as pairs; 16-byte accesses where there are as many bytes.
template <int P, typename T>
__device__ __forceinline__ void load_twos(Two (&o)[P], const T *p)
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (P % 2 == 0) {
#pragma unroll
            for (int i = 0; i < P / 2; ++i) {
                const float4 x = reinterpret_cast<const float4 *>(p)[i];
                o[2 * i] = two(x.x, x.y);
                o[2 * i + 1] = two(x.z, x.w);
            }
        }
    } else {
        Pack<uint32_t, P> x = *reinterpret_cast<const Pack<uint32_t, P> *>(p);
#pragma unroll
        for (int i = 0; i < P; ++i) o[i] = widen(x.v[i], T());
    }
}
template <int P, typename T>
__device__ __forceinline__ void store_twos(T *p, const Two (&x)[P])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < P / 2; ++i) {
            const float2 a = parts(x[2 * i]), b = parts(x[2 * i + 1]);
            reinterpret_cast<float4 *>(p)[i] = make_float4(a.x, a.y, b.x, b.y);
        }
    } else {
        Pack<uint32_t, P> o;
#pragma unroll
        for (int i = 0; i < P; ++i) o.v[i] = narrow(x[i], T());
        *reinterpret_cast<Pack<uint32_t, P> *>(p) = o;
    }
}

// The greater of two, a NaN if either is one.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ double warp_sum(double x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
#endif

}  // namespace rcd
