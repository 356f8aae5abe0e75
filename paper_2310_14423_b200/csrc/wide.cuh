// Device helpers shared by the operators that work in the caller's own number types: 16- and 32-byte accesses, bf16 /
// fp16 / E4M3 to fp32 and back, warp reductions.
#ifndef QSR_WIDE_CUH_
#define QSR_WIDE_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cstdint>

#include "internal.h"

namespace qsr {

__device__ __forceinline__ float rcp_1(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sqrt_1(float x)
{
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float exp2_1(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The larger operand; NaN if either is NaN (fmaxf drops a NaN).
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float infinity() { return __uint_as_float(0x7f800000u); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fffffffu); }

// Eight consecutive elements as they lie in memory: 32 bytes of fp32 (all eight words) or 16 bytes of a 16-bit type
// (the first four).  Loading and widening are separate so that a thread can issue the loads of all its operands before
// it waits for the first one.
struct Raw8 { uint32_t w[8]; };

// One 256-bit load / store (sm_100): 32-byte aligned.  Streamed data: nothing is kept in L1.
__device__ __forceinline__ void load32(Raw8 &r, const void *p)
{
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                 : "l"(p) : "memory");
}
__device__ __forceinline__ void store32(void *p, const Raw8 &r)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]),
                 "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]) : "memory");
}
__device__ __forceinline__ void load16(Raw8 &r, const void *p)
{
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store16(void *p, const Raw8 &r)
{
    asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]) : "memory");
}

__device__ __forceinline__ float2 widen2(uint32_t w, int type)
{
    if (type == QSR_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
// Rounds to nearest even, once.
__device__ __forceinline__ uint32_t narrow2(float a, float b, int type)
{
    if (type == QSR_BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// `type` is the same for all threads of a warp, so these branches do not diverge.
__device__ __forceinline__ void load8(Raw8 &r, const void *base, int64_t i, int type)
{
    if (type == QSR_F32) load32(r, static_cast<const float *>(base) + i);
    else load16(r, static_cast<const uint16_t *>(base) + i);
}
__device__ __forceinline__ void widen8(float (&x)[8], const Raw8 &r, int type)
{
    if (type == QSR_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = widen2(r.w[i], type);
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    }
}
__device__ __forceinline__ void store8(void *base, int64_t i, const float (&x)[8], int type)
{
    Raw8 r;
    if (type == QSR_F32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.w[j] = __float_as_uint(x[j]);
        store32(static_cast<float *>(base) + i, r);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) r.w[j] = narrow2(x[2 * j], x[2 * j + 1], type);
        store16(static_cast<uint16_t *>(base) + i, r);
    }
}
// One element as it lies in memory, widened by widen1.
__device__ __forceinline__ uint32_t load1(const void *base, int64_t i, int type)
{
    if (type == QSR_F32) return static_cast<const uint32_t *>(base)[i];
    return static_cast<const uint16_t *>(base)[i];
}
__device__ __forceinline__ float widen1(uint32_t w, int type)
{
    if (type == QSR_F32) return __uint_as_float(w);
    return widen2(w, type).x;
}
__device__ __forceinline__ void store1(void *base, int64_t i, float x, int type)
{
    if (type == QSR_F32) static_cast<float *>(base)[i] = x;
    else static_cast<uint16_t *>(base)[i] = uint16_t(narrow2(x, 0.0f, type));
}

// E4M3: four exponent bits, three mantissa bits, no infinity, largest value 448, smallest positive 2^-9.  Rounds to
// nearest even; beyond 448 (infinity included) saturates; NaN stays NaN.
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t w)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(w), __NV_E4M3);
    return __half22float2(__half2(h));
}

// Four codes at once, low byte first.
__device__ __forceinline__ uint32_t to_e4m3x4(float2 a, float2 b)
{
    uint32_t w;
    asm("{.reg .b16 lo, hi; cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1; cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3; mov.b32 %0, {lo, hi};}"
        : "=r"(w) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return w;
}
__device__ __forceinline__ void from_e4m3x4(float2 &a, float2 &b, uint32_t w)
{
    uint32_t x, y;
    asm("{.reg .b16 lo, hi; mov.b32 {lo, hi}, %2; cvt.rn.f16x2.e4m3x2 %0, lo; cvt.rn.f16x2.e4m3x2 %1, hi;}" : "=r"(x), "=r"(y) : "r"(w));
    a = __half22float2(*reinterpret_cast<const __half2 *>(&x));
    b = __half22float2(*reinterpret_cast<const __half2 *>(&y));
}

// Three-operand extrema (sm_100); NaNs are passed over.
__device__ __forceinline__ float max3_abs(float a, float b, float c)
{
    float y;
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float min3(float a, float b, float c)
{
    float y;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

// Largest value over the warp; NaNs are passed over.  One instruction on sm_100a.
__device__ __forceinline__ float warp_max(float x)
{
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float warp_max_nan(float x)
{
    float y;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
// Sum over the warp in a fixed order, the same in every lane.
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}

}  // namespace qsr
#endif
