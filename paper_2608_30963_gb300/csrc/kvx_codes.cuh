// kvx_codes.cuh -- rows of 8-bit caches (library-internal): a row of d values is d e4m3 codes and one scale byte.
//
//   value = code * 2^(s - 127)
// Every value is exact in bf16 and fp32: a code has 4 significant bits and the scale is a power of two, which e4m3's relative
// precision does not depend on (a scale in 32 bits would not make a row more exact, only 3 bytes longer).
#pragma once

#include "kvx_decode.cuh"

namespace kvx {
namespace {

// Scale bytes that are written: values from 2^-126 (normal in 32 bits) up to 1.875 * 2^127.
constexpr int kMinScale = 10, kMaxScale = 247;

// The float that a scale byte stands for: 0 stands for 0, 255 for infinity.
__device__ __forceinline__ float scale_of(unsigned s) { return __uint_as_float(s << 23); }
// Its reciprocal, for bytes that are written.
__device__ __forceinline__ float inv_scale(unsigned s) { return __uint_as_float((254u - s) << 23); }
// The smallest scale s (clamped) with top <= 448 * 2^(s - 127): top = 1.f * 2^x takes 2^(x - 8), or twice that where 1.f is
// above 448 / 256.
__device__ __forceinline__ unsigned scale_for(float top)
{
    const unsigned b = __float_as_uint(top);
    const int s = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u);
    return (unsigned)min(max(s, kMinScale), kMaxScale);
}

// Two codes as floats.
__device__ __forceinline__ float2 codes_f32(unsigned short two)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
    float2 f;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
// Two values rounded to codes, to nearest even; above 448 they would be 448.
__device__ __forceinline__ uint32_t to_codes(float lo, float hi)
{
    unsigned short two;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(hi), "f"(lo));
    return two;
}
__device__ __forceinline__ uint2 pack_codes(const float (&x)[8])
{
    return make_uint2(to_codes(x[0], x[1]) | to_codes(x[2], x[3]) << 16, to_codes(x[4], x[5]) | to_codes(x[6], x[7]) << 16);
}
__device__ __forceinline__ void unpack_codes(uint2 w, float scale, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = codes_f32((unsigned short)((i < 2 ? w.x : w.y) >> (i & 1) * 16));
        x[2 * i] = f.x * scale;
        x[2 * i + 1] = f.y * scale;
    }
}

// Infinities become NaN, magnitudes at most 1.875 * 2^127 (the next code, 2^128, is no number in 32 bits).
__device__ __forceinline__ float tame(float x)
{
    return fabsf(x) <= 3.402823466e38f ? copysignf(fminf(fabsf(x), 1.875f * 0x1p127f), x) : __uint_as_float(0x7fffffffu);
}
// The scale of a row from its lanes' largest magnitudes (LANES lanes, consecutive, aligned).  Whole warps call it.
template <int LANES> __device__ __forceinline__ unsigned row_scale(float top)
{
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    return scale_for(top);
}
// A row's LANES lanes hold 16 of its values each: their codes and the row's scale.  Values that are not finite have no say in
// the scale and become NaN.
template <int LANES> __device__ __forceinline__ unsigned quantise_row(float (&a)[8], float (&b)[8], uint2& lo, uint2& hi)
{
    auto largest = [&] {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(a[i]), fabsf(b[i])));
        return top;
    };
    float top = largest();              // (a NaN does not count)
    if (top > 3.0e38f) {                // rare
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[i] = tame(a[i]);
            b[i] = tame(b[i]);
        }
        top = largest();
    }
    const unsigned s = row_scale<LANES>(top);
    const float f = inv_scale(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        a[i] *= f;
        b[i] *= f;
    }
    lo = pack_codes(a);
    hi = pack_codes(b);
    return s;
}

// Eight consecutive values of T.
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
        const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_f32<T>(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 w = __ldcs(reinterpret_cast<const float4*>(p + i));
            x[i] = w.x;
            x[i + 1] = w.y;
            x[i + 2] = w.z;
            x[i + 3] = w.w;
        }
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        uint4 w;
        T* e = reinterpret_cast<T*>(&w);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = from_f32<T>(x[i]);
        __stcs(reinterpret_cast<uint4*>(p), w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i += 4) __stcs(reinterpret_cast<float4*>(p + i), make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
    }
}

}  // namespace
}  // namespace kvx
