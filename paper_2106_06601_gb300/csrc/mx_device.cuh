// Device code of the microscaled formats (blocks of 32, power-of-two scales).
#pragma once

#include <cstdint>

#include <cuda_bf16.h>

#include "mx.h"

namespace costa {
namespace mx {

// 2^(biased - 127) for biased in 0 .. 254; NaN for 255.
__device__ __forceinline__ float pow2(int biased) {
    const uint32_t bits = biased == 0 ? 0x00400000u : biased == 255 ? 0x7fffffffu : uint32_t(biased) << 23;
    return __uint_as_float(bits);
}

// The scale byte of a block from the biased exponent of its largest magnitude:
// floor(log2) + 127 for normal numbers; subnormal ones and zero clamp to 0, where
// their exponent field already is.  255: an infinity or a NaN.
template <int FMT> __device__ __forceinline__ int scale_byte(int e) {
    if (e == 255) return 255;
    return FMT == COSTA_MX_E2M1 ? max(e - 2, 0) : e;
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Two E2M1 codes, a in the low half.  The conversion rounds to nearest even and saturates at 6.
__device__ __forceinline__ uint32_t e2m1x2(float a, float b) {
    uint32_t r;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %2, %1;\n\tmov.b32 %0, {t, 0, 0, 0};\n\t}" : "=r"(r) : "f"(a), "f"(b));
    return r;
}

// Codes of 8 elements x(0) .. x(7), for scale byte s; zero codes for 255.  What
// takes an element to its code's range is a normal power of two (two of them
// for I8 below 2^-121, where 2^(6 - E) is beyond a float), so the products are
// exact unless they are subnormal, far below half of the least code.
template <typename X> __device__ __forceinline__ uint32_t e2m1_of8(const X &x, int s) {
    if (s == 255) return 0;
    const float f = pow2(254 - s);  // s <= 252
    return e2m1x2(x(0) * f, x(1) * f) | e2m1x2(x(2) * f, x(3) * f) << 8 | e2m1x2(x(4) * f, x(5) * f) << 16 |
           e2m1x2(x(6) * f, x(7) * f) << 24;
}

// Added to 1.5 2^23 a number below 2^22 is rounded to an integer, to nearest
// even, in the low bits; they are clamped in pairs of 16 bits.
__device__ __forceinline__ uint32_t i8_of4(float a, float b, float c, float d, float f) {
    constexpr float kRound = 12582912.0f;
    uint32_t p = __byte_perm(__float_as_uint(fmaf(a, f, kRound)), __float_as_uint(fmaf(b, f, kRound)), 0x5410);
    uint32_t q = __byte_perm(__float_as_uint(fmaf(c, f, kRound)), __float_as_uint(fmaf(d, f, kRound)), 0x5410);
    p = __vmaxs2(__vmins2(p, 0x007f007fu), 0xff81ff81u);
    q = __vmaxs2(__vmins2(q, 0x007f007fu), 0xff81ff81u);
    return __byte_perm(p, q, 0x6420);
}
template <typename X> __device__ __forceinline__ uint2 i8_of8(const X &x, int s) {
    if (s == 255) return make_uint2(0, 0);
    if (s >= 6) {
        const float f = pow2(260 - s);
        return make_uint2(i8_of4(x(0), x(1), x(2), x(3), f), i8_of4(x(4), x(5), x(6), x(7), f));
    }
    const float f = pow2(254 - s);
    return make_uint2(i8_of4(x(0) * 64.0f, x(1) * 64.0f, x(2) * 64.0f, x(3) * 64.0f, f),
                      i8_of4(x(4) * 64.0f, x(5) * 64.0f, x(6) * 64.0f, x(7) * 64.0f, f));
}

// The value of an I8 code for scale byte s is q times this: 2^(s - 133), below 2^-126 for small s.
__device__ __forceinline__ float i8_unit(int s) {
    const uint32_t bits = s == 255 ? 0x7fffffffu : s <= 6 ? 1u << (s + 16) : uint32_t(s - 6) << 23;
    return __uint_as_float(bits);
}

// Values of 4 codes of E2M1 (the low 16 bits) and of I8.  The three low bits of
// an E2M1 code are the exponent and fraction of a float 2^126 times smaller (0.5
// a subnormal one); an I8 code q is taken as the float 2^23 + 128 + q.
__device__ __forceinline__ void e2m1_to4(uint32_t codes, float unit, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t top = codes << (28 - 4 * i);  // the code in the top four bits
        v[i] = __uint_as_float((top & 0x80000000u) | (top >> 6 & 0x01c00000u)) * 0x1p126f * unit;
    }
}
__device__ __forceinline__ void i8_to4(uint32_t codes, float unit, float (&v)[4]) {
    const uint32_t w = codes ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = unit * (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7540 | i)) - 8388736.0f);
}

// Byte of block j of row i in E2M1's scales.
__device__ __forceinline__ int64_t scale_at(int64_t i, int64_t j, int64_t tiles) {
    return ((i >> 7) * tiles + (j >> 2)) * 512 + (i & 31) * 16 + ((i >> 5) & 3) * 4 + (j & 3);
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Elements col .. col + 7 of a row of `cols`, 0 past its end.  vec: row + col
// is 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load8(const T *row, int64_t col, int64_t cols, bool vec, float (&x)[8]) {
    if (vec && col + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4 *>(row + col), b = *reinterpret_cast<const float4 *>(row + col + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4 *>(row + col);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = col + i < cols ? to_float(row[col + i]) : 0.0f;
    }
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

}  // namespace mx
}  // namespace costa
