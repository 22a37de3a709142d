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

// The scale byte of a block from the bits of its largest magnitude: the
// exponent field is floor(log2) + 127 for normal numbers; subnormal ones and
// zero clamp to 0, where their field already is.  255: an infinity or a NaN.
template <int FMT> __device__ __forceinline__ int scale_byte(uint32_t amax) {
    const int e = static_cast<int>(amax >> 23);
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

// What takes an element to its code's range for scale byte s (not 255): every
// factor is a normal power of two, so the products are exact unless they are
// below the smallest subnormal, far below half of the least code.
struct ToE2M1 {
    float f;
    __device__ explicit ToE2M1(int s) : f(pow2(254 - s)) {}  // s <= 252
    __device__ float operator()(float x) const { return x * f; }
};
struct ToI8 {
    float c, f;  // x 2^(6 - E); for the smallest scales that factor is beyond a float
    __device__ explicit ToI8(int s) : c(s < 6 ? 64.0f : 1.0f), f(pow2(s < 6 ? 254 - s : 260 - s)) {}
    __device__ int operator()(float x) const { return max(-127, min(127, __float2int_rn(x * c * f))); }
};

// The value of an I8 code for scale byte s is q times this: 2^(s - 133), below 2^-126 for small s.
__device__ __forceinline__ float i8_unit(int s) {
    const uint32_t bits = s == 255 ? 0x7fffffffu : s <= 6 ? 1u << (s + 16) : uint32_t(s - 6) << 23;
    return __uint_as_float(bits);
}

// Codes of 8 elements (4 or 8 bytes), for scale byte s; zero codes for 255.
__device__ __forceinline__ uint32_t e2m1_of8(const float (&x)[8], int s) {
    if (s == 255) return 0;
    const ToE2M1 to(s);
    return e2m1x2(to(x[0]), to(x[1])) | e2m1x2(to(x[2]), to(x[3])) << 8 | e2m1x2(to(x[4]), to(x[5])) << 16 |
           e2m1x2(to(x[6]), to(x[7])) << 24;
}
__device__ __forceinline__ uint2 i8_of8(const float (&x)[8], int s) {
    if (s == 255) return make_uint2(0, 0);
    const ToI8 to(s);
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        w[h] = __byte_perm(__byte_perm(to(x[4 * h]), to(x[4 * h + 1]), 0x0040),
                           __byte_perm(to(x[4 * h + 2]), to(x[4 * h + 3]), 0x0040), 0x5410);
    return make_uint2(w[0], w[1]);
}

// Values of 8 codes.
__device__ __forceinline__ void e2m1_to8(uint32_t codes, float unit, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = codes >> (4 * i);
        // exponent 1 .. 3 with one fraction bit, or 0 / 0.5: 2 |v| as an integer, 0 1 2 3 4 6 8 12
        const int twice = (0xC8643210u >> (4 * (c & 7))) & 15;
        const float m = 0.5f * unit * static_cast<float>(twice);
        v[i] = c & 8 ? -m : m;
    }
}
__device__ __forceinline__ void i8_to8(uint2 codes, float unit, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t w = i < 4 ? codes.x : codes.y;
        v[i] = unit * static_cast<float>(static_cast<int8_t>(w >> (8 * (i & 3))));
    }
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

template <typename T>
__device__ __forceinline__ void store8(T *row, int64_t col, int64_t cols, bool vec, const float (&x)[8]) {
    if (vec && col + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(row + col) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4 *>(row + col + 4) = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            *reinterpret_cast<uint4 *>(row + col) =
                make_uint4(bf16x2(x[0], x[1]), bf16x2(x[2], x[3]), bf16x2(x[4], x[5]), bf16x2(x[6], x[7]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = from_float<T>(x[i]);
    }
}

}  // namespace mx
}  // namespace costa
