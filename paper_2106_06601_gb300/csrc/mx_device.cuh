// Device code of the microscaled formats (blocks of 32, power-of-two scales).
#pragma once

#include <cstdint>

#include <cuda_bf16.h>

#include "mx.h"

namespace costa {
namespace mx {

// From here on the next kernel's blocks may start.  The first call of every
// kernel; in those that use tensor memory once they hold it: a kernel that waits
// for this one must not hold what this one still waits for.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// Before anything in global memory is read or written: what the kernels before this one wrote is there.  (A
// product brings weights as far as the L2 cache before it, which changes nothing that a kernel sees.)
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

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

// The larger magnitude (of each half), NaN if there is one: as floating
// comparisons, which take half the cycles of integer ones and no masking.
__device__ __forceinline__ float larger(float a, float x) {
    asm("{\n\t.reg .f32 t;\n\tabs.f32 t, %1;\n\tmax.NaN.f32 %0, %0, t;\n\t}" : "+f"(a) : "f"(x));
    return a;
}
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t x) {
    asm("{\n\t.reg .b32 t;\n\tabs.bf16x2 t, %1;\n\tmax.NaN.bf16x2 %0, %0, t;\n\t}" : "+r"(a) : "r"(x));
    return a;
}

// E2M1 codes of 8 numbers x(0) .. x(7), the first in the low bits; the
// conversion rounds to nearest even and saturates at 6.
template <typename X> __device__ __forceinline__ uint32_t e2m1_of8(const X &x) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(x(0)), "f"(x(1)), "f"(x(2)), "f"(x(3)), "f"(x(4)), "f"(x(5)), "f"(x(6)), "f"(x(7)));
    return r;
}

// What takes a block's elements to its codes' range: a normal power of two, so
// the products are exact unless they are subnormal, far below half of the least
// code (as are bf16 products); 0 for NaN blocks, whose codes are then cleared.
// I8 below 2^-121, where 2^(6 - E) is beyond a float, takes 2^6 apart.
__device__ __forceinline__ float e2m1_factor(int s) { return s == 255 ? 0.0f : pow2(254 - s); }  // s <= 252
__device__ __forceinline__ __nv_bfloat162 halves(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
__device__ __forceinline__ uint32_t word(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t *>(&v); }
__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Added to 1.5 2^23 a number below 2^22 is rounded to an integer, to nearest
// even, in the low bits; they are clamped in pairs of 16 bits.
__device__ __forceinline__ uint32_t clamp127(uint32_t pair) {
    asm("min.s16x2 %0, %0, %1;" : "+r"(pair) : "r"(0x007f007fu));
    asm("max.s16x2 %0, %0, %1;" : "+r"(pair) : "r"(0xff81ff81u));
    return pair;
}
__device__ __forceinline__ uint32_t i8_of4(float a, float b, float c, float d, float f) {
    constexpr float kRound = 12582912.0f;
    uint32_t p = __byte_perm(__float_as_uint(fmaf(a, f, kRound)), __float_as_uint(fmaf(b, f, kRound)), 0x5410);
    uint32_t q = __byte_perm(__float_as_uint(fmaf(c, f, kRound)), __float_as_uint(fmaf(d, f, kRound)), 0x5410);
    p = clamp127(p);
    q = clamp127(q);
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

// Values of 4 codes of E2M1 (the low 16 bits) as bf16 pairs.  A byte permutation
// looks up the high and the low bytes of 0, 0.5, 1, 1.5, 2, 3, 4, 6 by three bits
// of each code; one with the whole code gives 0x40, or 0 (the selected byte's
// sign throughout) where the sign is set.
__device__ __forceinline__ void e2m1_to4(uint32_t codes, __nv_bfloat162 unit, uint32_t (&v)[2]) {
    const uint32_t which = codes & 0x7777u;
    uint32_t high = __byte_perm(0x3f3f3f00u, 0x40404040u, which);
    const uint32_t low = __byte_perm(0xc0800000u, 0xc0804000u, which);
    uint32_t plus;
    asm("prmt.b32 %0, %1, %1, %2;" : "=r"(plus) : "r"(0x40404040u), "r"(codes));
    high |= ~(plus << 1) & 0x80808080u;
    v[0] = word(__hmul2(halves(__byte_perm(low, high, 0x5140)), unit));
    v[1] = word(__hmul2(halves(__byte_perm(low, high, 0x7362)), unit));
}
// The unit of E2M1 codes with scale byte s, 2^(s - 127), as a bf16 pair.
__device__ __forceinline__ __nv_bfloat162 e2m1_unit(int s) {
    return halves((s == 0 ? 0x0040u : s == 255 ? 0x7fffu : uint32_t(s) << 7) * 0x10001u);
}

// Values of 4 codes of I8: a code q is taken as the float 2^23 + 128 + q.
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

// N elements of T from p, which need not be aligned, as words.  load() brings
// the whole 16-byte chunks that hold one of the first `count`; place() shifts
// them into place and clears the elements after those.
template <typename T, int N> struct Unaligned {
    static constexpr int kWords = N * sizeof(T) / 4;
    uint32_t c[kWords + 4];
    __device__ static uint32_t offset(const T *p) { return static_cast<uint32_t>(reinterpret_cast<uint64_t>(p)) & 15; }
    __device__ void load(const T *p, uint32_t off, int count) {
        const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) - off);
        const int bytes = count > 0 ? static_cast<int>(off) + count * static_cast<int>(sizeof(T)) : 0;
#pragma unroll
        for (int j = 0; j <= kWords / 4; ++j) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (16 * j < bytes) v = from[j];
            c[4 * j] = v.x;
            c[4 * j + 1] = v.y;
            c[4 * j + 2] = v.z;
            c[4 * j + 3] = v.w;
        }
    }
    __device__ void load_whole(const T *p, uint32_t off) {  // all N exist
        const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) - off);
#pragma unroll
        for (int j = 0; j <= kWords / 4; ++j) {
            if (j == kWords / 4 && off == 0) break;
            const uint4 v = from[j];
            c[4 * j] = v.x;
            c[4 * j + 1] = v.y;
            c[4 * j + 2] = v.z;
            c[4 * j + 3] = v.w;
        }
    }
    template <int FROM> __device__ void shift(uint32_t bits, uint32_t (&w)[kWords]) const {  // from word FROM
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            w[i] = sizeof(T) == 2 ? __funnelshift_r(c[i + FROM], c[i + FROM + 1], bits) : c[i + FROM];
    }
    // `off` is the same in (nearly) all warps' lanes: a branch costs less than selecting words.
    __device__ void place(uint32_t off, int count, uint32_t (&w)[kWords]) const {
        const uint32_t bits = (off & 2) * 8;
        if (off == 0) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = c[i];
        } else if (off < 4) {
            shift<0>(bits, w);
        } else if (off < 8) {
            shift<1>(bits, w);
        } else if (off < 12) {
            shift<2>(bits, w);
        } else {
            shift<3>(bits, w);
        }
        if (count >= N) return;
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 2) {
                if (2 * i >= count) w[i] = 0;
                if (2 * i + 1 >= count) w[i] &= 0xffffu;
            } else {
                if (i >= count) w[i] = 0;
            }
        }
    }
};

// How many of the `n` elements from column `col` a row of `cols` has.
__device__ __forceinline__ int count_from(int64_t col, int64_t cols, int n) {
    return static_cast<int>(max(int64_t(0), min(int64_t(n), cols - col)));
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

}  // namespace mx
}  // namespace costa
