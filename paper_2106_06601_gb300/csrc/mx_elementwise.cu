// Kernels that make and read microscaled codes element by element: the
// quantisation of op(X), its inverse, and activations with 8-bit checkpoints.
//
// All read and write each byte once, so memory bounds them where they issue few
// enough instructions: of 16 elements to a thread, in 32-byte accesses, they
// have 8 to 18 an element (first versions had 50 and ran at a third of the copy
// rate).  Rates below are of the bytes of inputs, codes and outputs, where a
// copy reaches 6786 GB/s.
#include <algorithm>

#include "costa_internal.h"
#include "mx_device.cuh"
#include "mx_host.h"

namespace costa {
namespace mx {
namespace {

constexpr int kThreads = 256;

// Rows cut into groups of 16 elements, half a block, one to a thread: two
// neighbouring lanes share a block, a warp takes 16 of them.  gpr: groups of a
// row, even (so a block's lanes lie in one warp).
struct Groups {
    int64_t gpr, total;
    uint32_t mul, shift;  // x / gpr = (x mul >> 32) >> shift for x < 2^31
    // This thread's group; past the last one a place without elements (col = none).
    __device__ bool at(int64_t none, int64_t &row, int64_t &col) const {
        const int64_t g = int64_t(blockIdx.x) * kThreads + threadIdx.x;
        row = 0;
        col = none;
        if (g >= total) return false;
        if (total <= 0x7fffffff) {
            const uint32_t r = __umulhi(static_cast<uint32_t>(g), mul) >> shift;
            row = r;
            col = (static_cast<uint32_t>(g) - r * static_cast<uint32_t>(gpr)) * 16;
        } else {
            row = g / gpr;
            col = (g - row * gpr) * 16;
        }
        return true;
    }
};

Groups groups_of(int64_t rows, int64_t gpr) {
    Groups g{gpr, rows * gpr, 0, 0};
    if (g.total > 0x7fffffff) return g;
    // 2^(s-1) < gpr <= 2^s and gpr even, so s >= 1: ceil(2^(31+s) / gpr) < 2^32 is exact for 31 bits
    uint32_t s = 1;
    while ((int64_t(1) << s) < gpr) ++s;
    g.mul = static_cast<uint32_t>(((uint64_t(1) << (31 + s)) + gpr - 1) / gpr);
    g.shift = s - 1;
    return g;
}

int64_t blocks_for(const Groups &g) { return mx_ceil(g.total, kThreads); }

template <typename T> struct Dense {
    T *p;
    int64_t ld;
    int align;  // rows start on boundaries of 32 bytes (2), of 16 (1) or any (0)
};

template <typename T> Dense<T> dense(const costa_mx_dense &d) {
    const uint64_t bits = reinterpret_cast<uint64_t>(d.ptr) | static_cast<uint64_t>(d.ld) * sizeof(T);
    return {static_cast<T *>(d.ptr), d.ld, bits % 32 == 0 ? 2 : bits % 16 == 0 ? 1 : 0};
}

// 16 elements as they lie in memory.
template <typename T> struct Sixteen;
template <> struct Sixteen<float> {
    uint32_t w[16];
    __device__ float operator()(int i) const { return __uint_as_float(w[i]); }
    __device__ void set(int i, float x) { w[i] = __float_as_uint(x); }
    __device__ int exponent() const {  // biased, of the largest magnitude
        float a = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) a = larger(a, (*this)(i));
        return __float_as_uint(a) >> 23;
    }
    __device__ uint2 e2m1(float f) const {
        return make_uint2(e2m1_of8([&](int i) { return (*this)(i) * f; }), e2m1_of8([&](int i) { return (*this)(i + 8) * f; }));
    }
    __device__ void set_pairs(int i, const uint32_t (&v)[2]) {
        w[i] = v[0] << 16;
        w[i + 1] = v[0] & 0xffff0000u;
        w[i + 2] = v[1] << 16;
        w[i + 3] = v[1] & 0xffff0000u;
    }
};
template <> struct Sixteen<__nv_bfloat16> {
    uint32_t w[8];
    __device__ float operator()(int i) const { return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
    __device__ void set(int i, float x) {  // in order: a whole word at odd i
        if (i % 2 == 0)
            w[i / 2] = __float_as_uint(x);
        else
            w[i / 2] = bf16x2(__uint_as_float(w[i / 2]), x);
    }
    __device__ int exponent() const {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = larger2(a, w[i]);
        return max(a & 0xffffu, a >> 16) >> 7;
    }
    __device__ uint2 e2m1(float f) const {
        const __nv_bfloat162 ff = __float2bfloat162_rn(f);
        uint32_t t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = word(__hmul2(halves(w[i]), ff));
        auto at = [&](int i) { return i % 2 ? high_of(t[i / 2]) : low_of(t[i / 2]); };
        return make_uint2(e2m1_of8(at), e2m1_of8([&](int i) { return at(i + 8); }));
    }
    __device__ void set_pairs(int i, const uint32_t (&v)[2]) {
        w[i / 2] = v[0];
        w[i / 2 + 1] = v[1];
    }
};

// 32 bytes at a 32-byte boundary
__device__ __forceinline__ void load32(const void *p, uint32_t *w) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
}
__device__ __forceinline__ void store32(void *p, const uint32_t *w) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

// This thread's 16 elements, 0 past the row's end.
template <typename T>
__device__ __forceinline__ void get(const Dense<const T> &X, int64_t row, int64_t col, int64_t cols, Sixteen<T> &x) {
    constexpr int kWords = sizeof(x.w) / 4;
    const T *p = X.p + row * X.ld + col;
    const int count = count_from(col, cols, 16);
    if (X.align == 2 && count == 16) {
#pragma unroll
        for (int i = 0; i < kWords; i += 8) load32(reinterpret_cast<const char *>(p) + 4 * i, x.w + i);
    } else if (X.align == 1 && count == 16) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4)
            *reinterpret_cast<uint4 *>(x.w + i) = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) + 4 * i);
    } else {
        Unaligned<T, 16> u;
        const uint32_t off = u.offset(p);
        u.load(p, off, count);
        u.place(off, count, x.w);
    }
}

// The elements of a warp's 32 groups on their way to rows that are not aligned
// or end inside a group: the lanes write a block's 32 elements together, from 2
// KB of shared memory of the warp.  Lane 2 i holds block i's place and how many
// of its elements exist; in most warps the blocks are one run in memory: they
// follow each other, and each but the last with elements is whole.  (Where rows
// are apart by whole blocks the next row also follows a block that is cut short.)
struct Blocks {
    int64_t place, first;
    int count, left;
    bool run;
    __device__ Blocks(int64_t row, int64_t col, int64_t cols, int64_t ld)
        : place(row * ld + col), count(count_from(col, cols, 32)) {
        const int lane = threadIdx.x % 32;
        first = __shfl_sync(~0u, place, 0);
        const uint32_t some = __ballot_sync(~0u, lane % 2 == 0 && count > 0), cut = __ballot_sync(~0u, count < 32);
        run = __all_sync(~0u, place == first + 16 * lane || count == 0) && (some & cut << 2) == 0;
        // elements from the first on: whole blocks, then one that may end, then none
        left = __reduce_add_sync(~0u, lane % 2 ? 0 : count);
    }
    // f(i, place) for this lane's element of each block i, where it exists.
    template <typename F> __device__ void each(F f) const {
        const int lane = threadIdx.x % 32;
        if (run) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (32 * i + lane < left) f(i, first + lane + 32 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t p = __shfl_sync(~0u, place, 2 * i);
                if (lane < __shfl_sync(~0u, count, 2 * i)) f(i, p + lane);
            }
        }
    }
};

// Where a lane's q-th four elements lie in the warp's shared memory (the four
// are exchanged so that 8 lanes fill all banks), and where element `lane` of
// block i does.
__device__ __forceinline__ int four_at(int lane, int q) { return 16 * lane + 4 * (q ^ (lane >> 1 & 3)); }
__device__ __forceinline__ int element_at(int i, int lane) {
    return 32 * i + (lane & 16) + 4 * ((lane >> 2 & 3) ^ (i & 3)) + (lane & 3);
}

// Writes this thread's 16 elements, those of the row.  Whole warps call this.
template <typename T>
__device__ __forceinline__ void put(const Dense<T> &Y, int64_t row, int64_t col, int64_t cols, float *stage,
                                    const Sixteen<T> &x) {
    constexpr int kWords = sizeof(x.w) / 4;
    if (Y.align && __all_sync(~0u, col + 16 <= cols || col >= cols)) {
        if (col >= cols) return;
        char *p = reinterpret_cast<char *>(Y.p + row * Y.ld + col);
        if (Y.align == 2) {
#pragma unroll
            for (int i = 0; i < kWords; i += 8) store32(p + 4 * i, x.w + i);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4 *>(p + 4 * i) = *reinterpret_cast<const uint4 *>(x.w + i);
        }
        return;
    }
    const int lane = threadIdx.x % 32;
    const Blocks b(row, col, cols, Y.ld);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4 *>(stage + four_at(lane, i / 4)) = make_float4(x(i), x(i + 1), x(i + 2), x(i + 3));
    __syncwarp();
    b.each([&](int i, int64_t at) { Y.p[at] = from_float<T>(stage[element_at(i, lane)]); });
}

#define COSTA_MX_STAGE                                        \
    __shared__ __align__(16) float stages[kThreads / 32][512]; \
    float *const stage = stages[threadIdx.x / 32]

struct Codes {
    uint8_t *codes, *scales;
    int64_t ld;
    int64_t unit;  // E2M1: scale tiles of a band of rows; I8: bytes of a row of scales
};

Codes codes(const costa_mx_matrix &q) {
    return {static_cast<uint8_t *>(q.codes), static_cast<uint8_t *>(q.scales), q.ld,
            q.format == COSTA_MX_E2M1 ? mx_scale_tiles(q.cols) : mx_scale_pitch(q.cols)};
}

// Writes the codes of 16 elements at (row, col) and returns the block's scale
// byte; whole warps call this.  Only columns of existing blocks are written.
template <int FMT, typename T>
__device__ __forceinline__ int put_codes(const Codes &q, bool in, int64_t row, int64_t col, int64_t cols,
                                         const Sixteen<T> &x) {
    const int e = x.exponent();
    const int s = scale_byte<FMT>(max(e, __shfl_xor_sync(~0u, e, 1)));
    if (in && col < ((cols + 31) & ~int64_t(31))) {
        if constexpr (FMT == COSTA_MX_E2M1) {
            uint2 w = x.e2m1(e2m1_factor(s));
            if (s == 255) w = make_uint2(0, 0);
            *reinterpret_cast<uint2 *>(q.codes + row * q.ld + col / 2) = w;
        } else {
            auto low = [&](int i) { return x(i); };
            auto high = [&](int i) { return x(i + 8); };
            const uint2 a = i8_of8(low, s), b = i8_of8(high, s);
            *reinterpret_cast<uint4 *>(q.codes + row * q.ld + col) = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
    return s;
}

// The same with the scale.  E2M1: `col` may lie in the padding of the last scale tile.
template <int FMT, typename T>
__device__ __forceinline__ void put16(const Codes &q, bool in, int64_t row, int64_t col, int64_t cols,
                                      const Sixteen<T> &x) {
    const int s = put_codes<FMT>(q, in, row, col, cols, x);
    if (!in || (col & 31) != 0) return;
    if constexpr (FMT == COSTA_MX_E2M1)
        q.scales[scale_at(row, col >> 5, q.unit)] = static_cast<uint8_t>(s);
    else
        q.scales[row * q.unit + (col >> 5)] = static_cast<uint8_t>(s);
}

// 16 codes of I8 and what they are multiples of.
struct Coded {
    uint32_t w[4];
    float unit;
    __device__ void load(const Codes &q, int64_t row, int64_t col) {
        const uint4 v = *reinterpret_cast<const uint4 *>(q.codes + row * q.ld + col);
        w[0] = v.x;
        w[1] = v.y;
        w[2] = v.z;
        w[3] = v.w;
        unit = i8_unit(q.scales[row * q.unit + (col >> 5)]);
    }
    __device__ void four(int i, float (&v)[4]) const { i8_to4(w[i], unit, v); }  // values of codes 4 i .. 4 i + 3
};

// Groups of a row of codes: whole blocks, and for E2M1 whole scale tiles.
Groups groups(const costa_mx_matrix &q, bool tiles) {
    return groups_of(q.rows,
                     tiles && q.format == COSTA_MX_E2M1 ? mx_scale_tiles(q.cols) * 8 : mx_blocks(q.cols) * 2);
}

// Quantisation along rows: the largest magnitude of a block from two lanes, one
// shuffle; a power-of-two factor, exact; one conversion.  8192 x 8192 bf16 to
// E2M1 27 us (6180 GB/s), to I8 31 us (6530); f32 43 us (7030).
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) quantize_n_kernel(Dense<const T> X, Codes Q, int64_t cols, Groups gr) {
    int64_t row, col;
    let_next_start();
    const bool in = gr.at(cols, row, col);
    Sixteen<T> x;
    after_previous();
    get(X, row, col, cols, x);
    put16<FMT>(Q, in, row, col, cols, x);
}

// The values of codes, exact in either type: 8192 x 8192 E2M1 to bf16 27 us (6220
// GB/s), to f32 45 us (6800); to f32 rows of an odd stride, through shared
// memory, 2777 x 4093 11 us (4650).
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(Codes Q, Dense<T> Y, int64_t cols, Groups gr) {
    COSTA_MX_STAGE;
    int64_t row, col;
    let_next_start();
    const bool in = gr.at(cols, row, col);
    Sixteen<T> y;
    after_previous();
    if constexpr (FMT == COSTA_MX_E2M1) {
        uint2 w{};
        __nv_bfloat162 unit = e2m1_unit(0);
        if (in) {
            w = *reinterpret_cast<const uint2 *>(Q.codes + row * Q.ld + col / 2);
            unit = e2m1_unit(Q.scales[scale_at(row, col >> 5, Q.unit)]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t v[2];
            e2m1_to4((i < 2 ? w.x : w.y) >> (i % 2 * 16), unit, v);
            y.set_pairs(4 * i, v);
        }
    } else {
        Coded q{};
        if (in) q.load(Q, row, col);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[4];
            q.four(i, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) y.set(4 * i + j, v[j]);
        }
    }
    put(Y, row, col, cols, stage, y);
}

// Quantisation across rows: a block is 32 rows of one column, which one thread
// holds.  A thread block takes 128 rows x 128 columns, which is a tile of
// E2M1's scales in either order; a warp 32 rows x 64 columns, two to a lane
// (neighbours where bf16 rows are 4-byte aligned, else 32 apart).  The codes go
// through shared memory so that each column's 4 blocks (64 or 128 bytes of a
// row of QT) are written together.  Neighbouring thread blocks take
// neighbouring columns, for the memory's pages.  With BOTH the same rows are
// then read again, from the cache, 8 lanes to a row.  8192 x 8192 bf16 to E2M1
// 27 us (6290 GB/s); both orders 41 us (4970 GB/s), where it issues 16
// instructions an element, 67% of the issue slots; two calls take 55.
constexpr int kTile = 128;

// The codes of a block of 32 elements x(0) .. x(31) with scale byte s (E2M1: taken
// to the codes' range already), to shared memory.
template <int FMT, typename F> __device__ __forceinline__ void block_codes(uint8_t *to, int s, F x) {
    constexpr int kWords = FMT == COSTA_MX_E2M1 ? 4 : 8;
    uint32_t w[kWords];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        auto y = [&](int i) { return x(8 * k + i); };
        if constexpr (FMT == COSTA_MX_E2M1) {
            w[k] = s == 255 ? 0 : e2m1_of8(y);
        } else {
            const uint2 u = i8_of8(y, s);
            w[2 * k] = u.x;
            w[2 * k + 1] = u.y;
        }
    }
#pragma unroll
    for (int k = 0; k < kWords; k += 4) reinterpret_cast<uint4 *>(to)[k / 4] = make_uint4(w[k], w[k + 1], w[k + 2], w[k + 3]);
}

template <typename T, int FMT, bool BOTH>
__global__ void __launch_bounds__(kThreads, 4) quantize_t_kernel(Dense<const T> X, bool pairs, int64_t rows, int64_t cols,
                                                                 Codes QN, Codes QT, unsigned col_tiles) {
    constexpr int kBlockBytes = FMT == COSTA_MX_E2M1 ? 16 : 32, kPitch = 4 * kBlockBytes + 16;
    __shared__ __align__(16) uint8_t codes[kTile * kPitch];
    __shared__ __align__(16) uint8_t sc[2][kTile][4];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, block = warp % 4, left = warp / 4 * 64;
    const int64_t r0 = int64_t(blockIdx.x / col_tiles) * kTile, c0 = int64_t(blockIdx.x % col_tiles) * kTile;
    const int in_rows = static_cast<int>(max(int64_t(0), min(int64_t(32), rows - r0 - 32 * block)));
    let_next_start();
    after_previous();
    // Whole tiles: rows at uniform addresses, this thread's elements at a 32-bit distance (8192 x 8192 bf16 to E2M1 29.5
    // -> 27.0 us, both orders 43.9 -> 41.3; f32 in both orders would have no registers for it: 58.9, 62.3).
    const bool whole = (sizeof(T) == 2 || !BOTH) && r0 + kTile <= rows && c0 + kTile <= cols && X.ld < (1 << 21);
    const char *const tile = reinterpret_cast<const char *>(X.p + r0 * X.ld + c0);
    if (sizeof(T) == 2 && pairs) {
        const uint32_t place = (32 * block * static_cast<uint32_t>(X.ld) + left + 2 * lane) * 2;
        const int64_t c = c0 + left + 2 * lane;
        const T *p = X.p + (r0 + 32 * block) * X.ld + c;
        const int in_cols = static_cast<int>(max(int64_t(0), min(int64_t(2), cols - c)));
        uint32_t v[32], a = 0;
        if (whole) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = *reinterpret_cast<const uint32_t *>(tile + i * X.ld * 2 + place);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i, p += X.ld) {
                v[i] = 0;
                if (i < in_rows && in_cols == 2)
                    v[i] = *reinterpret_cast<const uint32_t *>(p);
                else if (i < in_rows && in_cols == 1)
                    v[i] = *reinterpret_cast<const uint16_t *>(p);
            }
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) a = larger2(a, v[i]);
        const int sc2[2] = {scale_byte<FMT>((a & 0xffffu) >> 7), scale_byte<FMT>(a >> 23)};
        if constexpr (FMT == COSTA_MX_E2M1) {
            const __nv_bfloat162 f = __floats2bfloat162_rn(e2m1_factor(sc2[0]), e2m1_factor(sc2[1]));
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = word(__hmul2(halves(v[i]), f));
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int col = left + 2 * lane + h;
            sc[0][col][block] = static_cast<uint8_t>(sc2[h]);
            block_codes<FMT>(codes + col * kPitch + block * kBlockBytes, sc2[h],
                             [&](int i) { return h ? high_of(v[i]) : low_of(v[i]); });
        }
    } else {
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int col = left + lane + 32 * h;
            const T *p = X.p + (r0 + 32 * block) * X.ld + c0 + col;
            const int in = c0 + col < cols ? in_rows : 0;
            const uint32_t place = (32 * block * static_cast<uint32_t>(X.ld) + col) * sizeof(T);
            float x[32];
            float a = 0.0f;
            if (whole) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    x[i] = to_float(*reinterpret_cast<const T *>(tile + i * X.ld * static_cast<int64_t>(sizeof(T)) + place));
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i, p += X.ld) x[i] = i < in ? to_float(*p) : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) a = larger(a, x[i]);
            const int s = scale_byte<FMT>(__float_as_uint(a) >> 23);
            sc[0][col][block] = static_cast<uint8_t>(s);
            const float f = FMT == COSTA_MX_E2M1 ? e2m1_factor(s) : 1.0f;
            block_codes<FMT>(codes + col * kPitch + block * kBlockBytes, s,
                             [&](int i) { return FMT == COSTA_MX_E2M1 ? x[i] * f : x[i]; });
        }
    }
    __syncthreads();
    const int64_t nb = (rows + 31) >> 5, b0 = r0 >> 5;  // blocks of a row of QT; the first of these
    constexpr int kChunks = 4 * kBlockBytes / 16;       // 16-byte pieces of a column's codes
#pragma unroll
    for (int j = 0; j < kTile * kChunks / kThreads; ++j) {
        const int k = j * kThreads + threadIdx.x, col = k / kChunks, piece = k % kChunks;
        if (c0 + col < cols && b0 + piece * 16 / kBlockBytes < nb)
            *reinterpret_cast<uint4 *>(QT.codes + (c0 + col) * QT.ld + b0 * kBlockBytes + piece * 16) =
                *reinterpret_cast<const uint4 *>(codes + col * kPitch + piece * 16);
    }
    // The 4 scales of row `row` of a matrix of codes of `q_rows` x `q_cols`, from `from`.
    auto put_scales = [](const Codes &q, int64_t row, int64_t q_rows, int64_t q_cols, int64_t first, const uint8_t *from) {
        if (row >= q_rows) return;
        if constexpr (FMT == COSTA_MX_E2M1) {
            *reinterpret_cast<uint32_t *>(q.scales + scale_at(row, first, q.unit)) = *reinterpret_cast<const uint32_t *>(from);
        } else {
            uint8_t *to = q.scales + row * q.unit + first;
            const int64_t left_over = ((q_cols + 31) >> 5) - first;
            if (left_over >= 4)
                *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(from);
            else
                for (int64_t i = 0; i < left_over; ++i) to[i] = from[i];
        }
    };
    if (threadIdx.x < kTile) put_scales(QT, c0 + threadIdx.x, cols, rows, b0, sc[0][threadIdx.x]);
    if constexpr (BOTH) {
        const int64_t col = c0 + lane % 8 * 16;
        Sixteen<T> y[2];
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int64_t row = r0 + 16 * warp + 4 * (i + k) + lane / 8;
                get(X, min(row, rows - 1), row < rows ? col : cols, cols, y[k]);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int64_t row = r0 + 16 * warp + 4 * (i + k) + lane / 8;
                const int s = put_codes<FMT>(QN, row < rows, row, col, cols, y[k]);
                if (lane % 2 == 0) sc[1][row - r0][lane % 8 / 2] = static_cast<uint8_t>(s);
            }
        }
        __syncthreads();
        if (threadIdx.x < kTile) put_scales(QN, r0 + threadIdx.x, rows, cols, c0 >> 5, sc[1][threadIdx.x]);
    }
}

// SiLU and GELU are accurate to their own size, in the tails too.  f32: within 10
// and 19 units of 2^-24 of themselves, down to where e^-|x| or e^(-x^2 / 2) is
// subnormal.  bf16, whose rounding is off by up to 2^-8: within 2^-16 and 2^-15,
// with cheaper exponentials (8192 x 16384 gated, the f32 forms: SiLU forward 197
// us for 181, GELU 235 and backward 212 for 203 and 174); they flush to 0 what
// is below 2^-126, where the result is below |x| 2^-126.
template <typename T> constexpr bool kShort = sizeof(T) == 2;

__device__ __forceinline__ float fast_exp2(float x) {
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    return e;
}
__device__ __forceinline__ float fast_inverse(float x) {  // of x >= 1
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// s = 1 / (1 + e^-x) and rest = 1 - s; f32: both from e^-|x| <= 1, so that neither is a difference.
template <typename T> __device__ __forceinline__ float sigmoid(float x, float &rest) {
    if constexpr (kShort<T>) {
        const float s = fast_inverse(1.0f + fast_exp2(x * -1.4426950408889634f));
        rest = 1.0f - s;
        return s;
    } else {
        const float e = expf(-fabsf(x)), r = fast_inverse(1.0f + e), t = e * r;
        rest = x < 0.0f ? r : t;
        return x < 0.0f ? t : r;
    }
}

// The normal distribution's cdf at x, and e^(-x^2 / 2).  The tail beyond |x| is
// e^(-x^2 / 2) R(|x|); R falls slowly.  With t = 1 / (1 + p |x|), R / t is taken as
// a polynomial, in u = 1 - t from 1/2 at 0 (f32) or in t (bf16), fitted for the
// least relative error: 3.6e-8 on 0 .. 14.5, past which the tail is below 2^-149,
// and 4.7e-6 on 0 .. 13.2.  f32 takes x^2 with what its rounding leaves.
template <typename T> __device__ __forceinline__ float normal_cdf(float x, float &e) {
    float tail;
    if constexpr (kShort<T>) {
        const float t = fast_inverse(fmaf(fabsf(x), 0.31f, 1.0f));
        float s = fmaf(t, -0.0739290646f, 0.180450087f);
        s = fmaf(t, s, 0.0157450492f);
        s = fmaf(t, s, 0.133429573f);
        s = fmaf(t, s, 0.120441339f);
        s = fmaf(t, s, 0.123860695f);
        e = fast_exp2(x * x * (-0.5f * 1.4426950408889634f));
        tail = t * s * e;
    } else {
        const float a = fminf(fabsf(x), 16.0f), t = fast_inverse(fmaf(a, 0.35f, 1.0f)), u = 1.0f - t;
        float s = fmaf(u, -0.0289184507f, 0.0883767232f);
        s = fmaf(u, s, -0.0627829507f);
        s = fmaf(u, s, -0.0170807354f);
        s = fmaf(u, s, -0.0637271628f);
        s = fmaf(u, s, 0.102527089f);
        s = fmaf(u, s, 0.261060268f);
        s = fmaf(u, s, -0.639832914f);
        s = fmaf(u, s, 0.5f);
        const float square = a * a, left = fmaf(a, a, -square);
        e = expf(-0.5f * square);
        e = fmaf(e, -0.5f * left, e);
        tail = t * s * e;
    }
    return x < 0.0f ? tail : 1.0f - tail;
}

// act(x) and act'(x), for results of type T.
template <int ACT, typename T> __device__ __forceinline__ float act(float x) {
    float unused;
    if constexpr (ACT == COSTA_MX_SILU) return x * sigmoid<T>(x, unused);
    if constexpr (ACT == COSTA_MX_GELU) return x * normal_cdf<T>(x, unused);
    return x > 0.0f || x != x ? x : 0.0f;
}
template <int ACT, typename T> __device__ __forceinline__ void act_both(float x, float &y, float &slope) {
    if constexpr (ACT == COSTA_MX_SILU) {
        float rest;
        const float s = sigmoid<T>(x, rest);
        y = x * s;
        slope = kShort<T> ? s * (1.0f + x * rest) : fmaf(y, rest, s);
    } else if constexpr (ACT == COSTA_MX_GELU) {
        float e;
        const float c = normal_cdf<T>(x, e);
        y = x * c;
        slope = fmaf(x * e, 0.3989422804014327f, c);
    } else {
        y = act<ACT, T>(x);
        slope = x != x ? x : x > 0.0f ? 1.0f : 0.0f;
    }
}

// Y and the checkpoints from one pass over X (and G).  8192 x 16384, gated, bf16:
// SiLU 181 us (5980 GB/s), GELU 203 us (5330), whose cdf is beside the traffic; f32:
// 266 us (7080) and 276 us (6840).
template <typename T, int ACT, bool GATED>
__global__ void __launch_bounds__(kThreads, 4) act_forward_kernel(Dense<const T> X, Dense<const T> G, Dense<T> Y, Codes QX,
                                                               Codes QG, int64_t cols, Groups gr) {
    COSTA_MX_STAGE;
    int64_t row, col;
    let_next_start();
    const bool in = gr.at(cols, row, col);
    Sixteen<T> x, g, y;
    after_previous();
    get(X, row, col, cols, x);
    if constexpr (GATED) get(G, row, col, cols, g);
#pragma unroll
    for (int i = 0; i < 16; ++i) y.set(i, GATED ? act<ACT, T>(x(i)) * g(i) : act<ACT, T>(x(i)));
    put(Y, row, col, cols, stage, y);
    put16<COSTA_MX_I8>(QX, in, row, col, cols, x);
    if constexpr (GATED) put16<COSTA_MX_I8>(QG, in, row, col, cols, g);
}

// The gradients from the checkpoints, nothing else kept.  8192 x 16384, gated, bf16:
// SiLU 163 us (6640 GB/s; with five blocks of an SM 171), GELU 174 us (6220); f32:
// 272 us (6950) and 280 us (6730).
template <typename T, int ACT, bool GATED>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 6 : 4) act_backward_kernel(Codes QX, Codes QG, Dense<const T> dY, Dense<T> dX,
                                                                Dense<T> dG, int64_t cols, Groups gr) {
    COSTA_MX_STAGE;
    int64_t row, col;
    let_next_start();
    const bool in = gr.at(cols, row, col);
    Sixteen<T> d, dx, dg;
    Coded x{}, g{};
    after_previous();
    if (in) {
        x.load(QX, row, col);
        if constexpr (GATED) g.load(QG, row, col);
    }
    get(dY, row, col, cols, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float xs[4], gs[4];
        x.four(i, xs);
        if constexpr (GATED) g.four(i, gs);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = 4 * i + j;
            float y, slope;
            act_both<ACT, T>(xs[j], y, slope);
            if constexpr (GATED) {
                dg.set(k, d(k) * y);
                dx.set(k, d(k) * gs[j] * slope);
            } else {
                dx.set(k, d(k) * slope);
            }
        }
    }
    put(dX, row, col, cols, stage, dx);
    if constexpr (GATED) put(dG, row, col, cols, stage, dg);
}

template <typename T, int ACT>
cudaError_t forward(const costa_mx_dense &X, const costa_mx_dense *G, const costa_mx_dense &Y, const costa_mx_matrix &QX,
                    const costa_mx_matrix *QG, cudaStream_t s) {
    const Groups gr = groups(QX, false);
    return mx_launch(G ? act_forward_kernel<T, ACT, true> : act_forward_kernel<T, ACT, false>, blocks_for(gr), kThreads, 0,
                     1, s, dense<const T>(X), G ? dense<const T>(*G) : Dense<const T>{}, dense<T>(Y), codes(QX),
                     QG ? codes(*QG) : Codes{}, X.cols, gr);
}

template <typename T, int ACT>
cudaError_t backward(const costa_mx_matrix &QX, const costa_mx_matrix *QG, const costa_mx_dense &dY,
                     const costa_mx_dense &dX, const costa_mx_dense *dG, cudaStream_t s) {
    const Groups gr = groups(QX, false);
    return mx_launch(QG ? act_backward_kernel<T, ACT, true> : act_backward_kernel<T, ACT, false>, blocks_for(gr), kThreads,
                     0, 1, s, codes(QX), QG ? codes(*QG) : Codes{}, dense<const T>(dY), dense<T>(dX),
                     dG ? dense<T>(*dG) : Dense<T>{}, dY.cols, gr);
}

template <typename F> cudaError_t by_type(int type, F f) {
    return type == COSTA_MX_F32 ? f(float{}) : f(__nv_bfloat16{});
}

}  // namespace
}  // namespace mx

using namespace mx;

cudaError_t launch_mx_quantize_n(const costa_mx_dense &X, const costa_mx_matrix &Q, cudaStream_t s) {
    return by_type(X.type, [&](auto t) {
        using T = decltype(t);
        const Groups gr = groups(Q, true);
        return mx_launch(Q.format == COSTA_MX_E2M1 ? quantize_n_kernel<T, COSTA_MX_E2M1> : quantize_n_kernel<T, COSTA_MX_I8>,
                         blocks_for(gr), kThreads, 0, 1, s, dense<const T>(X), codes(Q), X.cols, gr);
    });
}

cudaError_t launch_mx_quantize_t(const costa_mx_dense &X, const costa_mx_matrix *QN, const costa_mx_matrix &QT,
                                 cudaStream_t s) {
    return by_type(X.type, [&](auto t) {
        using T = decltype(t);
        const int64_t col_tiles = mx_ceil(X.cols, kTile);
        const bool pairs = reinterpret_cast<uint64_t>(X.ptr) % 4 == 0 && X.ld % 2 == 0, e2m1 = QT.format == COSTA_MX_E2M1;
        return mx_launch(QN ? (e2m1 ? quantize_t_kernel<T, COSTA_MX_E2M1, true> : quantize_t_kernel<T, COSTA_MX_I8, true>)
                            : (e2m1 ? quantize_t_kernel<T, COSTA_MX_E2M1, false> : quantize_t_kernel<T, COSTA_MX_I8, false>),
                         col_tiles * mx_ceil(X.rows, kTile), kThreads, 0, 1, s, dense<const T>(X), pairs, X.rows, X.cols,
                         QN ? codes(*QN) : Codes{}, codes(QT), static_cast<unsigned>(col_tiles));
    });
}

cudaError_t launch_mx_dequantize(const costa_mx_matrix &Q, const costa_mx_dense &Y, cudaStream_t s) {
    return by_type(Y.type, [&](auto t) {
        using T = decltype(t);
        const Groups gr = groups(Q, false);
        return mx_launch(Q.format == COSTA_MX_E2M1 ? dequantize_kernel<T, COSTA_MX_E2M1> : dequantize_kernel<T, COSTA_MX_I8>,
                         blocks_for(gr), kThreads, 0, 1, s, codes(Q), dense<T>(Y), Y.cols, gr);
    });
}

cudaError_t launch_mx_act_forward(int a, const costa_mx_dense &X, const costa_mx_dense *G, const costa_mx_dense &Y,
                                  const costa_mx_matrix &QX, const costa_mx_matrix *QG, cudaStream_t s) {
    return by_type(X.type, [&](auto t) {
        using T = decltype(t);
        return a == COSTA_MX_SILU   ? forward<T, COSTA_MX_SILU>(X, G, Y, QX, QG, s)
               : a == COSTA_MX_GELU ? forward<T, COSTA_MX_GELU>(X, G, Y, QX, QG, s)
                                    : forward<T, COSTA_MX_RELU>(X, G, Y, QX, QG, s);
    });
}

cudaError_t launch_mx_act_backward(int a, const costa_mx_matrix &QX, const costa_mx_matrix *QG,
                                   const costa_mx_dense &dY, const costa_mx_dense &dX, const costa_mx_dense *dG,
                                   cudaStream_t s) {
    return by_type(dY.type, [&](auto t) {
        using T = decltype(t);
        return a == COSTA_MX_SILU   ? backward<T, COSTA_MX_SILU>(QX, QG, dY, dX, dG, s)
               : a == COSTA_MX_GELU ? backward<T, COSTA_MX_GELU>(QX, QG, dY, dX, dG, s)
                                    : backward<T, COSTA_MX_RELU>(QX, QG, dY, dX, dG, s);
    });
}

}  // namespace costa
