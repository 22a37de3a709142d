// Kernels that make and read microscaled codes element by element: the
// quantisation of op(X), its inverse, and activations with 8-bit checkpoints.
// All are bound by memory traffic.
#include <algorithm>

#include "costa_internal.h"
#include "mx_device.cuh"

namespace costa {
namespace mx {
namespace {

constexpr int kThreads = 256;

// Rows cut into groups of 8 elements, one to a thread; 4 lanes share a block.
// gpr: groups of a row, a multiple of 4 (a block's lanes lie in one warp).
struct Groups {
    int64_t gpr, total;
    __device__ bool at(int64_t &row, int64_t &col) const {
        const int64_t g = int64_t(blockIdx.x) * kThreads + threadIdx.x;
        if (total <= 0x7fffffff) {
            const uint32_t r = static_cast<uint32_t>(g) / static_cast<uint32_t>(gpr);
            row = r;
            col = (static_cast<uint32_t>(g) - r * static_cast<uint32_t>(gpr)) * 8;
        } else {
            row = g / gpr;
            col = (g - row * gpr) * 8;
        }
        return g < total;
    }
};

unsigned blocks_for(const Groups &g) { return static_cast<unsigned>(mx_ceil(g.total, kThreads)); }

template <typename T> struct Dense {
    T *p;
    int64_t ld;
    bool vec;  // rows start on 16-byte boundaries
};

template <typename T> Dense<T> dense(const costa_mx_dense &d) {
    return {static_cast<T *>(d.ptr), d.ld,
            reinterpret_cast<uint64_t>(d.ptr) % 16 == 0 && (d.ld * static_cast<int64_t>(sizeof(T))) % 16 == 0};
}

struct Codes {
    uint8_t *codes, *scales;
    int64_t ld;
    int64_t unit;  // E2M1: scale tiles of a band of rows; I8: bytes of a row of scales
};

Codes codes(const costa_mx_matrix &q) {
    return {static_cast<uint8_t *>(q.codes), static_cast<uint8_t *>(q.scales), q.ld,
            q.format == COSTA_MX_E2M1 ? mx_scale_tiles(q.cols) : mx_scale_pitch(q.cols)};
}

// The largest magnitude of a block whose 32 elements 4 neighbouring lanes hold.
__device__ __forceinline__ uint32_t block_amax(const float (&x)[8], unsigned lanes) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, magnitude(x[i]));
    a = max(a, __shfl_xor_sync(lanes, a, 1));
    return max(a, __shfl_xor_sync(lanes, a, 2));
}

// Writes the codes of 8 elements at (row, col) and, by the block's first lane,
// the scale.  E2M1: `col` may lie in the padding of the last scale tile.
template <int FMT>
__device__ __forceinline__ void put8(const Codes &q, int64_t row, int64_t col, int64_t cols, const float (&x)[8],
                                     unsigned lanes) {
    const int s = scale_byte<FMT>(block_amax(x, lanes));
    const bool inside = col < ((cols + 31) & ~int64_t(31));
    if constexpr (FMT == COSTA_MX_E2M1) {
        if (inside) *reinterpret_cast<uint32_t *>(q.codes + row * q.ld + col / 2) = e2m1_of8(x, s);
        if ((col & 31) == 0) q.scales[scale_at(row, col >> 5, q.unit)] = static_cast<uint8_t>(s);
    } else {
        if (inside) *reinterpret_cast<uint2 *>(q.codes + row * q.ld + col) = i8_of8(x, s);
        if (inside && (col & 31) == 0) q.scales[row * q.unit + (col >> 5)] = static_cast<uint8_t>(s);
    }
}

template <int FMT>
__device__ __forceinline__ void get8(const Codes &q, int64_t row, int64_t col, float (&v)[8]) {
    if constexpr (FMT == COSTA_MX_E2M1) {
        const float unit = pow2(q.scales[scale_at(row, col >> 5, q.unit)]);
        e2m1_to8(*reinterpret_cast<const uint32_t *>(q.codes + row * q.ld + col / 2), unit, v);
    } else {
        const float unit = i8_unit(q.scales[row * q.unit + (col >> 5)]);
        i8_to8(*reinterpret_cast<const uint2 *>(q.codes + row * q.ld + col), unit, v);
    }
}

// Groups of a row of codes: whole blocks, and for E2M1 whole scale tiles.
Groups groups(const costa_mx_matrix &q, bool tiles) {
    const int64_t gpr = tiles && q.format == COSTA_MX_E2M1 ? mx_scale_tiles(q.cols) * 16 : mx_blocks(q.cols) * 4;
    return {gpr, q.rows * gpr};
}

template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) quantize_n_kernel(Dense<const T> X, Codes Q, int64_t cols, Groups gr) {
    int64_t row, col;
    const bool in = gr.at(row, col);
    const unsigned lanes = __ballot_sync(~0u, in);
    if (!in) return;
    float x[8];
    load8(X.p + row * X.ld, col, cols, X.vec, x);
    put8<FMT>(Q, row, col, cols, x, lanes);
}

template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(Codes Q, Dense<T> Y, int64_t cols, Groups gr) {
    int64_t row, col;
    if (!gr.at(row, col)) return;
    float v[8];
    get8<FMT>(Q, row, col, v);
    store8(Y.p + row * Y.ld, col, cols, Y.vec, v);
}

// Quantisation across rows: a block is 32 rows of one column, which one thread
// holds.  A thread block takes 256 rows x 64 columns; a warp 32 rows, two
// columns to a lane.  The codes go through shared memory so that each column's
// 8 blocks (128 or 256 bytes of a row of QT) are written together.
constexpr int kTRows = 256, kTCols = 64;

template <typename T, int FMT, bool BOTH>
__global__ void __launch_bounds__(kThreads) quantize_t_kernel(Dense<const T> X, int64_t rows, int64_t cols, Codes QN,
                                                              Codes QT, unsigned row_tiles) {
    constexpr int kBlockBytes = FMT == COSTA_MX_E2M1 ? 16 : 32, kPitch = 8 * kBlockBytes + 16;
    __shared__ __align__(16) uint8_t stage[kTCols * kPitch];
    __shared__ uint8_t sc[kTCols][8];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t r0 = int64_t(blockIdx.x % row_tiles) * kTRows, c0 = int64_t(blockIdx.x / row_tiles) * kTCols;
    const int64_t rw = r0 + warp * 32, c = c0 + 2 * lane;
    float x[2][32];
    const bool pair = X.vec && c + 2 <= cols;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const T *p = X.p + (rw + i) * X.ld + c;
        x[0][i] = x[1][i] = 0.0f;
        if (rw + i < rows) {
            if (pair) {
                if constexpr (sizeof(T) == 4) {
                    const float2 v = *reinterpret_cast<const float2 *>(p);
                    x[0][i] = v.x;
                    x[1][i] = v.y;
                } else {
                    const uint32_t v = *reinterpret_cast<const uint32_t *>(p);
                    x[0][i] = __uint_as_float(v << 16);
                    x[1][i] = __uint_as_float(v & 0xffff0000u);
                }
            } else {
                if (c < cols) x[0][i] = to_float(p[0]);
                if (c + 1 < cols) x[1][i] = to_float(p[1]);
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) a = max(a, magnitude(x[h][i]));
        const int s = scale_byte<FMT>(a);
        uint8_t *to = stage + (2 * lane + h) * kPitch + warp * kBlockBytes;
        sc[2 * lane + h][warp] = static_cast<uint8_t>(s);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[h][8 * k + i];
            if constexpr (FMT == COSTA_MX_E2M1)
                *reinterpret_cast<uint32_t *>(to + 4 * k) = e2m1_of8(y, s);
            else
                *reinterpret_cast<uint2 *>(to + 8 * k) = i8_of8(y, s);
        }
    }
    __syncthreads();
    const int64_t nb = (rows + 31) >> 5, b0 = r0 >> 5;  // blocks of a row of QT; the first of these
    constexpr int kChunks = 8 * kBlockBytes / 16;       // 16-byte pieces of a column's codes
    for (int k = threadIdx.x; k < kTCols * kChunks; k += kThreads) {
        const int col = k / kChunks, piece = k % kChunks;
        if (c0 + col < cols && b0 + piece * 16 / kBlockBytes < nb)
            *reinterpret_cast<uint4 *>(QT.codes + (c0 + col) * QT.ld + b0 * kBlockBytes + piece * 16) =
                *reinterpret_cast<const uint4 *>(stage + col * kPitch + piece * 16);
    }
    for (int k = threadIdx.x; k < kTCols * 8; k += kThreads) {
        const int col = k / 8;
        const int64_t b = b0 + k % 8;
        if (c0 + col >= cols) continue;
        if constexpr (FMT == COSTA_MX_E2M1) {
            if (b < QT.unit * 4) QT.scales[scale_at(c0 + col, b, QT.unit)] = sc[col][k % 8];
        } else {
            if (b < nb) QT.scales[(c0 + col) * QT.unit + b] = sc[col][k % 8];
        }
    }
    if constexpr (BOTH) {  // the same rows again, along the columns: 8 lanes to a row (read from the cache)
#pragma unroll 4
        for (int i = 0; i < 32; i += 4) {
            const int64_t row = rw + i + lane / 8, col = c0 + (lane % 8) * 8;
            const bool in = row < rows && col < (FMT == COSTA_MX_E2M1 ? QN.unit * 128 : ((cols + 31) & ~int64_t(31)));
            const unsigned lanes = __ballot_sync(~0u, in);
            if (in) {
                float y[8];
                load8(X.p + row * X.ld, col, cols, X.vec, y);
                put8<FMT>(QN, row, col, cols, y, lanes);
            }
        }
    }
}

// act(x) and act'(x).
template <int ACT> __device__ __forceinline__ float act(float x) {
    if constexpr (ACT == COSTA_MX_SILU) return x / (1.0f + expf(-x));
    if constexpr (ACT == COSTA_MX_GELU) return x * normcdff(x);
    return x > 0.0f || x != x ? x : 0.0f;
}
template <int ACT> __device__ __forceinline__ void act_both(float x, float &y, float &slope) {
    if constexpr (ACT == COSTA_MX_SILU) {
        const float s = 1.0f / (1.0f + expf(-x));
        y = x * s;
        slope = s * (1.0f + x * (1.0f - s));
    } else if constexpr (ACT == COSTA_MX_GELU) {
        const float c = normcdff(x);
        y = x * c;
        slope = c + x * expf(-0.5f * x * x) * 0.3989422804014327f;
    } else {
        y = act<ACT>(x);
        slope = x != x ? x : x > 0.0f ? 1.0f : 0.0f;
    }
}

template <typename T, int ACT, bool GATED>
__global__ void __launch_bounds__(kThreads) act_forward_kernel(Dense<const T> X, Dense<const T> G, Dense<T> Y, Codes QX,
                                                               Codes QG, int64_t cols, Groups gr) {
    int64_t row, col;
    const bool in = gr.at(row, col);
    const unsigned lanes = __ballot_sync(~0u, in);
    if (!in) return;
    float x[8], g[8], y[8];
    load8(X.p + row * X.ld, col, cols, X.vec, x);
    if constexpr (GATED) load8(G.p + row * G.ld, col, cols, G.vec, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = act<ACT>(x[i]);
        if constexpr (GATED) y[i] *= g[i];
    }
    store8(Y.p + row * Y.ld, col, cols, Y.vec, y);
    put8<COSTA_MX_I8>(QX, row, col, cols, x, lanes);
    if constexpr (GATED) put8<COSTA_MX_I8>(QG, row, col, cols, g, lanes);
}

template <typename T, int ACT, bool GATED>
__global__ void __launch_bounds__(kThreads) act_backward_kernel(Codes QX, Codes QG, Dense<const T> dY, Dense<T> dX,
                                                                Dense<T> dG, int64_t cols, Groups gr) {
    int64_t row, col;
    if (!gr.at(row, col)) return;
    float x[8], g[8], d[8], dg[8];
    load8(dY.p + row * dY.ld, col, cols, dY.vec, d);
    get8<COSTA_MX_I8>(QX, row, col, x);
    if constexpr (GATED) get8<COSTA_MX_I8>(QG, row, col, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float y, slope;
        act_both<ACT>(x[i], y, slope);
        if constexpr (GATED) {
            dg[i] = d[i] * y;
            d[i] *= g[i];
        }
        d[i] *= slope;
    }
    store8(dX.p + row * dX.ld, col, cols, dX.vec, d);
    if constexpr (GATED) store8(dG.p + row * dG.ld, col, cols, dG.vec, dg);
}

cudaError_t launched() {
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

template <typename T, int ACT>
cudaError_t forward(const costa_mx_dense &X, const costa_mx_dense *G, const costa_mx_dense &Y, const costa_mx_matrix &QX,
                    const costa_mx_matrix *QG, cudaStream_t s) {
    const Groups gr = groups(QX, false);
    if (G)
        act_forward_kernel<T, ACT, true><<<blocks_for(gr), kThreads, 0, s>>>(
            dense<const T>(X), dense<const T>(*G), dense<T>(Y), codes(QX), codes(*QG), X.cols, gr);
    else
        act_forward_kernel<T, ACT, false><<<blocks_for(gr), kThreads, 0, s>>>(dense<const T>(X), {}, dense<T>(Y),
                                                                              codes(QX), {}, X.cols, gr);
    return launched();
}

template <typename T, int ACT>
cudaError_t backward(const costa_mx_matrix &QX, const costa_mx_matrix *QG, const costa_mx_dense &dY,
                     const costa_mx_dense &dX, const costa_mx_dense *dG, cudaStream_t s) {
    const Groups gr = groups(QX, false);
    if (QG)
        act_backward_kernel<T, ACT, true><<<blocks_for(gr), kThreads, 0, s>>>(
            codes(QX), codes(*QG), dense<const T>(dY), dense<T>(dX), dense<T>(*dG), dY.cols, gr);
    else
        act_backward_kernel<T, ACT, false><<<blocks_for(gr), kThreads, 0, s>>>(
            codes(QX), {}, dense<const T>(dY), dense<T>(dX), {}, dY.cols, gr);
    return launched();
}

template <typename T, int FMT>
cudaError_t quantize_t(const costa_mx_dense &X, const costa_mx_matrix *QN, const costa_mx_matrix &QT, cudaStream_t s) {
    const unsigned row_tiles = static_cast<unsigned>(mx_ceil(X.rows, kTRows));
    // with QN also the columns that fill its last scale tile
    const int64_t col_tiles = QN ? mx_scale_tiles(X.cols) * (128 / kTCols) : mx_ceil(X.cols, kTCols);
    const unsigned grid = static_cast<unsigned>(row_tiles * col_tiles);
    if (QN)
        quantize_t_kernel<T, FMT, true>
            <<<grid, kThreads, 0, s>>>(dense<const T>(X), X.rows, X.cols, codes(*QN), codes(QT), row_tiles);
    else
        quantize_t_kernel<T, FMT, false>
            <<<grid, kThreads, 0, s>>>(dense<const T>(X), X.rows, X.cols, {}, codes(QT), row_tiles);
    return launched();
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
        if (Q.format == COSTA_MX_E2M1)
            quantize_n_kernel<T, COSTA_MX_E2M1>
                <<<blocks_for(gr), kThreads, 0, s>>>(dense<const T>(X), codes(Q), X.cols, gr);
        else
            quantize_n_kernel<T, COSTA_MX_I8>
                <<<blocks_for(gr), kThreads, 0, s>>>(dense<const T>(X), codes(Q), X.cols, gr);
        return launched();
    });
}

cudaError_t launch_mx_quantize_t(const costa_mx_dense &X, const costa_mx_matrix *QN, const costa_mx_matrix &QT,
                                 cudaStream_t s) {
    return by_type(X.type, [&](auto t) {
        using T = decltype(t);
        return QT.format == COSTA_MX_E2M1 ? quantize_t<T, COSTA_MX_E2M1>(X, QN, QT, s)
                                          : quantize_t<T, COSTA_MX_I8>(X, QN, QT, s);
    });
}

cudaError_t launch_mx_dequantize(const costa_mx_matrix &Q, const costa_mx_dense &Y, cudaStream_t s) {
    return by_type(Y.type, [&](auto t) {
        using T = decltype(t);
        const Groups gr = groups(Q, false);
        if (Q.format == COSTA_MX_E2M1)
            dequantize_kernel<T, COSTA_MX_E2M1><<<blocks_for(gr), kThreads, 0, s>>>(codes(Q), dense<T>(Y), Y.cols, gr);
        else
            dequantize_kernel<T, COSTA_MX_I8><<<blocks_for(gr), kThreads, 0, s>>>(codes(Q), dense<T>(Y), Y.cols, gr);
        return launched();
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
