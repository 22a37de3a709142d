// dW = alpha dY^T X + beta dW with X from its 8-bit checkpoint.
#include "costa_internal.h"
#include "mx_device.cuh"
#include "mx_host.h"

namespace costa {
namespace mx {
namespace {

constexpr int kTile = 32;

template <typename T, typename W>
__global__ void __launch_bounds__(256) grad_kernel(const T *dY, int64_t ldy, costa_mx_matrix Q, int64_t pitch,
                                                   float alpha, float beta, W *dW, int64_t ldw, int64_t n,
                                                   unsigned col_tiles) {
    __shared__ float a[kTile][33], b[kTile][33];  // tokens x columns
    const int64_t i0 = int64_t(blockIdx.x / col_tiles) * kTile, j0 = int64_t(blockIdx.x % col_tiles) * kTile;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
    const uint8_t *codes = static_cast<const uint8_t *>(Q.codes), *scales = static_cast<const uint8_t *>(Q.scales);
    for (int64_t t0 = 0; t0 < Q.rows; t0 += kTile) {
        for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + ty + 8 * i;
            a[ty + 8 * i][tx] = t < Q.rows && i0 + tx < n ? to_float(dY[t * ldy + i0 + tx]) : 0.0f;
            b[ty + 8 * i][tx] = 0.0f;
            if (t < Q.rows && j0 + tx < Q.cols)
                b[ty + 8 * i][tx] = i8_unit(scales[t * pitch + (j0 >> 5)]) *
                                    static_cast<float>(static_cast<int8_t>(codes[t * Q.ld + j0 + tx]));
        }
        __syncthreads();
        for (int q = 0; q < kTile; ++q)
            for (int i = 0; i < 4; ++i) acc[i] += a[q][ty + 8 * i] * b[q][tx];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int64_t row = i0 + ty + 8 * i, col = j0 + tx;
        if (row < n && col < Q.cols) {
            W *c = dW + row * ldw + col;
            *c = from_float<W>(beta == 0.0f ? alpha * acc[i] : alpha * acc[i] + beta * to_float(*c));
        }
    }
}

template <typename T, typename W>
void launch(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta, const costa_mx_dense &dW,
            cudaStream_t s) {
    const unsigned cols = static_cast<unsigned>(mx_ceil(dW.cols, kTile));
    const unsigned grid = static_cast<unsigned>(cols * mx_ceil(dW.rows, kTile));
    grad_kernel<T, W><<<grid, 256, 0, s>>>(static_cast<const T *>(dY.ptr), dY.ld, Q, mx_scale_pitch(Q.cols), alpha, beta,
                                           static_cast<W *>(dW.ptr), dW.ld, dW.rows, cols);
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_weight_grad(const costa_mx_dense &dY, const costa_mx_matrix &Q, float alpha, float beta,
                                  const costa_mx_dense &dW, cudaStream_t s) {
    if (dY.rows == 0) return launch_mx_scale(beta, dW, s);
    using bf16 = __nv_bfloat16;
    const bool wf = dW.type == COSTA_MX_F32;
    if (dY.type == COSTA_MX_F32)
        wf ? mx::launch<float, float>(dY, Q, alpha, beta, dW, s) : mx::launch<float, bf16>(dY, Q, alpha, beta, dW, s);
    else
        wf ? mx::launch<bf16, float>(dY, Q, alpha, beta, dW, s) : mx::launch<bf16, bf16>(dY, Q, alpha, beta, dW, s);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

cudaError_t mx_grad_failures(unsigned *count) {
    *count = 0;
    return cudaSuccess;
}

}  // namespace costa
