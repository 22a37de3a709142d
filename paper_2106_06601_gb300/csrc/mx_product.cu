// C = alpha A B^T + beta C with A and B in E2M1.
#include "costa_internal.h"
#include "mx_device.cuh"

namespace costa {
namespace mx {
namespace {

constexpr int kTile = 32;

template <typename T>
__global__ void __launch_bounds__(256) product_kernel(costa_mx_matrix A, costa_mx_matrix B, float alpha, float beta,
                                                      T *C, int64_t ldc, unsigned col_tiles) {
    __shared__ float a[kTile][33], b[kTile][33];
    const int64_t i0 = int64_t(blockIdx.x / col_tiles) * kTile, j0 = int64_t(blockIdx.x % col_tiles) * kTile;
    const int64_t tiles = (((A.cols + 31) >> 5) + 3) >> 2;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
    for (int64_t k = 0; k < A.cols; k += 32) {
        {
            const bool is_a = threadIdx.x < 128;
            const int t = threadIdx.x & 127, r = t / 4, g = t % 4;
            const costa_mx_matrix &M = is_a ? A : B;
            const int64_t row = (is_a ? i0 : j0) + r;
            float v[8] = {};
            if (row < M.rows) {
                const float unit = pow2(static_cast<const uint8_t *>(M.scales)[scale_at(row, k >> 5, tiles)]);
                e2m1_to8(*reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(M.codes) + row * M.ld + k / 2 +
                                                             4 * g),
                         unit, v);
            }
            for (int i = 0; i < 8; ++i) (is_a ? a : b)[r][8 * g + i] = v[i];
        }
        __syncthreads();
        for (int q = 0; q < 32; ++q)
            for (int i = 0; i < 4; ++i) acc[i] += a[ty + 8 * i][q] * b[tx][q];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int64_t row = i0 + ty + 8 * i, col = j0 + tx;
        if (row < A.rows && col < B.rows) {
            T *c = C + row * ldc + col;
            *c = from_float<T>(beta == 0.0f ? alpha * acc[i] : alpha * acc[i] + beta * to_float(*c));
        }
    }
}

}  // namespace
}  // namespace mx

cudaError_t launch_mx_product(const costa_mx_matrix &A, const costa_mx_matrix &B, float alpha, float beta,
                              const costa_mx_dense &C, cudaStream_t s) {
    const unsigned cols = static_cast<unsigned>(mx_ceil(C.cols, mx::kTile));
    const unsigned grid = static_cast<unsigned>(cols * mx_ceil(C.rows, mx::kTile));
    if (C.type == COSTA_MX_F32)
        mx::product_kernel<<<grid, 256, 0, s>>>(A, B, alpha, beta, static_cast<float *>(C.ptr), C.ld, cols);
    else
        mx::product_kernel<<<grid, 256, 0, s>>>(A, B, alpha, beta, static_cast<__nv_bfloat16 *>(C.ptr), C.ld, cols);
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace costa
