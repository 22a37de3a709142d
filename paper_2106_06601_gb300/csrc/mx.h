// Low-bit matrices: what the entry points (mx.cpp) pass to the kernels
// (mx_elementwise.cu, mx_product.cu, mx_grad.cu).  All arguments are checked
// and no extent is zero unless a launcher says so.
#pragma once

#include <cstdint>

#include <cuda_runtime_api.h>

#include "costa_gb300.h"

namespace costa {

// Blocks of 32 elements in a row, and what pads them in storage.
constexpr int64_t mx_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t mx_blocks(int64_t cols) { return mx_ceil(cols, 32); }
// E2M1: tiles of 128 rows x 4 blocks; I8: bytes of a row of scales.
constexpr int64_t mx_scale_tiles(int64_t cols) { return mx_ceil(mx_blocks(cols), 4); }
constexpr int64_t mx_scale_pitch(int64_t cols) { return mx_ceil(mx_blocks(cols), 8) * 8; }

cudaError_t launch_mx_quantize_n(const costa_mx_dense &X, const costa_mx_matrix &Q, cudaStream_t s);
// QN may be null.
cudaError_t launch_mx_quantize_t(const costa_mx_dense &X, const costa_mx_matrix *QN, const costa_mx_matrix &QT,
                                 cudaStream_t s);
cudaError_t launch_mx_dequantize(const costa_mx_matrix &Q, const costa_mx_dense &Y, cudaStream_t s);
// G, QG (forward) and QG, dG (backward) may be null.
cudaError_t launch_mx_act_forward(int act, const costa_mx_dense &X, const costa_mx_dense *G, const costa_mx_dense &Y,
                                  const costa_mx_matrix &QX, const costa_mx_matrix *QG, cudaStream_t s);
cudaError_t launch_mx_act_backward(int act, const costa_mx_matrix &QX, const costa_mx_matrix *QG,
                                   const costa_mx_dense &dY, const costa_mx_dense &dX, const costa_mx_dense *dG,
                                   cudaStream_t s);
// The reduced extent (A's columns, dY's rows) may be zero.
cudaError_t launch_mx_product(const costa_mx_matrix &A, const costa_mx_matrix &B, float alpha, float beta,
                              const costa_mx_dense &C, cudaStream_t s);
cudaError_t launch_mx_weight_grad(const costa_mx_dense &dY, const costa_mx_matrix &QX, float alpha, float beta,
                                  const costa_mx_dense &dW, cudaStream_t s);

}  // namespace costa
