// Low-bit matrices: what the entry points (mx.cpp) pass to the kernels
// (mx_elementwise.cu, mx_product.cu, mx_grad.cu); and what stands around them:
// mx_layer.cpp to mx_norm.cu, mx_experts.cu and mx_distill.cu.  All arguments are checked
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

// Blocks of the norm's gradients at most, each with partial sums of dW: four to an SM up to 1024 columns, else two.
constexpr int64_t mx_norm_parts(int64_t cols) { return cols <= 1024 ? 608 : 304; }
// R with H may be null; and any of Y, Q4, Q8 and S.
cudaError_t launch_mx_norm_forward(const costa_mx_dense &X, const costa_mx_dense *R, const costa_mx_dense &W, float eps,
                                   const costa_mx_dense *H, const costa_mx_dense *Y, const costa_mx_matrix *Q4,
                                   const costa_mx_matrix *Q8, const costa_mx_dense *S, cudaStream_t s);
// dH may be null, and dW; no rows are allowed where dW is not.
cudaError_t launch_mx_norm_backward(const costa_mx_dense &dY, const costa_mx_dense &H, const costa_mx_dense &S,
                                    const costa_mx_dense &W, const costa_mx_dense *dH, const costa_mx_dense &dX,
                                    const costa_mx_dense *dW, void *work, cudaStream_t s);
// No tokens and no experts of a token are allowed.
cudaError_t launch_mx_expert_sort(const costa_mx_index &experts, int n_experts, int align, const costa_mx_index &place,
                                  const costa_mx_index &starts, const costa_mx_index &counts, cudaStream_t s);
// rows: those that places may name.  Any of Y, Q4 and Q8 may be null.
cudaError_t launch_mx_dispatch(const costa_mx_dense &X, const costa_mx_index &place, int64_t rows, const costa_mx_dense *Y,
                               const costa_mx_matrix *Q4, const costa_mx_matrix *Q8, cudaStream_t s);
// W may be null; a token may have no experts, and Z no rows.
cudaError_t launch_mx_combine(const costa_mx_dense &Z, const costa_mx_index &place, const costa_mx_dense *W,
                              const costa_mx_dense &Y, cudaStream_t s);
// Z with dW may be null, and dZ and Q4; no columns are allowed.
cudaError_t launch_mx_combine_backward(const costa_mx_dense &dY, const costa_mx_dense *Z, const costa_mx_index &place,
                                       int64_t rows, const costa_mx_dense &W, const costa_mx_dense *dZ,
                                       const costa_mx_matrix *Q4, const costa_mx_dense *dW, cudaStream_t s);
// loss null: the gradient from stats; G and dZ null: no gradient.  No columns and no entries are allowed.
cudaError_t launch_mx_distill(const costa_mx_dense &Z, const costa_mx_index &ids, const costa_mx_dense &T, float tau,
                              const costa_mx_dense *loss, const costa_mx_dense &stats, const costa_mx_dense *G,
                              const costa_mx_dense *dZ, cudaStream_t s);

}  // namespace costa
