// Host helpers of the low-bit products' launchers.
#pragma once

#include <cstdint>

#include <cuda.h>
#include <cuda_runtime_api.h>

#include "costa_gb300.h"

namespace costa {

// The 2-D tensor map of bytes (128-byte swizzle, zeros outside): `width` bytes
// x `rows`, `pitch` bytes from row to row, boxes of 128 bytes x `box_rows`.
cudaError_t mx_byte_map(CUtensorMap *map, const void *base, uint64_t width, uint64_t rows, uint64_t pitch,
                        uint32_t box_rows);
// C = beta C (0 without reading C for beta == 0): products over nothing.
cudaError_t launch_mx_scale(float beta, const costa_mx_dense &C, cudaStream_t s);
// Waits that gave up, on the current device since the library was loaded.
cudaError_t mx_product_failures(unsigned *count);
cudaError_t mx_grad_failures(unsigned *count);

}  // namespace costa
