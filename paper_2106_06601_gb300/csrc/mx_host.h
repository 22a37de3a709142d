// Host helpers of the low-bit products' launchers.
#pragma once

#include <cstdint>

#include <cuda.h>
#include <cuda_runtime_api.h>

#include "costa_gb300.h"

namespace costa {

// 2-D tensor maps, zeros outside, 128-byte swizzle: of bytes, `width` bytes x
// `rows`, `pitch` bytes from row to row, in boxes of 128 bytes x `box_rows`
// (swizzled or not); of bf16, in boxes of 64 elements.
cudaError_t mx_byte_map(CUtensorMap *map, const void *base, uint64_t width, uint64_t rows, uint64_t pitch,
                        uint32_t box_rows, bool swizzle);
cudaError_t mx_bf16_map(CUtensorMap *map, const void *base, uint64_t cols, uint64_t rows, uint64_t ld,
                        uint32_t box_rows);
// Of tiles of scales (512 bytes), in boxes of `box_tiles`, not swizzled.
cudaError_t mx_scale_map(CUtensorMap *map, const void *base, uint64_t tiles, uint32_t box_tiles);
// C = beta C (0 without reading C for beta == 0): products over nothing.
cudaError_t launch_mx_scale(float beta, const costa_mx_dense &C, cudaStream_t s);
// Waits that gave up, on the current device since the library was loaded.
cudaError_t mx_product_failures(unsigned *count);
cudaError_t mx_grad_failures(unsigned *count);

}  // namespace costa
