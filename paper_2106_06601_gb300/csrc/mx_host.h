// Host helpers of the low-bit products' launchers.
#pragma once

#include <cstdint>

#include <cuda.h>
#include <cuda_runtime_api.h>

#include "costa_gb300.h"
#include "costa_internal.h"

namespace costa {

// Dynamic shared memory of a launch, and the most that any launch of its kernel
// takes.  A kernel is always allowed the latter: what it is allowed is one number
// for all host threads, and a thread that lowered it between another's asking and
// launching would have that launch refused.
struct MxShared {
    size_t bytes, most;
    MxShared(size_t always) : bytes(always), most(always) {}
    MxShared(size_t bytes_, size_t most_) : bytes(bytes_), most(most_) {}
};

// Launches a kernel of the low-bit operators, in clusters of `cluster` blocks,
// as a dependent of the kernel before it on the stream: its blocks may start
// when that one's have all started (or, for a kernel that says nothing, ended),
// set themselves up, and wait in after_previous() until it is complete and its
// writes are visible.  Measured on GB300, two launches that follow each other
// (a token's quantisation and its inverse): 3.9 -> 2.4 us each.
template <typename... P, typename... A>
cudaError_t mx_launch(void (*kernel)(P...), int64_t blocks, int threads, MxShared smem, int cluster, cudaStream_t s,
                      A &&...args) {
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem.bytes;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {static_cast<unsigned>(cluster), 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    cudaError_t e = cudaSuccess;
    // (48 KB are granted unasked, the kernel's static shared memory among them, which is below 16 KB)
    if (smem.bytes > 32 * 1024)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem.most));
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
    if (e == cudaSuccess)
        count_launch();
    else
        cudaGetLastError();
    return e;
}

// 2-D tensor maps, zeros outside, 128-byte swizzle: of bytes, `width` bytes x
// `rows`, `pitch` bytes from row to row, in boxes of 128 bytes x `box_rows`; of
// bf16, in boxes of 64 elements.
cudaError_t mx_byte_map(CUtensorMap *map, const void *base, uint64_t width, uint64_t rows, uint64_t pitch,
                        uint32_t box_rows);
cudaError_t mx_bf16_map(CUtensorMap *map, const void *base, uint64_t cols, uint64_t rows, uint64_t ld,
                        uint32_t box_rows);
// Of tiles of scales (512 bytes), in boxes of `box_tiles`, not swizzled.
cudaError_t mx_scale_map(CUtensorMap *map, const void *base, uint64_t tiles, uint32_t box_tiles);
// How many clusters of `size` blocks (1, 2, 4 or 8) the current device runs at a
// time, with one block to an SM or two: fewer than its SMs would hold, as a
// cluster stays within one group of SMs (152 SMs: 76 of 2, 36 of 4, 15 of 8).
int mx_clusters(int size, int blocks_per_sm);
// C = beta C (0 without reading C for beta == 0): products over nothing.
cudaError_t launch_mx_scale(float beta, const costa_mx_dense &C, cudaStream_t s);
// Waits that gave up, on the current device since the library was loaded.
cudaError_t mx_product_failures(unsigned *count);
cudaError_t mx_grad_failures(unsigned *count);

}  // namespace costa
