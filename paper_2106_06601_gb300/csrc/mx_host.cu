// Host helpers of the low-bit products, and C = beta C.
#include <atomic>

#include "costa_internal.h"
#include "mx_device.cuh"
#include "mx_host.h"

namespace costa {
namespace {

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                              const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                              CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
    static const EncodeFn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeFn>(f);
    }();
    return fn;
}

cudaError_t tensor_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, uint64_t width, uint64_t rows,
                       uint64_t pitch, uint32_t box_width, uint32_t box_rows, bool swizzle) {
    const EncodeFn encode = encode_fn();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {width, rows}, strides[1] = {pitch};
    const cuuint32_t box[2] = {box_width, box_rows}, step[2] = {1, 1};
    const CUresult r = encode(map, type, 2, const_cast<void *>(base), dims, strides, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE,
                              swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// Stands for a kernel with as much shared memory in questions about clusters; never launched.
__global__ void no_kernel() {}

template <typename T> __global__ void scale_kernel(T *c, int64_t ld, int64_t rows, int64_t cols, float beta) {
    mx::let_next_start();
    mx::after_previous();
    for (int64_t i = blockIdx.x; i < rows; i += gridDim.x)
        for (int64_t j = threadIdx.x; j < cols; j += blockDim.x) {
            T *at = c + i * ld + j;
            *at = mx::from_float<T>(beta == 0.0f ? 0.0f : beta * mx::to_float(*at));
        }
}

}  // namespace

cudaError_t mx_byte_map(CUtensorMap *map, const void *base, uint64_t width, uint64_t rows, uint64_t pitch,
                        uint32_t box_rows) {
    return tensor_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, width, rows, pitch, 128, box_rows, true);
}

cudaError_t mx_bf16_map(CUtensorMap *map, const void *base, uint64_t cols, uint64_t rows, uint64_t ld,
                        uint32_t box_rows) {
    return tensor_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, cols, rows, 2 * ld, 64, box_rows, true);
}

cudaError_t mx_scale_map(CUtensorMap *map, const void *base, uint64_t tiles, uint32_t box_tiles) {
    return tensor_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, base, 128, tiles, 512, 128, box_tiles, false);
}

int mx_clusters(int size, int blocks_per_sm) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices][2][4];  // a property of the device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    const int which = size >= 8 ? 3 : size >= 4 ? 2 : size >= 2 ? 1 : 0, two = blocks_per_sm > 1;
    if (dev < kDevices)
        if (const int n = known[dev][two][which].load(std::memory_order_relaxed)) return n;
    const int smem = (two ? 104 : 160) * 1024;
    int n = 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(size));
    cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = static_cast<size_t>(smem);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {static_cast<unsigned>(size), 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(no_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, no_kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = 1;
    }
    if (dev < kDevices) known[dev][two][which].store(n, std::memory_order_relaxed);
    return n;
}

cudaError_t launch_mx_scale(float beta, const costa_mx_dense &C, cudaStream_t s) {
    const int64_t blocks = C.rows < 65536 ? C.rows : 65536;
    if (C.type == COSTA_MX_F32)
        return mx_launch(scale_kernel<float>, blocks, 256, 0, 1, s, static_cast<float *>(C.ptr), C.ld, C.rows, C.cols, beta);
    return mx_launch(scale_kernel<__nv_bfloat16>, blocks, 256, 0, 1, s, static_cast<__nv_bfloat16 *>(C.ptr), C.ld, C.rows,
                     C.cols, beta);
}

}  // namespace costa
