// Tensor maps (descriptors of tiled asynchronous copies), encoded through the driver's entry point.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>
#include <atomic>
#include "common.cuh"

namespace ttsgpt {

// dims and box: innermost first; strides: bytes, of every dimension but the innermost
inline cudaError_t tensor_map_encode(CUtensorMap *map, CUtensorMapDataType type, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
                                     const cuuint32_t *box, CUtensorMapSwizzle swizzle) {
  static std::atomic<PFN_cuTensorMapEncodeTiled> known{nullptr};   // the same address whoever looks it up first
  PFN_cuTensorMapEncodeTiled encode = known.load(std::memory_order_acquire);
  if (!encode) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
    encode = (PFN_cuTensorMapEncodeTiled)fn;
    known.store(encode, std::memory_order_release);
  }
  const cuuint32_t step[5] = {1, 1, 1, 1, 1};
  return encode(map, type, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace ttsgpt
