// Host side of the operators' tensor-core kernels: tensor maps of bf16 operands, and how many clusters a device runs at a time.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "mote_common.cuh"

namespace mote {

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// bf16 [rows, cols] with a row stride in elements; box [box_rows, 64], 128-byte swizzle
static inline bool make_operand_map(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t stride, int box_rows) {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(p);
  });
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Clusters of `ctas` (2, 4 or 8) CTAs of a kernel that the current device runs at a time; 0 where the query fails.  Where a CTA fills an SM,
// that depends on how the SMs are grouped: 74, 33 and 15 on a B200 of 148.  The kernel's shared-memory limit has to be set already.
struct ResidentClusters {
  std::atomic<int> n[kMaxDevices][9];
  template <typename K>
  int get(K kernel, int threads, int smem, int ctas) {
    const int dev = current_device();
    const bool known = dev >= 0 && dev < kMaxDevices;
    int v = known ? n[dev][ctas].load(std::memory_order_relaxed) : 0;
    if (v == 0) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(ctas);
      cfg.blockDim = dim3(threads);
      cfg.dynamicSmemBytes = smem;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = (unsigned)ctas;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&v, kernel, &cfg) != cudaSuccess) { (void)cudaGetLastError(); v = 0; }
      v = v > 0 ? v : -1;
      if (known) n[dev][ctas].store(v, std::memory_order_relaxed);
    }
    return v > 0 ? v : 0;
  }
};

}  // namespace mote
