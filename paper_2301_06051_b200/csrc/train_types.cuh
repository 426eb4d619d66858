// Storage types of the training operators (norm.cu, segment.cu): float, bfloat16 and float16 rows, float arithmetic.
#pragma once
#include <cuda_fp16.h>

#include "dsvt_common.cuh"

namespace dsvt_train {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

static inline int type_size(int type) { return type == DSVT_TYPE_F32 ? 4 : 2; }
static inline bool type_known(int type) { return type == DSVT_TYPE_F32 || type == DSVT_TYPE_BF16 || type == DSVT_TYPE_F16; }

// A call runs on its context's device, whichever is current.
struct DeviceGuard {
  int before = -1;
  explicit DeviceGuard(int device) {
    if (cudaGetDevice(&before) != cudaSuccess || before == device || cudaSetDevice(device) != cudaSuccess) before = -1;
  }
  ~DeviceGuard() { if (before >= 0) cudaSetDevice(before); }
};

}  // namespace dsvt_train
