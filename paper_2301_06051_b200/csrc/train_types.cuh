// Storage types of the training operators (norm.cu, segment.cu): float, bfloat16 and float16 rows, float arithmetic.
#pragma once
#include <cuda_fp16.h>

#include <atomic>

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

// Two floats in neighbouring registers: sm_100 adds and multiplies them in one instruction, each rounded as alone.
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 pair(float x, float y) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 parts(F2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ F2 add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
// The same for one float, so that code for either can be written once.
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float mul(float a, float b) { return a * b; }
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float sum_of(float a) { return a; }
__device__ __forceinline__ float sum_of(F2 a) { const float2 p = parts(a); return p.x + p.y; }

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

// Lets a kernel have `bytes` of shared memory.  That is the process's state and not a call's: always the same number for a kernel, so that calls
// of several threads never take from one another.  (Once per kernel and device: the call costs more than a launch's share of it.)
template <auto kernel>
static int allow_smem(dsvt_ctx* ctx, int bytes) {
  static std::atomic<uint64_t> done{0};
  const uint64_t bit = (uint64_t)1 << (ctx->device & 63);
  if (ctx->device < 64 && (done.load(std::memory_order_relaxed) & bit)) return DSVT_OK;
  DSVT_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  done.fetch_or(bit, std::memory_order_relaxed);
  return DSVT_OK;
}

}  // namespace dsvt_train
