// Host-side pieces shared by the stand-alone operators (attention over packed sequences, token log probabilities, clipping).
#pragma once
#include "pm_common.cuh"

namespace pm {

// Sets the message that pm_last_error(NULL) returns to this thread; never throws.
pm_status ops_fail(pm_status s, const char* format, ...) noexcept;
inline pm_status ops_cuda(cudaError_t e, const char* what) noexcept {
  if (e == cudaSuccess) return PM_OK;
  cudaGetLastError();                             // reported here: not left for whoever asks the runtime next
  return ops_fail(PM_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 2^x (relative error about 2^-22, results below 2^-126 are zero)
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

}  // namespace pm
