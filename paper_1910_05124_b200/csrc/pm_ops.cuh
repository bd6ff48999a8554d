// Host-side pieces shared by the stand-alone operators (attention over packed sequences, token log probabilities, clipping).
#pragma once
#include <algorithm>
#include <utility>

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

// Where a tensor's elements lie: n_outer x n_inner pieces of `bytes` bytes, `outer` and `inner` bytes apart.  128 bits: any strides.
struct Extent {
  __int128 at, outer, n_outer, inner, n_inner, bytes;
};
inline Extent dense_extent(const void* p, int64_t bytes) { return Extent{(__int128)reinterpret_cast<uintptr_t>(p), 0, 1, 0, 1, p ? bytes : 0}; }
inline Extent rows_extent(const void* p, int64_t rows, int64_t row_stride, int64_t columns, int size) {
  return Extent{(__int128)reinterpret_cast<uintptr_t>(p), (__int128)row_stride * size, rows, 0, 1, (__int128)columns * size};
}
// The same bytes in as few pieces as possible, the larger stride outside.
inline Extent joined(Extent x) {
  if (x.n_inner > 1 && (x.outer < x.inner || x.n_outer == 1)) { std::swap(x.outer, x.inner); std::swap(x.n_outer, x.n_inner); }
  if (x.inner <= x.bytes) { x.bytes += x.inner * (x.n_inner - 1); x.n_inner = 1; }
  if (x.n_inner == 1 && x.outer <= x.bytes) { x.bytes += x.outer * (x.n_outer - 1); x.n_outer = 1; }
  return x;
}
inline bool joined_share(Extent a, Extent b) {
  constexpr int kMost = 1024;                     // pairs of pieces that are looked at: 0.1 ms
  if (a.at >= b.at + b.outer * (b.n_outer - 1) + b.inner * (b.n_inner - 1) + b.bytes) return false;
  if (b.at >= a.at + a.outer * (a.n_outer - 1) + a.inner * (a.n_inner - 1) + a.bytes) return false;
  if (a.n_outer == 1) a.outer = b.outer;          // one piece has any stride
  if (b.n_outer == 1) b.outer = a.outer;
  if (a.outer != b.outer) {
    if (a.n_outer * a.n_inner > b.n_outer * b.n_inner) std::swap(a, b);
    if (a.n_outer * a.n_inner * b.n_inner > kMost) return false;
    for (int i = 0; i < a.n_outer; ++i)
      if (joined_share(Extent{a.at + i * a.outer, 0, 1, a.inner, a.n_inner, a.bytes}, b)) return true;
    return false;
  }
  if (a.inner == b.inner ? a.n_inner + b.n_inner > kMost : a.n_inner * b.n_inner > kMost) return false;
  auto floor_div = [](__int128 x, __int128 y) { return x / y - (x % y < 0); };
  auto meet = [&](int i, int j) {                 // inner pieces i and j for some distance of t rows
    const __int128 d = a.at + i * a.inner - (b.at + j * b.inner);
    if (a.outer == 0) return d < b.bytes && -d < a.bytes;
    const __int128 lo = -floor_div(a.bytes - 1 + d, a.outer), hi = floor_div(b.bytes - 1 - d, a.outer);
    return std::max(lo, 1 - b.n_outer) <= std::min(hi, a.n_outer - 1);
  };
  for (int i = 0; i < a.n_inner; ++i)
    for (int j = 0; j < (a.inner == b.inner && i > 0 ? 1 : b.n_inner); ++j)          // with one stride i - j decides
      if (meet(i, j)) return true;
  return false;
}
// Whether two tensors have a byte in common.  Exact, but for two strided tensors of different row strides and more pairs of pieces than
// are looked at: those pass.
inline bool extents_share(const Extent& a, const Extent& b) {
  if (a.n_outer < 1 || a.n_inner < 1 || a.bytes < 1 || b.n_outer < 1 || b.n_inner < 1 || b.bytes < 1) return false;
  return joined_share(joined(a), joined(b));
}

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
