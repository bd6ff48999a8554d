// Dropout whose mask is formed from a counter-based generator wherever it is needed, with the sum into a residual stream.
//
//   bits_i = 16 bits of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with the key
//            `seed` and the counter `first + i / 8`: eight elements to a counter, the lower half of a word before its upper half
//   kept_i = bits_i >= T,  T = p 2^16 to the nearest whole number;   y_i = residual_i + (kept_i ? x_i 2^16 / (2^16 - T) : 0)
//
// Bound by memory: x (and the residual) read, y written, nothing stored for the backward pass, which is the same call on the gradient.
// 16 bits to an element, so a counter's ten rounds serve a whole 16-byte vector of bf16: 32 bits to an element would take twice the
// multiplications, which are then as long as the memory takes.
#include <type_traits>

#include "pm_ops.cuh"

namespace pm {

// Vectors of eight elements to a thread at a time and blocks to an SM: 64 to 96 bytes under way for each thread.  16384 x 1024 bf16, us on the
// device with the residual / without it: three vectors 16.2 / 12.4, two 18.6 / 15.4, four 16.0 / 13.3, one (six blocks) 19.7 / 14.7.
constexpr int kDropThreads = 256, kDropVectors = 3;
template <typename T, bool RES> constexpr int kDropBlocks = RES || sizeof(T) == 4 ? 3 : 4;

// The keys of the ten rounds, formed once for a thread's counters.
struct RoundKeys {
  uint2 k[10];
  __device__ __forceinline__ explicit RoundKeys(uint64_t key) {
    k[0] = make_uint2((uint32_t)key, (uint32_t)(key >> 32));
#pragma unroll
    for (int i = 1; i < 10; ++i) k[i] = make_uint2(k[i - 1].x + 0x9E3779B9u, k[i - 1].y + 0xBB67AE85u);
  }
};
__device__ __forceinline__ uint4 philox(uint64_t counter, const RoundKeys& keys) {
  uint4 c = make_uint4((uint32_t)counter, (uint32_t)(counter >> 32), 0u, 0u);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)0xD2511F53u * c.x, b = (uint64_t)0xCD9E8D57u * c.z;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ keys.k[i].x, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ keys.k[i].y, (uint32_t)a);
  }
  return c;
}

// Eight values as they lie in memory.
template <typename T> struct Eight {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void load(const T* p, int64_t n) {                  // of which n exist; any alignment
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : from_f<T>(0.f);
    memcpy(w, v, sizeof(w));
  }
  __device__ __forceinline__ void spread(float (&v)[8]) const {
    const T* p = reinterpret_cast<const T*>(w);
    load8<T>(p, v);
  }
};

// VEC: every tensor starts at a 16-byte boundary.  x and y may be one tensor, so nothing is declared read-only.  The generator works while
// the loads are under way; as many blocks as run at a time, whose threads form the round keys once.
template <typename T, bool VEC, bool RES, int U>
__global__ void __launch_bounds__(kDropThreads, kDropBlocks<T, RES>) dropout_kernel(const T* x, const T* residual, T* y, int64_t n, const uint64_t* rng, uint32_t dropped, float scale) {
  const uint64_t counter = rng[1];
  const RoundKeys keys(rng[0]);
  const uint32_t border = dropped << 16;
  for (int64_t first = (int64_t)blockIdx.x * kDropThreads * U + threadIdx.x; first * 8 < n; first += (int64_t)gridDim.x * kDropThreads * U) {
    Eight<T> a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = (first + u * kDropThreads) * 8;
      if (VEC && at + 8 <= n) {
        a[u].load(x + at);
        if (RES) b[u].load(residual + at);
      } else {
        a[u].load(x + at, n - at);
        if (RES) b[u].load(residual + at, n - at);
      }
    }
    uint4 words[U];
#pragma unroll
    for (int u = 0; u < U; ++u) words[u] = philox(counter + (uint64_t)(first + u * kDropThreads), keys);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = (first + u * kDropThreads) * 8;
      if (at >= n) break;
      const uint32_t w[4] = {words[u].x, words[u].y, words[u].z, words[u].w};
      float v[8], r[8];
      a[u].spread(v);
      if (RES) b[u].spread(r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {               // chosen, not multiplied: what is dropped may be anything
        const bool kept = (e & 1 ? w[e / 2] : w[e / 2] << 16) >= border;         // the half as the upper one: the lower bits decide nothing
        v[e] = kept ? (RES ? fmaf(v[e], scale, r[e]) : v[e] * scale) : (RES ? r[e] : 0.f);
      }
      if (VEC && at + 8 <= n) {
        store8<T>(y + at, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (at + e < n) y[at + e] = from_f<T>(v[e]);
      }
    }
  }
}

template <typename T> static cudaError_t dropout_run(const void* x, const void* residual, void* y, int64_t n, const int64_t* rng, uint32_t dropped, cudaStream_t st) {
  const bool vec = aligned_to(x, 16) && aligned_to(residual, 16) && aligned_to(y, 16);
  const float scale = 65536.f / (float)(65536u - dropped);                       // rounded: off by 2^-24 of itself at most, all elements alike
  const int64_t groups = (n + 8 * kDropThreads - 1) / (8 * kDropThreads);        // blocks with one vector to a thread
  auto go = [&](auto kernel, int64_t blocks) {
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kDropThreads), 0, st, false, static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<T*>(y), n,
                      reinterpret_cast<const uint64_t*>(rng), dropped, scale);
  };
  auto with = [&](auto res) {
    constexpr bool RES = decltype(res)::value;
    constexpr int kMost = kDropBlocks<T, RES> * kSms, V = kDropVectors;
    // tensors whose vectors all have a thread at the same time take one each
    if (groups <= kMost) return go(vec ? dropout_kernel<T, true, RES, 1> : dropout_kernel<T, false, RES, 1>, groups);
    return go(vec ? dropout_kernel<T, true, RES, V> : dropout_kernel<T, false, RES, V>, std::min<int64_t>((groups + V - 1) / V, kMost));
  };
  return residual ? with(std::true_type{}) : with(std::false_type{});
}

static pm_status dropout_call(const void* x, const void* residual, int32_t dtype, int64_t n, double p, const int64_t* rng, void* y, const char* what, void* stream) {
  if (dtype != PM_F32 && dtype != PM_BF16) return ops_fail(PM_ERR_INVALID_ARG, "unknown element type");
  if (n < 0) return ops_fail(PM_ERR_INVALID_ARG, "negative size");
  if (n > (int64_t)1 << 42) return ops_fail(PM_ERR_SHAPE, "too many elements");
  if (!(p >= 0.0) || p >= 1.0 - 1.0 / 131072) return ops_fail(PM_ERR_INVALID_ARG, "p must be 0 to below 1 - 2^-17");
  if (n == 0) return PM_OK;
  const int size = dtype == PM_BF16 ? 2 : 4;
  if (!x || !y || !rng) return ops_fail(PM_ERR_INVALID_ARG, "null pointer");
  if (!aligned_to(x, size) || !aligned_to(residual, size) || !aligned_to(y, size)) return ops_fail(PM_ERR_INVALID_ARG, "pointer not aligned to its element type");
  if (!aligned_to(rng, 8)) return ops_fail(PM_ERR_INVALID_ARG, "rng must be 8-byte aligned");
  auto apart = [&](const void* in) { return in == y || !dense_share(y, n * size, in, n * size); };
  if (!apart(x) || !apart(residual) || dense_share(y, n * size, rng, 16))
    return ops_fail(PM_ERR_INVALID_ARG, "the output overlaps an input without being the same tensor");
  const uint32_t dropped = (uint32_t)(p * 65536.0 + 0.5);
  const cudaStream_t st = (cudaStream_t)stream;
  return ops_cuda(dtype == PM_BF16 ? dropout_run<__nv_bfloat16>(x, residual, y, n, rng, dropped, st) : dropout_run<float>(x, residual, y, n, rng, dropped, st), what);
}

}  // namespace pm

using namespace pm;

extern "C" {

pm_status pm_dropout(const void* x, const void* residual, int32_t dtype, int64_t n, double p, const int64_t* rng, void* y, void* stream) {
  return dropout_call(x, residual, dtype, n, p, rng, y, "dropout", stream);
}

pm_status pm_dropout_backward(const void* d_y, int32_t dtype, int64_t n, double p, const int64_t* rng, void* d_x, void* stream) {
  return dropout_call(d_y, nullptr, dtype, n, p, rng, d_x, "dropout backward", stream);
}

}  // extern "C"
