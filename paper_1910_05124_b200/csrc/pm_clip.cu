// Global gradient norm over many tensors, and clipping into their destinations.
//
//   norm = sqrt(sum over every element g^2),   scale = min(1, max_norm / norm),   dst = scale g
//
// Two launches.  The first reads every tensor once and leaves one 64-bit partial sum per block; the second adds the partial
// sums in a fixed order in every block (a few kilobytes from L2, cheaper than a launch between the two) and writes the
// destinations.  No atomics: the same tensors give the same bits.  Bound by memory: one read, and a read and a write, of which
// the second read walks each block's range backwards so that what the first pass read last is still in the 126 MB L2.
//
// The list of tensors travels as a kernel parameter (32 bytes a tensor, up to 1000 a launch), so a call copies nothing to the
// device and can be captured into a graph.  Each tensor is cut into chunks of kChunk elements, a block takes a contiguous range
// of chunks.
#include <cfloat>
#include <cmath>

#include "pm_ops.cuh"

namespace pm {

constexpr int kClipThreads = 256;
constexpr int kChunk = 8192;                      // elements: four (bf16) or eight (fp32) 16-byte loads per thread
// Blocks of 256 threads per SM: the norm keeps eight 16-byte loads a thread in flight and takes the registers of four blocks, the second
// pass runs with six (185 M bf16 gradients into fp32: 186 us, with four 189).
constexpr int kNormBlocks = 4 * kSms, kScaleBlocks = 6 * kSms;
constexpr int kClipCap = 1000;                    // tensors per launch: the parameter space holds 32764 bytes

enum { CF_SRC_BF16 = 1, CF_DST_BF16 = 2, CF_SRC_VEC = 4, CF_DST_VEC = 8, CF_IN_PLACE = 16 };

struct ClipEntry {
  const void* src;
  void* dst;
  uint64_t count;
  uint32_t first_chunk;                           // of this launch's chunks
  uint32_t flags;
};
template <int CAP> struct ClipTable {
  uint32_t n, chunks;
  ClipEntry e[CAP];
};

// the entry whose chunks include `chunk`
template <int CAP> __device__ __forceinline__ uint32_t clip_find(const ClipTable<CAP>& t, uint32_t chunk) {
  uint32_t lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) / 2;
    if (t.e[mid].first_chunk <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Sum of squares of eight values.  Squares leave the range of fp32 at 2^64 and lose bits below 2^-63, so eight values whose
// largest lies outside 2^-50 .. 2^60 are squared in 64 bits; among the others what underflows is below 2^-25 of the sum.
// (A NaN passes the test with its neighbours or not; either way it reaches the sum.)
__device__ __forceinline__ double square8(const float (&v)[8]) {
  float m = fabsf(v[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  if ((m >= 8.8817842e-16f && m <= 1.1529215e18f) || m == 0.f)
    return (double)(((v[0] * v[0] + v[1] * v[1]) + (v[2] * v[2] + v[3] * v[3])) + ((v[4] * v[4] + v[5] * v[5]) + (v[6] * v[6] + v[7] * v[7])));
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += (double)v[i] * v[i];
  return sum;
}

__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}

// the thread's part of the squares of N 16-byte vectors per thread
template <int N> __device__ __forceinline__ double square_chunk(const __nv_bfloat16* p) {
  uint4 q[N];
#pragma unroll
  for (int i = 0; i < N; ++i) q[i] = reinterpret_cast<const uint4*>(p)[i * kClipThreads + threadIdx.x];
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float v[8];
    unpack8(q[i], v);
    sum += square8(v);
  }
  return sum;
}

// block-wide sum in a fixed order; valid in thread 0
__device__ __forceinline__ double block_sum(double v, double* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = scratch[0];
    for (int w = 1; w < kClipThreads / 32; ++w) v += scratch[w];
  }
  return v;
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads, 4) clip_norm_kernel(const __grid_constant__ ClipTable<CAP> t, double* partials) {
  __shared__ double scratch[kClipThreads / 32];
  const uint32_t c0 = (uint32_t)((uint64_t)t.chunks * blockIdx.x / gridDim.x), c1 = (uint32_t)((uint64_t)t.chunks * (blockIdx.x + 1) / gridDim.x);
  double acc = 0.0;
  if (c0 < c1) {
    uint32_t e = clip_find(t, c0);
    for (uint32_t c = c0; c < c1; ++c) {
      while (e + 1 < t.n && t.e[e + 1].first_chunk <= c) ++e;
      const uint64_t begin = (uint64_t)(c - t.e[e].first_chunk) * kChunk;
      const int n = (int)min((uint64_t)kChunk, t.e[e].count - begin);
      const uint32_t flags = t.e[e].flags;
      if (flags & CF_SRC_BF16) {
        const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(t.e[e].src) + begin;
        if (c + 1 < c1 && begin + 2 * kChunk <= t.e[e].count && (flags & CF_SRC_VEC)) {
          acc += square_chunk<kChunk / 4 / kClipThreads>(p);           // two chunks: as many loads in flight as for one of fp32
          ++c;
        } else if (n == kChunk && (flags & CF_SRC_VEC)) {
          acc += square_chunk<kChunk / 8 / kClipThreads>(p);
        } else {
          for (int i = threadIdx.x; i < n; i += kClipThreads) { const double x = __bfloat162float(p[i]); acc += x * x; }
        }
      } else {
        const float* p = static_cast<const float*>(t.e[e].src) + begin;
        if (n == kChunk && (flags & CF_SRC_VEC)) {
          float4 q[kChunk / 4 / kClipThreads];
#pragma unroll
          for (int i = 0; i < kChunk / 4 / kClipThreads; ++i) q[i] = reinterpret_cast<const float4*>(p)[i * kClipThreads + threadIdx.x];
#pragma unroll
          for (int i = 0; i < kChunk / 4 / kClipThreads; i += 2)
            acc += square8({q[i].x, q[i].y, q[i].z, q[i].w, q[i + 1].x, q[i + 1].y, q[i + 1].z, q[i + 1].w});
        } else {
          for (int i = threadIdx.x; i < n; i += kClipThreads) { const double x = p[i]; acc += x * x; }
        }
      }
    }
  }
  const double sum = block_sum(acc, scratch);
  if (threadIdx.x == 0) partials[blockIdx.x] = sum;
  pdl_wait();
  pdl_trigger();
}

__device__ __forceinline__ void store4(__nv_bfloat16* p, float a, float b, float c, float d) {
  __nv_bfloat162 lo = __floats2bfloat162_rn(a, b), hi = __floats2bfloat162_rn(c, d);
  uint2 w;
  w.x = *reinterpret_cast<uint32_t*>(&lo); w.y = *reinterpret_cast<uint32_t*>(&hi);
  *reinterpret_cast<uint2*>(p) = w;
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }

// Four elements a thread and step: 8 or 16 bytes in, 8 or 16 bytes out, whole 32-byte sectors per warp in every case.
template <typename S, typename D>
__device__ __forceinline__ void clip_chunk(const S* src, D* dst, int n, bool vec, float scale) {
  if (n == kChunk && vec) {
    constexpr int kSteps = kChunk / 4 / kClipThreads;
    float v[kSteps][4];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int at = (i * kClipThreads + threadIdx.x) * 4;
      if constexpr (sizeof(S) == 2) {
        const uint2 q = *reinterpret_cast<const uint2*>(src + at);
        v[i][0] = __uint_as_float(q.x << 16); v[i][1] = __uint_as_float(q.x & 0xFFFF0000u);
        v[i][2] = __uint_as_float(q.y << 16); v[i][3] = __uint_as_float(q.y & 0xFFFF0000u);
      } else {
        const float4 q = *reinterpret_cast<const float4*>(src + at);
        v[i][0] = q.x; v[i][1] = q.y; v[i][2] = q.z; v[i][3] = q.w;
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      store4(dst + (i * kClipThreads + threadIdx.x) * 4, v[i][0] * scale, v[i][1] * scale, v[i][2] * scale, v[i][3] * scale);
  } else {
    for (int i = threadIdx.x; i < n; i += kClipThreads) dst[i] = from_f<D>(to_f<S>(src[i]) * scale);
  }
}

// The same with a factor below the normal range of fp32, where its own rounding would be that of a few bits: products in 64 bits,
// rounded to fp32 as the others.  Out of line: such a norm is above 2^126 max_norm, the other path keeps its registers.
template <typename S, typename D> __device__ __noinline__ void clip_chunk_tiny(const S* src, D* dst, int n, double factor) {
  for (int i = threadIdx.x; i < n; i += kClipThreads) dst[i] = from_f<D>((float)((double)to_f<S>(src[i]) * factor));
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads, 6) clip_scale_kernel(const __grid_constant__ ClipTable<CAP> t, const double* partials, int n_partials,
                                                                    double max_norm, float* norm_out, float* scale_out) {
  __shared__ double scratch[kClipThreads / 32];
  __shared__ float s_scale;
  __shared__ double s_factor;
  pdl_wait();
  pdl_trigger();
  double acc = 0.0;
  for (int i = threadIdx.x; i < n_partials; i += kClipThreads) acc += partials[i];
  acc = block_sum(acc, scratch);
  if (threadIdx.x == 0) {
    const double norm = sqrt(acc);
    // an infinite or undefined norm clips nothing: the caller sees it in norm_out (what counts is the norm as reported, in fp32)
    const double factor = norm > max_norm && isfinite((float)norm) ? max_norm / norm : 1.0;
    const float scale = (float)factor;
    s_scale = scale;
    s_factor = factor;
    if (blockIdx.x == 0 && norm_out) { *norm_out = (float)norm; *scale_out = scale; }
  }
  __syncthreads();
  const float scale = s_scale;
  auto clip = [&](auto* src, auto* dst, int n, bool vec) {
    if (scale < FLT_MIN) clip_chunk_tiny(src, dst, n, s_factor);
    else clip_chunk(src, dst, n, vec, scale);
  };
  const uint32_t c0 = (uint32_t)((uint64_t)t.chunks * blockIdx.x / gridDim.x), c1 = (uint32_t)((uint64_t)t.chunks * (blockIdx.x + 1) / gridDim.x);
  if (c0 >= c1) return;
  uint32_t e = clip_find(t, c1 - 1);
  for (uint32_t c = c1; c-- > c0;) {
    while (t.e[e].first_chunk > c) --e;
    const uint32_t flags = t.e[e].flags;
    if (scale == 1.f && (flags & CF_IN_PLACE)) continue;
    const uint64_t begin = (uint64_t)(c - t.e[e].first_chunk) * kChunk;
    const int n = (int)min((uint64_t)kChunk, t.e[e].count - begin);
    const bool vec = (flags & CF_SRC_VEC) && (flags & CF_DST_VEC);
    const bool sb = flags & CF_SRC_BF16, db = flags & CF_DST_BF16;
    if (sb) {
      const __nv_bfloat16* s = static_cast<const __nv_bfloat16*>(t.e[e].src) + begin;
      if (db) clip(s, static_cast<__nv_bfloat16*>(t.e[e].dst) + begin, n, vec);
      else clip(s, static_cast<float*>(t.e[e].dst) + begin, n, vec);
    } else {
      const float* s = static_cast<const float*>(t.e[e].src) + begin;
      if (db) clip(s, static_cast<__nv_bfloat16*>(t.e[e].dst) + begin, n, vec);
      else clip(s, static_cast<float*>(t.e[e].dst) + begin, n, vec);
    }
  }
}

// entries with empty tensors are left out
template <int CAP> static int clip_fill(ClipTable<CAP>& t, const pm_tensor_pair* tensors, int n) {
  uint64_t chunks = 0;
  int m = 0;
  for (int i = 0; i < n; ++i) {
    const pm_tensor_pair& p = tensors[i];
    if (p.count == 0) continue;
    const bool sb = p.src_dtype == PM_BF16, db = p.dst_dtype == PM_BF16;
    uint32_t flags = (sb ? CF_SRC_BF16 : 0) | (db ? CF_DST_BF16 : 0);
    if (aligned_to(p.src, 16)) flags |= CF_SRC_VEC;
    if (aligned_to(p.dst, 16)) flags |= CF_DST_VEC;
    if (p.src == p.dst) flags |= CF_IN_PLACE;
    t.e[m++] = ClipEntry{p.src, p.dst, p.count, (uint32_t)chunks, flags};
    chunks += (p.count + kChunk - 1) / kChunk;
  }
  t.n = (uint32_t)m;
  t.chunks = (uint32_t)chunks;
  return m;
}

struct ClipCall {
  double* partials;
  int n_partials;                                 // of all launches
  double max_norm;
  float *norm, *scale;
  cudaStream_t stream;
};
enum { CLIP_NORM = 1, CLIP_SCALE = 2 };           // passes: both where one launch holds all tensors
template <int CAP>
static cudaError_t clip_launch(const pm_tensor_pair* tensors, int n, int passes, int first_partial, const ClipCall& c, bool writes) {
  ClipTable<CAP> t;
  clip_fill(t, tensors, n);
  auto blocks = [&](int most) { return t.chunks < 1 ? 1 : t.chunks < (uint32_t)most ? (int)t.chunks : most; };
  cudaError_t e = cudaSuccess;
  if (passes & CLIP_NORM) e = launch_pdl(clip_norm_kernel<CAP>, dim3(blocks(kNormBlocks)), dim3(kClipThreads), 0, c.stream, false, t, c.partials + first_partial);
  if (e == cudaSuccess && (passes & CLIP_SCALE))
    e = launch_pdl(clip_scale_kernel<CAP>, dim3(blocks(kScaleBlocks)), dim3(kClipThreads), 0, c.stream, writes, t, c.partials, c.n_partials, c.max_norm,
                   writes ? c.norm : nullptr, writes ? c.scale : nullptr);
  return e;
}

static cudaError_t clip_dispatch(const pm_tensor_pair* tensors, int n, int passes, int first_partial, const ClipCall& c, bool writes) {
  if (n <= 64) return clip_launch<64>(tensors, n, passes, first_partial, c, writes);
  if (n <= 256) return clip_launch<256>(tensors, n, passes, first_partial, c, writes);
  return clip_launch<kClipCap>(tensors, n, passes, first_partial, c, writes);
}

// blocks of the first pass over these tensors
static int clip_partials(const pm_tensor_pair* tensors, int n) {
  uint64_t chunks = 0;
  for (int i = 0; i < n; ++i) chunks += (tensors[i].count + kChunk - 1) / kChunk;
  return (int)(chunks < 1 ? 1 : chunks < (uint64_t)kNormBlocks ? chunks : (uint64_t)kNormBlocks);
}

}  // namespace pm

using namespace pm;

extern "C" {

uint64_t pm_clip_gradients_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 1) return 0;
  return (uint64_t)((n_tensors + kClipCap - 1) / kClipCap) * kNormBlocks * sizeof(double);
}

pm_status pm_clip_gradients(const pm_tensor_pair* tensors, int32_t n_tensors, double max_norm, float* norm, float* scale, void* workspace,
                            uint64_t workspace_bytes, void* stream) {
  if (!tensors || !norm || !scale) return ops_fail(PM_ERR_INVALID_ARG, "null argument");
  if (n_tensors < 1) return ops_fail(PM_ERR_INVALID_ARG, "n_tensors must be positive");
  if (!(max_norm > 0)) return ops_fail(PM_ERR_INVALID_ARG, "max_norm must be positive");
  uint64_t total = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const pm_tensor_pair& p = tensors[i];
    if ((p.src_dtype != PM_F32 && p.src_dtype != PM_BF16) || (p.dst_dtype != PM_F32 && p.dst_dtype != PM_BF16))
      return ops_fail(PM_ERR_INVALID_ARG, "tensor %d: unknown element type", i);
    if (p.count > 0 && (!p.src || !p.dst)) return ops_fail(PM_ERR_INVALID_ARG, "tensor %d: null pointer", i);
    if (p.count > ((uint64_t)1 << 42) || (total += p.count) > ((uint64_t)1 << 42)) return ops_fail(PM_ERR_SHAPE, "more than 2^42 elements");
    if (p.count > 0 && (!aligned_to(p.src, p.src_dtype == PM_BF16 ? 2 : 4) || !aligned_to(p.dst, p.dst_dtype == PM_BF16 ? 2 : 4)))
      return ops_fail(PM_ERR_INVALID_ARG, "tensor %d: pointer not aligned to its element type", i);
    if (p.count > 0 && p.src == p.dst && p.src_dtype != p.dst_dtype)
      return ops_fail(PM_ERR_INVALID_ARG, "tensor %d: source and destination of different types share their memory", i);
  }
  const uint64_t need = pm_clip_gradients_workspace_bytes(n_tensors);
  if (!workspace || workspace_bytes < need) return ops_fail(PM_ERR_NOMEM, "workspace too small: need %llu bytes", (unsigned long long)need);
  if (!aligned_to(workspace, 8)) return ops_fail(PM_ERR_INVALID_ARG, "workspace must be 8-byte aligned");
  ClipCall c{static_cast<double*>(workspace), 0, max_norm, norm, scale, (cudaStream_t)stream};
  if (n_tensors <= kClipCap) {
    c.n_partials = clip_partials(tensors, n_tensors);
    return ops_cuda(clip_dispatch(tensors, n_tensors, CLIP_NORM | CLIP_SCALE, 0, c, true), "gradient clipping");
  }
  // several launches a pass: the first of the second pass writes norm and scale
  for (int at = 0; at < n_tensors; at += kClipCap) {
    const int n = n_tensors - at < kClipCap ? n_tensors - at : kClipCap;
    if (const pm_status s = ops_cuda(clip_dispatch(tensors + at, n, CLIP_NORM, c.n_partials, c, false), "gradient norm")) return s;
    c.n_partials += clip_partials(tensors + at, n);
  }
  for (int at = 0; at < n_tensors; at += kClipCap) {
    const int n = n_tensors - at < kClipCap ? n_tensors - at : kClipCap;
    if (const pm_status s = ops_cuda(clip_dispatch(tensors + at, n, CLIP_SCALE, 0, c, at == 0), "gradient clipping")) return s;
  }
  return PM_OK;
}

}  // extern "C"
