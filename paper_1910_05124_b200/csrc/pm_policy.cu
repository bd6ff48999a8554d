// The clipped policy loss of sampled tokens with a KL term and an entropy bonus, and its gradients.
//
//   delta = logprob - old_logprob,  ratio = e^delta,  A the advantage
//   policy = -min(ratio A, clip(ratio, 1 - low, 1 + high) A),  kl = e^d - d - 1 with d = ref_logprob - logprob
//   loss = sum_i share_i (policy_i + kl_coef kl_i - entropy_coef entropy_i),   share = weight / sum of the weights, or the weight itself
//   d_logprob = share ([not clipped] (-ratio A) - kl_coef (e^d - 1)),   d_entropy = -entropy_coef share
//
// Short lists: one cluster of blocks, whose threads hold their tokens while the sum of the weights and the sums of the terms cross the
// cluster's shared memory; one launch, bound by its latency.  Long lists: a launch that adds the weights, and one that does the rest, in
// which the block that ends last adds the blocks' sums, in their order.  Bound by memory: each input once, the weights twice (the second
// time from L2).  4096 tokens 3.9 us, 1048576 12.4 us (33 MB: 5.2 at the rate of a copy; the ends of two launches are the rest).  Sums in
// 64 bits; which side of a border a ratio is on is decided by delta in 64 bits, where the difference of two fp32 numbers is all but
// exact, so that no rounding of an exponential moves a gradient across the border.
#include <cmath>

#include <cooperative_groups.h>

#include "pm_ops.cuh"

namespace pm {
namespace cg = cooperative_groups;

constexpr int kPolicySums = 5;                    // of the weights, policy, kl, entropy and clipped terms
constexpr int kPolicyThreads = 512, kPolicyHeld = 4, kPolicyCluster = 8;         // short lists: tokens to a thread, blocks
constexpr int64_t kPolicyShort = (int64_t)kPolicyThreads * kPolicyHeld * kPolicyCluster;
// Long lists: blocks of the launch that adds the weights; threads, consecutive tokens to a thread and most blocks of the one that does the rest.
constexpr int kWeightBlocks = kSms, kPolicyLong = 256, kPolicyRun = 4, kPolicyBlocks = 4 * kSms;

struct PolicyArgs {
  const float *logprob, *old_logprob, *advantage, *ref_logprob, *entropy, *weight;
  float *stats, *d_logprob, *d_entropy;
  double* sums;                                   // long lists: of the weights [kWeightBlocks], then of the terms [blocks][4]
  unsigned* ended;
  int64_t n;
  double log_low, log_high;                       // borders of delta
  float bound_low, bound_high;                    // 1 - low, 1 + high
  double kl_coef, entropy_coef;
  int mean;
};

struct PolicyToken {
  float lp, old, adv, ref, ent, w;
  __device__ __forceinline__ void load(const PolicyArgs& a, int64_t i) {
    const bool in = i < a.n;
    w = !in ? 0.f : a.weight ? a.weight[i] : 1.f;
    lp = in ? a.logprob[i] : 0.f;
    old = in ? a.old_logprob[i] : 0.f;
    adv = in ? a.advantage[i] : 0.f;
    ref = in && a.ref_logprob ? a.ref_logprob[i] : 0.f;
    ent = in && a.entropy ? a.entropy[i] : 0.f;
  }
  // four tokens from 16-byte loads
  static __device__ __forceinline__ void load4(PolicyToken (&t)[4], const PolicyArgs& a, int64_t i) {
    auto four = [&](const float* p, float other) { return p ? *reinterpret_cast<const float4*>(p + i) : make_float4(other, other, other, other); };
    const float4 w = four(a.weight, 1.f), lp = four(a.logprob, 0.f), old = four(a.old_logprob, 0.f), adv = four(a.advantage, 0.f), ref = four(a.ref_logprob, 0.f),
                 ent = four(a.entropy, 0.f);
    t[0] = PolicyToken{lp.x, old.x, adv.x, ref.x, ent.x, w.x};
    t[1] = PolicyToken{lp.y, old.y, adv.y, ref.y, ent.y, w.y};
    t[2] = PolicyToken{lp.z, old.z, adv.z, ref.z, ent.z, w.z};
    t[3] = PolicyToken{lp.w, old.w, adv.w, ref.w, ent.w, w.w};
  }
  // adds the token's terms; returns its gradient but for the share
  __device__ __forceinline__ float terms(const PolicyArgs& a, double (&sums)[kPolicySums]) const {
    if (w == 0.f) return 0.f;                     // padding: whatever its values are
    const double delta = (double)lp - (double)old;
    const bool high = delta > a.log_high, low = delta < a.log_low;
    const bool clipped = (high && adv > 0.f) || (low && adv < 0.f);
    const float ratio = expf((float)delta);
    const float policy = adv == 0.f ? 0.f : -(clipped ? (high ? a.bound_high : a.bound_low) : ratio) * adv;
    float grad = clipped || adv == 0.f ? 0.f : -ratio * adv;
    sums[0] += w;
    sums[1] += (double)w * policy;
    if (clipped) sums[4] += w;
    if (a.ref_logprob) {
      const float d = ref - lp;
      // e^d - 1 and e^d - 1 - d.  The second loses its bits for small d: there its series d^2 (1/2 + d/6 + ...), the next term below 2^-27 of
      // the sum.  From 1 on it has the exponential's own error e^d / (e^d - 1 - d) times, at most 3.8, and the first 1.6 times; behind -1
      // neither has more than the exponential.  (From 1/2 on it would be 11 times.)
      float s = 1.f / 39916800.f;
      s = fmaf(s, d, 1.f / 3628800.f);
      s = fmaf(s, d, 1.f / 362880.f);
      s = fmaf(s, d, 1.f / 40320.f);
      s = fmaf(s, d, 1.f / 5040.f);
      s = fmaf(s, d, 1.f / 720.f);
      s = fmaf(s, d, 1.f / 120.f);
      s = fmaf(s, d, 1.f / 24.f);
      s = fmaf(s, d, 1.f / 6.f);
      s = fmaf(s, d, 0.5f);
      const bool near = fabsf(d) < 1.f;
      const float far = expf(d) - 1.f, kl = near ? d * d * s : far - d, slope = near ? d + kl : far;
      sums[2] += (double)w * kl;
      if (a.kl_coef != 0.0) grad -= (float)a.kl_coef * slope;        // measured alone: an infinite slope has no part of the gradient
    }
    if (a.entropy) sums[3] += (double)w * ent;
    return grad;
  }
  __device__ __forceinline__ float lp_gradient(float grad, double share) const { return w == 0.f ? 0.f : (float)((double)w * share) * grad; }
  __device__ __forceinline__ float entropy_gradient(const PolicyArgs& a, double share) const {
    return w == 0.f ? 0.f : (float)(-a.entropy_coef * ((double)w * share));
  }
  __device__ __forceinline__ void store(const PolicyArgs& a, int64_t i, float grad, double share) const {
    if (i >= a.n) return;
    if (a.d_logprob) a.d_logprob[i] = lp_gradient(grad, share);
    if (a.d_entropy) a.d_entropy[i] = entropy_gradient(a, share);
  }
};

// what a weight is multiplied with; weights that add up to nothing give nothing
__device__ __forceinline__ double policy_share(const PolicyArgs& a, double weights) { return !a.mean ? 1.0 : weights == 0.0 ? 0.0 : 1.0 / weights; }

__device__ __forceinline__ void policy_stats(const PolicyArgs& a, const double (&sums)[kPolicySums], double share) {
  const double policy = sums[1] * share, kl = sums[2] * share, entropy = sums[3] * share;
  a.stats[0] = (float)(policy + (a.kl_coef != 0.0 ? a.kl_coef * kl : 0.0) - (a.entropy_coef != 0.0 ? a.entropy_coef * entropy : 0.0));
  a.stats[1] = (float)policy;
  a.stats[2] = (float)kl;
  a.stats[3] = (float)entropy;
  a.stats[4] = (float)(sums[4] * share);
}

// Block-wide sums of N values in a fixed order, in scratch [warps][N] and then, by thread i < N, returned.
template <int N> __device__ __forceinline__ double policy_block_sum(const double (&v)[N], double (*scratch)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    double x = v[k];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5][k] = x;
  }
  __syncthreads();
  double sum = 0.0;
  if (threadIdx.x < N)
    for (int w = 0; w < (int)blockDim.x / 32; ++w) sum += scratch[w][threadIdx.x];
  return sum;
}

__global__ void __launch_bounds__(kPolicyThreads) policy_short_kernel(const __grid_constant__ PolicyArgs a) {
  __shared__ double scratch[kPolicyThreads / 32][kPolicySums];
  __shared__ double mine[kPolicySums], total[kPolicySums];
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int64_t first = (int64_t)rank * kPolicyThreads + threadIdx.x, step = (int64_t)blocks * kPolicyThreads;
  PolicyToken t[kPolicyHeld];
  float grad[kPolicyHeld];
#pragma unroll
  for (int i = 0; i < kPolicyHeld; ++i) t[i].load(a, first + i * step);
  double sums[kPolicySums] = {};
#pragma unroll
  for (int i = 0; i < kPolicyHeld; ++i) grad[i] = t[i].terms(a, sums);
  const double sum = policy_block_sum(sums, scratch);
  if (threadIdx.x < kPolicySums) mine[threadIdx.x] = sum;
  cluster.sync();
  if (threadIdx.x < kPolicySums) {
    double v = 0.0;
    for (int b = 0; b < blocks; ++b) v += cluster.map_shared_rank(mine, b)[threadIdx.x];
    total[threadIdx.x] = v;
  }
  cluster.sync();                                 // also: the others have read this block's sums
  const double share = policy_share(a, total[0]);
#pragma unroll
  for (int i = 0; i < kPolicyHeld; ++i) t[i].store(a, first + i * step, grad[i], share);
  if (rank == 0 && threadIdx.x == 0) policy_stats(a, total, share);
}

// Sum of the weights, a part to a block, and the counter of the next launch.
template <bool VEC> __global__ void __launch_bounds__(kPolicyThreads) policy_weights_kernel(const __grid_constant__ PolicyArgs a) {
  __shared__ double scratch[kPolicyThreads / 32][1];
  pdl_trigger();
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.ended = 0;
  if (!a.weight || !a.mean) return;
  double sum[1] = {};
  const int64_t first = (int64_t)blockIdx.x * kPolicyThreads + threadIdx.x, step = (int64_t)gridDim.x * kPolicyThreads, whole = VEC ? a.n / 4 : 0;
  if (VEC)
#pragma unroll 4
    for (int64_t i = first; i < whole; i += step) {
      const float4 w = reinterpret_cast<const float4*>(a.weight)[i];
      sum[0] += ((double)w.x + w.y) + ((double)w.z + w.w);
    }
  for (int64_t i = whole * 4 + first; i < a.n; i += step) sum[0] += a.weight[i];
  const double v = policy_block_sum(sum, scratch);
  if (threadIdx.x == 0) a.sums[blockIdx.x] = v;
}

// VEC: every tensor starts at a 16-byte boundary.
template <bool VEC> __global__ void __launch_bounds__(kPolicyLong, 4) policy_long_kernel(const __grid_constant__ PolicyArgs a) {
  __shared__ double scratch[kPolicyLong / 32][kPolicySums];
  __shared__ double total[kPolicySums];
  __shared__ bool last;
  constexpr int R = kPolicyRun;
  const int64_t step = (int64_t)gridDim.x * kPolicyLong * R;
  int64_t i = ((int64_t)blockIdx.x * kPolicyLong + threadIdx.x) * R;
  PolicyToken t[R];
  auto load = [&]() {
    if (VEC && i + R <= a.n) {
      PolicyToken::load4(t, a, i);
    } else {
#pragma unroll
      for (int e = 0; e < R; ++e) t[e].load(a, i + e);
    }
  };
  load();                                         // the first tokens while the weights are added
  double sums[kPolicySums] = {};
  float grad[R];
#pragma unroll
  for (int e = 0; e < R; ++e) grad[e] = t[e].terms(a, sums);
  pdl_wait();
  if (threadIdx.x < 32) {
    double v = 0.0;
    if (a.weight && a.mean)
      for (int b = threadIdx.x; b < kWeightBlocks; b += 32) v += a.sums[b];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threadIdx.x == 0) total[0] = a.weight && a.mean ? v : (double)a.n;
  }
  __syncthreads();
  const double weights = total[0], share = policy_share(a, weights);
  for (;;) {
    if (VEC && i + R <= a.n) {
      auto four = [&](auto value) { return make_float4(value(0), value(1), value(2), value(3)); };
      if (a.d_logprob) *reinterpret_cast<float4*>(a.d_logprob + i) = four([&](int e) { return t[e].lp_gradient(grad[e], share); });
      if (a.d_entropy) *reinterpret_cast<float4*>(a.d_entropy + i) = four([&](int e) { return t[e].entropy_gradient(a, share); });
    } else {
#pragma unroll
      for (int e = 0; e < R; ++e) t[e].store(a, i + e, grad[e], share);
    }
    i += step;
    if (i >= a.n) break;
    load();
#pragma unroll
    for (int e = 0; e < R; ++e) grad[e] = t[e].terms(a, sums);
  }
  const double sum = policy_block_sum(sums, scratch);
  double* const terms = a.sums + kWeightBlocks;
  if (threadIdx.x > 0 && threadIdx.x < kPolicySums) __stcg(terms + (int64_t)blockIdx.x * 4 + threadIdx.x - 1, sum);
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(a.ended, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  {                                               // a lane in four to a term
    const int k = threadIdx.x & 3;
    double v = 0.0;
#pragma unroll 8
    for (int b = threadIdx.x >> 2; b < (int)gridDim.x; b += kPolicyLong / 4) v += __ldcg(terms + (int64_t)b * 4 + k);
#pragma unroll
    for (int o = 16; o >= 4; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) < 4) scratch[threadIdx.x >> 5][k] = v;
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    double v = 0.0;
    for (int w = 0; w < kPolicyLong / 32; ++w) v += scratch[w][threadIdx.x];
    total[threadIdx.x + 1] = v;
  }
  __syncthreads();
  if (threadIdx.x == 0) policy_stats(a, total, share);
}

}  // namespace pm

using namespace pm;

extern "C" {

uint64_t pm_policy_loss_workspace_bytes(int64_t n) {
  return n <= kPolicyShort ? 0 : (uint64_t)(kWeightBlocks + kPolicyBlocks * 4 + 1) * sizeof(double);
}

pm_status pm_policy_loss(const pm_policy_desc* d, int64_t n, const float* logprob, const float* old_logprob, const float* advantage, const float* ref_logprob,
                         const float* entropy, const float* weight, float* stats, float* d_logprob, float* d_entropy, void* workspace,
                         uint64_t workspace_bytes, void* stream) {
  if (!d) return ops_fail(PM_ERR_INVALID_ARG, "null argument");
  if (n < 0) return ops_fail(PM_ERR_INVALID_ARG, "negative size");
  if (n > (int64_t)1 << 40) return ops_fail(PM_ERR_SHAPE, "too many tokens");
  if (!(d->clip_low >= 0.0 && d->clip_low <= 1.0)) return ops_fail(PM_ERR_INVALID_ARG, "clip_low must be 0 to 1");
  if (!(d->clip_high >= 0.0)) return ops_fail(PM_ERR_INVALID_ARG, "clip_high must not be negative");
  if (!std::isfinite(d->kl_coef) || !std::isfinite(d->entropy_coef)) return ops_fail(PM_ERR_INVALID_ARG, "coefficients must be finite");
  if (d->kl_coef != 0.0 && !ref_logprob && n) return ops_fail(PM_ERR_INVALID_ARG, "kl_coef without ref_logprob");
  if (d->entropy_coef != 0.0 && !entropy && n) return ops_fail(PM_ERR_INVALID_ARG, "entropy_coef without entropy");
  if (!stats) return ops_fail(PM_ERR_INVALID_ARG, "null stats");
  if (n && (!logprob || !old_logprob || !advantage)) return ops_fail(PM_ERR_INVALID_ARG, "null pointer");
  const int64_t bytes = 4 * n;
  const struct { const void* p; int64_t bytes; } all[] = {{stats, 20}, {d_logprob, bytes}, {d_entropy, bytes}, {logprob, bytes}, {old_logprob, bytes},
                                                          {advantage, bytes}, {ref_logprob, bytes}, {entropy, bytes}, {weight, bytes}};
  for (const auto& x : all) if (!aligned_to(x.p, 4)) return ops_fail(PM_ERR_INVALID_ARG, "pointer not aligned to its element type");
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < 9; ++j)
      if (i != j && dense_share(all[i].p, all[i].bytes, all[j].p, all[j].bytes))
        return ops_fail(PM_ERR_INVALID_ARG, j < 3 ? "two outputs overlap" : "an output overlaps one of the inputs");
  const uint64_t need = pm_policy_loss_workspace_bytes(n);
  if (need) {
    if (!workspace || workspace_bytes < need) return ops_fail(PM_ERR_NOMEM, "workspace too small: need %llu bytes", (unsigned long long)need);
    if (!aligned_to(workspace, 8)) return ops_fail(PM_ERR_INVALID_ARG, "workspace must be 8-byte aligned");
    for (const auto& x : all)
      if (dense_share(workspace, (int64_t)need, x.p, x.bytes)) return ops_fail(PM_ERR_INVALID_ARG, "the workspace overlaps a tensor");
  }
  PolicyArgs a{};
  a.logprob = logprob; a.old_logprob = old_logprob; a.advantage = advantage; a.ref_logprob = ref_logprob; a.entropy = entropy; a.weight = weight;
  a.stats = stats; a.d_logprob = d_logprob; a.d_entropy = d_entropy; a.n = n; a.mean = d->mean != 0;
  a.log_low = std::log1p(-d->clip_low); a.log_high = std::log1p(d->clip_high);
  a.bound_low = (float)(1.0 - d->clip_low); a.bound_high = (float)(1.0 + d->clip_high);
  a.kl_coef = d->kl_coef; a.entropy_coef = d->entropy_coef;
  const cudaStream_t st = (cudaStream_t)stream;
  if (!need) {
    // one block's tokens at a time, up to the cluster's
    int blocks = 1;
    while (blocks < kPolicyCluster && (int64_t)blocks * kPolicyThreads < n) blocks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(kPolicyThreads); cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = blocks; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return ops_cuda(cudaLaunchKernelEx(&cfg, policy_short_kernel, a), "policy loss");
  }
  a.sums = static_cast<double*>(workspace);
  a.ended = reinterpret_cast<unsigned*>(a.sums + kWeightBlocks + kPolicyBlocks * 4);
  bool vec = true;
  for (const void* p : {(const void*)logprob, (const void*)old_logprob, (const void*)advantage, (const void*)ref_logprob, (const void*)entropy, (const void*)weight,
                        (const void*)d_logprob, (const void*)d_entropy})
    vec = vec && aligned_to(p, 16);
  const dim3 first(weight && a.mean ? kWeightBlocks : 1), rest((unsigned)std::min<int64_t>((n + kPolicyLong * kPolicyRun - 1) / (kPolicyLong * kPolicyRun), kPolicyBlocks));
  cudaError_t e = launch_pdl(vec ? policy_weights_kernel<true> : policy_weights_kernel<false>, first, dim3(kPolicyThreads), 0, st, false, a);
  if (e == cudaSuccess) e = launch_pdl(vec ? policy_long_kernel<true> : policy_long_kernel<false>, rest, dim3(kPolicyLong), 0, st, true, a);
  return ops_cuda(e, "policy loss");
}

}  // extern "C"
