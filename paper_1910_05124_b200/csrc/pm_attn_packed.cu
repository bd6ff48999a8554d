// Attention over packed sequences with shared key/value heads, forward and backward, on the CUDA cores: fp32, and bf16 head widths
// or layouts that the tensor-core kernels do not take.
//
//   s_ij = scale q_i . k_j (j <= i where causal),  lse_i = log sum_j e^(s_ij),  o_i = sum_j e^(s_ij - lse_i) v_j
//   p_ij = e^(s_ij - lse_i),  ds_ij = p_ij (do_i . v_j - do_i . o_i)
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_{h, i} ds_ij q_i,   dv_j = sum_{h, i} p_ij do_i    (h: the heads that share k, v)
//
// Tiles of 64 x 64 scores by 256 threads, a thread holds 4 x 4 of them; operands are fp32 in shared memory whatever their type
// (exact for bf16), all sums fp32.  Forward: one block per 64 query rows and head, one pass over the keys with the running
// maximum and sum.  Backward: a block owns query rows (dq), or key rows (dk, dv) and walks the query tiles of every head of
// its group, so each gradient is summed by one block in a fixed order, without atomics, at the price of forming the
// scores twice.
#include <atomic>

#include <cooperative_groups.h>

#include "pm_attn_packed.cuh"

namespace pm {
namespace cg = cooperative_groups;

constexpr int PK_T = 64, PK_LDP = PK_T + 4;       // rows of a streamed tile

// A block owns R rows, 64 or 32, with 4 R threads.

template <int DP> constexpr int kPkLd = DP + 4;
// `own` tiles of R rows, `streamed` ones of 64, `squares` of R x 64, and two values to each streamed row
template <int DP, int R> constexpr int pk_smem(int own, int streamed, int squares) {
  return ((own * R + streamed * PK_T) * kPkLd<DP> + squares * R * PK_LDP + 2 * PK_T) * 4;
}

// ROWS rows of a head from row0 on, zeros outside the sequence and behind the head's width: four consecutive values to a register
// quadruple, all of a thread's loads in flight before the first is put into the tile.  VEC: one load brings the four.
template <typename T, int DP, bool VEC, int ROWS, int THREADS> struct PkRows {
  static constexpr int kN = ROWS * DP / 4 / THREADS;
  float4 v[kN];
  __device__ __forceinline__ void fetch(const HeadView& x, const SeqTile& s, int row0, int head, int dim) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int at = i * THREADS + threadIdx.x, r = at / (DP / 4), c = at % (DP / 4) * 4;
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row0 + r >= s.len || c >= dim) continue;
      const T* p = head_row<T>(x, s.begin + row0 + r, head) + c;
      if constexpr (VEC && sizeof(T) == 4) {
        v[i] = *reinterpret_cast<const float4*>(p);
      } else if constexpr (VEC) {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        v[i] = make_float4(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16), __uint_as_float(q.y & 0xFFFF0000u));
      } else {
        v[i].x = to_f<T>(p[0]);
        if (c + 1 < dim) v[i].y = to_f<T>(p[1]);
        if (c + 2 < dim) v[i].z = to_f<T>(p[2]);
        if (c + 3 < dim) v[i].w = to_f<T>(p[3]);
      }
    }
  }
  __device__ __forceinline__ void put(float* tile) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int at = i * THREADS + threadIdx.x;
      *reinterpret_cast<float4*>(tile + at / (DP / 4) * kPkLd<DP> + at % (DP / 4) * 4) = v[i];
    }
  }
};
// A tile of each of two tensors per step.  The next step's are fetched while this one's are worked on, where registers allow.
template <typename T, int DP, bool VEC, int ROWS, int THREADS> struct PkPair {
  static constexpr bool kAhead = DP <= 64;
  PkRows<T, DP, VEC, ROWS, THREADS> x, y;
  __device__ __forceinline__ void fetch(const HeadView& a, const HeadView& b, const SeqTile& s, int row0, int head, int dim) {
    x.fetch(a, s, row0, head, dim);
    y.fetch(b, s, row0, head, dim);
  }
};

// acc[i][j] += A[4 ty + i] . B[tx + 16 j]
template <int DP> __device__ __forceinline__ void pk_abt(float (&acc)[4][4], const float* A, const float* B) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 4
  for (int d = 0; d < DP; d += 4) {
    float4 a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(A + (4 * ty + i) * kPkLd<DP> + d);
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(B + (tx + 16 * j) * kPkLd<DP> + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[i].w, b[j].w, fmaf(a[i].z, b[j].z, fmaf(a[i].y, b[j].y, fmaf(a[i].x, b[j].x, acc[i][j]))));
  }
}
// the thread's columns of a DP-wide row: 2 tx, 2 tx + 1 (DP = 32), else 4 tx .. 4 tx + 3 of every 64
template <int DP> __device__ __forceinline__ int pk_col(int c) {
  const int tx = threadIdx.x & 15;
  return DP == 32 ? 2 * tx + c : (c >> 2) * 64 + 4 * tx + (c & 3);
}
// acc[i][c] += sum_k P[4 ty + i][k] B[k][column c]
template <int DP> __device__ __forceinline__ void pk_pb(float (&acc)[4][DP / 16], const float* P, const float* B) {
  const int ty = threadIdx.x >> 4;
#pragma unroll 2
  for (int k = 0; k < PK_T; k += 4) {
    float p[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(P + (4 * ty + i) * PK_LDP + k);
      p[i][0] = v.x; p[i][1] = v.y; p[i][2] = v.z; p[i][3] = v.w;
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      float b[DP / 16];
      const float* row = B + (k + kk) * kPkLd<DP>;
      if constexpr (DP == 32) {
        const float2 v = *reinterpret_cast<const float2*>(row + pk_col<DP>(0));
        b[0] = v.x; b[1] = v.y;
      } else {
#pragma unroll
        for (int g = 0; g < DP / 64; ++g) {
          const float4 v = *reinterpret_cast<const float4*>(row + pk_col<DP>(4 * g));
          b[4 * g] = v.x; b[4 * g + 1] = v.y; b[4 * g + 2] = v.z; b[4 * g + 3] = v.w;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) acc[i][c] = fmaf(p[i][kk], b[c], acc[i][c]);
    }
  }
}
template <typename T, int DP>
__device__ __forceinline__ void pk_store(const HeadView& x, const SeqTile& s, int row0, int head, int dim, const float (&acc)[4][DP / 16], const float (&f)[4]) {
  const int ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = row0 + 4 * ty + i;
    if (r >= s.len) continue;
    T* out = head_row_out<T>(x, s.begin + r, head);
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) if (pk_col<DP>(c) < dim) out[pk_col<DP>(c)] = from_f<T>(acc[i][c] * f[i]);
  }
}
// tiles are counted from a sequence's end where the last ones see the most keys: the longest blocks start first
template <int R> __device__ __forceinline__ int pk_from_end(const SeqTile& s) { return (s.len + R - 1) / R - 1 - s.tile; }
template <int R> constexpr int kLog = R == 64 ? 6 : 5;
template <int R> constexpr bool pk_split = R == 32;  // blocks of 64 rows are launched where there are enough of them: they are not shared

// Where there are few blocks, a cluster of them shares one block's rows: each takes a part of what is streamed, leaves its sums in its
// shared memory, and finishes a part of the rows from everybody's, added in the order of the parts.
template <int DP> __device__ __forceinline__ void pk_leave(float* sums, const float (&acc)[4][DP / 16]) {
  const int ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) sums[(4 * ty + i) * kPkLd<DP> + pk_col<DP>(c)] = acc[i][c];
}
template <typename T, int DP, int R, typename W>
__device__ __forceinline__ void pk_finish(const HeadView& x, const SeqTile& s, int row0, int head, int dim, float* sums, int part, int parts, W weight) {
  cg::cluster_group cluster = cg::this_cluster();
  const int r0 = R * part / parts, r1 = R * (part + 1) / parts;
  for (int i = threadIdx.x; i < (r1 - r0) * (DP / 4); i += 4 * R) {
    const int r = r0 + i / (DP / 4), c = i % (DP / 4) * 4;
    if (row0 + r >= s.len || c >= dim) continue;
    float v[4] = {};
    for (int p = 0; p < parts; ++p) {
      const float4 u = *reinterpret_cast<const float4*>(cluster.map_shared_rank(sums + r * kPkLd<DP> + c, p));
      const float f = weight(r, p);
      v[0] += f * u.x; v[1] += f * u.y; v[2] += f * u.z; v[3] += f * u.w;
    }
    T* out = head_row_out<T>(x, s.begin + row0 + r, head) + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) if (c + e < dim) out[e] = from_f<T>(v[e]);
  }
}

template <typename T, int DP, bool VEC, int R>
__global__ void __launch_bounds__(4 * R, R == 64 && DP <= 64 ? 2 : 1) attn_packed_fwd_kernel(PackedArgs a) {
  cg::cluster_group cluster = cg::this_cluster();
  const int parts = pk_split<R> ? (int)cluster.num_blocks() : 1, part = pk_split<R> ? (int)cluster.block_rank() : 0, block = blockIdx.x / parts;
  const SeqTile s = find_tile(a.cu, a.n_seqs, a.tokens, block / a.heads, kLog<R>);
  if (s.tile < 0) return;
  extern __shared__ float sm[];
  float *sQ = sm, *sK = sQ + R * kPkLd<DP>, *sV = sK + PK_T * kPkLd<DP>, *sP = sV + PK_T * kPkLd<DP>;
  const int h = block % a.heads, hk = h / a.group, q0 = pk_from_end<R>(s) * R;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int all = a.causal ? min(s.len, q0 + R) : s.len, tiles = (all + PK_T - 1) / PK_T;
  const int begin = tiles * part / parts * PK_T, end = min(all, tiles * (part + 1) / parts * PK_T);
  PkPair<T, DP, VEC, PK_T, 4 * R> next;
  {
    PkRows<T, DP, VEC, R, 4 * R> q;
    q.fetch(a.q, s, q0, h, a.dim);
    if (next.kAhead) next.fetch(a.k, a.v, s, begin, hk, a.dim);
    q.put(sQ);
  }
  float o[4][DP / 16] = {}, m[4], l[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = -INFINITY;
  for (int k0 = begin; k0 < end; k0 += PK_T) {
    if (!next.kAhead) next.fetch(a.k, a.v, s, k0, hk, a.dim);
    __syncthreads();
    next.x.put(sK);
    next.y.put(sV);
    __syncthreads();
    if (next.kAhead && k0 + PK_T < end) next.fetch(a.k, a.v, s, k0 + PK_T, hk, a.dim);
    float acc[4][4] = {};
    pk_abt<DP>(acc, sQ, sK);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = q0 + 4 * ty + i;
      float mx = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = k0 + tx + 16 * j;
        acc[i][j] = c < s.len && (!a.causal || c <= r) ? acc[i][j] * a.scale : -INFINITY;
        mx = max_nan(mx, acc[i][j]);
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, x));
      // -infinity: no key of this part yet
      const float base = mx == -INFINITY ? 0.f : mx, f = ex2((m[i] - base) * kLog2e);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = ex2((acc[i][j] - base) * kLog2e);
        sum += e;
        sP[(4 * ty + i) * PK_LDP + tx + 16 * j] = e;
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      l[i] = l[i] * f + sum;
      m[i] = mx;
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) o[i][c] *= f;
    }
    __syncthreads();
    pk_pb<DP>(o, sP, sV);
  }
  if (pk_split<R> && parts > 1) {
    float* stats = sP;                            // maximum, sum [2][R]
    __syncthreads();
    pk_leave<DP>(sK, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) if (tx == 0) { stats[4 * ty + i] = m[i]; stats[R + 4 * ty + i] = l[i]; }
    cluster.sync();
    // row r's maximum, what its exponentials are relative to (zero where every score is -infinity: their difference would be NaN, the
    // sum is zero), and the sum over the parts
    auto total = [&](int r, float& top, float& base, float& sum) {
      top = -INFINITY;
      for (int p = 0; p < parts; ++p) top = max_nan(top, cluster.map_shared_rank(stats, p)[r]);
      base = top == -INFINITY ? 0.f : top;
      sum = 0.f;
      for (int p = 0; p < parts; ++p) sum += ex2((cluster.map_shared_rank(stats, p)[r] - base) * kLog2e) * cluster.map_shared_rank(stats, p)[R + r];
    };
    // weights of the parts, once per row of this block's share: [parts][R] behind the statistics
    float* weights = stats + 2 * R;
    const int r0 = R * part / parts, r1 = R * (part + 1) / parts;
    for (int r = r0 + threadIdx.x; r < r1; r += 4 * R) {
      float top, base, sum;
      total(r, top, base, sum);
      for (int p = 0; p < parts; ++p) weights[p * R + r] = ex2((cluster.map_shared_rank(stats, p)[r] - base) * kLog2e) / sum;
      if (a.lse && q0 + r < s.len) a.lse[(int64_t)h * a.tokens + s.begin + q0 + r] = top + logf(sum);
    }
    __syncthreads();
    pk_finish<T, DP, R>(a.o, s, q0, h, a.dim, sK, part, parts, [&](int r, int p) { return weights[p * R + r]; });
    cluster.sync();                               // the others have read this block's sums
    return;
  }
  float inv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    inv[i] = 1.f / l[i];
    const int r = q0 + 4 * ty + i;
    if (a.lse && tx == 0 && r < s.len) a.lse[(int64_t)h * a.tokens + s.begin + r] = m[i] + logf(l[i]);
  }
  pk_store<T, DP>(a.o, s, q0, h, a.dim, o, inv);
}

// delta_i = do_i . o_i, one warp per row and head; rows outside the sequences get a value that nothing reads
template <typename T>
__global__ void __launch_bounds__(256) attn_packed_delta_kernel(PackedArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (i < a.tokens * a.heads) {
    const int64_t token = i / a.heads;
    const int h = (int)(i - token * a.heads);
    const T *x = head_row<T>(a.o, token, h), *y = head_row<T>(a.d_o, token, h);
    float sum = 0.f;
    for (int c = lane; c < a.dim; c += 32) sum = fmaf(to_f<T>(x[c]), to_f<T>(y[c]), sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) a.delta[(int64_t)h * a.tokens + token] = sum;
  }
}

template <typename T, int DP, bool VEC, int R> __device__ __forceinline__ void pk_dq_block(const PackedArgs& a, int block, int part, int parts) {
  const SeqTile s = find_tile(a.cu, a.n_seqs, a.tokens, block / a.heads, kLog<R>);
  if (s.tile < 0) { pdl_wait(); return; }
  extern __shared__ float sm[];
  float *sQ = sm, *sO = sQ + R * kPkLd<DP>, *sK = sO + R * kPkLd<DP>, *sV = sK + PK_T * kPkLd<DP>, *sS = sV + PK_T * kPkLd<DP>;
  const int h = block % a.heads, hk = h / a.group, q0 = pk_from_end<R>(s) * R;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int all = a.causal ? min(s.len, q0 + R) : s.len, tiles = (all + PK_T - 1) / PK_T;
  const int begin = tiles * part / parts * PK_T, end = min(all, tiles * (part + 1) / parts * PK_T);
  PkPair<T, DP, VEC, PK_T, 4 * R> next;
  {
    PkPair<T, DP, VEC, R, 4 * R> own;
    own.fetch(a.q, a.d_o, s, q0, h, a.dim);
    if (next.kAhead) next.fetch(a.k, a.v, s, begin, hk, a.dim);
    own.x.put(sQ);
    own.y.put(sO);
  }
  pdl_wait();                                     // delta
  float lse[4], delta[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = q0 + 4 * ty + i;
    lse[i] = r < s.len ? a.lse[(int64_t)h * a.tokens + s.begin + r] : 0.f;
    delta[i] = r < s.len ? a.delta[(int64_t)h * a.tokens + s.begin + r] : 0.f;
  }
  float dq[4][DP / 16] = {};
  for (int k0 = begin; k0 < end; k0 += PK_T) {
    if (!next.kAhead) next.fetch(a.k, a.v, s, k0, hk, a.dim);
    __syncthreads();
    next.x.put(sK);
    next.y.put(sV);
    __syncthreads();
    if (next.kAhead && k0 + PK_T < end) next.fetch(a.k, a.v, s, k0 + PK_T, hk, a.dim);
    float acc[4][4] = {}, dp[4][4] = {};
    pk_abt<DP>(acc, sQ, sK);
    pk_abt<DP>(dp, sO, sV);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = k0 + tx + 16 * j, r = q0 + 4 * ty + i;
        const float p = ex2((acc[i][j] * a.scale - lse[i]) * kLog2e);
        sS[(4 * ty + i) * PK_LDP + tx + 16 * j] = c < s.len && r < s.len && (!a.causal || c <= r) ? p * (dp[i][j] - delta[i]) : 0.f;
      }
    __syncthreads();
    pk_pb<DP>(dq, sS, sK);
  }
  if (pk_split<R> && parts > 1) {
    __syncthreads();
    pk_leave<DP>(sK, dq);
    cg::this_cluster().sync();
    pk_finish<T, DP, R>(a.dq, s, q0, h, a.dim, sK, part, parts, [&](int, int) { return a.scale; });
    cg::this_cluster().sync();                    // the others have read this block's sums
    return;
  }
  const float f[4] = {a.scale, a.scale, a.scale, a.scale};
  pk_store<T, DP>(a.dq, s, q0, h, a.dim, dq, f);
}

template <typename T, int DP, bool VEC, int R> __device__ __forceinline__ void pk_dkv_block(const PackedArgs& a, int block, int part, int parts) {
  const SeqTile s = find_tile(a.cu, a.n_seqs, a.tokens, block / a.kv_heads, kLog<R>);
  if (s.tile < 0) { pdl_wait(); return; }
  extern __shared__ float sm[];
  float *sK = sm, *sV = sK + R * kPkLd<DP>, *sQ = sV + R * kPkLd<DP>, *sO = sQ + PK_T * kPkLd<DP>, *sP = sO + PK_T * kPkLd<DP>,
        *sS = sP + R * PK_LDP, *sR = sS + R * PK_LDP;
  const int hk = block % a.kv_heads, k0 = s.tile * R;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int first = a.causal ? k0 : 0, per_head = (s.len - first + PK_T - 1) / PK_T;
  const int it0 = per_head * a.group * part / parts, it1 = per_head * a.group * (part + 1) / parts;
  int h = hk * a.group + it0 / per_head, q0 = first + it0 % per_head * PK_T;
  // a query tile's lse (threads 0 .. 63) and delta (64 .. 127) travel with it
  auto row_value = [&](int h, int q0) {
    const int r = q0 + (threadIdx.x & 63);
    if (threadIdx.x >= 128 || r >= s.len || it0 >= it1) return 0.f;
    return (threadIdx.x < 64 ? a.lse : a.delta)[(int64_t)h * a.tokens + s.begin + r];
  };
  PkPair<T, DP, VEC, PK_T, 4 * R> next;
  {
    PkPair<T, DP, VEC, R, 4 * R> own;
    own.fetch(a.k, a.v, s, k0, hk, a.dim);
    pdl_wait();                                   // delta
    if (next.kAhead && it0 < it1) next.fetch(a.q, a.d_o, s, q0, h, a.dim);
    own.x.put(sK);
    own.y.put(sV);
  }
  float next_row = row_value(h, q0);
  float dk[4][DP / 16] = {}, dv[4][DP / 16] = {};
  for (int it = it0; it < it1; ++it) {
    if (!next.kAhead) next.fetch(a.q, a.d_o, s, q0, h, a.dim);
    __syncthreads();
    next.x.put(sQ);
    next.y.put(sO);
    if (threadIdx.x < 128) sR[threadIdx.x] = next_row;
    __syncthreads();
    const int r0 = q0;
    q0 += PK_T;
    if (q0 >= s.len) { q0 = first; ++h; }
    if (it + 1 < it1) {
      next_row = row_value(h, q0);
      if (next.kAhead) next.fetch(a.q, a.d_o, s, q0, h, a.dim);
    }
    float acc[4][4] = {}, dp[4][4] = {};
    pk_abt<DP>(acc, sK, sQ);                      // rows: keys, columns: queries
    pk_abt<DP>(dp, sV, sO);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = r0 + tx + 16 * j;
      const float lse = sR[tx + 16 * j], delta = sR[64 + tx + 16 * j];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = k0 + 4 * ty + i;
        const bool in = c < s.len && r < s.len && (!a.causal || c <= r);
        const float p = in ? ex2((acc[i][j] * a.scale - lse) * kLog2e) : 0.f;
        sP[(4 * ty + i) * PK_LDP + tx + 16 * j] = p;
        sS[(4 * ty + i) * PK_LDP + tx + 16 * j] = in ? p * (dp[i][j] - delta) : 0.f;
      }
    }
    __syncthreads();
    pk_pb<DP>(dv, sP, sO);
    pk_pb<DP>(dk, sS, sQ);
  }
  if (pk_split<R> && parts > 1) {
    float* const other = sQ + R * kPkLd<DP>;
    __syncthreads();
    pk_leave<DP>(sQ, dk);
    pk_leave<DP>(other, dv);
    cg::this_cluster().sync();
    pk_finish<T, DP, R>(a.dk, s, k0, hk, a.dim, sQ, part, parts, [&](int, int) { return a.scale; });
    pk_finish<T, DP, R>(a.dv, s, k0, hk, a.dim, other, part, parts, [&](int, int) { return 1.f; });
    cg::this_cluster().sync();                    // the others have read this block's sums
    return;
  }
  const float f[4] = {a.scale, a.scale, a.scale, a.scale}, one[4] = {1.f, 1.f, 1.f, 1.f};
  pk_store<T, DP>(a.dk, s, k0, hk, a.dim, dk, f);
  pk_store<T, DP>(a.dv, s, k0, hk, a.dim, dv, one);
}

// The blocks of dk and dv, and behind them those of dq.
template <typename T, int DP, bool VEC, int R>
__global__ void __launch_bounds__(4 * R) attn_packed_bwd_kernel(PackedArgs a, int dkv_blocks) {
  const int parts = pk_split<R> ? (int)cg::this_cluster().num_blocks() : 1, part = pk_split<R> ? (int)cg::this_cluster().block_rank() : 0;
  const int block = blockIdx.x / parts;
  if (block < dkv_blocks) pk_dkv_block<T, DP, VEC, R>(a, block, part, parts);
  else pk_dq_block<T, DP, VEC, R>(a, block - dkv_blocks, part, parts);
}

// raises a kernel's shared-memory limit once per device
template <typename K> static cudaError_t pk_allow(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || dev > 63 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev <= 63) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return e;
}

template <typename T, int DP, bool VEC, int R> static cudaError_t pk_forward(const PackedArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int smem = pk_smem<DP, R>(1, 2, 1);
  const int64_t blocks = most_tiles(a.tokens, a.n_seqs, R) * a.heads;
  if (!launchable(blocks)) return cudaErrorInvalidConfiguration;
  const cudaError_t e = pk_allow(attn_packed_fwd_kernel<T, DP, VEC, R>, smem, done);
  if (e != cudaSuccess) return e;
  return launch_clusters(attn_packed_fwd_kernel<T, DP, VEC, R>, blocks, 4 * R, smem, st, false, pk_split<R> ? packed_parts(blocks, a, PK_T, 1, 4 * kSms, 3) : 1, a);
}
template <typename T, int DP, bool VEC, int R> static cudaError_t pk_backward(const PackedArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  constexpr int smem = pk_smem<DP, R>(2, 2, 2);
  const int64_t tiles = most_tiles(a.tokens, a.n_seqs, R), blocks = tiles * (a.heads + a.kv_heads);
  if (!launchable(blocks)) return cudaErrorInvalidConfiguration;
  cudaError_t e = pk_allow(attn_packed_bwd_kernel<T, DP, VEC, R>, smem, done);
  if (e == cudaSuccess) e = launch_pdl(attn_packed_delta_kernel<T>, dim3((unsigned)((a.tokens * a.heads + 7) / 8)), dim3(256), 0, st, false, a);
  if (e == cudaSuccess)
    e = launch_clusters(attn_packed_bwd_kernel<T, DP, VEC, R>, blocks, 4 * R, smem, st, true, pk_split<R> ? packed_parts(blocks, a, PK_T, a.group, 4 * kSms, 2) : 1, a,
                  (int)(tiles * a.kv_heads));
  return e;
}
template <typename T, int DP, bool VEC> static cudaError_t pk_rows(const PackedArgs& a, bool backward, cudaStream_t st) {
  // 32 rows to a block where blocks of 64 would leave SMs without one (as a rule on the most tiles that the lengths can make)
  const bool small = most_tiles(a.tokens, a.n_seqs, PK_T) * (a.heads + (backward ? a.kv_heads : 0)) < 2 * kSms;
  if (small) return backward ? pk_backward<T, DP, VEC, 32>(a, st) : pk_forward<T, DP, VEC, 32>(a, st);
  return backward ? pk_backward<T, DP, VEC, 64>(a, st) : pk_forward<T, DP, VEC, 64>(a, st);
}
template <typename T, int DP> static cudaError_t pk_width(const PackedArgs& a, bool backward, cudaStream_t st) {
  // four elements at a time where every row of the inputs starts at such a boundary
  const size_t bytes = 4 * sizeof(T);
  bool vec = a.dim % 4 == 0;
  for (const HeadView* x : {&a.q, &a.k, &a.v, backward ? &a.d_o : &a.q}) vec = vec && aligned_to(x->data, bytes) && x->token % 4 == 0 && x->head % 4 == 0;
  return vec ? pk_rows<T, DP, true>(a, backward, st) : pk_rows<T, DP, false>(a, backward, st);
}
template <typename T> static cudaError_t pk_run(const PackedArgs& a, bool backward, cudaStream_t st) {
  if (a.dim <= 32) return pk_width<T, 32>(a, backward, st);
  return a.dim <= 64 ? pk_width<T, 64>(a, backward, st) : pk_width<T, 128>(a, backward, st);
}

static pm_status pk_check(const pm_attention_desc* d) {
  if (!d) return ops_fail(PM_ERR_INVALID_ARG, "null argument");
  if (d->dtype != PM_F32 && d->dtype != PM_BF16) return ops_fail(PM_ERR_INVALID_ARG, "unknown element type");
  if (d->n_heads < 1 || d->n_kv_heads < 1 || d->n_heads % d->n_kv_heads) return ops_fail(PM_ERR_INVALID_ARG, "n_heads must be a positive multiple of n_kv_heads");
  if (d->n_heads > 65535) return ops_fail(PM_ERR_SHAPE, "at most 65535 heads");
  if (d->head_dim < 1) return ops_fail(PM_ERR_INVALID_ARG, "head_dim must be positive");
  if (d->head_dim > 128) return ops_fail(PM_ERR_UNSUPPORTED, "heads wider than 128");
  if (d->n_seqs < 0 || d->n_tokens < 0) return ops_fail(PM_ERR_INVALID_ARG, "negative size");
  if (d->n_tokens > 0x7fffffff - 128 || d->n_seqs > (1 << 24) || d->n_tokens * d->n_heads > ((int64_t)1 << 33))
    return ops_fail(PM_ERR_SHAPE, "too many tokens, sequences or rows");
  // the kernels work with scale log2(e), which has to be finite too
  if (!(d->scale > 0) || d->scale >= 2e38f) return ops_fail(PM_ERR_INVALID_ARG, "scale must be positive and below 2e38");
  return PM_OK;
}
static pm_status pk_view(HeadView& out, const pm_head_view* v, const char* name, int size) {
  if (!v || !v->data) return ops_fail(PM_ERR_INVALID_ARG, "%s: null pointer", name);
  if (!aligned_to(v->data, size)) return ops_fail(PM_ERR_INVALID_ARG, "%s: pointer not aligned to its element type", name);
  if (v->token_stride < 0 || v->head_stride < 0) return ops_fail(PM_ERR_INVALID_ARG, "%s: negative stride", name);
  out = HeadView{v->data, v->token_stride, v->head_stride};
  return PM_OK;
}
static Extent pk_extent(const HeadView& x, int64_t tokens, int heads, int dim, int size) {
  return Extent{(__int128)reinterpret_cast<uintptr_t>(x.data), (__int128)x.token * size, tokens, (__int128)x.head * size, heads, (__int128)dim * size};
}
// what is written shares no memory with the other tensors
static pm_status pk_apart(const Extent* written, int n_written, const Extent* read, int n_read) {
  for (int i = 0; i < n_written; ++i) {
    for (int j = 0; j < n_read; ++j) if (extents_share(written[i], read[j])) return ops_fail(PM_ERR_INVALID_ARG, "an output overlaps one of the inputs");
    for (int j = 0; j < i; ++j) if (extents_share(written[i], written[j])) return ops_fail(PM_ERR_INVALID_ARG, "two outputs overlap or are the same tensor");
  }
  return PM_OK;
}
static pm_status pk_result(cudaError_t e, const char* what) {
  if (e != cudaErrorInvalidConfiguration) return ops_cuda(e, what);
  cudaGetLastError();                             // as ops_cuda does
  return ops_fail(PM_ERR_SHAPE, "%s: more blocks than a launch has: too many sequences for so many heads", what);
}
static PackedArgs pk_args(const pm_attention_desc* d, const int32_t* cu, float* lse) {
  PackedArgs a{};
  a.cu = cu; a.lse = lse; a.tokens = d->n_tokens; a.n_seqs = d->n_seqs; a.heads = d->n_heads; a.kv_heads = d->n_kv_heads;
  a.group = d->n_heads / d->n_kv_heads; a.dim = d->head_dim; a.causal = d->causal != 0; a.scale = d->scale;
  return a;
}

}  // namespace pm

using namespace pm;

extern "C" {

pm_status pm_attention_packed_forward(const pm_attention_desc* d, const pm_head_view* q, const pm_head_view* k, const pm_head_view* v,
                                      const int32_t* cu_seqlens, const pm_head_view* o, float* lse, void* stream) {
  if (const pm_status s = pk_check(d)) return s;
  if (d->n_tokens == 0 || d->n_seqs == 0) return PM_OK;
  if (!cu_seqlens) return ops_fail(PM_ERR_INVALID_ARG, "null cu_seqlens");
  PackedArgs a = pk_args(d, cu_seqlens, lse);
  const int size = d->dtype == PM_BF16 ? 2 : 4;
  if (const pm_status s = pk_view(a.q, q, "q", size)) return s;
  if (const pm_status s = pk_view(a.k, k, "k", size)) return s;
  if (const pm_status s = pk_view(a.v, v, "v", size)) return s;
  if (const pm_status s = pk_view(a.o, o, "o", size)) return s;
  auto all = [&](const HeadView& x, int heads) { return pk_extent(x, a.tokens, heads, a.dim, size); };
  const Extent written[] = {all(a.o, a.heads), dense_extent(lse, 4 * a.tokens * a.heads)};
  const Extent read[] = {all(a.q, a.heads), all(a.k, a.kv_heads), all(a.v, a.kv_heads), dense_extent(cu_seqlens, 4 * ((int64_t)a.n_seqs + 1))};
  if (const pm_status s = pk_apart(written, 2, read, 4)) return s;
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = attn_packed_tc_takes(a, d->dtype, false) ? attn_packed_tc_forward(a, st)
                        : d->dtype == PM_BF16 ? pk_run<__nv_bfloat16>(a, false, st) : pk_run<float>(a, false, st);
  return pk_result(e, "packed attention");
}

uint64_t pm_attention_packed_workspace_bytes(const pm_attention_desc* d) {
  return !d || d->n_heads < 1 || d->n_tokens < 0 ? 0 : (uint64_t)d->n_heads * (uint64_t)d->n_tokens * sizeof(float);
}

pm_status pm_attention_packed_backward(const pm_attention_desc* d, const pm_head_view* q, const pm_head_view* k, const pm_head_view* v,
                                       const pm_head_view* o, const float* lse, const pm_head_view* d_o, const int32_t* cu_seqlens,
                                       const pm_head_view* dq, const pm_head_view* dk, const pm_head_view* dv, void* workspace,
                                       uint64_t workspace_bytes, void* stream) {
  if (const pm_status s = pk_check(d)) return s;
  if (d->n_tokens == 0 || d->n_seqs == 0) return PM_OK;
  if (!cu_seqlens || !lse) return ops_fail(PM_ERR_INVALID_ARG, "null cu_seqlens or lse");
  PackedArgs a = pk_args(d, cu_seqlens, const_cast<float*>(lse));
  const int size = d->dtype == PM_BF16 ? 2 : 4;
  if (const pm_status s = pk_view(a.q, q, "q", size)) return s;
  if (const pm_status s = pk_view(a.k, k, "k", size)) return s;
  if (const pm_status s = pk_view(a.v, v, "v", size)) return s;
  if (const pm_status s = pk_view(a.o, o, "o", size)) return s;
  if (const pm_status s = pk_view(a.d_o, d_o, "d_o", size)) return s;
  if (const pm_status s = pk_view(a.dq, dq, "dq", size)) return s;
  if (const pm_status s = pk_view(a.dk, dk, "dk", size)) return s;
  if (const pm_status s = pk_view(a.dv, dv, "dv", size)) return s;
  auto all = [&](const HeadView& x, int heads) { return pk_extent(x, a.tokens, heads, a.dim, size); };
  const Extent others[] = {all(a.dq, a.heads), all(a.dk, a.kv_heads), all(a.dv, a.kv_heads), all(a.q, a.heads), all(a.k, a.kv_heads), all(a.v, a.kv_heads),
                           all(a.o, a.heads), all(a.d_o, a.heads), dense_extent(lse, 4 * a.tokens * a.heads),
                           dense_extent(cu_seqlens, 4 * ((int64_t)a.n_seqs + 1))};
  if (const pm_status s = pk_apart(others, 3, others + 3, 7)) return s;
  const uint64_t need = pm_attention_packed_workspace_bytes(d);
  if (!workspace || workspace_bytes < need) return ops_fail(PM_ERR_NOMEM, "workspace too small: need %llu bytes", (unsigned long long)need);
  if (!aligned_to(workspace, 4)) return ops_fail(PM_ERR_INVALID_ARG, "workspace must be 4-byte aligned");
  for (const Extent& x : others) if (extents_share(dense_extent(workspace, (int64_t)need), x)) return ops_fail(PM_ERR_INVALID_ARG, "the workspace overlaps a tensor");
  a.delta = static_cast<float*>(workspace);
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = attn_packed_tc_takes(a, d->dtype, true) ? attn_packed_tc_backward(a, st)
                        : d->dtype == PM_BF16 ? pk_run<__nv_bfloat16>(a, true, st) : pk_run<float>(a, true, st);
  return pk_result(e, "packed attention backward");
}

pm_status pm_attention_packed_selftest_wait_timeout(int64_t limit_cycles, void* stream) {
  if (limit_cycles < 1 || limit_cycles > 1000000000) return ops_fail(PM_ERR_INVALID_ARG, "limit_cycles must be 1 to 10^9");
  return ops_cuda(attn_packed_wait_probe(limit_cycles, (cudaStream_t)stream), "packed attention wait self-test");
}

pm_status pm_attention_packed_status(void* stream) {
  int code = 0;
  if (const pm_status s = ops_cuda(attn_packed_status(&code, (cudaStream_t)stream), "packed attention status")) return s;
  return code ? ops_fail(PM_ERR_TIMEOUT, "packed attention: device-side wait %d ran out", code) : PM_OK;
}

}  // extern "C"
