// Norms of queries and keys for each head, and the rotation by their positions, in one pass; backward with the gains' gradients.
//
//   r = (mean_i x_i^2 + eps)^(-1/2),  n_i = g_i x_i r,  y = R(position) n
//   (y_a, y_b) = (n_a cos - n_b sin, n_b cos + n_a sin) for pair i of the first rotary_dim dimensions at the angle position f_i
//   u = R^T dy,  dg = sum u x r,  dx = r (g u - x r^2 mean_i(g_i u_i x_i))
//
// Bound by memory: each row is read once and written once.  A group of lanes takes all heads of a token in turn, so the sines and cosines
// of a token are formed once, in registers, by the lanes whose dimensions they turn; both dimensions of a pair lie in one lane, and
// only the sum of squares crosses lanes.  Where there are few tokens, several groups share a token's heads.
//
// The angle is a fraction of a turn in 64 bits: position times the frequency in units of 2^-64 turns wraps as angles do, so it is exact
// to 2^-33 turns at every position; the nearest quarter turn is taken off it before it becomes a float (at most an eighth of a turn, rounded
// by 2.4e-8 radians).
#include "pm_ops.cuh"
#include "pm_attn_packed.cuh"

namespace pm {

constexpr int kNormThreads = 256, kNormMostPairs = 64;

struct NormSide {
  HeadView x, y, dx;                              // y: the output, or in the backward pass its gradient
  const float* gain;
  int heads;
};
struct NormArgs {
  NormSide side[2];                               // queries, keys
  const int32_t* positions;
  float* partials;                                // [block][dim] of the gains' gradients, the keys' blocks behind the queries'
  int64_t tokens;
  int dim, rotary, parts;                         // parts: groups to a token
  int blocks[2], side_parts[2];                   // backward pass: blocks of each side, groups to a token there
  float eps;
  uint64_t turns[kNormMostPairs];                 // frequency of each pair, 2^-64 turns per position
};

// cos and sin of position times a frequency
__device__ __forceinline__ float2 turn_of(int32_t position, uint64_t turns) {
  const uint64_t a = (uint64_t)(int64_t)position * turns + (1ull << 61);         // an eighth of a turn on: the quarter is the nearest one
  const int quarter = (int)(a >> 62);
  const int32_t rest = (int32_t)((int64_t)((a & ((1ull << 62) - 1)) - (1ull << 61)) >> 30);   // 2^-34 turns
  float s, c;
  sincospif((float)rest * 1.1641532182693481e-10f, &s, &c);          // half turns: 2^-33
  const float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
  return quarter & 2 ? make_float2(-x, -y) : make_float2(x, y);
}

template <typename T> constexpr int kVec = 16 / sizeof(T);           // elements of a 16-byte vector

template <typename T> __device__ __forceinline__ void unpack(const uint4& w, float* v) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      v[i] = __uint_as_float(u[i]);
    } else {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
}
template <typename T> __device__ __forceinline__ uint4 packed(const float* v) {
  if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  } else {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
}

// What a lane of a group holds of every row: two vectors, at columns a and b.  Without INTER a pair is an element of each, with INTER
// it is two neighbours; behind the rotated dimensions the angle is zero.
template <typename T, bool INTER> struct NormLane {
  static constexpr int V = kVec<T>;
  int a, b;
  bool on;                                        // a group may have more lanes than a row has vectors
  __device__ __forceinline__ NormLane(int c, int dim, int rotary) {
    on = c < dim / (2 * V);
    if (!on) c = 0;
    if (INTER || c * 2 * V >= rotary) { a = 2 * c * V; b = a + V; }
    else { a = c * V; b = rotary / 2 + c * V; }
  }
  // pair of the e-th angle
  __device__ __forceinline__ int pair(int e) const {
    if (INTER) return e < V / 2 ? a / 2 + e : b / 2 + e - V / 2;
    return a + e;
  }
  __device__ __forceinline__ void angles(float2 (&cs)[V], const NormArgs& p, int32_t position) const {
#pragma unroll
    for (int e = 0; e < V; ++e) cs[e] = a < p.rotary ? turn_of(position, p.turns[pair(e)]) : make_float2(1.f, 0.f);
  }
  // v (both vectors one behind the other) turned forth or (BACK) back
  template <bool BACK> static __device__ __forceinline__ void turn(float (&v)[2 * V], const float2 (&cs)[V]) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int i = INTER ? 2 * e : e, j = INTER ? 2 * e + 1 : V + e;
      const float c = cs[e].x, s = BACK ? -cs[e].y : cs[e].y, x = v[i], y = v[j];
      v[i] = x * c - y * s;
      v[j] = y * c + x * s;
    }
  }
  __device__ __forceinline__ void load(float (&v)[2 * V], const T* row) const {
    unpack<T>(*reinterpret_cast<const uint4*>(row + a), v);
    unpack<T>(*reinterpret_cast<const uint4*>(row + b), v + V);
  }
  __device__ __forceinline__ void fetch(uint4 (&v)[2], const T* row) const {
    v[0] = *reinterpret_cast<const uint4*>(row + a);
    v[1] = *reinterpret_cast<const uint4*>(row + b);
  }
  static __device__ __forceinline__ void spread(float (&v)[2 * V], const uint4 (&raw)[2]) {
    unpack<T>(raw[0], v);
    unpack<T>(raw[1], v + V);
  }
  __device__ __forceinline__ void gains(float (&g)[2 * V], const float* gain) const {
#pragma unroll
    for (int e = 0; e < V; ++e) { g[e] = gain[a + e]; g[V + e] = gain[b + e]; }
  }
};

template <int L> __device__ __forceinline__ uint32_t group_mask() {
  return L == 32 ? 0xffffffffu : ((1u << (L & 31)) - 1) << (threadIdx.x & 31 & ~(L - 1));
}
template <int L> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(group_mask<L>(), v, o);
  return v;
}

// The heads of `side` that part `part` of `parts` takes, of both sides' heads in a row.
__device__ __forceinline__ void heads_of(const NormArgs& p, int side, int part, int& h0, int& h1) {
  const int n = p.side[0].heads, all = n + p.side[1].heads;
  const int first = (int)((int64_t)all * part / p.parts), last = (int)((int64_t)all * (part + 1) / p.parts);
  h0 = side ? max(first - n, 0) : min(first, n);
  h1 = side ? max(last - n, 0) : min(last, n);
}

template <typename T, int L, bool INTER>
__global__ void __launch_bounds__(kNormThreads) head_norm_kernel(const __grid_constant__ NormArgs p) {
  constexpr int V = kVec<T>, U = 2;               // heads in flight
  const int64_t group = ((int64_t)blockIdx.x * kNormThreads + threadIdx.x) / L, token = group / p.parts;
  if (token >= p.tokens) return;
  const NormLane<T, INTER> at(threadIdx.x % L, p.dim, p.rotary);
  float2 cs[V];
  at.angles(cs, p, p.rotary ? p.positions[token] : 0);
  const float per = 1.f / p.dim;
  for (int side = 0; side < 2; ++side) {
    const NormSide& s = p.side[side];
    int h0, h1;
    heads_of(p, side, (int)(group - token * p.parts), h0, h1);
    if (h0 >= h1) continue;
    float g[2 * V];
    at.gains(g, s.gain);
    for (int h = h0; h < h1; h += U) {
      float x[U][2 * V];
#pragma unroll
      for (int i = 0; i < U; ++i) at.load(x[i], head_row<T>(s.x, token, min(h + i, h1 - 1)));
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (h + i >= h1) break;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) sum = fmaf(x[i][e], x[i][e], sum);
        const float r = rsqrtf(group_sum<L>(at.on ? sum : 0.f) * per + p.eps);
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) x[i][e] *= r * g[e];
        at.template turn<false>(x[i], cs);
        T* out = head_row_out<T>(s.y, token, h + i);
        if (at.on) {
          *reinterpret_cast<uint4*>(out + at.a) = packed<T>(x[i]);
          *reinterpret_cast<uint4*>(out + at.b) = packed<T>(x[i] + V);
        }
      }
    }
  }
}

// The block's sums of the gains' gradients, over its groups in a fixed order, to row `block` of the partial sums.
template <int L, int N, typename COL>
__device__ __forceinline__ void leave_gains(const NormArgs& p, int block, const float (&acc)[N], bool on, COL col) {
  __shared__ float sums[kNormThreads / 32][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float v = acc[e];
#pragma unroll
    for (int o = L; o < 32; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane < L && on && col(e) < p.dim) sums[warp][col(e)] = v;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.dim; i += kNormThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kNormThreads / 32; ++w) v += sums[w][i];
    p.partials[(int64_t)block * p.dim + i] = v;
  }
}

// A block has rows of queries or rows of keys alone, so that it needs the sums of one gain; the next head's rows are fetched while this
// one's are worked on.
template <typename T, int L, bool INTER>
__global__ void __launch_bounds__(kNormThreads, 2) head_norm_bwd_kernel(const __grid_constant__ NormArgs p) {
  constexpr int V = kVec<T>;
  pdl_trigger();
  const int side = blockIdx.x >= p.blocks[0], block = blockIdx.x - (side ? p.blocks[0] : 0), parts = p.side_parts[side];
  const NormSide& s = p.side[side];
  const int64_t groups = p.tokens * parts, step = (int64_t)p.blocks[side] * (kNormThreads / L);
  const NormLane<T, INTER> at(threadIdx.x % L, p.dim, p.rotary);
  const float per = 1.f / p.dim;
  float acc[2 * V] = {}, g[2 * V];
  at.gains(g, s.gain);
  for (int64_t group = ((int64_t)block * kNormThreads + threadIdx.x) / L; group < groups; group += step) {
    const int64_t token = group / parts;
    const int part = (int)(group - token * parts), h0 = s.heads * part / parts, h1 = s.heads * (part + 1) / parts;
    const T *x_row = head_row<T>(s.x, token, h0), *u_row = head_row<T>(s.y, token, h0);
    T* out = head_row_out<T>(s.dx, token, h0);
    uint4 next_x[2], next_u[2];
    at.fetch(next_x, x_row);
    at.fetch(next_u, u_row);
    float2 cs[V];
    at.angles(cs, p, p.rotary ? p.positions[token] : 0);
    for (int h = h0; h < h1; ++h) {
      float x[2 * V], u[2 * V];
      at.spread(x, next_x);
      at.spread(u, next_u);
      if (h + 1 < h1) {
        x_row += s.x.head;
        u_row += s.y.head;
        at.fetch(next_x, x_row);
        at.fetch(next_u, u_row);
      }
      at.template turn<true>(u, cs);
      float square = 0.f, dot = 0.f;
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) { square = fmaf(x[e], x[e], square); dot = fmaf(x[e], u[e] * g[e], dot); }
      const float r = rsqrtf(group_sum<L>(at.on ? square : 0.f) * per + p.eps);
      const float f = group_sum<L>(at.on ? dot : 0.f) * per * r * r;
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        acc[e] = fmaf(u[e], x[e] * r, acc[e]);
        x[e] = r * (g[e] * u[e] - x[e] * f);
      }
      if (at.on) {
        *reinterpret_cast<uint4*>(out + at.a) = packed<T>(x);
        *reinterpret_cast<uint4*>(out + at.b) = packed<T>(x + V);
      }
      out += s.dx.head;
    }
  }
  if (p.partials) leave_gains<L>(p, blockIdx.x, acc, at.on, [&](int e) { return e < V ? at.a + e : at.b + e - V; });
}

// Rows of any width, alignment and pairing: a warp to a row, an element to a lane, the other of a pair through shared memory.
template <typename T, bool BACKWARD>
__global__ void __launch_bounds__(kNormThreads) head_norm_any_kernel(const __grid_constant__ NormArgs p, int interleaved) {
  __shared__ float rows[kNormThreads / 32][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = p.rotary / 2;
  float* const row = rows[warp];
  const int only = BACKWARD && blockIdx.x >= p.blocks[0], block = blockIdx.x - (only ? p.blocks[0] : 0), parts = BACKWARD ? p.side_parts[only] : p.parts;
  const int64_t groups = p.tokens * parts, step = (int64_t)(BACKWARD ? p.blocks[only] : (int)gridDim.x) * (kNormThreads / 32);
  const float per = 1.f / p.dim;
  float acc[4] = {};
  if (BACKWARD) pdl_trigger();
  for (int64_t group = (int64_t)block * (kNormThreads / 32) + warp; group < groups; group += step) {
    const int64_t token = group / parts;
    const int32_t position = p.rotary ? p.positions[token] : 0;
    float c[4], sn[4];
    int other[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = lane + 32 * j;
      const bool turned = i < p.rotary, second = interleaved ? i & 1 : i >= half;
      const int pair = interleaved ? i / 2 : second ? i - half : i;
      const float2 t = turned ? turn_of(position, p.turns[pair]) : make_float2(1.f, 0.f);
      other[j] = turned ? (interleaved ? i ^ 1 : second ? i - half : i + half) : 0;
      c[j] = t.x;
      sn[j] = second != BACKWARD ? t.y : -t.y;    // what the other element of the pair is multiplied with
    }
    auto turn = [&](float (&v)[4]) {
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 4; ++j) row[lane + 32 * j] = v[j];
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 4; ++j) if (lane + 32 * j < p.rotary) v[j] = v[j] * c[j] + row[other[j]] * sn[j];
    };
    const int part = (int)(group - token * parts);
    for (int side = only; side < (BACKWARD ? only + 1 : 2); ++side) {
      const NormSide& s = p.side[side];
      int h0, h1;
      if (BACKWARD) { h0 = s.heads * part / parts; h1 = s.heads * (part + 1) / parts; }
      else heads_of(p, side, part, h0, h1);
      for (int h = h0; h < h1; ++h) {
        float x[4], g[4], u[4];
        float square = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = lane + 32 * j;
          x[j] = i < p.dim ? to_f<T>(head_row<T>(s.x, token, h)[i]) : 0.f;
          u[j] = BACKWARD && i < p.dim ? to_f<T>(head_row<T>(s.y, token, h)[i]) : 0.f;
          g[j] = i < p.dim ? s.gain[i] : 0.f;
          square = fmaf(x[j], x[j], square);
        }
        const float r = rsqrtf(group_sum<32>(square) * per + p.eps);
        if constexpr (BACKWARD) {
          turn(u);
#pragma unroll
          for (int j = 0; j < 4; ++j) dot = fmaf(x[j], u[j] * g[j], dot);
          const float f = group_sum<32>(dot) * per * r * r;
          T* out = head_row_out<T>(s.dx, token, h);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            acc[j] = fmaf(u[j], x[j] * r, acc[j]);
            if (lane + 32 * j < p.dim) out[lane + 32 * j] = from_f<T>(r * (g[j] * u[j] - x[j] * f));
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] *= r * g[j];
          turn(x);
          T* out = head_row_out<T>(s.y, token, h);
#pragma unroll
          for (int j = 0; j < 4; ++j) if (lane + 32 * j < p.dim) out[lane + 32 * j] = from_f<T>(x[j]);
        }
      }
    }
  }
  if (BACKWARD && p.partials) leave_gains<32>(p, blockIdx.x, acc, true, [&](int e) { return lane + 32 * e; });
}

// Sums of the blocks' parts in a fixed order, in 64 bits: 32 columns of a side to a block, 32 rows at a time.
__global__ void __launch_bounds__(1024) head_norm_gains_kernel(const float* partials, int blocks_q, int blocks_k, int dim, float* d_gain_q, float* d_gain_k) {
  __shared__ double sums[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, side = blockIdx.y, col = blockIdx.x * 32 + x, blocks = side ? blocks_k : blocks_q;
  float* const out = side ? d_gain_k : d_gain_q;
  pdl_wait();
  if (!out) return;
  if (side) partials += (int64_t)blocks_q * dim;
  double v = 0.0;
  if (col < dim)
#pragma unroll 4
    for (int b = y; b < blocks; b += 32) v += partials[(int64_t)b * dim + col];
  sums[y][x] = v;
  __syncthreads();
  v = sums[x][y];                                 // a warp to a column
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (x == 0 && blockIdx.x * 32 + y < dim) out[blockIdx.x * 32 + y] = (float)v;
}

constexpr int kNormBwdBlocks = 2 * kSms;          // as many as run at a time; the two sides share them

// lanes to a row: the vectors of half a row, rounded up to a power of two
static int norm_lanes(int dim, int vec) {
  int lanes = 1;
  while (lanes * 2 * vec < dim) lanes *= 2;
  return lanes;
}
// Groups to a token: one where tokens alone fill the SMs with 512 threads each, else as many as that takes and there are heads.
static int norm_parts(int64_t tokens, int heads, int lanes) {
  const int64_t want = (int64_t)512 * kSms / lanes;
  return (int)std::min<int64_t>(heads, std::max<int64_t>(1, (want + tokens - 1) / tokens));
}

template <typename T, int L, bool INTER> static cudaError_t norm_vec(const NormArgs& p, bool backward, int64_t blocks, cudaStream_t st) {
  return backward ? launch_pdl(head_norm_bwd_kernel<T, L, INTER>, dim3((unsigned)blocks), dim3(kNormThreads), 0, st, false, p)
                  : launch_pdl(head_norm_kernel<T, L, INTER>, dim3((unsigned)blocks), dim3(kNormThreads), 0, st, false, p);
}
template <typename T, bool INTER> static cudaError_t norm_width(const NormArgs& p, int lanes, bool backward, int64_t blocks, cudaStream_t st) {
  switch (lanes) {
    case 1: return norm_vec<T, 1, INTER>(p, backward, blocks, st);
    case 2: return norm_vec<T, 2, INTER>(p, backward, blocks, st);
    case 4: return norm_vec<T, 4, INTER>(p, backward, blocks, st);
    case 8: return norm_vec<T, 8, INTER>(p, backward, blocks, st);
    default: break;
  }
  if constexpr (sizeof(T) == 4) return norm_vec<T, 16, INTER>(p, backward, blocks, st);
  return cudaErrorInvalidValue;
}

template <typename T> static cudaError_t norm_run(NormArgs& p, bool interleaved, bool backward, float* d_gain_q, float* d_gain_k, cudaStream_t st) {
  constexpr int V = kVec<T>;
  bool vec = p.dim % (2 * V) == 0 && p.rotary % (2 * V) == 0;
  auto whole = [&](const HeadView& x) { vec = vec && aligned_to(x.data, 16) && x.token % V == 0 && x.head % V == 0; };
  for (const NormSide& s : p.side)
    if (s.heads) {
      whole(s.x);
      whole(s.y);
      if (backward) whole(s.dx);
    }
  const int lanes = vec ? norm_lanes(p.dim, V) : 32, heads = p.side[0].heads + p.side[1].heads;
  const int64_t per_block = kNormThreads / lanes;
  int64_t blocks;
  if (backward) {
    // both sides' groups, and the blocks, by their heads
    blocks = 0;
    for (int i = 0; i < 2; ++i) {
      const int n = p.side[i].heads;
      if (!n) continue;
      const int share = std::max(1, (int)((int64_t)kNormBwdBlocks * n / heads));
      p.side_parts[i] = norm_parts(p.tokens, n, lanes);
      p.blocks[i] = (int)std::min<int64_t>((p.tokens * p.side_parts[i] + per_block - 1) / per_block, share);
      blocks += p.blocks[i];
    }
  } else {
    p.parts = norm_parts(p.tokens, heads, lanes);
    blocks = (p.tokens * p.parts + per_block - 1) / per_block;
  }
  if (!launchable(blocks)) return cudaErrorInvalidConfiguration;
  cudaError_t e;
  if (!vec)
    e = backward ? launch_pdl(head_norm_any_kernel<T, true>, dim3((unsigned)blocks), dim3(kNormThreads), 0, st, false, p, (int)interleaved)
                 : launch_pdl(head_norm_any_kernel<T, false>, dim3((unsigned)blocks), dim3(kNormThreads), 0, st, false, p, (int)interleaved);
  else
    e = interleaved ? norm_width<T, true>(p, lanes, backward, blocks, st) : norm_width<T, false>(p, lanes, backward, blocks, st);
  if (e == cudaSuccess && p.partials)
    e = launch_pdl(head_norm_gains_kernel, dim3((p.dim + 31) / 32, 2), dim3(1024), 0, st, true, (const float*)p.partials, p.blocks[0], p.blocks[1], p.dim,
                   d_gain_q, d_gain_k);
  return e;
}

static pm_status norm_check(NormArgs& p, const pm_head_norm_desc* d) {
  if (!d) return ops_fail(PM_ERR_INVALID_ARG, "null argument");
  if (d->dtype != PM_F32 && d->dtype != PM_BF16) return ops_fail(PM_ERR_INVALID_ARG, "unknown element type");
  if (d->head_dim < 1) return ops_fail(PM_ERR_INVALID_ARG, "head_dim must be positive");
  if (d->head_dim > 128) return ops_fail(PM_ERR_UNSUPPORTED, "heads wider than 128");
  if (d->n_heads < 0 || d->n_kv_heads < 0 || d->n_heads + (int64_t)d->n_kv_heads < 1) return ops_fail(PM_ERR_INVALID_ARG, "neither queries nor keys");
  if (d->n_heads > 65535 || d->n_kv_heads > 65535) return ops_fail(PM_ERR_SHAPE, "at most 65535 heads");
  if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 2) return ops_fail(PM_ERR_INVALID_ARG, "rotary_dim must be even and at most head_dim");
  if (d->rotary_dim && !d->turns) return ops_fail(PM_ERR_INVALID_ARG, "null turns");
  if (d->n_tokens < 0) return ops_fail(PM_ERR_INVALID_ARG, "negative size");
  if (d->n_tokens > 0x7fffffff) return ops_fail(PM_ERR_SHAPE, "too many tokens");
  if (!(d->eps >= 0) || d->eps > 1e30f) return ops_fail(PM_ERR_INVALID_ARG, "eps must not be negative");
  p.tokens = d->n_tokens; p.dim = d->head_dim; p.rotary = d->rotary_dim; p.eps = d->eps;
  p.side[0].heads = d->n_heads; p.side[1].heads = d->n_kv_heads;
  for (int i = 0; i < d->rotary_dim / 2; ++i) p.turns[i] = d->turns[i];
  return PM_OK;
}
static pm_status norm_view(HeadView& out, const pm_head_view* v, const char* name, int size) {
  if (!v || !v->data) return ops_fail(PM_ERR_INVALID_ARG, "%s: null pointer", name);
  if (!aligned_to(v->data, size)) return ops_fail(PM_ERR_INVALID_ARG, "%s: pointer not aligned to its element type", name);
  if (v->token_stride < 0 || v->head_stride < 0) return ops_fail(PM_ERR_INVALID_ARG, "%s: negative stride", name);
  out = HeadView{v->data, v->token_stride, v->head_stride};
  return PM_OK;
}
static bool same_view(const HeadView& a, const HeadView& b) { return a.data == b.data && a.token == b.token && a.head == b.head; }

}  // namespace pm

using namespace pm;

extern "C" {

pm_status pm_rotation_turns(int32_t rotary_dim, double base, uint64_t* turns) {
  if (!turns || rotary_dim < 0 || rotary_dim % 2 || rotary_dim > 2 * kNormMostPairs) return ops_fail(PM_ERR_INVALID_ARG, "rotary_dim must be even, 0 to 128");
  if (!(base >= 1.0) || base > 1e300) return ops_fail(PM_ERR_INVALID_ARG, "base must be at least 1");
  const long double turn = 2.0L * 3.14159265358979323846264338327950288L;
  for (int i = 0; i < rotary_dim / 2; ++i)
    turns[i] = (uint64_t)(powl((long double)base, -2.0L * i / rotary_dim) / turn * 18446744073709551616.0L + 0.5L);
  return PM_OK;
}

pm_status pm_head_norm_rotate(const pm_head_norm_desc* d, const pm_head_view* q, const pm_head_view* k, const int32_t* positions, const float* q_gain,
                              const float* k_gain, const pm_head_view* q_out, const pm_head_view* k_out, void* stream) {
  NormArgs p{};
  if (const pm_status s = norm_check(p, d)) return s;
  if (p.tokens == 0) return PM_OK;
  const int size = d->dtype == PM_BF16 ? 2 : 4;
  const pm_head_view *x[2] = {q, k}, *y[2] = {q_out, k_out};
  const float* gain[2] = {q_gain, k_gain};
  const char *names[2] = {"q", "k"}, *out_names[2] = {"q_out", "k_out"};
  Extent in[2] = {}, out[2] = {};
  for (int i = 0; i < 2; ++i) {
    NormSide& s = p.side[i];
    if (!s.heads) continue;
    if (const pm_status e = norm_view(s.x, x[i], names[i], size)) return e;
    if (const pm_status e = norm_view(s.y, y[i], out_names[i], size)) return e;
    if (!gain[i] || !aligned_to(gain[i], 4)) return ops_fail(PM_ERR_INVALID_ARG, "%s_gain: null or misaligned pointer", names[i]);
    s.gain = gain[i];
    in[i] = Extent{(__int128)reinterpret_cast<uintptr_t>(s.x.data), (__int128)s.x.token * size, p.tokens, (__int128)s.x.head * size, s.heads, (__int128)p.dim * size};
    out[i] = Extent{(__int128)reinterpret_cast<uintptr_t>(s.y.data), (__int128)s.y.token * size, p.tokens, (__int128)s.y.head * size, s.heads, (__int128)p.dim * size};
  }
  if (p.rotary && (!positions || !aligned_to(positions, 4))) return ops_fail(PM_ERR_INVALID_ARG, "positions: null or misaligned pointer");
  p.positions = positions;
  for (int i = 0; i < 2; ++i) {
    for (int j = 0; j < 2; ++j) {
      if (extents_share(out[i], in[j]) && !(i == j && same_view(p.side[i].x, p.side[i].y))) return ops_fail(PM_ERR_INVALID_ARG, "an output overlaps one of the inputs");
      if (p.side[j].heads && extents_share(out[i], dense_extent(gain[j], 4 * (int64_t)p.dim))) return ops_fail(PM_ERR_INVALID_ARG, "an output overlaps one of the inputs");
    }
    if (p.rotary && extents_share(out[i], dense_extent(positions, 4 * p.tokens))) return ops_fail(PM_ERR_INVALID_ARG, "an output overlaps one of the inputs");
  }
  if (extents_share(out[0], out[1])) return ops_fail(PM_ERR_INVALID_ARG, "two outputs overlap");
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = d->dtype == PM_BF16 ? norm_run<__nv_bfloat16>(p, d->interleaved != 0, false, nullptr, nullptr, st)
                                            : norm_run<float>(p, d->interleaved != 0, false, nullptr, nullptr, st);
  return ops_cuda(e, "head norms and rotation");
}

uint64_t pm_head_norm_rotate_workspace_bytes(const pm_head_norm_desc* d) {
  return !d || d->head_dim < 1 || d->head_dim > 128 ? 0 : (uint64_t)(kNormBwdBlocks + 1) * d->head_dim * sizeof(float);
}

pm_status pm_head_norm_rotate_backward(const pm_head_norm_desc* d, const pm_head_view* q, const pm_head_view* k, const int32_t* positions,
                                       const float* q_gain, const float* k_gain, const pm_head_view* d_q_out, const pm_head_view* d_k_out,
                                       const pm_head_view* dq, const pm_head_view* dk, float* d_q_gain, float* d_k_gain, void* workspace,
                                       uint64_t workspace_bytes, void* stream) {
  NormArgs p{};
  if (const pm_status s = norm_check(p, d)) return s;
  const cudaStream_t st = (cudaStream_t)stream;
  const int size = d->dtype == PM_BF16 ? 2 : 4;
  const pm_head_view *x[2] = {q, k}, *y[2] = {d_q_out, d_k_out}, *dx[2] = {dq, dk};
  const float* gain[2] = {q_gain, k_gain};
  float* d_gain[2] = {d_q_gain, d_k_gain};
  const char *names[2] = {"q", "k"}, *out_names[2] = {"d_q_out", "d_k_out"}, *grad_names[2] = {"dq", "dk"};
  Extent written[5] = {}, read[7] = {};           // dq, dk, d_q_gain, d_k_gain, workspace;  x, y, gain of both, positions
  const bool gains = d_q_gain || d_k_gain;
  const uint64_t need = gains ? pm_head_norm_rotate_workspace_bytes(d) : 0;
  for (int i = 0; i < 2; ++i) {
    NormSide& s = p.side[i];
    if (!s.heads) {
      if (d_gain[i]) return ops_fail(PM_ERR_INVALID_ARG, "d_%s_gain without %s", names[i], names[i]);
      continue;
    }
    if (!aligned_to(d_gain[i], 4)) return ops_fail(PM_ERR_INVALID_ARG, "d_%s_gain: misaligned pointer", names[i]);
    written[2 + i] = dense_extent(d_gain[i], 4 * (int64_t)p.dim);
    if (p.tokens == 0) continue;
    if (const pm_status e = norm_view(s.x, x[i], names[i], size)) return e;
    if (const pm_status e = norm_view(s.y, y[i], out_names[i], size)) return e;
    if (const pm_status e = norm_view(s.dx, dx[i], grad_names[i], size)) return e;
    if (!gain[i] || !aligned_to(gain[i], 4)) return ops_fail(PM_ERR_INVALID_ARG, "%s_gain: null or misaligned pointer", names[i]);
    s.gain = gain[i];
    auto all = [&](const HeadView& v) {
      return Extent{(__int128)reinterpret_cast<uintptr_t>(v.data), (__int128)v.token * size, p.tokens, (__int128)v.head * size, s.heads, (__int128)p.dim * size};
    };
    written[i] = all(s.dx);
    read[3 * i] = all(s.x);
    read[3 * i + 1] = all(s.y);
    read[3 * i + 2] = dense_extent(gain[i], 4 * (int64_t)p.dim);
  }
  if (p.tokens == 0) {                            // sums of nothing
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < 2; ++i) if (d_gain[i] && e == cudaSuccess) e = cudaMemsetAsync(d_gain[i], 0, sizeof(float) * p.dim, st);
    return ops_cuda(e, "head norms and rotation backward");
  }
  if (p.rotary && (!positions || !aligned_to(positions, 4))) return ops_fail(PM_ERR_INVALID_ARG, "positions: null or misaligned pointer");
  p.positions = positions;
  if (p.rotary) read[6] = dense_extent(positions, 4 * p.tokens);
  if (need) {
    if (!workspace || workspace_bytes < need) return ops_fail(PM_ERR_NOMEM, "workspace too small: need %llu bytes", (unsigned long long)need);
    if (!aligned_to(workspace, 4)) return ops_fail(PM_ERR_INVALID_ARG, "workspace must be 4-byte aligned");
    written[4] = dense_extent(workspace, (int64_t)need);
  }
  for (int i = 0; i < 5; ++i) {
    for (int j = 0; j < 7; ++j)
      if (extents_share(written[i], read[j]) && !(i < 2 && j == 3 * i + 1 && same_view(p.side[i].dx, p.side[i].y)))
        return ops_fail(PM_ERR_INVALID_ARG, "an output overlaps one of the inputs");
    for (int j = 0; j < i; ++j) if (extents_share(written[i], written[j])) return ops_fail(PM_ERR_INVALID_ARG, "two outputs overlap");
  }
  p.partials = gains ? static_cast<float*>(workspace) : nullptr;
  const cudaError_t e = d->dtype == PM_BF16 ? norm_run<__nv_bfloat16>(p, d->interleaved != 0, true, d_q_gain, d_k_gain, st)
                                            : norm_run<float>(p, d->interleaved != 0, true, d_q_gain, d_k_gain, st);
  return ops_cuda(e, "head norms and rotation backward");
}

}  // extern "C"
