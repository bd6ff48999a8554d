// Norms of queries and keys for each head, and the rotation by their positions, in one pass; backward with the gains' gradients.
//
//   r = (mean_i x_i^2 + eps)^(-1/2),  n_i = g_i x_i r,  y = R(position) n
//   (y_a, y_b) = (n_a cos - n_b sin, n_b cos + n_a sin) for pair i of the first rotary_dim dimensions at the angle position f_i
//   u = R^T dy,  dg = sum u x r,  dx = r (g u - x r^2 mean_i(g_i u_i x_i))
//
// Bound by memory: each row is read once and written once.  A group of lanes takes a row, and the groups of a warp take the same head of
// consecutive tokens, then the next head: the sines and cosines of a token are formed once or twice, in registers, by the lanes whose
// dimensions they turn, at the same time in the whole warp.  Both dimensions of a pair lie in one lane, and only the sum of squares
// crosses lanes.  A lane's constants and values fill 100 registers, so few warps run at a time: what is under way is kept in shared
// memory, each lane copying its own part of the next rows there.  12291 tokens, 16 + 2 heads of 128, bf16: forward 22 us, 5.1 TB/s, backward 33 us,
// 5.2 TB/s; 16 tokens forward 3.3 us, of which the launch and the loads of starts and rows are most.
//
// The angle is a fraction of a turn in 64 bits: position times the frequency in units of 2^-64 turns wraps as angles do, so it is exact
// to 2^-33 turns at every position; the nearest quarter turn is taken off it before it becomes a float (at most an eighth of a turn, rounded
// by 7e-8 radians), and sine and cosine of that are their series.
#include <atomic>
#include <cmath>

#include "pm_attn_packed.cuh"
#include "pm_ptx.cuh"

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
  int dim, rotary;
  int blocks[2];                                  // of each side
  float eps;
  uint64_t turns[kNormMostPairs];                 // frequency of each pair, 2^-64 turns per position
};

// What is left of position times a frequency beside its nearest quarter turn, in radians, and that quarter.
__device__ __forceinline__ float rest_of(int32_t position, uint64_t turns, int& quarter) {
  const uint64_t a = (uint64_t)(int64_t)position * turns + (1ull << 61);         // an eighth of a turn on: the quarter is the nearest one
  quarter = (int)(a >> 62);
  const int32_t rest = (int32_t)((uint32_t)(a >> 30) - (1u << 31));              // 2^-34 turns
  return (float)rest * 3.6572951e-10f;                                           // 2 pi 2^-34
}
// cosines (x) and sines of two angles of at most pi / 4: the series up to x^10 and x^9, whose next terms are below 2e-10 and 2e-9
__device__ __forceinline__ void series(float2 x, float2& c, float2& s) {
  auto k = [](float v) { return make_float2(v, v); };
  const float2 q = mul_f32x2(x, x);
  c = fma_f32x2(q, k(-1.f / 3628800.f), k(1.f / 40320.f));
  s = fma_f32x2(q, k(1.f / 362880.f), k(-1.f / 5040.f));
  c = fma_f32x2(c, q, k(-1.f / 720.f));
  s = fma_f32x2(s, q, k(1.f / 120.f));
  c = fma_f32x2(c, q, k(1.f / 24.f));
  s = fma_f32x2(s, q, k(-1.f / 6.f));
  c = fma_f32x2(c, q, k(-0.5f));
  s = mul_f32x2(s, q);
  c = fma_f32x2(c, q, k(1.f));
  s = fma_f32x2(s, x, x);
}
// cos and sin from those of the rest
__device__ __forceinline__ void turn_quarters(float& c, float& s, int quarter) {
  const float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
  c = quarter & 2 ? -x : x;
  s = quarter & 2 ? -y : y;
}
__device__ __forceinline__ float2 turn_of(int32_t position, uint64_t turns) {
  int quarter;
  float2 x = make_float2(rest_of(position, turns, quarter), 0.f), c, s;
  series(x, c, s);
  turn_quarters(c.x, s.x, quarter);
  return make_float2(c.x, s.x);
}

template <typename T> constexpr int kVec = 16 / sizeof(T);           // elements of a 16-byte vector
// V elements: 16 bytes, or 8 where that is what divides rows and their rotated part
template <typename T, int V> using NormVector = std::conditional_t<V * sizeof(T) == 16, uint4, uint2>;
template <int BYTES> __device__ __forceinline__ void norm_copy(void* dst, const void* src) {
  if constexpr (BYTES == 16) cp_async16(dst, src);
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// V pairs: the first elements and the second ones, two pairs to a register pair of the packed arithmetic.
template <int V> struct Pairs {
  float2 f[V / 2], s[V / 2];
};

// What a lane of a group holds of every row: two vectors, at columns a and b, which are V pairs.  Without INTER a pair is an element of
// each, with INTER it is two neighbours; behind the rotated dimensions the angle is zero.  b is half of the rotated dimensions, or of the
// others, from a, so that the lanes' vectors lie side by side (fp32, 12000 tokens, 8 + 2 heads of 128, 64 rotated: forward 21 us, backward
// 35; with a lane's two vectors side by side 28 and 46).
template <typename T, int V, bool INTER> struct NormLane {
  using Vector = NormVector<T, V>;
  static constexpr int kWords = sizeof(Vector) / 4;
  int a, b;
  bool on;                                        // a group may have more lanes than a row has vectors
  __device__ __forceinline__ NormLane(int c, int dim, int rotary) {
    on = c < dim / (2 * V);
    if (!on) c = 0;
    const int turned = rotary / (2 * V), from = c < turned ? 0 : rotary;         // lanes of the rotated dimensions, then those of the rest
    a = from + (c < turned ? c : c - turned) * V;
    b = a + (c < turned ? rotary : dim - rotary) / 2;
  }
  // columns of the e-th pair
  __device__ __forceinline__ int first(int e) const { return INTER ? (e < V / 2 ? a + 2 * e : b + 2 * e - V) : a + e; }
  __device__ __forceinline__ int second(int e) const { return INTER ? first(e) + 1 : b + e; }
  // cos in f, sin in s
  __device__ __forceinline__ void angles(Pairs<V>& cs, const NormArgs& p, int32_t position) const {
    if (a >= p.rotary) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) { cs.f[i] = make_float2(1.f, 1.f); cs.s[i] = make_float2(0.f, 0.f); }
      return;
    }
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      const int pair = INTER ? first(2 * i) / 2 : a + 2 * i;       // of which the next one is the lane's next one, too
      int qx, qy;
      float2 x;
      x.x = rest_of(position, p.turns[pair], qx);
      x.y = rest_of(position, p.turns[pair + 1], qy);
      series(x, cs.f[i], cs.s[i]);
      turn_quarters(cs.f[i].x, cs.s[i].x, qx);
      turn_quarters(cs.f[i].y, cs.s[i].y, qy);
    }
  }
  __device__ __forceinline__ void gains(Pairs<V>& g, const float* gain) const {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      (e & 1 ? g.f[e / 2].y : g.f[e / 2].x) = gain[first(e)];
      (e & 1 ? g.s[e / 2].y : g.s[e / 2].x) = gain[second(e)];
    }
  }
  static __device__ __forceinline__ void spread(Pairs<V>& v, const Vector* slot) {
    const Vector lo = slot[0], hi = slot[kNormThreads];
    uint32_t w[2 * kWords];
    memcpy(w, &lo, sizeof(lo));
    memcpy(w + kWords, &hi, sizeof(hi));
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v.f[i] = INTER ? make_float2(__uint_as_float(w[4 * i]), __uint_as_float(w[4 * i + 2])) : make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        v.s[i] = INTER ? make_float2(__uint_as_float(w[4 * i + 1]), __uint_as_float(w[4 * i + 3]))
                       : make_float2(__uint_as_float(w[4 + 2 * i]), __uint_as_float(w[5 + 2 * i]));
      }
    } else {
      auto low = [](uint32_t u) { return __uint_as_float(u << 16); };
      auto high = [](uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); };
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        v.f[i] = INTER ? make_float2(low(w[2 * i]), low(w[2 * i + 1])) : make_float2(low(w[i]), high(w[i]));
        v.s[i] = INTER ? make_float2(high(w[2 * i]), high(w[2 * i + 1])) : make_float2(low(w[kWords + i]), high(w[kWords + i]));
      }
    }
  }
  // to the lane's columns, of which `row` is the first; the other vector is `apart` elements on
  static __device__ __forceinline__ void store(T* row, int apart, const Pairs<V>& v) {
    uint32_t w[2 * kWords];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float x[4] = {v.f[i].x, v.f[i].y, v.s[i].x, v.s[i].y};
        w[INTER ? 4 * i : 2 * i] = __float_as_uint(x[0]);
        w[INTER ? 4 * i + 2 : 2 * i + 1] = __float_as_uint(x[1]);
        w[INTER ? 4 * i + 1 : 4 + 2 * i] = __float_as_uint(x[2]);
        w[INTER ? 4 * i + 3 : 5 + 2 * i] = __float_as_uint(x[3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        w[INTER ? 2 * i : i] = INTER ? pack_bf16(v.f[i].x, v.s[i].x) : pack_bf16(v.f[i].x, v.f[i].y);
        w[INTER ? 2 * i + 1 : kWords + i] = INTER ? pack_bf16(v.f[i].y, v.s[i].y) : pack_bf16(v.s[i].x, v.s[i].y);
      }
    }
    Vector lo, hi;
    memcpy(&lo, w, sizeof(lo));
    memcpy(&hi, w + kWords, sizeof(hi));
    *reinterpret_cast<Vector*>(row) = lo;
    *reinterpret_cast<Vector*>(row + apart) = hi;
  }
};
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 minus(float2 x) { return make_float2(-x.x, -x.y); }

// over the L lanes of a group; the whole warp takes part
template <int L> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The rows that a warp takes in turn, those of `tokens` consecutive tokens at a time: its share of one side's, heads within tokens.
struct NormWalk {
  int64_t token, left;
  int h, heads, tokens;
  __device__ __forceinline__ NormWalk(const NormArgs& p, int side, int block, int tokens) : heads(p.side[side].heads), tokens(tokens) {
    const int64_t all = (p.tokens + tokens - 1) / tokens * heads, warps = (int64_t)p.blocks[side] * (kNormThreads / 32);
    const int64_t at = (int64_t)block * (kNormThreads / 32) + (threadIdx.x >> 5), first = all * at / warps;
    left = all * (at + 1) / warps - first;
    token = first / heads;
    h = (int)(first - token * heads);
    token = token * tokens + (threadIdx.x & 31) / (32 / tokens);
  }
  // whether the next row is another token's
  __device__ __forceinline__ bool next() {
    --left;
    if (++h < heads) return false;
    h = 0;
    token += tokens;
    return true;
  }
};

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

// Rows ahead of the one that is worked on, of two vectors of BYTES a lane or, with their gradients, four.
template <bool BACKWARD, int BYTES> constexpr int kNormAhead = (BACKWARD ? 4 : 6) * 16 / BYTES - 1;
template <bool BACKWARD> constexpr int kNormSmem = (kNormAhead<BACKWARD, 16> + 1) * (BACKWARD ? 4 : 2) * kNormThreads * 16;

// A block has rows of queries or rows of keys alone: one gain, and the sums of one.
template <typename T, int V, int L, bool INTER, bool BACKWARD>
__global__ void __launch_bounds__(kNormThreads, BACKWARD ? 2 : 3) head_norm_kernel(const __grid_constant__ NormArgs p) {
  constexpr int kBytes = V * sizeof(T), A = kNormAhead<BACKWARD, kBytes>, W = BACKWARD ? 4 : 2;  // W: vectors of a row in shared memory
  using Vector = NormVector<T, V>;
  extern __shared__ uint4 norm_ring[];
  if (BACKWARD) pdl_trigger();
  const int side = blockIdx.x >= p.blocks[0], block = blockIdx.x - (side ? p.blocks[0] : 0);
  const NormSide& s = p.side[side];
  const NormLane<T, V, INTER> at(threadIdx.x % L, p.dim, p.rotary);
  const float per = 1.f / p.dim;
  NormWalk now(p, side, block, 32 / L), ahead = now;
  // a group behind the last token takes that one's rows and writes nothing
  auto row_of = [&](const HeadView& v, const NormWalk& w) { return head_row<T>(v, min(w.token, p.tokens - 1), w.h) + at.a; };
  const T *x_row = row_of(s.x, ahead), *u_row = BACKWARD ? row_of(s.y, ahead) : nullptr;
  const HeadView& result = BACKWARD ? s.dx : s.y;
  T* out = nullptr;
  const int apart = at.b - at.a;
  Vector* const mine = reinterpret_cast<Vector*>(norm_ring) + threadIdx.x;
  int put = 0, get = 0;                           // places in the ring, in vectors
  constexpr int kPlace = W * kNormThreads, kPlaces = (A + 1) * kPlace;
  auto copy_next = [&]() {                        // a group of copies even where there is no row left: they are counted
    if (ahead.left > 0) {
      norm_copy<kBytes>(mine + put, x_row);
      norm_copy<kBytes>(mine + put + kNormThreads, x_row + apart);
      x_row += s.x.head;
      if (BACKWARD) {
        norm_copy<kBytes>(mine + put + 2 * kNormThreads, u_row);
        norm_copy<kBytes>(mine + put + 3 * kNormThreads, u_row + apart);
        u_row += s.y.head;
      }
      if (ahead.next()) {
        x_row = row_of(s.x, ahead);
        if (BACKWARD) u_row = row_of(s.y, ahead);
      }
    }
    cp_async_commit();
    put = put + kPlace == kPlaces ? 0 : put + kPlace;
  };
#pragma unroll
  for (int i = 0; i < A; ++i) copy_next();
  Pairs<V> g, acc = {}, cs, gs;
  if (BACKWARD) at.gains(g, s.gain);
  for (bool fresh = true; now.left > 0; fresh = now.next()) {
    const bool on = at.on && now.token < p.tokens;
    if (fresh) {
      out = const_cast<T*>(row_of(result, now));
      at.angles(cs, p, p.rotary && on ? p.positions[now.token] : 0);
      if (!BACKWARD) {                            // gains times cosines (in cs, first and second element) and sines
        at.gains(g, s.gain);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          gs.f[i] = mul_f32x2(g.f[i], cs.s[i]);
          gs.s[i] = mul_f32x2(g.s[i], minus(cs.s[i]));
          cs.s[i] = mul_f32x2(g.s[i], cs.f[i]);
          cs.f[i] = mul_f32x2(g.f[i], cs.f[i]);
        }
      }
    }
    copy_next();
    cp_async_wait<A>();                           // this row's copies, the oldest
    const Vector* const slot = mine + get;
    get = get + kPlace == kPlaces ? 0 : get + kPlace;
    Pairs<V> x;
    at.spread(x, slot);
    float2 square = both(0.f);
    if constexpr (!BACKWARD) {
#pragma unroll
      for (int e = 0; e < V / 2; ++e) square = fma_f32x2(x.s[e], x.s[e], fma_f32x2(x.f[e], x.f[e], square));
      const float2 r = both(rsqrtf(group_sum<L>(on ? square.x + square.y : 0.f) * per + p.eps));
      if (r.x == 0.f)                             // the squares left the range of fp32, and a product might before r makes it zero
#pragma unroll
        for (int e = 0; e < V / 2; ++e) { x.f[e] = mul_f32x2(x.f[e], r); x.s[e] = mul_f32x2(x.s[e], r); }
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {           // y_a = r (x_a g_a cos - x_b g_b sin), y_b = r (x_b g_b cos + x_a g_a sin)
        const float2 f = mul_f32x2(r, fma_f32x2(x.f[e], cs.f[e], mul_f32x2(x.s[e], gs.s[e])));
        x.s[e] = mul_f32x2(r, fma_f32x2(x.s[e], cs.s[e], mul_f32x2(x.f[e], gs.f[e])));
        x.f[e] = f;
      }
      if (on) at.store(out, apart, x);
    } else {
      Pairs<V> u;
      at.spread(u, slot + 2 * kNormThreads);
      float2 dot = both(0.f);
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        const float2 f = fma_f32x2(u.f[e], cs.f[e], mul_f32x2(u.s[e], cs.s[e]));
        u.s[e] = fma_f32x2(u.s[e], cs.f[e], mul_f32x2(u.f[e], minus(cs.s[e])));
        u.f[e] = f;
        square = fma_f32x2(x.s[e], x.s[e], fma_f32x2(x.f[e], x.f[e], square));
        dot = fma_f32x2(mul_f32x2(x.s[e], u.s[e]), g.s[e], fma_f32x2(mul_f32x2(x.f[e], u.f[e]), g.f[e], dot));
      }
      const float r = rsqrtf(group_sum<L>(on ? square.x + square.y : 0.f) * per + p.eps);
      // x r before it meets anything else: r^2 mean by itself leaves the normal range of fp32 where rows are large and gradients small (1e17 and
      // 1e-6).  With r = 0 the sum of products may have left it, too.
      const float mean = group_sum<L>(on ? dot.x + dot.y : 0.f) * per;
      const float2 rr = both(on ? r : 0.f), f = both(r == 0.f ? 0.f : mean * -r);
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        x.f[e] = mul_f32x2(x.f[e], rr);
        x.s[e] = mul_f32x2(x.s[e], rr);
        acc.f[e] = fma_f32x2(u.f[e], x.f[e], acc.f[e]);
        acc.s[e] = fma_f32x2(u.s[e], x.s[e], acc.s[e]);
        u.f[e] = mul_f32x2(fma_f32x2(x.f[e], f, mul_f32x2(u.f[e], g.f[e])), rr);
        u.s[e] = mul_f32x2(fma_f32x2(x.s[e], f, mul_f32x2(u.s[e], g.s[e])), rr);
      }
      if (on) at.store(out, apart, u);
    }
    out += result.head;
  }
  cp_async_wait<0>();
  if constexpr (BACKWARD) {
    if (!p.partials) return;
    float sums[2 * V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sums[e] = e & 1 ? acc.f[e / 2].y : acc.f[e / 2].x;
      sums[V + e] = e & 1 ? acc.s[e / 2].y : acc.s[e / 2].x;
    }
    leave_gains<L>(p, blockIdx.x, sums, at.on, [&](int e) { return e < V ? at.first(e) : at.second(e - V); });
  }
}

// Rows of any width, alignment and pairing: a warp to a row, an element to a lane, the other of a pair through shared memory.
template <typename T, bool BACKWARD>
__global__ void __launch_bounds__(kNormThreads) head_norm_any_kernel(const __grid_constant__ NormArgs p, int interleaved) {
  __shared__ float rows[kNormThreads / 32][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = p.rotary / 2;
  float* const row = rows[warp];
  const int side = blockIdx.x >= p.blocks[0], block = blockIdx.x - (side ? p.blocks[0] : 0);
  const NormSide& s = p.side[side];
  const float per = 1.f / p.dim;
  float acc[4] = {};
  if (BACKWARD) pdl_trigger();
  NormWalk now(p, side, block, 1);
  float c[4], sn[4];
  int other[4];
  auto turn = [&](float (&v)[4]) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) row[lane + 32 * j] = v[j];
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) if (lane + 32 * j < p.rotary) v[j] = v[j] * c[j] + row[other[j]] * sn[j];
  };
  for (bool fresh = true; now.left > 0; fresh = now.next()) {
    if (fresh) {
      const int32_t position = p.rotary ? p.positions[now.token] : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = lane + 32 * j;
        const bool turned = i < p.rotary, second = interleaved ? i & 1 : i >= half;
        const int pair = interleaved ? i / 2 : second ? i - half : i;
        const float2 t = turned ? turn_of(position, p.turns[pair]) : make_float2(1.f, 0.f);
        other[j] = turned ? (interleaved ? i ^ 1 : second ? i - half : i + half) : 0;
        c[j] = t.x;
        sn[j] = second != BACKWARD ? t.y : -t.y;  // what the other element of the pair is multiplied with
      }
    }
    float x[4], g[4], u[4];
    float square = 0.f, dot = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = lane + 32 * j;
      x[j] = i < p.dim ? to_f<T>(head_row<T>(s.x, now.token, now.h)[i]) : 0.f;
      u[j] = BACKWARD && i < p.dim ? to_f<T>(head_row<T>(s.y, now.token, now.h)[i]) : 0.f;
      g[j] = i < p.dim ? s.gain[i] : 0.f;
      square = fmaf(x[j], x[j], square);
    }
    const float r = rsqrtf(group_sum<32>(square) * per + p.eps);
    if constexpr (BACKWARD) {
      turn(u);
#pragma unroll
      for (int j = 0; j < 4; ++j) dot = fmaf(x[j], u[j] * g[j], dot);
      const float mean = group_sum<32>(dot) * per, f = r == 0.f ? 0.f : mean * r * r;         // with r the sum of products may have left the range, too
      T* out = head_row_out<T>(s.dx, now.token, now.h);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[j] = fmaf(u[j], x[j] * r, acc[j]);
        if (lane + 32 * j < p.dim) out[lane + 32 * j] = from_f<T>(r * (g[j] * u[j] - x[j] * f));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] *= r * g[j];
      turn(x);
      T* out = head_row_out<T>(s.y, now.token, now.h);
#pragma unroll
      for (int j = 0; j < 4; ++j) if (lane + 32 * j < p.dim) out[lane + 32 * j] = from_f<T>(x[j]);
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

// As many blocks as run at a time; the two sides share them.
template <bool BACKWARD> constexpr int kNormBlocks = (BACKWARD ? 2 : 3) * kSms;

// lanes to a row: the vectors of half a row, rounded up to a power of two
static int norm_lanes(int dim, int vec) {
  int lanes = 1;
  while (lanes * 2 * vec < dim) lanes *= 2;
  return lanes;
}

// raises a kernel's shared-memory limit once per device
template <typename K> static cudaError_t norm_allow(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev > 63 || !(done.load(std::memory_order_relaxed) >> dev & 1))) {
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev <= 63) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return e;
}
template <typename T, int V, int L, bool INTER, bool BACKWARD> static cudaError_t norm_launch(const NormArgs& p, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = norm_allow(head_norm_kernel<T, V, L, INTER, BACKWARD>, kNormSmem<BACKWARD>, done);
  if (e != cudaSuccess) return e;
  return launch_pdl(head_norm_kernel<T, V, L, INTER, BACKWARD>, dim3(p.blocks[0] + p.blocks[1]), dim3(kNormThreads), kNormSmem<BACKWARD>, st, false, p);
}
template <typename T, int V, int L> static cudaError_t norm_vec(const NormArgs& p, bool interleaved, bool backward, cudaStream_t st) {
  if (interleaved) return backward ? norm_launch<T, V, L, true, true>(p, st) : norm_launch<T, V, L, true, false>(p, st);
  return backward ? norm_launch<T, V, L, false, true>(p, st) : norm_launch<T, V, L, false, false>(p, st);
}
template <typename T, int V> static cudaError_t norm_width(const NormArgs& p, int lanes, bool interleaved, bool backward, cudaStream_t st) {
  switch (lanes) {
    case 1: return norm_vec<T, V, 1>(p, interleaved, backward, st);
    case 2: return norm_vec<T, V, 2>(p, interleaved, backward, st);
    case 4: return norm_vec<T, V, 4>(p, interleaved, backward, st);
    case 8: return norm_vec<T, V, 8>(p, interleaved, backward, st);
    default: break;
  }
  if constexpr (V == 4) return norm_vec<T, V, 16>(p, interleaved, backward, st);
  return cudaErrorInvalidValue;
}

template <typename T> static cudaError_t norm_run(NormArgs& p, bool interleaved, bool backward, float* d_gain_q, float* d_gain_k, cudaStream_t st) {
  // the longest vectors that divide rows, their rotated part and strides
  auto divides = [&](int v) {
    bool all = p.dim % (2 * v) == 0 && p.rotary % (2 * v) == 0;
    auto whole = [&](const HeadView& x) { all = all && aligned_to(x.data, v * (int)sizeof(T)) && x.token % v == 0 && x.head % v == 0; };
    for (const NormSide& s : p.side)
      if (s.heads) {
        whole(s.x);
        whole(s.y);
        if (backward) whole(s.dx);
      }
    return all;
  };
  const int vec = divides(kVec<T>) ? kVec<T> : divides(4) ? 4 : 1;
  const int lanes = vec > 1 ? norm_lanes(p.dim, vec) : 32;
  // the blocks that run at a time go to the sides by their work: heads, and a token's angles, which take about as long as two rows.  By heads alone
  // the smaller side's blocks are the last by far, one to four rows are alike (12291 tokens, us forward / backward with none, one, two, four, bf16: 16 + 2
  // heads of 128 25 / 38, 22 / 33, 22 / 33, 23 / 33; 40 + 1 of 64 35 / 51, 26 / 38, 26 / 38, 26 / 38; 32 + 8 of 128 52 / 73, 51 / 72, 51 / 72, 50 / 71; fp32, 8 + 1 of
  // 128, 64 rotated, 23 / 36, 18 / 31, 18 / 31, 19 / 31)
  auto weight = [&](int n) { return n ? n + (p.rotary ? 2 : 0) : 0; };
  const int64_t per_block = kNormThreads / lanes;
  for (int i = 0; i < 2; ++i) {
    const int n = p.side[i].heads;
    if (!n) continue;
    const int64_t rows = (p.tokens + 32 / lanes - 1) / (32 / lanes) * (32 / lanes) * n;
    p.blocks[i] = (int)std::min<int64_t>((rows + per_block - 1) / per_block, std::max(1, (int)((int64_t)(backward ? kNormBlocks<true> : kNormBlocks<false>) * weight(n) / (weight(p.side[0].heads) + weight(p.side[1].heads)))));
  }
  cudaError_t e;
  if (vec == kVec<T>) {
    e = norm_width<T, kVec<T>>(p, lanes, interleaved, backward, st);
  } else if (vec == 4) {
    e = norm_width<T, 4>(p, lanes, interleaved, backward, st);
  } else {
    const dim3 grid(p.blocks[0] + p.blocks[1]);
    e = backward ? launch_pdl(head_norm_any_kernel<T, true>, grid, dim3(kNormThreads), 0, st, false, p, (int)interleaved)
                 : launch_pdl(head_norm_any_kernel<T, false>, grid, dim3(kNormThreads), 0, st, false, p, (int)interleaved);
  }
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
  return !d || d->head_dim < 1 || d->head_dim > 128 ? 0 : (uint64_t)(kNormBlocks<true> + 1) * d->head_dim * sizeof(float);
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
