// Log probabilities of given tokens, the distribution's entropy and its most likely alternatives, and their gradient.
//
//   lse = m + log sum e^(x - m),   logprob = x_y - lse,   H = log sum e^(x - m) - sum (x - m) e^(x - m) / sum e^(x - m)
//   dx_j = g_l ([j = y] - p_j) - g_H p_j (log p_j + H),   p_j = e^(x_j - lse)
//
// Forward: one pass over the logits.  A thread keeps the running maximum of its elements and the two sums relative to it; the
// threads' triples are joined at the end.  A row belongs to a cluster of 1, 2, 4 or 8 blocks that join through distributed shared
// memory, so that a few long rows still occupy the GPU and nothing needs a workspace.  Bound by memory (one read).
//
// The alternatives cost one comparison per element, the maximum that the softmax needs anyway: the k-th largest of 32 maxima
// over disjoint parts of the segment is a value that at least k elements reach, so only threads whose own maximum reaches it read
// their elements again (from L2) and list those that do; the list, a few dozen entries, is ranked by counting.  Rows with so many
// equal values that the list overflows take k passes over the segment instead.
#include <cfloat>

#include <cooperative_groups.h>

#include "pm_ops.cuh"

namespace pm {
namespace cg = cooperative_groups;

constexpr int kLpThreads = 256;
constexpr int kLpWarps = kLpThreads / 32;
constexpr int kLpMaxK = 32;
// Candidates of a block or warp.  Of independent logits 32 (1/32 + 1/31 + ... + 1/(33 - k)) reach the threshold on average: 9 for k = 8,
// 31 for 20, 130 for 32, there with a spread of 39; more than n with the chance that 33 - k of 32 parts have a maximum of e^(-n/32) of the
// elements.  512 are too few in 4 rows of a million at k = 32.
constexpr int kLpList = 512;
constexpr int kLpMaxCluster = 8;

struct LogprobArgs {
  const void* logits;
  int64_t rows, row_stride;
  int vocab, top_k;
  const int32_t* targets;
  float *logprob, *entropy, *lse, *top_logprob;
  int32_t* top_ids;
};

template <typename T> struct Vec { static constexpr int n = 16 / sizeof(T); };

__device__ __forceinline__ void unpack16(const uint4& q, float (&v)[4]) {
  v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack16(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}

// A row as 16-byte vectors at 16-byte boundaries: vector j holds elements j * n - shift ...; the first and the last may reach over the
// row's ends, where they are put together from single elements (-infinity outside).
template <typename T> struct RowVectors {
  const T* row;
  int vocab, shift, count;
  __device__ __forceinline__ RowVectors(const T* r, int v) : row(r), vocab(v) {
    shift = (int)((reinterpret_cast<uintptr_t>(r) & 15) / sizeof(T));
    count = (v + shift + Vec<T>::n - 1) / Vec<T>::n;
  }
  __device__ __forceinline__ int first(int j) const { return j * Vec<T>::n - shift; }
  __device__ __forceinline__ bool whole(int j) const { return first(j) >= 0 && first(j) + Vec<T>::n <= vocab; }
  __device__ __forceinline__ uint4 load(int j) const { return *reinterpret_cast<const uint4*>(row + first(j)); }
  __device__ __forceinline__ void get(int j, float (&v)[Vec<T>::n]) const {
    if (whole(j)) { unpack16(load(j), v); return; }
#pragma unroll
    for (int i = 0; i < Vec<T>::n; ++i) { const int at = first(j) + i; v[i] = at >= 0 && at < vocab ? to_f<T>(row[at]) : -INFINITY; }
  }
};

struct Sums { float m, s, t; };
// the sums relative to another maximum (never below the own one); a maximum of -infinity has empty sums
__device__ __forceinline__ void rebase(Sums& a, float m) {
  if (a.m == m || a.m == -INFINITY) { a.m = m; return; }
  const float d = fmaxf(a.m - m, -200.f), f = ex2(d * kLog2e);
  a.t = f * (a.t + d * a.s);                      // sum (x - m') e^(x - m') from sum (x - m) e^(x - m)
  a.s *= f;
  a.m = m;
}
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = max_nan(a.m, b.m);
  rebase(a, m); rebase(b, m);
  return Sums{m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ bool beats(float v, int id, float w, int other) { return v > w || (v == w && id < other); }

template <int THREADS> struct LpShared {
  Sums warp[THREADS / 32];
  Sums block[kLpMaxCluster];                      // of the cluster's blocks, in its first
  float lane_max[THREADS / 32][32];
  uint8_t hit[THREADS / 32][32];
  float threshold;
  int n_list;
  float list_v[kLpList];
  int list_id[kLpList];
  float top_v[kLpMaxK];                           // this block's best, in order
  int top_id[kLpMaxK];
  float all_v[kLpMaxCluster * kLpMaxK];           // the blocks' best, in the cluster's first
  int all_id[kLpMaxCluster * kLpMaxK];
};

// bitonic sort over the lanes, descending
__device__ __forceinline__ float sorted_down(float v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int size = 2; size <= 32; size *= 2)
#pragma unroll
    for (int step = size / 2; step > 0; step /= 2) {
      const float o = __shfl_xor_sync(0xffffffffu, v, step);
      v = ((lane & size) == 0) == ((lane & step) == 0) ? fmaxf(v, o) : fminf(v, o);
    }
  return v;
}
// the best of vector j's elements that come after (last_v, last_id), and of (bv, bid)
template <typename T> __device__ __forceinline__ void best_after(const RowVectors<T>& x, int j, float last_v, int last_id, float& bv, int& bid) {
  float v[Vec<T>::n];
  x.get(j, v);
#pragma unroll
  for (int i = 0; i < Vec<T>::n; ++i) {
    const int id = x.first(j) + i;
    if (id >= 0 && id < x.vocab && beats(last_v, last_id, v[i], id) && beats(v[i], id, bv, bid)) { bv = v[i]; bid = id; }
  }
}
__device__ __forceinline__ void warp_best(float& bv, int& bid) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float ov = __shfl_xor_sync(0xffffffffu, bv, o);
    const int oid = __shfl_xor_sync(0xffffffffu, bid, o);
    if (beats(ov, oid, bv, bid)) { bv = ov; bid = oid; }
  }
}

// What a row's sums say.
struct RowResult {
  float m, log_s, entropy;
  bool none, empty;                               // a NaN or +infinity in the row: no distribution; nothing but -infinity
  __device__ __forceinline__ explicit RowResult(const Sums& st)
      : m(st.m), log_s(logf(st.s)), entropy(log_s - st.t / st.s), none(!(st.m < INFINITY)), empty(st.m == -INFINITY) {}
  __device__ __forceinline__ float log_p(float v) const { return none ? NAN : empty ? -INFINITY : (v - m) - log_s; }
  template <typename T> __device__ __forceinline__ void write(const LogprobArgs& a, const RowVectors<T>& x, int64_t row) const {
    if (a.lse) a.lse[row] = none ? NAN : empty ? -INFINITY : m + log_s;
    if (a.entropy) a.entropy[row] = none ? NAN : empty ? 0.f : entropy;
    if (a.targets) {
      const int y = a.targets[row];
      a.logprob[row] = y >= a.vocab ? NAN : y < 0 ? 0.f : log_p(to_f<T>(x.row[y]));
    }
  }
  __device__ __forceinline__ void write_top(const LogprobArgs& a, int64_t row, int rank, float v, int id) const {
    a.top_logprob[row * a.top_k + rank] = log_p(v);
    a.top_ids[row * a.top_k + rank] = none ? -1 : id;
  }
};

__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// The k best of the block's vectors [j0, j1) in order into sh.top_*: value descending, then index ascending.  `mine` is the largest
// value of the thread's own vectors j0 + threadIdx.x, + THREADS, ...  Missing entries are (-infinity, vocab).
template <int THREADS, typename T> __device__ void block_top(LpShared<THREADS>& sh, const RowVectors<T>& x, int j0, int j1, int k, float mine) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  sh.lane_max[warp][lane] = mine;
  if (tid == 0) sh.n_list = 0;
  if (tid < kLpMaxK) { sh.top_v[tid] = -INFINITY; sh.top_id[tid] = x.vocab; }
  __syncthreads();
  if (warp == 0) {
    float v = sh.lane_max[0][lane];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) v = fmaxf(v, sh.lane_max[w][lane]);
    const float th = __shfl_sync(0xffffffffu, sorted_down(v), k - 1);
    if (lane == 0) sh.threshold = th;
  }
  __syncthreads();
  const float th = sh.threshold;
  // the vectors of the threads that reach the threshold, read again by their whole warp: (thread, vector) pairs over the lanes
  const unsigned hits = __ballot_sync(0xffffffffu, mine >= th);
  if (mine >= th) sh.hit[warp][__popc(hits & ((1u << lane) - 1))] = (uint8_t)lane;
  __syncwarp();
  const int each = (j1 - j0 + THREADS - 1) / THREADS;
  for (int p = lane; p < __popc(hits) * each; p += 32) {
    const int j = j0 + warp * 32 + sh.hit[warp][p / each] + p % each * THREADS;
    if (j >= j1) continue;
    float v[Vec<T>::n];
    x.get(j, v);
#pragma unroll
    for (int i = 0; i < Vec<T>::n; ++i) {
      const int id = x.first(j) + i;
      if (v[i] >= th && id >= 0 && id < x.vocab) {
        const int at = atomicAdd(&sh.n_list, 1);
        if (at < kLpList) { sh.list_v[at] = v[i]; sh.list_id[at] = id; }
      }
    }
  }
  __syncthreads();
  const int n = sh.n_list;
  if (n <= kLpList) {
    for (int a = tid; a < n; a += THREADS) {
      const float v = sh.list_v[a];
      const int id = sh.list_id[a];
      int rank = 0;
      for (int b = 0; b < n; ++b) rank += beats(sh.list_v[b], sh.list_id[b], v, id);
      if (rank < k) { sh.top_v[rank] = v; sh.top_id[rank] = id; }
    }
    __syncthreads();
    return;
  }
  float last_v = INFINITY;
  int last_id = -1;
  for (int r = 0; r < k; ++r) {                    // the best of what comes after the last one found
    float bv = -INFINITY;
    int bid = x.vocab;
    for (int j = j0 + tid; j < j1; j += THREADS) best_after(x, j, last_v, last_id, bv, bid);
    warp_best(bv, bid);
    if (lane == 0) { sh.list_v[warp] = bv; sh.list_id[warp] = bid; }
    __syncthreads();
    bv = sh.list_v[0]; bid = sh.list_id[0];
    for (int w = 1; w < THREADS / 32; ++w) if (beats(sh.list_v[w], sh.list_id[w], bv, bid)) { bv = sh.list_v[w]; bid = sh.list_id[w]; }
    if (tid == 0) { sh.top_v[r] = bv; sh.top_id[r] = bid; }
    last_v = bv; last_id = bid;
    __syncthreads();
  }
}

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// the largest value of 16 bytes of logits and what came before
__device__ __forceinline__ float max_of(const uint4& q, float m, float) {
  return max_nan(max_nan(m, max_nan(__uint_as_float(q.x), __uint_as_float(q.y))), max_nan(__uint_as_float(q.z), __uint_as_float(q.w)));
}
__device__ __forceinline__ float max_of(const uint4& q, float m, __nv_bfloat16) {
  const uint32_t r = max_nan_bf16x2(max_nan_bf16x2(q.x, q.y), max_nan_bf16x2(q.z, q.w));
  return max_nan(m, max_nan(__uint_as_float(r << 16), __uint_as_float(r & 0xFFFF0000u)));
}

// Sums of a thread's vectors.  ENTROPY: with the sum that it needs, and a floor under x - m: at -200 the exponential is zero and its
// product with the difference too, at -infinity the product would not be.
template <typename T, bool ENTROPY, int U> __device__ __forceinline__ void take(Sums& st, const uint4 (&q)[U]) {
  constexpr int N = Vec<T>::n;
  float m = st.m;
#pragma unroll
  for (int u = 0; u < U; ++u) m = max_of(q[u], m, T());
  if (m != st.m) rebase(st, m);
  const float base = m == -INFINITY ? 0.f : m;
  float2 s = make_float2(0.f, 0.f), t = make_float2(0.f, 0.f);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float v[N];
    unpack16(q[u], v);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float2 d = add2(make_float2(v[i], v[i + 1]), make_float2(-base, -base));
      if (ENTROPY) d = make_float2(fmaxf(d.x, -200.f), fmaxf(d.y, -200.f));
      const float2 x = fma2(d, make_float2(kLog2e, kLog2e), make_float2(0.f, 0.f));
      const float2 e = make_float2(ex2(x.x), ex2(x.y));
      s = add2(s, e);
      if (ENTROPY) t = fma2(e, d, t);
    }
  }
  st.s += s.x + s.y;
  if (ENTROPY) st.t += t.x + t.y;
}

// 1536 threads to an SM, in six blocks or twelve: the end of a row (joining the sums, ranking the alternatives) is a chain of short steps that
// the other blocks' loads run beside.
template <typename T, int THREADS, bool TOP, bool ENTROPY>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) logprob_kernel(LogprobArgs a) {
  __shared__ LpShared<THREADS> sh;
  constexpr int U = 4;
  cg::cluster_group cluster = cg::this_cluster();
  const int parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int64_t row = blockIdx.x / parts;
  const int tid = threadIdx.x, lane = tid & 31;
  if (parts > 1) cluster_arrive_relaxed();        // this block has begun: the others may write to its shared memory
  const RowVectors<T> x(static_cast<const T*>(a.logits) + row * a.row_stride, a.vocab);
  const int j0 = (int)((int64_t)x.count * part / parts), j1 = (int)((int64_t)x.count * (part + 1) / parts);

  Sums st{-INFINITY, 0.f, 0.f};
  const uint32_t none2 = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;   // -infinity, or two of them
  for (int j = j0 + tid; j < j1; j += U * THREADS) {
    uint4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = j + u * THREADS;
      q[u] = at < j1 && x.whole(at) ? x.load(at) : make_uint4(none2, none2, none2, none2);
    }
    take<T, ENTROPY>(st, q);
  }
  // the vectors that reach over the row's ends, by the threads whose turn they are
  for (int e = 0; e < 2; ++e) {
    const int j = e ? x.count - 1 : 0;
    if (j < j0 || j >= j1 || (j - j0) % THREADS != tid || x.whole(j) || (e && x.count == 1)) continue;
    float v[Vec<T>::n];
    x.get(j, v);
#pragma unroll
    for (int i = 0; i < Vec<T>::n; ++i) {
      const Sums one{v[i], v[i] == -INFINITY ? 0.f : 1.f, 0.f};
      st = join(st, one);
    }
  }
  const float mine = st.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o)};
    st = lane & o ? join(b, st) : join(st, b);
  }
  if (lane == 0) sh.warp[tid >> 5] = st;
  __syncthreads();
  if (TOP) block_top(sh, x, j0, j1, a.top_k, mine);
  if (parts > 1) {
    cluster_wait();                               // all blocks have begun
    if (tid == 0) {
      st = sh.warp[0];
      for (int w = 1; w < THREADS / 32; ++w) st = join(st, sh.warp[w]);
      *cluster.map_shared_rank(&sh.block[part], 0) = st;
    }
    if (TOP && tid < a.top_k) {
      cluster.map_shared_rank(sh.all_v, 0)[part * a.top_k + tid] = sh.top_v[tid];
      cluster.map_shared_rank(sh.all_id, 0)[part * a.top_k + tid] = sh.top_id[tid];
    }
    cluster_arrive();
    cluster_wait();
    if (part != 0) return;
    st = sh.block[0];
    for (int c = 1; c < parts; ++c) st = join(st, sh.block[c]);
  } else {
    st = sh.warp[0];
    for (int w = 1; w < THREADS / 32; ++w) st = join(st, sh.warp[w]);
  }
  const RowResult r(st);
  if (tid == 0) r.write<T>(a, x, row);
  if (TOP) {
    const int k = a.top_k, n = parts * k;
    const float* bv = parts > 1 ? sh.all_v : sh.top_v;
    const int* bid = parts > 1 ? sh.all_id : sh.top_id;
    for (int i = tid; i < n; i += THREADS) {
      int rank = i;
      if (parts > 1) {
        // entries of blocks with fewer than k elements are equal among themselves and come behind every element
        rank = 0;
        for (int b = 0; b < n; ++b) rank += beats(bv[b], bid[b], bv[i], bid[i]);
      }
      if (rank < k && bid[i] < a.vocab) r.write_top(a, row, rank, bv[i], bid[i]);
    }
    if (r.none && tid < k) r.write_top(a, row, tid, 0.f, 0);
  }
}

// Short rows: a warp to each, nothing shared between warps; for rows of up to 4 KB, and of up to 16 KB where there are many.  us with a warp / a
// block to a row, fp32, five alternatives: 16 x 200 4.4 / 6.3, 300 x 1000 6.3 / 6.3, 1200 x 2000 8.5 / 10.4, 2400 x 4000 15.6 / 18.6; but 40 x 3000 9.2 / 6.4 and 1345 x 8191 30.9 / 27.3.
constexpr int kLpShortBytes = 4096, kLpMidBytes = 16384, kLpMidRows = 1024;
// Candidates of a warp: 160 are too few in 3 rows of a million at k = 28, but in 18 of a hundred at k = 32, and the launch waits for such a row's
// k passes: 2400 x 4000 fp32, k = 32, 350 us with 160, 90 with 512.  Longer lists leave less of L1 to the rows: k = 20, 37 with 512, 33 with 160.
constexpr int kLpShortList = 160, kLpShortK = 28;
__host__ __device__ constexpr int lp_short_list(int k) { return k <= kLpShortK ? kLpShortList : kLpList; }
__host__ __device__ constexpr int lp_short_bytes(int list) { return list * 8 + 32; }       // of a warp

template <typename T, bool TOP, bool ENTROPY>
__global__ void __launch_bounds__(kLpThreads) logprob_short_kernel(LogprobArgs a) {
  extern __shared__ float lp_lists[];             // of each warp: the candidates' values, their ids, and the lanes that reach the threshold
  constexpr int U = 4, N = Vec<T>::n;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * kLpWarps + warp;
  if (row >= a.rows) return;
  const RowVectors<T> x(static_cast<const T*>(a.logits) + row * a.row_stride, a.vocab);
  Sums st{-INFINITY, 0.f, 0.f};
  const uint32_t none2 = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;   // -infinity, or two of them
  for (int j = lane; j < x.count; j += U * 32) {
    uint4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = j + u * 32;
      q[u] = at < x.count && x.whole(at) ? x.load(at) : make_uint4(none2, none2, none2, none2);
    }
    take<T, ENTROPY>(st, q);
  }
  for (int e = 0; e < 2; ++e) {                   // the vectors that reach over the row's ends
    const int j = e ? x.count - 1 : 0;
    if (j % 32 != lane || x.whole(j) || (e && x.count == 1)) continue;
    float v[N];
    x.get(j, v);
#pragma unroll
    for (int i = 0; i < N; ++i) st = join(st, Sums{v[i], v[i] == -INFINITY ? 0.f : 1.f, 0.f});
  }
  const float mine = st.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Sums b{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), __shfl_xor_sync(0xffffffffu, st.t, o)};
    st = lane & o ? join(b, st) : join(st, b);
  }
  const RowResult r(st);
  if (lane == 0) r.write<T>(a, x, row);
  if constexpr (TOP) {
    const int k = a.top_k;
    if (r.none) {
      if (lane < k) r.write_top(a, row, lane, 0.f, 0);
      return;
    }
    const int list = lp_short_list(k);
    float* const list_v = lp_lists + warp * (lp_short_bytes(list) / 4);
    int* const list_id = reinterpret_cast<int*>(list_v + list);
    uint8_t* const hit = reinterpret_cast<uint8_t*>(list_id + list);
    const float th = __shfl_sync(0xffffffffu, sorted_down(mine), k - 1);
    const unsigned hits = __ballot_sync(0xffffffffu, mine >= th);
    if (mine >= th) hit[__popc(hits & ((1u << lane) - 1))] = (uint8_t)lane;
    __syncwarp();
    const int each = (x.count + 31) / 32, pairs = __popc(hits) * each;
    int n = 0;
    for (int base = 0; base < pairs; base += 32) {   // the vectors of the lanes that reach the threshold: (lane, vector) pairs over the lanes
      const int p = base + lane, at = p < pairs ? hit[p / each] + p % each * 32 : x.count;
      float v[N];
      if (at < x.count) x.get(at, v);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int id = x.first(at) + i;
        const bool in = at < x.count && id >= 0 && id < x.vocab && v[i] >= th;
        const unsigned all = __ballot_sync(0xffffffffu, in);
        const int to = n + __popc(all & ((1u << lane) - 1));
        if (in && to < list) { list_v[to] = v[i]; list_id[to] = id; }
        n += __popc(all);
      }
    }
    __syncwarp();
    if (n <= list) {
      for (int i = lane; i < n; i += 32) {
        const float v = list_v[i];
        const int id = list_id[i];
        int rank = 0;
        for (int b = 0; b < n; ++b) rank += beats(list_v[b], list_id[b], v, id);
        if (rank < k) r.write_top(a, row, rank, v, id);
      }
      return;
    }
    float last_v = INFINITY;
    int last_id = -1;
    for (int rank = 0; rank < k; ++rank) {        // the best of what comes after the last one found
      float bv = -INFINITY;
      int bid = x.vocab;
      for (int j = lane; j < x.count; j += 32) best_after(x, j, last_v, last_id, bv, bid);
      warp_best(bv, bid);
      if (lane == 0) r.write_top(a, row, rank, bv, bid);
      last_v = bv; last_id = bid;
    }
  }
}

struct LogprobBwdArgs {
  const void* logits;
  int64_t row_stride, grad_stride;
  int vocab, per_row;                             // blocks per row
  const int32_t* targets;
  const float *lse, *entropy, *d_logprob, *d_entropy;
  void* d_logits;
};

constexpr int kLbVectors = 4;                     // 16-byte vectors per thread

// An lse beyond this magnitude no longer resolves log p (its rounding alone reaches 2^-12 there), as in a row whose every logit is a
// mask's lowest value.  Such a row is left to one block, which takes the maximum and the sum from the logits again.  Below, p is off by up to
// 2^-24 |lse| of itself: 6e-7 at an lse of 10, 1.2e-4 just below the limit.
constexpr float kLseCoarse = 4096.f;

__device__ __forceinline__ float logit_grad(float lp, float gl, float gh, float h) {
  lp = max_nan(lp, -200.f);                       // where p underflows the product below is zero
  return -ex2(lp * kLog2e) * fmaf(gh, lp + h, gl);
}

template <typename T> __device__ __noinline__ void coarse_row(const T* in, T* out, int vocab, int y, float gl, float gh, float h) {
  __shared__ Sums warp_sums[kLpWarps];
  Sums st{-INFINITY, 0.f, 0.f};
  for (int i = threadIdx.x; i < vocab; i += kLpThreads) {
    const float v = to_f<T>(in[i]);
    st = join(st, Sums{v, v == -INFINITY ? 0.f : 1.f, 0.f});
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Sums b{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), 0.f};
    st = threadIdx.x & o ? join(b, st) : join(st, b);
  }
  if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = st;
  __syncthreads();
  st = warp_sums[0];
  for (int w = 1; w < kLpWarps; ++w) st = join(st, warp_sums[w]);
  const float log_s = logf(st.s);
  for (int i = threadIdx.x; i < vocab; i += kLpThreads)
    out[i] = from_f<T>(logit_grad((to_f<T>(in[i]) - st.m) - log_s, gl, gh, h) + (i == y ? gl : 0.f));
}

// One read, one write: dx_j = -p_j (g_l + g_H (log p_j + H)), plus g_l at the target.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kLpThreads) logprob_bwd_kernel(LogprobBwdArgs a) {
  constexpr int N = Vec<T>::n;
  const int64_t row = blockIdx.x / a.per_row;
  const int part = (int)(blockIdx.x - row * a.per_row);
  const T* in = static_cast<const T*>(a.logits) + row * a.row_stride;
  T* out = static_cast<T*>(a.d_logits) + row * a.grad_stride;
  const float lse = a.lse[row];
  const int y = a.targets ? a.targets[row] : -1;
  float gl = a.d_logprob && y >= 0 ? a.d_logprob[row] : 0.f;
  if (a.d_logprob && y >= a.vocab) gl = NAN;
  const float gh = a.d_entropy ? a.d_entropy[row] : 0.f, h = a.d_entropy ? a.entropy[row] : 0.f;
  const bool empty = lse == -INFINITY;
  if (fabsf(lse) > kLseCoarse && !empty) {
    if (part == 0) coarse_row(in, out, a.vocab, y, gl, gh, h);
    return;
  }
  auto grad = [&](float v, int at) { return empty ? 0.f : logit_grad(v - lse, gl, gh, h) + (at == y ? gl : 0.f); };
  if (VEC) {
    const RowVectors<T> x(in, a.vocab);
    const int j0 = part * kLbVectors * kLpThreads + threadIdx.x;
    uint4 q[kLbVectors];
#pragma unroll
    for (int u = 0; u < kLbVectors; ++u) {
      const int j = j0 + u * kLpThreads;
      if (j < x.count && x.whole(j)) q[u] = x.load(j);
    }
#pragma unroll
    for (int u = 0; u < kLbVectors; ++u) {
      const int j = j0 + u * kLpThreads;
      if (j >= x.count) break;
      const int at = x.first(j);
      if (x.whole(j)) {
        float v[N];
        unpack16(q[u], v);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = grad(v[i], at + i);
        uint4 w;
        if constexpr (N == 4) {
          w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        } else {
          uint32_t p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            p[i] = *reinterpret_cast<const uint32_t*>(&b);
          }
          w = make_uint4(p[0], p[1], p[2], p[3]);
        }
        *reinterpret_cast<uint4*>(out + at) = w;
      } else {
        for (int i = 0; i < N; ++i)
          if (at + i >= 0 && at + i < a.vocab) out[at + i] = from_f<T>(grad(to_f<T>(in[at + i]), at + i));
      }
    }
  } else {
    const int e1 = min(a.vocab, (part + 1) * kLbVectors * kLpThreads * N);
    for (int i = part * kLbVectors * kLpThreads * N + threadIdx.x; i < e1; i += kLpThreads) out[i] = from_f<T>(grad(to_f<T>(in[i]), i));
  }
}

template <typename T, int THREADS> static cudaError_t logprob_launch_rows(const LogprobArgs& a, int parts, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.rows * parts)); cfg.blockDim = dim3(THREADS); cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = parts; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  void (*kernel)(LogprobArgs) = a.top_k ? (a.entropy ? logprob_kernel<T, THREADS, true, true> : logprob_kernel<T, THREADS, true, false>)
                                        : (a.entropy ? logprob_kernel<T, THREADS, false, true> : logprob_kernel<T, THREADS, false, false>);
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T> static cudaError_t logprob_launch(const LogprobArgs& a, int parts, cudaStream_t st) {
  const int bytes = a.vocab * (int)sizeof(T);
  if (bytes <= kLpShortBytes || (bytes <= kLpMidBytes && a.rows >= kLpMidRows)) {
    void (*kernel)(LogprobArgs) = a.top_k ? (a.entropy ? logprob_short_kernel<T, true, true> : logprob_short_kernel<T, true, false>)
                                          : (a.entropy ? logprob_short_kernel<T, false, true> : logprob_short_kernel<T, false, false>);
    const int smem = a.top_k ? kLpWarps * lp_short_bytes(lp_short_list(a.top_k)) : 0;
    return launch_pdl(kernel, dim3((unsigned)((a.rows + kLpWarps - 1) / kLpWarps)), dim3(kLpThreads), smem, st, false, a);
  }
  // Rows of up to 64 KB take 128 threads.  us with 128 / 256: 1345 x 8191 fp32, both passes, 27 / 29; 4096 x 32000 bf16 with eight
  // alternatives 76 / 78; but the same in fp32, rows of 128 KB, 121 / 103.
  return bytes <= 65536 ? logprob_launch_rows<T, 128>(a, parts, st) : logprob_launch_rows<T, 256>(a, parts, st);
}

static pm_status logprob_shape(int32_t dtype, int64_t rows, int32_t vocab, int64_t row_stride, const void* logits) {
  if (dtype != PM_F32 && dtype != PM_BF16) return ops_fail(PM_ERR_INVALID_ARG, "unknown element type");
  if (rows < 0 || vocab < 1) return ops_fail(PM_ERR_INVALID_ARG, "rows must be >= 0 and vocab positive");
  if (rows > (1 << 24) || vocab > (1 << 24)) return ops_fail(PM_ERR_SHAPE, "at most 2^24 rows and 2^24 tokens of vocabulary");
  if (row_stride < vocab) return ops_fail(PM_ERR_INVALID_ARG, "row stride below the vocabulary size");
  if (!aligned_to(logits, dtype == PM_BF16 ? 2 : 4)) return ops_fail(PM_ERR_INVALID_ARG, "pointer not aligned to its element type");
  return PM_OK;
}

}  // namespace pm

using namespace pm;

extern "C" {

pm_status pm_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int32_t vocab, int64_t row_stride, const int32_t* targets,
                            float* logprob, float* entropy, float* lse, int32_t top_k, float* top_logprob, int32_t* top_ids, void* stream) {
  if (const pm_status s = logprob_shape(dtype, rows, vocab, row_stride, logits)) return s;
  if (rows == 0) return PM_OK;
  if (!logits) return ops_fail(PM_ERR_INVALID_ARG, "null logits");
  if ((targets == nullptr) != (logprob == nullptr)) return ops_fail(PM_ERR_INVALID_ARG, "targets and logprob are given together or not at all");
  if (top_k < 0 || top_k > kLpMaxK || top_k > vocab) return ops_fail(PM_ERR_INVALID_ARG, "top_k must be 0 to 32 and at most the vocabulary size");
  if (top_k > 0 && (!top_logprob || !top_ids)) return ops_fail(PM_ERR_INVALID_ARG, "top_k without a place for the alternatives");
  const Extent outs[] = {dense_extent(logprob, 4 * rows), dense_extent(entropy, 4 * rows), dense_extent(lse, 4 * rows),
                         dense_extent(top_k > 0 ? top_logprob : nullptr, 4 * rows * top_k), dense_extent(top_k > 0 ? top_ids : nullptr, 4 * rows * top_k)};
  const Extent ins[] = {rows_extent(logits, rows, row_stride, vocab, dtype == PM_BF16 ? 2 : 4), dense_extent(targets, 4 * rows)};
  for (int i = 0; i < 5; ++i) {
    for (int j = 0; j < i; ++j) if (extents_share(outs[i], outs[j])) return ops_fail(PM_ERR_INVALID_ARG, "two results share their memory");
    for (const Extent& x : ins) if (extents_share(outs[i], x)) return ops_fail(PM_ERR_INVALID_ARG, "a result overlaps the logits or the targets");
  }
  // A cluster per row once the rows leave SMs without work, as long as each block keeps some vectors per thread.
  const int vectors = vocab / (dtype == PM_BF16 ? 8 : 4);
  int parts = 1;
  while (parts < kLpMaxCluster && rows * parts * 2 <= 2 * kSms && vectors / (parts * 2) >= 2 * kLpThreads) parts *= 2;
  const LogprobArgs a{logits, rows, row_stride, vocab, top_k, targets, logprob, entropy, lse, top_logprob, top_ids};
  const cudaError_t e = dtype == PM_BF16 ? logprob_launch<__nv_bfloat16>(a, parts, (cudaStream_t)stream) : logprob_launch<float>(a, parts, (cudaStream_t)stream);
  return ops_cuda(e, "token log probabilities");
}

pm_status pm_token_logprobs_backward(const void* logits, int32_t dtype, int64_t rows, int32_t vocab, int64_t row_stride, const int32_t* targets,
                                     const float* lse, const float* entropy, const float* d_logprob, const float* d_entropy, void* d_logits,
                                     int64_t grad_stride, void* stream) {
  if (const pm_status s = logprob_shape(dtype, rows, vocab, row_stride, logits)) return s;
  if (const pm_status s = logprob_shape(dtype, rows, vocab, grad_stride, d_logits)) return s;
  if (!d_logprob && !d_entropy) return ops_fail(PM_ERR_INVALID_ARG, "neither a gradient of logprob nor one of the entropy");
  if (rows == 0) return PM_OK;
  if (!logits || !lse || !d_logits) return ops_fail(PM_ERR_INVALID_ARG, "null argument");
  if (d_logprob && !targets) return ops_fail(PM_ERR_INVALID_ARG, "a gradient of logprob needs the targets");
  if (d_entropy && !entropy) return ops_fail(PM_ERR_INVALID_ARG, "a gradient of the entropy needs the entropy");
  const int size = dtype == PM_BF16 ? 2 : 4, per_block = kLbVectors * kLpThreads * 16 / size;
  const Extent out = rows_extent(d_logits, rows, grad_stride, vocab, size);
  const void* const per_row_inputs[] = {d_logprob ? targets : nullptr, lse, d_entropy ? entropy : nullptr, d_logprob, d_entropy};
  for (const void* p : per_row_inputs) if (extents_share(out, dense_extent(p, 4 * rows))) return ops_fail(PM_ERR_INVALID_ARG, "d_logits overlaps another input");
  if ((d_logits != logits || (rows > 1 && grad_stride != row_stride)) && extents_share(out, rows_extent(logits, rows, row_stride, vocab, size)))
    return ops_fail(PM_ERR_INVALID_ARG, "d_logits overlaps the logits without being them");
  // both rows at the same place within their 16-byte blocks, in every row: vectors; else single elements
  const bool vec = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(d_logits)) & 15) == 0 &&
                   ((row_stride - grad_stride) * size) % 16 == 0;
  const int per_row = (vocab + 16 / size - 1 + per_block - 1) / per_block;
  const LogprobBwdArgs a{logits, row_stride, grad_stride, vocab, per_row, d_logprob ? targets : nullptr, lse, entropy, d_logprob, d_entropy, d_logits};
  const dim3 grid((unsigned)(rows * per_row)), block(kLpThreads);
  if ((int64_t)rows * per_row > 0x7fffffff) return ops_fail(PM_ERR_SHAPE, "more than 2^31 blocks");
  void (*kernel)(LogprobBwdArgs) = dtype == PM_BF16 ? (vec ? logprob_bwd_kernel<__nv_bfloat16, true> : logprob_bwd_kernel<__nv_bfloat16, false>)
                                                    : (vec ? logprob_bwd_kernel<float, true> : logprob_bwd_kernel<float, false>);
  return ops_cuda(launch_pdl(kernel, grid, block, 0, (cudaStream_t)stream, false, a), "gradient of the log probabilities");
}

}  // extern "C"
