// Cross attention of few query rows: a decoding step, with a token or the few of a beam to each sequence.  bf16.
//
// Bound by memory: every key and value is read once and meets at most 16 query rows (tokens times the heads that share it), far too few
// for a 128-row tile of the large tensor-core products, whose chain of waits would set the pace.  Here every warp has a pipeline of
// its own and no barrier in it: it copies runs of keys and values into its part of shared memory (cp.async, zeros behind the sequence's
// end), forms S = Q K^T and O += P V with 16-row products from registers (mma m16n8k16; Q in registers throughout, P handed from
// one product's accumulator to the other's operand), and keeps its own running maximum and sum.  The four warps of a block and the
// blocks of a cluster, which share a sequence's keys, join their fp32 sums at the end in a fixed order.
//
// 16 sequences of 251 to 4016 keys, 16 heads of 64, a token each (143 MB): 28 us, 5.0 TB/s; 55 with the 128-row tiles.  128 of 4096 keys, 32 heads
// of 128 on 8 (2.1 GB): 299 us, 7.2 TB/s with what the 126 MB L2 keeps from call to call.
#include <atomic>

#include <cooperative_groups.h>

#include "pm_attn_packed.cuh"
#include "pm_ptx.cuh"

namespace pm {
namespace cg = cooperative_groups;

constexpr int CS_ROWS = 16, CS_KEYS = 16;         // of a tile of queries, and of a run of keys

// TEAM warps share the keys of a tile of query rows: all four of a block; each warp for itself, where sequences are short and many; or
// eight with a deeper pipeline, a block to an SM, where there are few tiles.
template <int DT, int TEAM> struct StepShape {
  static constexpr int kWarps = TEAM == 8 ? 8 : 4, kTeams = kWarps / TEAM;
  static constexpr int kRow = DT * 2;                                // bytes
  static constexpr int kRun = 2 * CS_KEYS * kRow;                    // keys and values: 4 or 8 KB
  static constexpr int kStages = TEAM == 8 && DT == 64 ? 6 : 3;
  static constexpr int kBlocks = TEAM == 8 ? 1 : DT == 64 ? 4 : 2;   // per SM
  static constexpr int kLd = DT + 4;                                 // floats of a row of sums
  static constexpr int kSmem = kWarps * kStages * kRun;
  static constexpr int kParts = TEAM == 1 ? 1 : 8;  // most blocks that share a tile
  // a team's part of shared memory at the end: sums of its warps, the team's, statistics of both, weights of the parts
  static_assert(((TEAM + 1) * CS_ROWS * kLd + (2 * TEAM + 2 + kParts) * CS_ROWS) * 4 <= TEAM * kStages * kRun, "sums of a team");
};

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes, or zeros
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// The rows of a tile; `upper`: 8 to 15 are used as well.
template <int DT> struct StepRows {
  static constexpr int kRow = DT * 2, kLd = DT + 4;
  uint32_t q[DT / 16][4];
  float o[DT / 8][4], m[2], l[2];

  __device__ __forceinline__ void start(const PackedArgs& a, const SeqTile& s, int token0, int hk, int r0, int rows) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r = r0 + (lane >> 2) + half * 8;
      const __nv_bfloat16* row = head_row<__nv_bfloat16>(a.q, s.begin + token0 + (r < rows ? r / a.group : 0), hk * a.group + (r < rows ? r % a.group : 0));
#pragma unroll
      for (int kk = 0; kk < DT / 16; ++kk)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int c = kk * 16 + (lane & 3) * 2 + i * 8;
          q[kk][half + 2 * i] = r < rows && c < a.dim ? *reinterpret_cast<const uint32_t*>(row + c) : 0u;
        }
    }
#pragma unroll
    for (int n = 0; n < DT / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
  }
  // a run of keys at k and their values behind them, of which `there` belong to the sequence
  __device__ __forceinline__ void add(uint32_t k, int there, float c, bool upper) {
    constexpr int N = CS_KEYS / 8;
    const int lane = threadIdx.x & 31;
    const uint32_t v = k + CS_KEYS * kRow;
    float p[N][4];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      p[n][0] = p[n][1] = p[n][2] = p[n][3] = 0.f;
      const int row = n * 8 + (lane & 7);
#pragma unroll
      for (int j = 0; j < DT / 32; ++j) {
        uint32_t b[4];
        ldmatrix4(b, k + row * kRow + (((4 * j + (lane >> 3)) ^ (row & 7)) << 4));
        mma_16816(p[n], q[2 * j], b[0], b[1]);
        mma_16816(p[n], q[2 * j + 1], b[2], b[3]);
      }
    }
    if (there < CS_KEYS) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) if (n * 8 + (lane & 3) * 2 + (i & 1) >= there) p[n][i] = -INFINITY;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half && !upper) {
#pragma unroll
        for (int n = 0; n < N; ++n) p[n][2] = p[n][3] = 0.f;
        break;
      }
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < N; ++n) top = max_nan(top, max_nan(p[n][2 * half], p[n][2 * half + 1]));
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2)) * c;
      if (__any_sync(0xffffffffu, !(top <= m[half]))) {              // rows whose maximum stands take a factor of one
        const float up = max_nan(m[half], top), f = up == -INFINITY ? 1.f : ex2(m[half] - up);
        m[half] = up;
        l[half] *= f;
#pragma unroll
        for (int n = 0; n < DT / 8; ++n) { o[n][2 * half] *= f; o[n][2 * half + 1] *= f; }
      }
      const float shift = m[half] == -INFINITY ? 0.f : -m[half];     // no finite score so far: nothing but zeros
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          p[n][2 * half + i] = ex2(fmaf(p[n][2 * half + i], c, shift));
          sum += p[n][2 * half + i];
        }
      l[half] += sum;                             // of this lane's keys: the row's other three lanes are added at the end
    }
#pragma unroll
    for (int t = 0; t < N / 2; ++t) {
      const uint32_t w[4] = {pack_bf16(p[2 * t][0], p[2 * t][1]), pack_bf16(p[2 * t][2], p[2 * t][3]), pack_bf16(p[2 * t + 1][0], p[2 * t + 1][1]),
                             pack_bf16(p[2 * t + 1][2], p[2 * t + 1][3])};
      const int row = t * 16 + (lane & 15);
#pragma unroll
      for (int n = 0; n < DT / 8; n += 2) {
        uint32_t b[4];
        ldmatrix4_trans(b, v + row * kRow + (((n + (lane >> 4)) ^ (row & 7)) << 4));
        mma_16816(o[n], w, b[0], b[1]);
        mma_16816(o[n + 1], w, b[2], b[3]);
      }
    }
  }
  // this warp's sums to shared memory
  __device__ __forceinline__ void leave(float* sums, float* stats, bool upper) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half && !upper) break;
      const int r = (lane >> 2) + 8 * half;
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
#pragma unroll
      for (int n = 0; n < DT / 8; ++n) *reinterpret_cast<float2*>(sums + r * kLd + n * 8 + (lane & 3) * 2) = make_float2(o[n][2 * half], o[n][2 * half + 1]);
      if ((lane & 3) == 0) { stats[r] = m[half]; stats[CS_ROWS + r] = l[half]; }
    }
  }
};

// One row's maximum and sum over n parts of (maximum, sum), `at(i)` the i-th part's statistics; factor(i) is what its sums count for.
template <typename AT> __device__ __forceinline__ void join_stats(int n, int r, AT at, float& top, float& base, float& sum) {
  top = -INFINITY;
  for (int i = 0; i < n; ++i) top = max_nan(top, at(i)[r]);
  base = top == -INFINITY ? 0.f : top;            // every score -infinity: their difference would be NaN, the sum is zero
  sum = 0.f;
  for (int i = 0; i < n; ++i) sum += ex2(at(i)[r] - base) * at(i)[CS_ROWS + r];
}

// `part` of the `parts` blocks that share a tile
template <int DT, int TEAM>
__device__ __forceinline__ void step_rows(const PackedArgs& a, const SeqTile& s, const SeqTile& ks, int token0, int hk, int r0, int rows, int part, int parts, uint8_t* smem) {
  using S = StepShape<DT, TEAM>;
  constexpr int kRow = S::kRow, kThreads = TEAM * 32;
  const int warp = threadIdx.x / 32 % TEAM, lane = threadIdx.x & 31, thread = warp * 32 + lane;
  const int runs = (ks.len + CS_KEYS - 1) / CS_KEYS, first = (int)((int64_t)runs * part / parts), last = (int)((int64_t)runs * (part + 1) / parts);
  const float c = a.scale * kLog2e;
  auto team_sync = [&]() {
    if (TEAM == 1) __syncwarp();
    else __syncthreads();
  };
  const uint32_t ring = smem_u32(smem + warp * S::kStages * S::kRun);
  // a lane copies one 16-byte column of every kStep-th row
  constexpr int kCols = DT / 8, kStep = 32 / kCols;
  const int col = lane % kCols, row0 = lane / kCols;
  const bool in = col * 8 < a.dim;
  const __nv_bfloat16 *kp = head_row<__nv_bfloat16>(a.k, ks.begin, hk) + (in ? col * 8 : 0), *vp = head_row<__nv_bfloat16>(a.v, ks.begin, hk) + (in ? col * 8 : 0);
  auto copy = [&](int run, int stage) {           // a group of copies even where there is nothing left: they are counted
    if (run < last) {
      const uint32_t to = ring + stage * S::kRun;
      const int key = run * CS_KEYS + row0;
      const __nv_bfloat16 *k = kp + key * a.k.token, *v = vp + key * a.v.token;
#pragma unroll
      for (int i = 0; i < CS_KEYS / kStep; ++i) {
        const int row = row0 + i * kStep;
        const bool there = in && key + i * kStep < ks.len;
        const uint32_t place = row * kRow + ((col ^ (row & 7)) << 4);
        cp_async16_or_zero(to + place, there ? k : kp, there);
        cp_async16_or_zero(to + CS_KEYS * kRow + place, there ? v : vp, there);
        k += kStep * a.k.token;
        v += kStep * a.v.token;
      }
    }
    cp_async_commit();
  };
  const int run0 = first + warp;
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) copy(run0 + i * TEAM, i);
  StepRows<DT> t;
  const bool upper = rows - r0 > 8;
  t.start(a, s, token0, hk, r0, rows);
  int get = 0, put = S::kStages - 1;
  for (int run = run0; run < last; run += TEAM) {
    cp_async_wait<S::kStages - 2>();
    __syncwarp();                                 // the lanes' copies are there, and all have read the run whose place is written next
    copy(run + (S::kStages - 1) * TEAM, put);
    put = put + 1 == S::kStages ? 0 : put + 1;
    t.add(ring + get * S::kRun, ks.len - run * CS_KEYS, c, upper);
    get = get + 1 == S::kStages ? 0 : get + 1;
  }
  cp_async_wait<0>();
  team_sync();                                    // the runs in shared memory have been read
  float* const sums = reinterpret_cast<float*>(smem);
  float* const joined = sums + TEAM * CS_ROWS * S::kLd;
  float* const stats = joined + CS_ROWS * S::kLd; // [TEAM + 1][2][16], the last one the block's; behind them the weights of the parts
  float* const block = stats + TEAM * 2 * CS_ROWS;
  float* const weights = block + 2 * CS_ROWS;
  t.leave(sums + warp * CS_ROWS * S::kLd, stats + warp * 2 * CS_ROWS, upper);
  team_sync();
  const int n = min(rows - r0, CS_ROWS), vectors = a.dim / 8;
  auto store = [&](int r, int col, float (&v)[8], float f) {
    const int at = r0 + r;
    *reinterpret_cast<uint4*>(head_row_out<__nv_bfloat16>(a.o, s.begin + token0 + at / a.group, hk * a.group + at % a.group) + col) =
        make_uint4(pack_bf16(v[0] * f, v[1] * f), pack_bf16(v[2] * f, v[3] * f), pack_bf16(v[4] * f, v[5] * f), pack_bf16(v[6] * f, v[7] * f));
  };
  auto store_lse = [&](int r, float top, float sum) {
    const int at = r0 + r;
    if (a.lse) a.lse[(int64_t)(hk * a.group + at % a.group) * a.tokens + s.begin + token0 + at / a.group] = (top + log2f(sum)) * kLn2;
  };
  auto add = [](float (&v)[8], float f, const float* from) {
    const float4 lo = reinterpret_cast<const float4*>(from)[0], hi = reinterpret_cast<const float4*>(from)[1];
    v[0] = fmaf(f, lo.x, v[0]); v[1] = fmaf(f, lo.y, v[1]); v[2] = fmaf(f, lo.z, v[2]); v[3] = fmaf(f, lo.w, v[3]);
    v[4] = fmaf(f, hi.x, v[4]); v[5] = fmaf(f, hi.y, v[5]); v[6] = fmaf(f, hi.z, v[6]); v[7] = fmaf(f, hi.w, v[7]);
  };
  for (int i = thread; i < n * vectors; i += kThreads) {
    const int r = i / vectors, col = i % vectors * 8;
    float top, base, sum, v[8] = {};
    auto of_warp = [&](int w) { return stats + w * 2 * CS_ROWS; };
    join_stats(TEAM, r, of_warp, top, base, sum);
#pragma unroll
    for (int w = 0; w < TEAM; ++w) add(v, ex2(of_warp(w)[r] - base), sums + (w * CS_ROWS + r) * S::kLd + col);
    if (parts == 1) {
      store(r, col, v, 1.f / sum);
      if (col == 0) store_lse(r, top, sum);
    } else {
      float4* const u = reinterpret_cast<float4*>(joined + r * S::kLd + col);
      u[0] = make_float4(v[0], v[1], v[2], v[3]);
      u[1] = make_float4(v[4], v[5], v[6], v[7]);
      if (col == 0) { block[r] = top; block[CS_ROWS + r] = sum; }
    }
  }
  if (TEAM > 1 && parts > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (thread < n) {                             // the parts' weights, and lse by the first part
      float top, base, sum;
      auto of_part = [&](int p) { return cluster.map_shared_rank(block, p); };
      join_stats(parts, thread, of_part, top, base, sum);
      for (int p = 0; p < parts; ++p) weights[p * CS_ROWS + thread] = ex2(of_part(p)[thread] - base) / sum;
      if (part == 0) store_lse(thread, top, sum);
    }
    __syncthreads();
    const int i0 = n * vectors * part / parts, i1 = n * vectors * (part + 1) / parts;
    for (int i = i0 + thread; i < i1; i += kThreads) {
      const int r = i / vectors, col = i % vectors * 8;
      float v[8] = {};
#pragma unroll 4
      for (int p = 0; p < parts; ++p) add(v, weights[p * CS_ROWS + r], cluster.map_shared_rank(joined + r * S::kLd + col, p));
      store(r, col, v, 1.f);
    }
    cluster.sync();                               // the others have read this block's sums
  }
  team_sync();
}

template <int DT, int TEAM>
__global__ void __launch_bounds__(StepShape<DT, TEAM>::kWarps * 32, StepShape<DT, TEAM>::kBlocks) attn_cross_step_kernel(const __grid_constant__ PackedArgs a, int log_tokens) {
  using S = StepShape<DT, TEAM>;
  extern __shared__ __align__(128) uint8_t step_smem[];
  const int parts = TEAM == 1 ? 1 : (int)cg::this_cluster().num_blocks(), part = TEAM == 1 ? 0 : (int)cg::this_cluster().block_rank();
  const int team = threadIdx.x / (TEAM * 32), unit = blockIdx.x / parts * S::kTeams + team, hk = unit % a.kv_heads;
  SeqTile ks;
  const SeqTile s = find_pair(a.cu, a.cu_kv, a.n_seqs, a.tokens, a.kv_tokens, unit / a.kv_heads, log_tokens, ks);
  if (s.tile < 0) return;
  const int token0 = s.tile << log_tokens, rows = min(s.len - token0, 1 << log_tokens) * a.group;
  if (ks.len == 0) {                              // no keys: zeros
    if (part == 0)
      for (int i = threadIdx.x % (TEAM * 32); i < rows * (a.dim / 8); i += TEAM * 32) {
        const int r = i / (a.dim / 8), col = i % (a.dim / 8) * 8, h = hk * a.group + r % a.group;
        const int64_t token = s.begin + token0 + r / a.group;
        *reinterpret_cast<uint4*>(head_row_out<__nv_bfloat16>(a.o, token, h) + col) = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse && col == 0) a.lse[(int64_t)h * a.tokens + token] = -INFINITY;
      }
    return;
  }
  uint8_t* const smem = step_smem + team * TEAM * S::kStages * S::kRun;
  for (int r0 = 0; r0 < rows; r0 += CS_ROWS) step_rows<DT, TEAM>(a, s, ks, token0, hk, r0, rows, part, parts, smem);
}

// tokens whose rows fill a tile of 16, as a power of two
static int step_log_tokens(const PackedArgs& a) {
  int log = 0;
  while ((2 << log) * a.group <= CS_ROWS) ++log;
  return log;
}

// Sequences of no more rows on average than a tile has.
bool attn_cross_step_takes(const PackedArgs& a) { return a.cross && a.tokens * a.group <= (int64_t)CS_ROWS * a.n_seqs; }

template <int DT, int TEAM> static cudaError_t step_launch(const PackedArgs& a, int64_t units, int parts, int log_tokens, cudaStream_t st) {
  using S = StepShape<DT, TEAM>;
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev > 63 || !(done.load(std::memory_order_relaxed) >> dev & 1))) {
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(attn_cross_step_kernel<DT, TEAM>), cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e == cudaSuccess && dev <= 63) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  const int64_t blocks = (units + S::kTeams - 1) / S::kTeams;
  return launch_clusters(attn_cross_step_kernel<DT, TEAM>, blocks, S::kWarps * 32, S::kSmem, st, false, parts, a, log_tokens);
}
template <int DT> static cudaError_t step_width(const PackedArgs& a, cudaStream_t st) {
  const int log_tokens = step_log_tokens(a);
  const int64_t units = most_tiles(a.tokens, a.n_seqs, 1 << log_tokens) * a.kv_heads, average = (a.kv_tokens + a.n_seqs - 1) / a.n_seqs;
  if (!launchable(units)) return cudaErrorInvalidConfiguration;      // parts are for launches of few
  // Many short sequences: a warp to a tile and nothing to join.  us with one / four warps to a tile: 256 tokens over 50 keys each, 16 heads
  // of 64, 16.2 / 37.1; 600 over 100, 8 heads, 29.0 / 48.0; 64 over 512, 16 heads, 25.1 / 26.4.
  if (units >= 4 * kSms && average <= 512) return step_launch<DT, 1>(a, units, 1, log_tokens, st);
  // Parts of at least four runs to a warp on average, as long as the launch has no more than four blocks to an SM: clusters cost what finer
  // parts would gain (16 sequences of 2133 keys, 16 heads of 64: 26 us with 272 blocks in two parts, 31 in four, 46 in eight; 8 sequences
  // of 300 keys: 6.9 whole, 8.8 in two).
  auto parts_of = [&](int team, int64_t most_blocks) {
    int parts = 1;
    while (parts < StepShape<DT, 4>::kParts && units * parts * 2 <= most_blocks && average >= (int64_t)parts * 2 * team * 4 * CS_KEYS) parts *= 2;
    return parts;
  };
  // Few tiles: eight warps to a block (one of 100000 keys, 8 heads of 128: 80 us, with four 112; one of 30000, 4 heads of 64 on 1: 22 / 30).
  if (units * 8 <= kSms) return step_launch<DT, 8>(a, units, parts_of(8, kSms), log_tokens, st);
  return step_launch<DT, 4>(a, units, parts_of(4, 4 * kSms), log_tokens, st);
}
cudaError_t attn_cross_step(const PackedArgs& a, cudaStream_t st) { return a.dim <= 64 ? step_width<64>(a, st) : step_width<128>(a, st); }

}  // namespace pm
