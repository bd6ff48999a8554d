// Cross attention of few query rows: a decoding step, with a token or the few of a beam to each sequence.  bf16 and fp32.
//
// Bound by memory: every key and value is read once for 16 query rows (tokens times the heads that share it), most often for all, far too few
// for a tile of the other kernels, whose chain of waits would set the pace.  Here every warp has a pipeline of its own and no barrier in it: it
// copies runs of keys and values into its part of shared memory (cp.async, zeros behind the sequence's end), forms S = Q K^T and
// O += P V, and keeps its own running maximum and sum.  bf16: 16-row products from registers (mma m16n8k16; Q in registers throughout, P
// handed from one product's accumulator to the other's operand).  fp32: a few lanes to a key for the scores, a few columns to a lane
// for O.  The warps of a block and the blocks of a cluster that share a sequence's keys join their fp32 sums at the end in a fixed order.
//
// 16 sequences of 251 to 4016 keys, 16 heads of 64, a token each, bf16 (143 MB): 28 us, 5.0 TB/s; 48 with the 128-row tiles.  128 of 4096 keys,
// 32 heads of 128 on 8 (2.1 GB): 296 us, 7.3 TB/s with what the 126 MB L2 keeps from call to call.
#include <algorithm>
#include <atomic>

#include <cooperative_groups.h>

#include "pm_attn_packed.cuh"
#include "pm_ptx.cuh"

namespace pm {
namespace cg = cooperative_groups;

constexpr int CS_ROWS = 16;                       // of a tile of queries, at most

// TEAM warps share the keys of a tile of query rows: all four of a block; each warp for itself, where sequences are short and many; or
// eight with a deeper pipeline, a block to an SM, where there are few tiles.  E: what is done with a run of keys (HalfRows, FloatRows).
template <typename E, int TEAM> struct StepShape {
  static constexpr int kWarps = TEAM == 8 ? 8 : 4, kTeams = kWarps / TEAM;
  static constexpr int kStages = TEAM == 8 && E::kRun < 8192 ? 6 : 3;
  static constexpr int kLd = E::kWidth + 4;                          // floats of a row of sums
  static constexpr int kRing = kWarps * kStages * E::kRun;
  static constexpr int kSmem = kRing + kTeams * E::kTeamBytes + kWarps * E::kWarpBytes;
  static constexpr int kFit = 227 * 1024 / (kSmem + 1024);
  static constexpr int kBlocks = TEAM == 8 ? 1 : kFit < E::kMostBlocks ? kFit : E::kMostBlocks;     // per SM
  static constexpr int kParts = TEAM == 1 ? 1 : 8;                   // most blocks that share a tile
  // a team's part of the ring at the end: sums of its warps, the team's, statistics of both, weights of the parts
  static_assert(((TEAM + 1) * kLd + 2 * TEAM + 2 + kParts) * E::kRows * 4 <= TEAM * kStages * E::kRun, "sums of a team");
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

// bf16, heads of up to DT
template <int DT> struct HalfRows {
  using T = __nv_bfloat16;
  static constexpr int kWidth = DT, kRows = CS_ROWS, kKeys = 16, kRow = DT * 2, kLd = DT + 4, kCols = 8;
  static constexpr int kRun = 2 * kKeys * kRow, kTeamBytes = 0, kWarpBytes = 0, kMostBlocks = DT == 64 ? 4 : 2, kShort = 512;
  bool upper;                                     // rows 8 to 15 are used as well

  // a lane copies one 16-byte column of every kStep-th row
  struct Copy {
    static constexpr int kColumns = DT / 8, kStep = 32 / kColumns;
    const T *kp, *vp;
    int64_t k_stride, v_stride;
    int len, row0;
    uint32_t place;
    bool in;
    __device__ __forceinline__ Copy(const PackedArgs& a, const SeqTile& ks, int hk) : k_stride(a.k.token), v_stride(a.v.token), len(ks.len) {
      const int lane = threadIdx.x & 31, col = lane % kColumns;
      row0 = lane / kColumns;
      in = col * 8 < a.dim;
      kp = head_row<T>(a.k, ks.begin, hk) + (in ? col * 8 : 0);
      vp = head_row<T>(a.v, ks.begin, hk) + (in ? col * 8 : 0);
      place = col;
    }
    __device__ __forceinline__ void run(int run, uint32_t to) const {
      const int key = run * kKeys + row0;
      const T *k = kp + key * k_stride, *v = vp + key * v_stride;
#pragma unroll
      for (int i = 0; i < kKeys / kStep; ++i) {
        const int row = row0 + i * kStep;
        const bool there = in && key + i * kStep < len;
        const uint32_t at = to + row * kRow + ((place ^ (row & 7)) << 4);
        cp_async16_or_zero(at, there ? k : kp, there);
        cp_async16_or_zero(at + kKeys * kRow, there ? v : vp, there);
        k += kStep * k_stride;
        v += kStep * v_stride;
      }
    }
  };
  static __device__ __forceinline__ void store(T* row, int col, int, const float (&v)[8], float f) {
    *reinterpret_cast<uint4*>(row + col) =
        make_uint4(pack_bf16(v[0] * f, v[1] * f), pack_bf16(v[2] * f, v[3] * f), pack_bf16(v[4] * f, v[5] * f), pack_bf16(v[6] * f, v[7] * f));
  }
  uint32_t q[DT / 16][4];
  float o[DT / 8][4], m[2], l[2];

  __device__ __forceinline__ void start(const PackedArgs& a, const SeqTile& s, int token0, int hk, int r0, int rows, float*, float*, int, int) {
    const int lane = threadIdx.x & 31;
    upper = rows - r0 > 8;
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
  __device__ __forceinline__ void add(const uint8_t* run, int there, float c) {
    constexpr int N = kKeys / 8;
    const int lane = threadIdx.x & 31;
    const uint32_t k = smem_u32(run), v = k + kKeys * kRow;
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
    if (there < kKeys) {
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
  __device__ __forceinline__ void leave(float* sums, float* stats) {
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

// 16 or 4 bytes, or zeros
__device__ __forceinline__ void cp_async4_or_zero(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}

// fp32, heads of up to DP.  VEC: rows start at 16-byte boundaries.  kPer lanes share a key and take every kPer-th four of its columns; a lane owns
// kOwn columns of O of ROWS rows, 4 or 16.  Columns of key j are put at their place exclusive-or kPer j, by fours, so that the lanes that read at a time meet no bank twice.
template <int DP, bool VEC, int ROWS> struct FloatRows {
  using T = float;
  // with few rows the runs are as short as 4 KB, so that more blocks fit an SM
  static constexpr int kWidth = DP, kRows = ROWS, kKeys = ROWS == 4 ? 512 / DP : DP == 128 ? 8 : 16, kPer = 32 / kKeys, kOwn = DP / 32, kLd = DP + 4, kCols = 4;
  static constexpr int kRun = 2 * kKeys * DP * 4, kTeamBytes = ROWS * DP * 4, kWarpBytes = kKeys * ROWS * 4, kMostBlocks = ROWS == 4 || DP == 32 ? 4 : 2, kShort = 128;
  float o[ROWS][kOwn], m[ROWS], l[ROWS];
  float *q, *p;                                   // the tile's rows, the team's; probabilities [key][row], the warp's
  int n;                                          // rows in use

  static __device__ __forceinline__ int place(int row, int four) { return row * DP + ((four ^ (row * kPer & 7)) << 2); }
  struct Copy {
    static constexpr int kColumns = VEC ? DP / 4 : DP, kStep = kColumns >= 32 ? 1 : 32 / kColumns, kEach = kColumns > 32 ? kColumns / 32 : 1;
    const T *kp, *vp;
    int64_t k_stride, v_stride;
    int len, dim;
    __device__ __forceinline__ Copy(const PackedArgs& a, const SeqTile& ks, int hk)
        : kp(head_row<T>(a.k, ks.begin, hk)), vp(head_row<T>(a.v, ks.begin, hk)), k_stride(a.k.token), v_stride(a.v.token), len(ks.len), dim(a.dim) {}
    __device__ __forceinline__ void run(int run, uint32_t to) const {
      const int lane = threadIdx.x & 31, row0 = kColumns >= 32 ? 0 : lane / kColumns;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int col = (kColumns >= 32 ? lane + 32 * e : lane % kColumns) * (VEC ? 4 : 1);
        const int key = run * kKeys + row0;
        const T *k = kp + key * k_stride + col, *v = vp + key * v_stride + col;
#pragma unroll
        for (int i = 0; i < kKeys / kStep; ++i) {
          const int row = row0 + i * kStep;
          const bool there = col < dim && key + i * kStep < len;
          const uint32_t at = to + (place(row, col >> 2) + (col & 3)) * 4;
          if (VEC) {
            cp_async16_or_zero(at, there ? k : kp, there);
            cp_async16_or_zero(at + kKeys * DP * 4, there ? v : vp, there);
          } else {
            cp_async4_or_zero(at, there ? k : kp, there);
            cp_async4_or_zero(at + kKeys * DP * 4, there ? v : vp, there);
          }
          k += kStep * k_stride;
          v += kStep * v_stride;
        }
      }
    }
  };
  static __device__ __forceinline__ void store(T* row, int col, int dim, const float (&v)[4], float f) {
    if (VEC) {
      *reinterpret_cast<float4*>(row + col) = make_float4(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) if (col + e < dim) row[col + e] = v[e] * f;
    }
  }
  // rows up to the next multiple of four are filled, with zeros behind the last; the team waits for one another before add
  __device__ __forceinline__ void start(const PackedArgs& a, const SeqTile& s, int token0, int hk, int r0, int rows, float* team, float* warp, int thread, int threads) {
    q = team;
    p = warp;
    n = min(rows - r0, ROWS);
    for (int i = thread; i < (n + 3) / 4 * 4 * DP; i += threads) {
      const int r = r0 + i / DP, c = i % DP;
      q[i] = r < rows && c < a.dim ? head_row<T>(a.q, s.begin + token0 + r / a.group, hk * a.group + r % a.group)[c] : 0.f;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int e = 0; e < kOwn; ++e) o[r][e] = 0.f;
    }
  }
  // R rows from r0 on: scores, maximum, probabilities
  template <int R> __device__ __forceinline__ void rows_of(const float* k, int r0, int there, float c) {
    const int lane = threadIdx.x & 31, key = lane / kPer, part = lane % kPer;
    float acc[R] = {};
#pragma unroll
    for (int i = 0; i < DP / 4 / kPer; ++i) {
      const int four = part + kPer * i;
      const float4 x = *reinterpret_cast<const float4*>(k + place(key, four));
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float4 y = *reinterpret_cast<const float4*>(q + (r0 + r) * DP + four * 4);
        acc[r] = fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, acc[r]))));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 1; i < kPer; i *= 2) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], i);
      if (key >= there) acc[r] = -INFINITY;
      float top = acc[r];
#pragma unroll
      for (int i = kPer; i < 32; i *= 2) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, i));
      top *= c;
      if (!(top <= m[r0 + r])) {                  // the same in all lanes; a maximum that stands takes a factor of one
        const float up = max_nan(m[r0 + r], top), f = up == -INFINITY ? 1.f : ex2(m[r0 + r] - up);
        m[r0 + r] = up;
        l[r0 + r] *= f;
#pragma unroll
        for (int e = 0; e < kOwn; ++e) o[r0 + r][e] *= f;
      }
      const float shift = m[r0 + r] == -INFINITY ? 0.f : -m[r0 + r];             // no finite score so far: nothing but zeros
      acc[r] = ex2(fmaf(acc[r], c, shift));
      if (part == 0) l[r0 + r] += acc[r];         // of this lane's keys: the others' are added at the end
    }
    if (part == 0) {
      if constexpr (R == 4) *reinterpret_cast<float4*>(p + key * ROWS + r0) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      else p[key * ROWS + r0] = acc[0];
    }
  }
  template <int R> __device__ __forceinline__ void values_of(const float (&v)[kOwn], const float* at, int r0) {
    float w[R];
    if constexpr (R == 4) {
      const float4 x = *reinterpret_cast<const float4*>(at + r0);
      w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else {
      w[0] = at[r0];
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < kOwn; ++e) o[r0 + r][e] = fmaf(w[r], v[e], o[r0 + r][e]);
  }
  __device__ __forceinline__ void add(const uint8_t* run, int there, float c) {
    const int lane = threadIdx.x & 31;
    const float *k = reinterpret_cast<const float*>(run), *v = k + kKeys * DP;
    if (n == 1) {
      rows_of<1>(k, 0, there, c);
    } else {
#pragma unroll
      for (int r0 = 0; r0 < ROWS; r0 += 4) if (r0 < n) rows_of<4>(k, r0, there, c);
    }
    __syncwarp();
#pragma unroll 4
    for (int key = 0; key < kKeys; ++key) {
      const int col = lane * kOwn;
      const float* from = v + place(key, col >> 2) + (col & 3);
      float x[kOwn];
      if constexpr (kOwn == 4) {
        const float4 y = *reinterpret_cast<const float4*>(from);
        x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
      } else if constexpr (kOwn == 2) {
        const float2 y = *reinterpret_cast<const float2*>(from);
        x[0] = y.x; x[1] = y.y;
      } else {
        x[0] = from[0];
      }
      if (n == 1) {
        values_of<1>(x, p + key * ROWS, 0);
      } else {
#pragma unroll
        for (int r0 = 0; r0 < ROWS; r0 += 4) if (r0 < n) values_of<4>(x, p + key * ROWS, r0);
      }
    }
    __syncwarp();                                 // the probabilities have been read
  }
  __device__ __forceinline__ void leave(float* sums, float* stats) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (r >= n) break;
#pragma unroll
      for (int i = 1; i < 32; i *= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], i);
#pragma unroll
      for (int e = 0; e < kOwn; ++e) sums[r * kLd + lane * kOwn + e] = o[r][e];
      if (lane == 0) { stats[r] = m[r]; stats[ROWS + r] = l[r]; }
    }
  }
};

// One row's maximum and sum over n parts of (maximum, sum), `at(i)` the i-th part's statistics; factor(i) is what its sums count for.
template <int ROWS, typename AT> __device__ __forceinline__ void join_stats(int n, int r, AT at, float& top, float& base, float& sum) {
  top = -INFINITY;
  for (int i = 0; i < n; ++i) top = max_nan(top, at(i)[r]);
  base = top == -INFINITY ? 0.f : top;            // every score -infinity: their difference would be NaN, the sum is zero
  sum = 0.f;
  for (int i = 0; i < n; ++i) sum += ex2(at(i)[r] - base) * at(i)[ROWS + r];
}

// `part` of the `parts` blocks that share a tile
template <typename E, int TEAM>
__device__ __forceinline__ void step_rows(const PackedArgs& a, const SeqTile& s, const SeqTile& ks, int token0, int hk, int r0, int rows, int part, int parts, uint8_t* smem, float* of_team,
                                          float* of_this_warp) {
  using S = StepShape<E, TEAM>;
  using T = typename E::T;
  constexpr int kThreads = TEAM * 32, C = E::kCols, R = E::kRows;
  const int warp = threadIdx.x / 32 % TEAM, lane = threadIdx.x & 31, thread = warp * 32 + lane;
  const int runs = (ks.len + E::kKeys - 1) / E::kKeys, first = (int)((int64_t)runs * part / parts), last = (int)((int64_t)runs * (part + 1) / parts);
  const float c = a.scale * kLog2e;
  auto team_sync = [&]() {
    if (TEAM == 1) __syncwarp();
    else __syncthreads();
  };
  uint8_t* const ring = smem + warp * S::kStages * E::kRun;
  const uint32_t ring_at = smem_u32(ring);
  const typename E::Copy from(a, ks, hk);
  auto copy = [&](int run, int stage) {           // a group of copies even where there is nothing left: they are counted
    if (run < last) from.run(run, ring_at + stage * E::kRun);
    cp_async_commit();
  };
  const int run0 = first + warp;
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) copy(run0 + i * TEAM, i);
  E t;
  t.start(a, s, token0, hk, r0, rows, of_team, of_this_warp, thread, kThreads);
  if (E::kTeamBytes) team_sync();
  int get = 0, put = S::kStages - 1;
  for (int run = run0; run < last; run += TEAM) {
    cp_async_wait<S::kStages - 2>();
    __syncwarp();                                 // the lanes' copies are there, and all have read the run whose place is written next
    copy(run + (S::kStages - 1) * TEAM, put);
    put = put + 1 == S::kStages ? 0 : put + 1;
    t.add(ring + get * E::kRun, ks.len - run * E::kKeys, c);
    get = get + 1 == S::kStages ? 0 : get + 1;
  }
  cp_async_wait<0>();
  team_sync();                                    // the runs in shared memory have been read
  float* const sums = reinterpret_cast<float*>(smem);
  float* const joined = sums + TEAM * R * S::kLd;
  float* const stats = joined + R * S::kLd; // [TEAM + 1][2][R], the last one the block's; behind them the weights of the parts
  float* const block = stats + TEAM * 2 * R;
  float* const weights = block + 2 * R;
  t.leave(sums + warp * R * S::kLd, stats + warp * 2 * R);
  team_sync();
  const int n = min(rows - r0, R), vectors = (a.dim + C - 1) / C;
  auto store = [&](int r, int col, const float (&v)[C], float f) {
    const int at = r0 + r;
    E::store(head_row_out<T>(a.o, s.begin + token0 + at / a.group, hk * a.group + at % a.group), col, a.dim, v, f);
  };
  auto store_lse = [&](int r, float top, float sum) {
    const int at = r0 + r;
    if (a.lse) a.lse[(int64_t)(hk * a.group + at % a.group) * a.tokens + s.begin + token0 + at / a.group] = (top + log2f(sum)) * kLn2;
  };
  auto add = [](float (&v)[C], float f, const float* from) {
#pragma unroll
    for (int e = 0; e < C; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(from + e);
      v[e] = fmaf(f, x.x, v[e]); v[e + 1] = fmaf(f, x.y, v[e + 1]); v[e + 2] = fmaf(f, x.z, v[e + 2]); v[e + 3] = fmaf(f, x.w, v[e + 3]);
    }
  };
  for (int i = thread; i < n * vectors; i += kThreads) {
    const int r = i / vectors, col = i % vectors * C;
    float top, base, sum, v[C] = {};
    auto of_warp = [&](int w) { return stats + w * 2 * R; };
    join_stats<R>(TEAM, r, of_warp, top, base, sum);
#pragma unroll
    for (int w = 0; w < TEAM; ++w) add(v, ex2(of_warp(w)[r] - base), sums + (w * R + r) * S::kLd + col);
    if (parts == 1) {
      store(r, col, v, 1.f / sum);
      if (col == 0) store_lse(r, top, sum);
    } else {
#pragma unroll
      for (int e = 0; e < C; e += 4) *reinterpret_cast<float4*>(joined + r * S::kLd + col + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
      if (col == 0) { block[r] = top; block[R + r] = sum; }
    }
  }
  if (TEAM > 1 && parts > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (thread < n) {                             // the parts' weights, and lse by the first part
      float top, base, sum;
      auto of_part = [&](int p) { return cluster.map_shared_rank(block, p); };
      join_stats<R>(parts, thread, of_part, top, base, sum);
      for (int p = 0; p < parts; ++p) weights[p * R + thread] = ex2(of_part(p)[thread] - base) / sum;
      if (part == 0) store_lse(thread, top, sum);
    }
    __syncthreads();
    const int i0 = n * vectors * part / parts, i1 = n * vectors * (part + 1) / parts;
    for (int i = i0 + thread; i < i1; i += kThreads) {
      const int r = i / vectors, col = i % vectors * C;
      float v[C] = {};
#pragma unroll 4
      for (int p = 0; p < parts; ++p) add(v, weights[p * R + r], cluster.map_shared_rank(joined + r * S::kLd + col, p));
      store(r, col, v, 1.f);
    }
    cluster.sync();                               // the others have read this block's sums
  }
  team_sync();
}

template <typename E, int TEAM>
__global__ void __launch_bounds__(StepShape<E, TEAM>::kWarps * 32, StepShape<E, TEAM>::kBlocks) attn_cross_step_kernel(const __grid_constant__ PackedArgs a, int log_tokens) {
  using S = StepShape<E, TEAM>;
  using T = typename E::T;
  extern __shared__ __align__(128) uint8_t step_smem[];
  const int parts = TEAM == 1 ? 1 : (int)cg::this_cluster().num_blocks(), part = TEAM == 1 ? 0 : (int)cg::this_cluster().block_rank();
  const int team = threadIdx.x / (TEAM * 32), unit = blockIdx.x / parts * S::kTeams + team, hk = unit % a.kv_heads;
  SeqTile ks;
  const SeqTile s = find_longest(a.cu, a.cu_kv, a.n_seqs, a.tokens, a.kv_tokens, unit / a.kv_heads, log_tokens, ks);
  if (s.tile < 0) return;
  const int token0 = s.tile << log_tokens, rows = min(s.len - token0, 1 << log_tokens) * a.group;
  if (ks.len == 0) {                              // no keys: zeros
    if (part == 0)
      for (int i = threadIdx.x % (TEAM * 32); i < rows * a.dim; i += TEAM * 32) {
        const int r = i / a.dim, col = i % a.dim, h = hk * a.group + r % a.group;
        const int64_t token = s.begin + token0 + r / a.group;
        head_row_out<T>(a.o, token, h)[col] = from_f<T>(0.f);
        if (a.lse && col == 0) a.lse[(int64_t)h * a.tokens + token] = -INFINITY;
      }
    return;
  }
  uint8_t* const smem = step_smem + team * TEAM * S::kStages * E::kRun;
  float* const of_team = reinterpret_cast<float*>(step_smem + S::kRing + team * E::kTeamBytes);
  float* const of_warp = reinterpret_cast<float*>(step_smem + S::kRing + S::kTeams * E::kTeamBytes + threadIdx.x / 32 * E::kWarpBytes);
  for (int r0 = 0; r0 < rows; r0 += E::kRows) step_rows<E, TEAM>(a, s, ks, token0, hk, r0, rows, part, parts, smem, of_team, of_warp);
}

// tokens whose rows fill a tile, as a power of two
static int step_log_tokens(const PackedArgs& a, int rows) {
  int log = 0;
  while ((2 << log) * a.group <= rows) ++log;
  return log;
}

// Rows (tokens times the heads that share a key) on average of a sequence that these kernels are the faster ones for; bf16 in what the tensor-core
// kernels take.  us with these / the others: bf16, 16 x 8 tokens over 1000 keys, 16 heads of 128 on 4 (32 rows) 15.1 / 22.4; 64 x 20 over 60, 8 heads
// of 64 (20) 8.0 / 11.6; 16 x 32 over 1000, 16 heads of 64 (32) 20.0 / 19.7; 16 x 64 (64) 34.7 / 19.6.  fp32, 16 x 8 over 1000, 16 heads of 128 on 4 125 / 164; 16 x 5
// over 3000, 32 heads of 128 on 8 (20) 490 / 1714; but 16 x 20 over 1000, 16 heads of 64 175 / 147: heads that share keys are what the others repeat.
bool attn_cross_step_takes(const PackedArgs& a, int dtype) {
  const int64_t rows = a.tokens * a.group;
  if (!a.cross || rows > (int64_t)32 * a.n_seqs) return false;
  if (dtype == PM_F32) return rows <= (int64_t)16 * a.n_seqs || a.tokens <= (int64_t)8 * a.n_seqs;
  return attn_packed_tc_takes(a, dtype, false);
}

template <typename E, int TEAM> static cudaError_t step_launch(const PackedArgs& a, int64_t units, int parts, int log_tokens, cudaStream_t st) {
  using S = StepShape<E, TEAM>;
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev > 63 || !(done.load(std::memory_order_relaxed) >> dev & 1))) {
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(attn_cross_step_kernel<E, TEAM>), cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e == cudaSuccess && dev <= 63) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) return e;
  const int64_t blocks = (units + S::kTeams - 1) / S::kTeams;
  return launch_clusters(attn_cross_step_kernel<E, TEAM>, blocks, S::kWarps * 32, S::kSmem, st, false, parts, a, log_tokens);
}
template <typename E> static cudaError_t step_run(const PackedArgs& a, cudaStream_t st) {
  const int log_tokens = step_log_tokens(a, E::kRows);
  const int64_t units = most_tiles(a.tokens, a.n_seqs, 1 << log_tokens) * a.kv_heads, average = (a.kv_tokens + a.n_seqs - 1) / a.n_seqs;
  if (!launchable(units)) return cudaErrorInvalidConfiguration;      // parts are for launches of few
  // Many short sequences: a warp to a tile and nothing to join.  us with one / four warps to a tile, bf16: 256 tokens over 50 keys each, 16 heads
  // of 64, 14 / 33; 600 over 100, 8 heads, 27 / 39; 64 over 512, 16 heads, 24.3 / 25.7.  fp32: 25 / 42, 50 / 55, 51 / 44.
  if (units >= 4 * kSms && average <= E::kShort) return step_launch<E, 1>(a, units, 1, log_tokens, st);
  // Parts of at least four runs to a warp on average, as long as the launch has no more than four blocks to an SM: clusters cost what finer
  // parts would gain (bf16, 16 sequences of 2133 keys, 16 heads of 64: 25 us whole, 26 with 272 blocks in two parts, 31 in four, 46 in eight; 8
  // sequences of 300 keys: 5.6 whole, 7.4 in two).  Blocks without a tile, of which there may be many, do not count.
  const int64_t tokens = (a.tokens + a.n_seqs - 1) / a.n_seqs, filled = std::min(units, (int64_t)a.n_seqs * ((tokens + (1 << log_tokens) - 1) >> log_tokens) * a.kv_heads);
  auto parts_of = [&](int team, int64_t most_blocks) {
    int parts = 1;
    while (parts < StepShape<E, 4>::kParts && filled * parts * 2 <= most_blocks && average >= (int64_t)parts * 2 * team * 4 * E::kKeys) parts *= 2;
    return parts;
  };
  // Few tiles: eight warps to a block (one of 100000 keys, 8 heads of 128: 70 us, with four 100; one of 30000, 4 heads of 64 on 1: 19 / 30).
  if (filled * 8 <= kSms) return step_launch<E, 8>(a, units, parts_of(8, kSms), log_tokens, st);
  return step_launch<E, 4>(a, units, parts_of(4, 4 * kSms), log_tokens, st);
}
template <bool VEC, int ROWS> static cudaError_t step_float(const PackedArgs& a, cudaStream_t st) {
  if (a.dim <= 32) return step_run<FloatRows<32, VEC, ROWS>>(a, st);
  return a.dim <= 64 ? step_run<FloatRows<64, VEC, ROWS>>(a, st) : step_run<FloatRows<128, VEC, ROWS>>(a, st);
}
cudaError_t attn_cross_step(const PackedArgs& a, int dtype, cudaStream_t st) {
  if (dtype == PM_BF16) return a.dim <= 64 ? step_run<HalfRows<64>>(a, st) : step_run<HalfRows<128>>(a, st);
  bool vec = a.dim % 4 == 0;
  for (const HeadView* x : {&a.q, &a.k, &a.v, &a.o}) vec = vec && aligned_to(x->data, 16) && x->token % 4 == 0 && x->head % 4 == 0;
  // tiles of four rows where sequences have no more on average: the sums of 16 take the registers of half the warps
  if (a.tokens * a.group <= (int64_t)4 * a.n_seqs) return vec ? step_float<true, 4>(a, st) : step_float<false, 4>(a, st);
  return vec ? step_float<true, 16>(a, st) : step_float<false, 16>(a, st);
}

}  // namespace pm
