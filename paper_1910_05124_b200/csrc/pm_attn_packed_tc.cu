// Attention over packed sequences on the tensor cores (tcgen05, TMEM, TMA): bf16, heads of up to 128 in steps of 8 (zero-filled to a
// tile of 64 or 128 by the copies).  The mathematics is that of pm_attn_packed.cu.
//
// Forward.  A block owns NT query tiles of 128 rows: two heads that share keys and values, or two consecutive tiles of one head; every
// key/value tile it copies serves both.  Four warps per query tile (thread = row = tensor-memory lane) do the softmax, one warp
// copies, one issues the products:
//   S = Q K^T (128 x 128 x D, operands in shared memory) -> p = 2^(c s - m) in fp32 -> bf16 P over S's columns in tensor memory
//   -> O += P V (A = P from tensor memory).
// While the softmax of one tile runs, the products of the other do.  The running maximum m is raised, and O and the row sum rescaled,
// only when the row outgrows it by 2^8: P then reaches at most 256, which bf16 holds as exactly as 1, and most key tiles
// leave O alone.
//
// Where P lies over S, products that read P are issued before the product that overwrites it, and products complete in the order of
// their issue, so a commit behind S(j + 1) also says that O holds tile j.
#include <atomic>
#include <mutex>

#include <cooperative_groups.h>

#include "pm_attn_packed.cuh"
#include "pm_ptx.cuh"

namespace pm {
namespace cg = cooperative_groups;

// A bounded wait that ran out (a defect): its code, kept until pm_attention_packed_status reads it.
__device__ int g_attn_packed_status;

constexpr int TC_ROWS = 128, TC_LOG_ROWS = 7;     // rows of a tile, of queries and of keys
constexpr int TC_SUB = TC_ROWS * 128;             // bytes of a [128 x 64] bf16 sub-tile, 128-byte swizzle

// A bounded wait in line: a call from a thread that holds a row of scores would have to put them away.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int code,
                                         long long limit_cycles = WAIT_LIMIT_CYCLES) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (*abort_flag) return false;
    if (clock64() - t0 > limit_cycles) {
      *abort_flag = 1;
      atomicCAS(status, 0, code);
      return false;
    }
  }
  return true;
}

template <int DT, int NT> struct FwdShape {
  static constexpr int kSub = DT / 64;            // sub-tiles of a tile
  static constexpr int kTile = kSub * TC_SUB;
  static_assert(NT == 1 || DT == 128, "two query tiles to a block are for heads of 128");
  static constexpr int kStages = NT == 1 && DT == 128 ? 1 : 2;
  static constexpr int kWarps = NT * 4;           // of the softmax: thread = row
  static constexpr int kThreads = kWarps * 32 + 128;
  static constexpr int kBlocks = NT == 1 ? 2 : 1; // per SM
  // Registers: a softmax thread holds a row of 128 scores, the warps that copy and issue need few.  NT = 2: 384 threads are launched
  // with 168, 256 x 224 + 128 x 56 is no more than that; NT = 1: 256 with 128, 128 x 208 + 128 x 48.
  // What does not fit while a row is held goes to local memory: 100 to 132 bytes of stores, 176 to 184 of loads.
  // (Two threads to a row, 64 scores each, took 332 us where this took 295: 8192 + 4099 tokens, 16 heads of 128 on 4.)
  static constexpr int kSoftmaxRegs = NT == 1 ? 208 : 224, kOtherRegs = NT == 1 ? 48 : 56;
  // Tensor-memory columns: S (128 for each tile), O (DT), and for heads of 64 P (64) beside S instead of over it, so that the
  // next scores are formed while the exponentials of these are (8192 tokens, 16 heads of 64, causal: 197 us, over S 205).
  static constexpr int kCols = NT * 256;
  static constexpr bool kApart = DT == 64;
  static constexpr int kBars = 1 + 4 * kStages + 5 * NT;
  static constexpr int kSmem = NT * kTile + 2 * kStages * kTile + 1024 + kBars * 8 + 16;
};

struct TcMaps { CUtensorMap q, k, v; };

// What a matrix descriptor takes of a shared-memory address: in a block of a cluster the address carries the block's rank above it.
__device__ __forceinline__ uint32_t own_address(uint32_t a) { return a & 0x3FFFFu; }

// 128 x N x DT product of two K-major tiles
template <int DT> __device__ __forceinline__ void mma_abt(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
  a = own_address(a); b = own_address(b);
  const uint64_t base = desc_base(16, 1024);
#pragma unroll
  for (int k = 0; k < DT / 16; ++k) {
    const uint32_t off = (k >> 2) * TC_SUB + (k & 3) * 32;
    tc_mma_bf16(d, desc_at(base, a + off), desc_at(base, b + off), idesc, k > 0);
  }
}
// 128 x DT x 64 product of half of A in tensor memory and half of a tile whose rows run along the depth
template <int DT> __device__ __forceinline__ void mma_ab(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate, int half) {
  b = own_address(b);
  const uint64_t base = desc_base(TC_SUB, 1024);
#pragma unroll
  for (int k = 0; k < 4; ++k) tc_mma_bf16_ta(d, a + (half * 4 + k) * 8, desc_at(base, b + (half * 4 + k) * 2048), idesc, accumulate || k > 0);
}

template <int DT> __device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int64_t token) {
#pragma unroll
  for (int i = 0; i < DT / 64; ++i) tma_load_3d(dst + i * TC_SUB, map, bar, i * 64, head, (int)token);
}

__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// A warp's 32 rows of an accumulator, 32 columns from c0 on, times f, to bf16 rows in memory.  Each lane has a row; through 2 KB of
// shared memory four lanes come to write 64 bytes of a row, a quarter of the transactions that a lane to a row would make.
// `rows`: how many of the warp's rows are the sequence's, from the first one on.  NaN where a wait ran out (ok is false).
__device__ __forceinline__ void store_rows(__nv_bfloat16* out, int64_t stride, int rows, uint32_t taddr, int c0, int dim, float f, bool ok, uint8_t* stage) {
  const int lane = threadIdx.x & 31;
  uint32_t o[32];
  tmem_ld32(taddr + c0, o);
  tmem_ld_wait(o);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(o[g * 8 + i]) * f;
    *reinterpret_cast<uint4*>(stage + lane * 64 + ((g ^ (lane >> 1 & 3)) << 4)) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 8 + (lane >> 2), g = lane & 3;
    uint4 w = *reinterpret_cast<const uint4*>(stage + r * 64 + ((g ^ (r >> 1 & 3)) << 4));
    if (!ok) w = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
    if (r < rows && c0 + g * 8 < dim) *reinterpret_cast<uint4*>(out + r * stride + c0 + g * 8) = w;
  }
  __syncwarp();
}

// Where there are few blocks, a cluster of them shares one block's rows: each takes a part of what is streamed, leaves its fp32 sums in its
// shared memory, and finishes a part of the rows from everybody's, added in the order of the parts.
template <int DT> constexpr int kSumLd = DT + 4;
// 32 columns of each lane's row, from the accumulator or, of a block that had nothing to do, zeros
template <int DT> __device__ __forceinline__ void leave_sums(float* row, uint32_t taddr, int c0, bool any) {
  uint32_t o[32];
  tmem_ld32(taddr + c0, o);
  tmem_ld_wait(o);
#pragma unroll
  for (int i = 0; i < 32; i += 4)
    *reinterpret_cast<uint4*>(row + c0 + i) = any ? make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]) : make_uint4(0u, 0u, 0u, 0u);
}
// this block's share of the rows, by its first `threads` threads
template <int DT, typename W>
__device__ __forceinline__ void finish_rows(const HeadView& x, const SeqTile& s, int row0, int head, int dim, float* sums, int part, int parts, int threads, W weight) {
  cg::cluster_group cluster = cg::this_cluster();
  const int r0 = TC_ROWS * part / parts, r1 = TC_ROWS * (part + 1) / parts;
  for (int i = threadIdx.x; i < (r1 - r0) * (DT / 8); i += threads) {
    const int r = r0 + i / (DT / 8), c = i % (DT / 8) * 8;
    if (row0 + r >= s.len || c >= dim) continue;
    float v[8] = {};
    for (int p = 0; p < parts; ++p) {
      const float4* u = reinterpret_cast<const float4*>(cluster.map_shared_rank(sums + r * kSumLd<DT> + c, p));
      const float4 lo = u[0], hi = u[1];
      const float f = weight(r, p);
      v[0] += f * lo.x; v[1] += f * lo.y; v[2] += f * lo.z; v[3] += f * lo.w;
      v[4] += f * hi.x; v[5] += f * hi.y; v[6] += f * hi.z; v[7] += f * hi.w;
    }
    *reinterpret_cast<uint4*>(head_row_out<__nv_bfloat16>(x, s.begin + row0 + r, head) + c) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
}

// 2^x for two values on the FMA units: x = n + f with n the nearest integer, 2^f by the polynomial of degree 4 through f(0) = 1 with the
// least relative error on [-1/2, 1/2] (2.9e-6, a 1300th of bf16's half step; found as a linear program over 4001 points), n added to the
// exponent.  The row sum takes the same values in fp32, so that o stays their weighted mean; lse carries their error, at most 2.9e-6 absolute.  x is at most 8 here.  At -127 and below, masked scores among them, the result is exactly zero (1.0's exponent less 127):
// a masked key's value counts for nothing however large.  Between -127 and -126 it is below 2^-126, and of a NaN it is zero: the row's
// other exponentials keep it.
__device__ __forceinline__ float2 ex2_fma(float2 x) {
  const float magic = 12582912.f;                 // 1.5 * 2^23: the sum's low bits are the nearest integer
  x.x = fmaxf(x.x, -127.f); x.y = fmaxf(x.y, -127.f);
  const float2 t = add_f32x2(x, make_float2(magic, magic)), n = add_f32x2(t, make_float2(-magic, -magic));
  const float2 f = fma_f32x2(n, make_float2(-1.f, -1.f), x);
  float2 p = fma_f32x2(make_float2(0.009582852945f, 0.009582852945f), f, make_float2(0.05590642616f, 0.05590642616f));
  p = fma_f32x2(p, f, make_float2(0.2402409911f, 0.2402409911f));
  p = fma_f32x2(p, f, make_float2(0.6931241751f, 0.6931241751f));
  p = fma_f32x2(p, f, make_float2(1.f, 1.f));
  return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)),
                     __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}

// Which of a thread's 16 pairs of a quarter row take the FMA units, as a mask: one in eight.  8192 tokens, 16 heads, causal, us for
// none / 1/8 / 1/4 / 3/8 / 1/2: heads of 128 230 / 231 / 229 / 235 / 244, heads of 64 211 / 191 / 200 / 198 / 206.
constexpr uint32_t FWD_FMA = 0x8080;

// X: the keys are those of other sequences (cross attention), which may have none; a template, so that the registers of a row of scores
// are as many as they are without.
template <int DT, int NT, bool X>
__global__ void __launch_bounds__(FwdShape<DT, NT>::kThreads, FwdShape<DT, NT>::kBlocks)
attn_packed_fwd_tc_kernel(const __grid_constant__ PackedArgs a, const __grid_constant__ TcMaps maps, int units, int pair_heads) {
  using S = FwdShape<DT, NT>;
  constexpr int kCopy = S::kWarps, kIssue = kCopy + 1;                 // the warps that copy and issue
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sptr = smem_raw + (base - raw);
  const uint32_t sQ = base, sK = sQ + NT * S::kTile, sV = sK + S::kStages * S::kTile, bars = sV + S::kStages * S::kTile;
  const uint32_t bar_q = bars;
  auto k_full = [&](int i) { return bars + 8 * (1 + i); };
  auto k_empty = [&](int i) { return bars + 8 * (1 + S::kStages + i); };
  auto v_full = [&](int i) { return bars + 8 * (1 + 2 * S::kStages + i); };
  auto v_empty = [&](int i) { return bars + 8 * (1 + 3 * S::kStages + i); };
  auto s_full = [&](int t) { return bars + 8 * (1 + 4 * S::kStages + t); };
  auto p_full = [&](int t) { return bars + 8 * (1 + 4 * S::kStages + NT + t); };
  auto o_full = [&](int t) { return bars + 8 * (1 + 4 * S::kStages + 2 * NT + t); };
  auto p_half = [&](int t) { return bars + 8 * (1 + 4 * S::kStages + 3 * NT + t); };
  auto s_read = [&](int t) { return bars + 8 * (1 + 4 * S::kStages + 4 * NT + t); };
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(sptr + (bars - base) + 8 * S::kBars);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* const status = &g_attn_packed_status;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // Barriers, tensor memory and the tile's place at the same time; the first copies go out as soon as the copying warp knows its tile.
  if (warp == kCopy && lane == 0) {
    mbar_init(bar_q, 1);
    for (int i = 0; i < S::kStages; ++i) { mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1); mbar_init(v_full(i), 1); mbar_init(v_empty(i), 1); }
    for (int t = 0; t < NT; ++t) { mbar_init(s_full(t), 1); mbar_init(s_read(t), 4); mbar_init(p_half(t), 4); mbar_init(p_full(t), 4); mbar_init(o_full(t), 1); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&maps.q);
    tma_prefetch_desc(&maps.k);
    tma_prefetch_desc(&maps.v);
  }
  if (warp == kIssue) {
    tmem_alloc(smem_u32(tmem_slot), S::kCols);
    tmem_relinquish();
  }
  const int log_rows = pair_heads ? TC_LOG_ROWS : TC_LOG_ROWS + NT - 1, rows = 1 << log_rows;
  const int parts = NT == 1 ? (int)cg::this_cluster().num_blocks() : 1, part = NT == 1 ? (int)cg::this_cluster().block_rank() : 0;
  const int block = blockIdx.x / parts, unit = block % units;
  SeqTile ks;
  SeqTile s;
  if constexpr (X) s = find_longest(a.cu, a.cu_kv, a.n_seqs, a.tokens, a.kv_tokens, block / units, log_rows, ks);
  else ks = s = find_tile(a.cu, a.n_seqs, a.tokens, block / units, log_rows);
  if (s.tile < 0) {
    __syncthreads();
    if (warp == kIssue) tmem_dealloc(*tmem_slot, S::kCols);
    return;
  }
  // the last tiles of a sequence see the most keys: they come first
  const int tile = ((s.len + rows - 1) >> log_rows) - 1 - s.tile;
  auto head_of = [&](int t) { return pair_heads ? unit * 2 + t : unit; };
  auto first_of = [&](int t) { return pair_heads ? tile * TC_ROWS : (tile * NT + t) * TC_ROWS; };
  auto keys_of = [&](int t) {                     // key tiles that query tile t sees
    const int q0 = first_of(t);
    return q0 >= s.len ? 0 : ((!X && a.causal ? min(s.len, q0 + TC_ROWS) : ks.len) + TC_ROWS - 1) / TC_ROWS;
  };
  const int hk = head_of(0) / a.group;
  // of the key tiles, this block's share
  const int j0 = NT == 1 ? keys_of(0) * part / parts : 0;
  const int n_keys = NT == 1 ? keys_of(0) * (part + 1) / parts - j0 : max(keys_of(0), keys_of(NT - 1));
  auto count_of = [&](int t) { return NT == 1 ? n_keys : keys_of(t); };

  auto copy_keys = [&](int j) {
    const int st = j % S::kStages;
    if (elect_one()) { mbar_arrive_expect_tx(k_full(st), S::kTile); load_tile<DT>(sK + st * S::kTile, &maps.k, k_full(st), hk, ks.begin + (j0 + j) * TC_ROWS); }
    __syncwarp();
  };
  auto copy_values = [&](int j) {
    const int st = j % S::kStages;
    if (elect_one()) { mbar_arrive_expect_tx(v_full(st), S::kTile); load_tile<DT>(sV + st * S::kTile, &maps.v, v_full(st), hk, ks.begin + (j0 + j) * TC_ROWS); }
    __syncwarp();
  };
  if (warp == kCopy && n_keys > 0) {
    __syncwarp();
    if (elect_one()) {
      int bytes = 0;
      for (int t = 0; t < NT; ++t) if (keys_of(t)) bytes += S::kTile;
      mbar_arrive_expect_tx(bar_q, bytes);
      for (int t = 0; t < NT; ++t)
        if (keys_of(t)) load_tile<DT>(sQ + t * S::kTile, &maps.q, bar_q, head_of(t), s.begin + first_of(t));
    }
    __syncwarp();
    copy_keys(0);
    copy_values(0);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto col_s = [&](int t) { return tmem + t * 128; };
  auto col_o = [&](int t) { return tmem + NT * 128 + t * DT; };
  auto col_p = [&](int t) { return S::kApart ? tmem + NT * (128 + DT) + t * 64 : col_s(t); };

  if (warp >= S::kWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kOtherRegs));
    if (n_keys == 0) {                              // nothing of a shared block's keys
    } else if (warp == kCopy) {                     // ---- copies
      int armed_k = 1, armed_v = 1;
      bool ok = true;
      for (int j = 1; j < n_keys && ok; ++j) {
        const int st = j % S::kStages;
        const uint32_t ph = (j / S::kStages - 1) & 1;
        if (j >= S::kStages) ok = wait_for(k_empty(st), ph, abort_flag, status, 31);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        copy_keys(j);
        ++armed_k;
        if (j >= S::kStages) ok = wait_for(v_empty(st), ph, abort_flag, status, 32);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        copy_values(j);
        ++armed_v;
      }
      if (*abort_flag) {                            // nothing may be in flight when the block ends
        volatile int never = 0;
        wait_for(bar_q, 0, &never, status, 33);
        for (int j = max(0, armed_k - S::kStages); j < armed_k; ++j) wait_for(k_full(j % S::kStages), (j / S::kStages) & 1, &never, status, 33);
        for (int j = max(0, armed_v - S::kStages); j < armed_v; ++j) wait_for(v_full(j % S::kStages), (j / S::kStages) & 1, &never, status, 33);
      }
    } else if (warp == kIssue) {                    // ---- products
      const uint32_t id_s = make_idesc_mn(128, 128, 0, 0), id_o = make_idesc_mn(128, DT, 0, 1);
      bool ok = wait_for(bar_q, 0, abort_flag, status, 34) && wait_for(k_full(0), 0, abort_flag, status, 35);
      if (ok) {
        tc_fence_after();
        if (elect_one()) {
          for (int t = 0; t < NT; ++t)
            if (count_of(t)) { mma_abt<DT>(col_s(t), sQ + t * S::kTile, sK, id_s); tc_commit(s_full(t)); }
          tc_commit(k_empty(0));
        }
        __syncwarp();
      }
      auto values = [&](int t, int j) {             // O += P V, the first half of the keys as soon as their probabilities are there
        const uint32_t v = sV + (j % S::kStages) * S::kTile;
        if (!wait_for(p_half(t), j & 1, abort_flag, status, 38)) return false;
        tc_fence_after();
        if (elect_one()) mma_ab<DT>(col_o(t), col_p(t), v, id_o, j > 0, 0);
        __syncwarp();
        if (!wait_for(p_full(t), j & 1, abort_flag, status, 38)) return false;
        tc_fence_after();
        if (elect_one()) mma_ab<DT>(col_o(t), col_p(t), v, id_o, true, 1);
        __syncwarp();
        return true;
      };
      auto scores = [&](int t, int j) {
        if (elect_one()) { mma_abt<DT>(col_s(t), sQ + t * S::kTile, sK + (j % S::kStages) * S::kTile, id_s); tc_commit(s_full(t)); }
        __syncwarp();
      };
      auto done = [&](uint32_t bar) {
        if (elect_one()) tc_commit(bar);
        __syncwarp();
      };
      for (int j = 0; j < n_keys && ok; ++j) {
        const int st = j % S::kStages, nx = (j + 1) % S::kStages;
        const bool more = j + 1 < n_keys;
        auto next_keys = [&]() { return wait_for(k_full(nx), ((j + 1) / S::kStages) & 1, abort_flag, status, 37); };
        if constexpr (S::kApart) {
          if (more) {
            ok = next_keys();
#pragma unroll
            for (int t = 0; t < NT; ++t)
              if (ok && j + 1 < count_of(t)) {
                ok = wait_for(s_read(t), j & 1, abort_flag, status, 42);
                tc_fence_after();
                if (ok) scores(t, j + 1);
              }
            if (!ok) break;
            done(k_empty(nx));
          }
          ok = wait_for(v_full(st), (j / S::kStages) & 1, abort_flag, status, 36);
#pragma unroll
          for (int t = 0; t < NT; ++t)
            if (ok && j < count_of(t)) {
              ok = values(t, j);
              if (ok) done(o_full(t));
            }
          if (!ok) break;
          done(v_empty(st));
        } else {
          ok = wait_for(v_full(st), (j / S::kStages) & 1, abort_flag, status, 36);
          // with one stage the next keys are copied only behind the previous product's commit: waited for below
          if (ok && more && S::kStages > 1) ok = next_keys();
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const int n = count_of(t);
            if (!ok || j >= n) continue;
            ok = values(t, j);
            if (ok && S::kStages == 1 && j + 1 < n) ok = next_keys();
            if (!ok) continue;
            tc_fence_after();
            if (j + 1 < n) scores(t, j + 1);
            else done(o_full(t));
          }
          if (!ok) break;
          done(v_empty(st));
          if (more) done(k_empty(nx));
        }
      }
    }
    if (NT == 1 && parts > 1) {
      __syncwarp();
      cluster_sync_all();
      cluster_sync_all();
    }
  } else {                                        // ---- softmax: thread = row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kSoftmaxRegs));
    const int t = warp >> 2, r = threadIdx.x & 127;
    const int n = count_of(t), q0 = first_of(t), row = q0 + r;
    if (X && ks.len == 0) {                       // no keys: zeros
      if (parts > 1) {                            // as the other warps do
        __syncwarp();
        cluster_sync_all();
        cluster_sync_all();
      }
      if (part == 0 && row < s.len) {
        const int h = head_of(t);
        uint4* const out = reinterpret_cast<uint4*>(head_row_out<__nv_bfloat16>(a.o, s.begin + row, h));
        for (int i = 0; i < a.dim / 8; ++i) out[i] = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse) a.lse[(int64_t)h * a.tokens + s.begin + row] = -INFINITY;
      }
    } else if (n > 0 || parts > 1) {
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t ts = col_s(t) + lanes, to = col_o(t) + lanes, tp = col_p(t) + lanes;
      const float c = a.scale * kLog2e;
      const int limit = !X && a.causal ? min(s.len, row + 1) : ks.len;      // keys this row sees
      float m = -INFINITY, l = 0.f;               // m: the maximum in use, times c
      bool ok = true;
      for (int j = 0; j < n; ++j) {
        ok = wait_for(s_full(t), j & 1, abort_flag, status, 39);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const int k0 = (j0 + j) * TC_ROWS;
        const bool edge = k0 + TC_ROWS > ks.len || (!X && a.causal && k0 + TC_ROWS > q0 + 1);
        // The rows behind the sequence's end of its last value tile belong to other sequences, or to none: zeros, as p is there, so
        // that nothing that is not finite meets a zero.  The first query tile that reads the tile clears it.
        if (k0 + TC_ROWS > ks.len && (t == 0 || keys_of(0) <= j)) {
          const int st = j % S::kStages, valid = ks.len - k0;
          ok = wait_for(v_full(st), (j / S::kStages) & 1, abort_flag, status, 40);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          for (int i = valid * 8 + r; i < TC_ROWS * 8; i += 128)
#pragma unroll
            for (int q = 0; q < S::kSub; ++q)
              *reinterpret_cast<uint4*>(sptr + (sV - base) + st * S::kTile + q * TC_SUB + i * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_async_smem();
        }
        uint32_t v[4][32];
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(ts + q * 32, v[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld_wait(v[q]);
        if (S::kApart) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(s_read(t));
        }
        if (edge) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (k0 + q * 32 + i >= limit) v[q][i] = 0xFF800000u;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 2)
#pragma unroll
          for (int q = 0; q < 4; ++q) mx[q] = max3_nan(mx[q], __uint_as_float(v[q][i]), __uint_as_float(v[q][i + 1]));
        // a NaN or +infinity among the scores: no distribution; the maximum says so to every exponential of the row
        float top = max3_nan(mx[0], mx[1], max_nan(mx[2], mx[3])) * c;
        if (top == INFINITY) top = NAN;
        if (S::kApart && j > 0) {                 // P's columns are free, and O holds the tiles before this one
          ok = wait_for(o_full(t), (j - 1) & 1, abort_flag, status, 43);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
        }
        if (j == 0) {
          m = top;
        } else if (__any_sync(0xffffffffu, !(top <= m + 8.f))) {
          // rows that need it not keep theirs, those without a finite score so far among them
          const float up = top <= m + 8.f ? m : max_nan(m, top), f = up == -INFINITY ? 1.f : ex2(m - up);
          m = up;
          l *= f;
#pragma unroll
          for (int q = 0; q < DT / 16; ++q) {
            uint32_t o[16];
            tmem_ld16(to + q * 16, o);
            tmem_ld_wait(o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st16(to + q * 16, o);
          }
        }
        float2 sum = make_float2(0.f, 0.f);
        const float shift = m == -INFINITY ? 0.f : -m;       // no finite score so far: nothing but zeros
        const float2 cc = make_float2(c, c), mm = make_float2(shift, shift);
        auto probabilities = [&](const uint32_t (&x)[32], int q) {
          uint32_t p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float2 e = fma_f32x2(make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), cc, mm);
            if (FWD_FMA >> i & 1) e = ex2_fma(e);
            else { e.x = ex2(e.x); e.y = ex2(e.y); }
            sum = add_f32x2(sum, e);
            p[i] = pack_bf16(e.x, e.y);
          }
          tmem_st16(tp + q * 16, p);
        };
        probabilities(v[0], 0);                   // P overwrites scores that are in registers
        probabilities(v[1], 1);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_half(t));
        probabilities(v[2], 2);
        probabilities(v[3], 3);
        l += sum.x + sum.y;
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(t));
      }
      if (ok && n > 0) ok = wait_for(o_full(t), S::kApart ? (n - 1) & 1 : 0, abort_flag, status, 41);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      const int h = head_of(t);
      if (NT == 1 && parts > 1) {                 // the tiles in shared memory have been read
        float* const sums = reinterpret_cast<float*>(sptr);
        float* const stats = sums + TC_ROWS * kSumLd<DT>;              // maximum, sum [2][128], then weights [parts][128]
        float* const weights = stats + 2 * TC_ROWS;
        static_assert((TC_ROWS * kSumLd<DT> + 10 * TC_ROWS) * 4 <= (NT + 2 * S::kStages) * S::kTile, "sums of a shared block");
        cg::cluster_group cluster = cg::this_cluster();
        for (int c0 = 0; c0 < DT; c0 += 32) leave_sums<DT>(sums + r * kSumLd<DT>, to, c0, n > 0);
        stats[r] = ok ? m : NAN;
        stats[TC_ROWS + r] = l;
        __syncwarp();
        cluster_sync_all();
        const int r0 = TC_ROWS * part / parts, r1 = TC_ROWS * (part + 1) / parts;
        if (r >= r0 && r < r1) {
          float top = -INFINITY, sum = 0.f;
          for (int p = 0; p < parts; ++p) {
            const float x = cluster.map_shared_rank(stats, p)[r];
            top = top != top || x != x ? NAN : fmaxf(top, x);
          }
          const float base = top == -INFINITY ? 0.f : top;             // every score -infinity: their difference would be NaN, the sum is zero
          for (int p = 0; p < parts; ++p) sum += ex2(cluster.map_shared_rank(stats, p)[r] - base) * cluster.map_shared_rank(stats, p)[TC_ROWS + r];
          for (int p = 0; p < parts; ++p) weights[p * TC_ROWS + r] = ex2(cluster.map_shared_rank(stats, p)[r] - base) / sum;
          if (a.lse && row < s.len) a.lse[(int64_t)h * a.tokens + s.begin + row] = (top + log2f(sum)) * kLn2;
        }
        asm volatile("barrier.cta.sync 1, 128;" ::: "memory");
        finish_rows<DT>(a.o, s, q0, h, a.dim, sums, part, parts, 128, [&](int at, int p) { return weights[p * TC_ROWS + at]; });
        __syncwarp();
        cluster_sync_all();                       // the others have read this block's sums
      } else {
        const float inv = 1.f / l;
        if (a.lse && row < s.len) a.lse[(int64_t)h * a.tokens + s.begin + row] = ok ? (m + log2f(l)) * kLn2 : NAN;
        const int first_row = q0 + (warp & 3) * 32;
#pragma unroll
        for (int q = 0; q < DT / 32; ++q)             // Q's tile has been read
          store_rows(head_row_out<__nv_bfloat16>(a.o, s.begin + first_row, h), a.o.token, s.len - first_row, to, q * 32, a.dim, inv, ok,
                     sptr + t * S::kTile + (warp & 3) * 2048);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssue) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kCols);
  }
}

// ---- forward, cross attention of heads of up to 64, more tiles than blocks run at a time -----------------------------
//
// The same work by blocks that stay: a block takes query tiles in turn, and the copies and products of the next tile run while the
// softmax warps bring the last one's rows out; in short sequences the ends of a tile (its place, the first copies, the barriers between
// the first products and the last rows) are most of its time.  16 x 256 tokens over 100 to 475 keys, 16 heads of 64: 19.1 us with a block to
// a tile, 17.0 with these; 100 x 100 over 300, 64 and 46; 4096 over 8192, 213 and 205.
//
// Key tiles are counted through all tiles of a block: g-th of all, in stage g mod 2, its barriers' phases by g.  The places of a block's
// tiles, 32 at most, are found at the start by all its warps.

struct StreamTile {
  int64_t row, key;                               // first rows of the sequence, in q and o and in k and v
  int len, q0, head, n_keys, key_len;             // rows of the sequence, the tile's first; key tiles and keys; -1 key tiles: no such tile
};
struct StreamShape {
  static constexpr int kTile = TC_SUB;            // [128 x 64]
  static constexpr int kStages = 2, kMost = 32;
  static constexpr int kCols = 256;               // S 128, O 64, P 64
  static constexpr int kThreads = 256;
  static constexpr int kStaging = 4 * 2048;
  static constexpr int kBars = 2 + 2 + 4 * kStages + 6;
  static constexpr int kSmem = 2 * kTile + 2 * kStages * kTile + kStaging + 1024 + kBars * 8 + kMost * (int)sizeof(StreamTile) + 16;
  static constexpr int kSoftmaxRegs = 208, kOtherRegs = 48;          // of 256 x 128 that are launched
};

// the block's i-th unit: forth through one round of blocks, back through the next, so that longer tiles and shorter ones behind them even out
__device__ __forceinline__ int64_t stream_unit(int i) { return (int64_t)i * gridDim.x + (i & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x); }

__global__ void __launch_bounds__(StreamShape::kThreads, 2)
attn_cross_stream_kernel(const __grid_constant__ PackedArgs a, const __grid_constant__ TcMaps maps, int units) {
  using S = StreamShape;
  constexpr int DT = 64, kCopy = 4, kIssue = 5;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sptr = smem_raw + (base - raw);
  const uint32_t sQ = base, sK = sQ + 2 * S::kTile, sV = sK + S::kStages * S::kTile, staging = sV + S::kStages * S::kTile, bars = staging + S::kStaging;
  auto q_full = [&](int i) { return bars + 8 * i; };
  auto q_empty = [&](int i) { return bars + 8 * (2 + i); };
  auto k_full = [&](int i) { return bars + 8 * (4 + i); };
  auto k_empty = [&](int i) { return bars + 8 * (6 + i); };
  auto v_full = [&](int i) { return bars + 8 * (8 + i); };
  auto v_empty = [&](int i) { return bars + 8 * (10 + i); };
  const uint32_t s_full = bars + 8 * 12, s_read = s_full + 8, p_half = s_full + 16, p_full = s_full + 24, o_full = s_full + 32, o_read = s_full + 40;
  static_assert(S::kBars == 18);
  StreamTile* const tiles = reinterpret_cast<StreamTile*>(sptr + (bars - base) + 8 * S::kBars);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(tiles + S::kMost);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* const status = &g_attn_packed_status;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == kCopy && lane == 0) {
    for (int i = 0; i < 2; ++i) { mbar_init(q_full(i), 1); mbar_init(q_empty(i), 1); mbar_init(k_full(i), 1); mbar_init(k_empty(i), 1); mbar_init(v_full(i), 1); mbar_init(v_empty(i), 1); }
    mbar_init(s_full, 1); mbar_init(s_read, 4); mbar_init(p_half, 4); mbar_init(p_full, 4); mbar_init(o_full, 1); mbar_init(o_read, 4);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&maps.q);
    tma_prefetch_desc(&maps.k);
    tma_prefetch_desc(&maps.v);
  }
  if (warp == kIssue) {
    tmem_alloc(smem_u32(tmem_slot), S::kCols);
    tmem_relinquish();
  }
  const int64_t all = (a.tokens / TC_ROWS + a.n_seqs) * units;       // as most_tiles counts them
  int n_tiles = 0;
  while (n_tiles < S::kMost && stream_unit(n_tiles) < all) ++n_tiles;
  for (int i = warp; i < n_tiles; i += S::kThreads / 32) {
    const int64_t unit = stream_unit(i);
    SeqTile ks;
    const SeqTile s = find_longest(a.cu, a.cu_kv, a.n_seqs, a.tokens, a.kv_tokens, (int)(unit / units), TC_LOG_ROWS, ks);
    if (lane == 0)
      tiles[i] = s.tile < 0 ? StreamTile{0, 0, 0, 0, 0, -1, 0}
                            : StreamTile{s.begin, ks.begin, s.len, s.tile * TC_ROWS, (int)(unit % units), (ks.len + TC_ROWS - 1) / TC_ROWS, ks.len};
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, col_s = tmem, col_o = tmem + 128, col_p = tmem + 192;

  if (warp >= 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::kOtherRegs));
    if (warp == kCopy) {                          // ---- places and copies
      int r = 0, g = 0;                           // tiles with keys, key tiles
      bool ok = true;
      for (int i = 0; i < n_tiles && ok; ++i) {
        const int n_keys = tiles[i].n_keys, hk = tiles[i].head / a.group;
        const int64_t key = tiles[i].key;
        if (n_keys <= 0) continue;
        if (r >= 2) ok = wait_for(q_empty(r & 1), (r / 2 - 1) & 1, abort_flag, status, 131);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (elect_one()) {
          mbar_arrive_expect_tx(q_full(r & 1), S::kTile);
          load_tile<DT>(sQ + (r & 1) * S::kTile, &maps.q, q_full(r & 1), tiles[i].head, tiles[i].row + tiles[i].q0);
        }
        __syncwarp();
        ++r;
        for (int j = 0; j < n_keys; ++j, ++g) {
          const int st = g & 1;
          const uint32_t ph = (g / 2 - 1) & 1;
          if (g >= 2) ok = wait_for(k_empty(st), ph, abort_flag, status, 132);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (elect_one()) { mbar_arrive_expect_tx(k_full(st), S::kTile); load_tile<DT>(sK + st * S::kTile, &maps.k, k_full(st), hk, key + j * TC_ROWS); }
          __syncwarp();
          if (g >= 2) ok = wait_for(v_empty(st), ph, abort_flag, status, 133);
          ok = __all_sync(0xffffffffu, ok);
          if (elect_one()) {                      // armed even when the wait ran out: as many values as keys have to be waited for
            mbar_arrive_expect_tx(v_full(st), ok ? S::kTile : 0);
            if (ok) load_tile<DT>(sV + st * S::kTile, &maps.v, v_full(st), hk, key + j * TC_ROWS);
          }
          __syncwarp();
          if (!ok) { ++g; break; }
        }
      }
      if (*abort_flag) {                          // nothing may be in flight when the block ends
        volatile int never = 0;
        for (int i = max(0, r - 2); i < r; ++i) wait_for(q_full(i & 1), (i / 2) & 1, &never, status, 134);
        for (int i = max(0, g - 2); i < g; ++i) {
          wait_for(k_full(i & 1), (i / 2) & 1, &never, status, 134);
          wait_for(v_full(i & 1), (i / 2) & 1, &never, status, 134);
        }
      }
    } else if (warp == kIssue) {                  // ---- products
      const uint32_t id_s = make_idesc_mn(128, 128, 0, 0);
      int n = 0, left = 0;                        // tiles so far; key tiles of the last of them without scores
      int r = -1, g_s = 0;                        // its number among those with keys; key tiles with scores
      // S of the next key tile of all, if there is one
      auto scores = [&](bool& any) {
        any = false;
        while (left == 0) {
          if (n == n_tiles) return true;
          left = max(tiles[n++].n_keys, 0);
          if (left == 0) continue;
          ++r;
          if (!wait_for(q_full(r & 1), (r / 2) & 1, abort_flag, status, 136)) return false;
        }
        if (!wait_for(k_full(g_s & 1), (g_s / 2) & 1, abort_flag, status, 137)) return false;
        if (g_s > 0 && !wait_for(s_read, (g_s - 1) & 1, abort_flag, status, 138)) return false;
        tc_fence_after();
        if (elect_one()) {
          mma_abt<DT>(col_s, sQ + (r & 1) * S::kTile, sK + (g_s & 1) * S::kTile, id_s);
          tc_commit(s_full);
          tc_commit(k_empty(g_s & 1));
          if (left == 1) tc_commit(q_empty(r & 1));
        }
        __syncwarp();
        --left;
        ++g_s;
        any = true;
        return true;
      };
      const uint32_t id_o = make_idesc_mn(128, DT, 0, 1);
      bool more;
      bool ok = scores(more);
      int first = 0, tile = 0;                    // key tiles before this tile's first; tiles whose values have begun
      int next_first = ok && more ? left + 1 : 0; // key tiles up to the end of the tile with the last scores
      for (int g = 0; ok && more; ++g) {
        const int end = next_first;               // of the tile that g belongs to, as its scores were the last
        ok = scores(more);
        if (!ok) break;
        if (more && g + 1 == end) next_first = end + left + 1;
        const uint32_t v = sV + (g & 1) * S::kTile;
        ok = wait_for(v_full(g & 1), (g / 2) & 1, abort_flag, status, 139) && wait_for(p_half, g & 1, abort_flag, status, 140);
        if (ok && g == first && tile > 0) ok = wait_for(o_read, (tile - 1) & 1, abort_flag, status, 141);      // the last tile's rows have left O
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) mma_ab<DT>(col_o, col_p, v, id_o, g > first, 0);
        __syncwarp();
        ok = wait_for(p_full, g & 1, abort_flag, status, 142);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          mma_ab<DT>(col_o, col_p, v, id_o, true, 1);
          tc_commit(o_full);
          tc_commit(v_empty(g & 1));
        }
        __syncwarp();
        if (g + 1 == end) { first = end; ++tile; }
      }
    }
  } else {                                        // ---- softmax: thread = row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::kSoftmaxRegs));
    const int row_in = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16, ts = col_s + lanes, to = col_o + lanes, tp = col_p + lanes;
    const float c = a.scale * kLog2e;
    int g = 0, n = 0;                             // key tiles, tiles
    bool ok = true;
    for (; n < n_tiles; ++n) {
      const StreamTile& t = tiles[n];
      const int n_keys = t.n_keys;
      if (n_keys < 0) continue;
      if (n_keys == 0) {                          // no keys: zeros
        const int row = t.q0 + row_in;
        if (row < t.len) {
          uint4* const out = reinterpret_cast<uint4*>(head_row_out<__nv_bfloat16>(a.o, t.row + row, t.head));
          for (int i = 0; i < a.dim / 8; ++i) out[i] = make_uint4(0u, 0u, 0u, 0u);
          if (a.lse) a.lse[(int64_t)t.head * a.tokens + t.row + row] = -INFINITY;
        }
        continue;
      }
      float m = -INFINITY, l = 0.f;               // m: the maximum in use, times c
      for (int j = 0; j < n_keys; ++j, ++g) {
        ok = wait_for(s_full, g & 1, abort_flag, status, 144);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const int valid = t.key_len - j * TC_ROWS;
        if (valid < TC_ROWS) {                    // rows behind the last key: zeros, as p is there
          ok = wait_for(v_full(g & 1), (g / 2) & 1, abort_flag, status, 145);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          for (int i = valid * 8 + row_in; i < TC_ROWS * 8; i += 128)
            *reinterpret_cast<uint4*>(sptr + (sV - base) + (g & 1) * S::kTile + i * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_async_smem();
        }
        uint32_t v[4][32];
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(ts + q * 32, v[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld_wait(v[q]);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_read);
        if (valid < TC_ROWS) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (q * 32 + i >= valid) v[q][i] = 0xFF800000u;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 2)
#pragma unroll
          for (int q = 0; q < 4; ++q) mx[q] = max3_nan(mx[q], __uint_as_float(v[q][i]), __uint_as_float(v[q][i + 1]));
        // a NaN or +infinity among the scores: no distribution; the maximum says so to every exponential of the row
        float top = max3_nan(mx[0], mx[1], max_nan(mx[2], mx[3])) * c;
        if (top == INFINITY) top = NAN;
        if (j > 0) {                              // P's columns are free, and O holds the tiles before this one
          ok = wait_for(o_full, (g - 1) & 1, abort_flag, status, 146);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
        }
        if (j == 0) {
          m = top;
        } else if (__any_sync(0xffffffffu, !(top <= m + 8.f))) {
          const float up = top <= m + 8.f ? m : max_nan(m, top), f = up == -INFINITY ? 1.f : ex2(m - up);
          m = up;
          l *= f;
#pragma unroll
          for (int q = 0; q < DT / 16; ++q) {
            uint32_t o[16];
            tmem_ld16(to + q * 16, o);
            tmem_ld_wait(o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st16(to + q * 16, o);
          }
        }
        float2 sum = make_float2(0.f, 0.f);
        const float shift = m == -INFINITY ? 0.f : -m;       // no finite score so far: nothing but zeros
        const float2 cc = make_float2(c, c), mm = make_float2(shift, shift);
        auto probabilities = [&](const uint32_t (&x)[32], int q) {
          uint32_t p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float2 e = fma_f32x2(make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), cc, mm);
            if (FWD_FMA >> i & 1) e = ex2_fma(e);
            else { e.x = ex2(e.x); e.y = ex2(e.y); }
            sum = add_f32x2(sum, e);
            p[i] = pack_bf16(e.x, e.y);
          }
          tmem_st16(tp + q * 16, p);
        };
        probabilities(v[0], 0);
        probabilities(v[1], 1);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_half);
        probabilities(v[2], 2);
        probabilities(v[3], 3);
        l += sum.x + sum.y;
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full);
      }
      if (ok) ok = wait_for(o_full, (g - 1) & 1, abort_flag, status, 147);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const int row = t.q0 + row_in, first_row = t.q0 + warp * 32, h = t.head;
      if (a.lse && row < t.len) a.lse[(int64_t)h * a.tokens + t.row + row] = (m + log2f(l)) * kLn2;
      const float inv = 1.f / l;
#pragma unroll
      for (int q = 0; q < DT / 32; ++q)
        store_rows(head_row_out<__nv_bfloat16>(a.o, t.row + first_row, h), a.o.token, t.len - first_row, to, q * 32, a.dim, inv, true,
                   sptr + (staging - base) + warp * 2048);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_read);
    }
    for (; n < n_tiles; ++n) {                    // where a wait ran out, the rows that are left: NaN
      const StreamTile& t = tiles[n];
      const int row = t.q0 + row_in;
      if (t.n_keys < 0 || row >= t.len) continue;
      uint4* const out = reinterpret_cast<uint4*>(head_row_out<__nv_bfloat16>(a.o, t.row + row, t.head));
      for (int q = 0; q < a.dim / 8; ++q) out[q] = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
      if (a.lse) a.lse[(int64_t)t.head * a.tokens + t.row + row] = NAN;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssue) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kCols);
  }
}

// ---- backward ---------------------------------------------------------------------------------------------------
//
// Two kinds of blocks, as on the CUDA cores: one owns 128 key rows (dk, dv), one 128 query rows (dq); every gradient is summed by one
// block in a fixed order.  Seven products a pair of tiles instead of the five that sharing the scores would take, and no atomics,
// no fp32 copy of dq in memory.  Both have the shape  two products -> 128 x BN values in registers -> bf16 factors in tensor
// memory -> one or two products that accumulate; a thread holds 32 values of one row.
//
// Keys:     S^T = K Q^T, dP^T = V dO^T;  P^T = 2^(c S^T - lse), dS^T = P^T (dP^T - delta);  dV += P^T dO,  dK += dS^T Q
//           Transposed, so that P^T and dS^T are what the products take from tensor memory and nothing is written to shared
//           memory; lse and delta go by column and are read from shared memory.  P^T overwrites S^T and dS^T dP^T, each part
//           of the columns its own.
// Queries:  S = Q K^T, dP = dO V^T;  dS as above, by rows;  dQ += dS K.  S is double-buffered; dS overwrites dP.
//
// Heads of 128: BN = 128, all 512 columns of tensor memory, one block of 18 warps per SM.  Heads of 64: BN = 64 and 256 columns, so
// that two blocks share an SM and one's copies and epilogue run under the other's work (most of the time of short sequences).

template <int DT> struct BwdShape {
  static constexpr int kCols = DT == 64 ? 64 : 128;                  // BN: columns of a tile of values
  static constexpr int kParts = kCols / 32;                          // threads to a row
  static constexpr int kBlocks = DT == 64 ? 2 : 1;                   // per SM
  static constexpr int kSub = DT / 64;
  static constexpr int kTile = kSub * TC_SUB;                        // a resident tile: 128 rows
  static constexpr int kStream = kSub * kCols * 128;                 // a streamed one: BN rows
  static constexpr int kStages = DT == 64 ? 3 : 2;
  static constexpr int kThreads = kParts * 128 + 64;
  static constexpr int kTmem = DT == 64 ? 256 : 512;
  static constexpr int kBars = 1 + 3 * kStages + 6;
  static constexpr int kRowBytes = kStages * 2 * kCols * 4;          // lse and delta of the query tiles in flight
  static constexpr int kSmem = 2 * kTile + 2 * kStages * kStream + kRowBytes + 1024 + kBars * 8 + 16;
};

// Copies of ROWS rows of a head, with boxes of BN rows.
template <int DT, int ROWS> __device__ __forceinline__ void copy_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int64_t token) {
  constexpr int kBox = BwdShape<DT>::kCols;
#pragma unroll
  for (int i = 0; i < DT / 64; ++i)
#pragma unroll
    for (int r = 0; r < ROWS; r += kBox) tma_load_3d(dst + (i * ROWS + r) * 128, map, bar, i * 64, head, (int)token + r);
}
// 128 x BN x DT product of a resident and a streamed tile
template <int DT> __device__ __forceinline__ void mma_scores(uint32_t d, uint32_t a, uint32_t b) {
  using S = BwdShape<DT>;
  a = own_address(a); b = own_address(b);
  const uint64_t base = desc_base(16, 1024);
  const uint32_t idesc = make_idesc_mn(128, S::kCols, 0, 0);
#pragma unroll
  for (int k = 0; k < DT / 16; ++k)
    tc_mma_bf16(d, desc_at(base, a + (k >> 2) * TC_SUB + (k & 3) * 32), desc_at(base, b + (k >> 2) * S::kCols * 128 + (k & 3) * 32), idesc, k > 0);
}
// 128 x DT x BN product of factors in tensor memory (16 columns of every 32) and a streamed tile whose rows run along the depth
template <int DT> __device__ __forceinline__ void mma_gradient(uint32_t d, uint32_t a, uint32_t b, bool accumulate) {
  using S = BwdShape<DT>;
  b = own_address(b);
  const uint64_t base = desc_base(S::kCols * 128, 1024);
  const uint32_t idesc = make_idesc_mn(128, DT, 0, 1);
#pragma unroll
  for (int k = 0; k < S::kCols / 16; ++k) tc_mma_bf16_ta(d, a + (k >> 1) * 32 + (k & 1) * 8, desc_at(base, b + k * 2048), idesc, accumulate || k > 0);
}
// zeros in rows `valid` .. BN - 1 of a streamed tile, by one warp
template <int DT> __device__ __forceinline__ void clear_rows(uint8_t* tile, int valid) {
  using S = BwdShape<DT>;
  for (int i = valid * 8 + (threadIdx.x & 31); i < S::kCols * 8; i += 32)
#pragma unroll
    for (int q = 0; q < S::kSub; ++q) *reinterpret_cast<uint4*>(tile + q * S::kCols * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
}
struct TcBwdMaps { CUtensorMap q, k, v, d_o; };

// 32 columns of a row
__device__ __forceinline__ void zero_columns(__nv_bfloat16* row, int c0, int dim) {
#pragma unroll
  for (int c = c0; c < c0 + 32; c += 8) if (c < dim) *reinterpret_cast<uint4*>(row + c) = make_uint4(0u, 0u, 0u, 0u);
}

template <int DT, bool X> __device__ __forceinline__ void dkv_block(const PackedArgs& a, const TcBwdMaps& maps, int block, int part, int parts) {
  using S = BwdShape<DT>;
  constexpr int BN = S::kCols, kCopy = S::kParts * 4, kIssue = kCopy + 1;        // the warps that copy and issue
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = block % a.kv_heads;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sptr = smem_raw + (base - raw);
  const uint32_t sK = base, sV = sK + S::kTile, sQ = sV + S::kTile, sO = sQ + S::kStages * S::kStream, srow = sO + S::kStages * S::kStream,
                 bars = srow + S::kRowBytes;
  float* const row_values = reinterpret_cast<float*>(sptr + (srow - base));      // [stage][lse, delta][BN]
  const uint32_t kv_full = bars;
  auto full = [&](int i) { return bars + 8 * (1 + i); };
  auto row_full = [&](int i) { return bars + 8 * (1 + S::kStages + i); };
  auto empty = [&](int i) { return bars + 8 * (1 + 2 * S::kStages + i); };
  const uint32_t s_full = bars + 8 * (1 + 3 * S::kStages), dp_full = s_full + 8, p_full = s_full + 16, ds_full = s_full + 24, acc_full = s_full + 32;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(sptr + (bars - base) + 8 * S::kBars);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* const status = &g_attn_packed_status;

  // barriers, tensor memory and the tile's place at the same time; the first copies go out as soon as the copying warp knows its tile
  if (warp == kCopy && lane == 0) {
    mbar_init(kv_full, 1);
    for (int i = 0; i < S::kStages; ++i) { mbar_init(full(i), 1); mbar_init(row_full(i), 32); mbar_init(empty(i), 1); }
    mbar_init(s_full, 1); mbar_init(dp_full, 1); mbar_init(p_full, S::kParts * 4); mbar_init(ds_full, S::kParts * 4); mbar_init(acc_full, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&maps.k); tma_prefetch_desc(&maps.v); tma_prefetch_desc(&maps.q); tma_prefetch_desc(&maps.d_o);
  }
  if (warp == kIssue) {
    tmem_alloc(smem_u32(tmem_slot), S::kTmem);
    tmem_relinquish();
  }
  SeqTile qs;
  SeqTile s;
  if constexpr (X) s = find_longest(a.cu_kv, a.cu, a.n_seqs, a.kv_tokens, a.tokens, block / a.kv_heads, TC_LOG_ROWS, qs);
  else qs = s = find_tile(a.cu_kv, a.n_seqs, a.kv_tokens, block / a.kv_heads, TC_LOG_ROWS);
  if (s.tile < 0) {
    __syncthreads();
    if (warp == kIssue) tmem_dealloc(*tmem_slot, S::kTmem);
    pdl_wait();
    return;
  }
  const int k0 = s.tile * TC_ROWS, first = !X && a.causal ? k0 : 0;
  // of the query tiles of all heads that share these keys, this block's share
  const int per_head = (qs.len - first + BN - 1) / BN, it0 = per_head * a.group * part / parts, n_it = per_head * a.group * (part + 1) / parts - it0;
  const int some = X ? max(per_head, 1) : per_head, h0 = hk * a.group + it0 / some, first_q0 = first + it0 % some * BN;
  auto copy_queries = [&](int it, int h, int q0) {
    const int st = it % S::kStages;
    if (elect_one()) {
      mbar_arrive_expect_tx(full(st), 2 * S::kStream);
      copy_rows<DT, BN>(sQ + st * S::kStream, &maps.q, full(st), h, qs.begin + q0);
      copy_rows<DT, BN>(sO + st * S::kStream, &maps.d_o, full(st), h, qs.begin + q0);
    }
    __syncwarp();
  };
  if (warp == kCopy && n_it > 0) {
    __syncwarp();
    if (elect_one()) {
      mbar_arrive_expect_tx(kv_full, 2 * S::kTile);
      copy_rows<DT, TC_ROWS>(sK, &maps.k, kv_full, hk, s.begin + k0);
      copy_rows<DT, TC_ROWS>(sV, &maps.v, kv_full, hk, s.begin + k0);
    }
    __syncwarp();
    copy_queries(0, h0, first_q0);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, col_s = tmem, col_dp = tmem + BN, col_dv = tmem + 2 * BN, col_dk = tmem + 2 * BN + DT;

  if (warp == kCopy) {                            // ---- copies
    int armed = 1, h = h0, q0 = first_q0;
    bool ok = true;
    pdl_wait();                                   // delta
    for (int it = 0; it < n_it; ++it) {
      const int st = it % S::kStages;
      if (it >= S::kStages) ok = wait_for(empty(st), (it / S::kStages - 1) & 1, abort_flag, status, 51);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (it > 0) {
        copy_queries(it, h, q0);
        ++armed;
      }
      float* rows = row_values + st * 2 * BN;
#pragma unroll
      for (int i = 0; i < BN; i += 32) {
        const int r = q0 + i + lane;
        const int64_t at = (int64_t)h * a.tokens + qs.begin + r;
        rows[i + lane] = r < qs.len ? a.lse[at] * kLog2e : INFINITY;              // no row: probability zero
        rows[BN + i + lane] = r < qs.len ? a.delta[at] : 0.f;
      }
      if (q0 + BN > qs.len) {                      // rows of other sequences, or of none: zeros, where P and dS are zero
        ok = wait_for(full(st), (it / S::kStages) & 1, abort_flag, status, 52);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        clear_rows<DT>(sptr + (sQ - base) + st * S::kStream, qs.len - q0);
        clear_rows<DT>(sptr + (sO - base) + st * S::kStream, qs.len - q0);
        fence_async_smem();
      }
      mbar_arrive(row_full(st));
      q0 += BN;
      if (q0 >= qs.len) { q0 = first; ++h; }
    }
    if (*abort_flag && n_it > 0) {                // nothing may be in flight when the block ends
      volatile int never = 0;
      wait_for(kv_full, 0, &never, status, 53);
      for (int it = max(0, armed - S::kStages); it < armed; ++it) wait_for(full(it % S::kStages), (it / S::kStages) & 1, &never, status, 53);
    }
  } else if (warp == kIssue) {                    // ---- products
    auto ready = [&](int it) {
      const int st = it % S::kStages;
      return wait_for(full(st), (it / S::kStages) & 1, abort_flag, status, 54) && wait_for(row_full(st), (it / S::kStages) & 1, abort_flag, status, 55);
    };
    bool ok = n_it > 0 && wait_for(kv_full, 0, abort_flag, status, 56) && ready(0);
    if (ok) {
      tc_fence_after();
      if (elect_one()) {
        mma_scores<DT>(col_s, sK, sQ);
        tc_commit(s_full);
        mma_scores<DT>(col_dp, sV, sO);
        tc_commit(dp_full);
      }
      __syncwarp();
    }
    for (int it = 0; it < n_it && ok; ++it) {
      const int st = it % S::kStages, nx = (it + 1) % S::kStages;
      const bool more = it + 1 < n_it;
      ok = wait_for(p_full, it & 1, abort_flag, status, 57);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) mma_gradient<DT>(col_dv, col_s, sO + st * S::kStream, it > 0);
      __syncwarp();
      if (more) {
        ok = ready(it + 1);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) { mma_scores<DT>(col_s, sK, sQ + nx * S::kStream); tc_commit(s_full); }
        __syncwarp();
      }
      ok = wait_for(ds_full, it & 1, abort_flag, status, 58);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        mma_gradient<DT>(col_dk, col_dp, sQ + st * S::kStream, it > 0);
        tc_commit(empty(st));
        if (more) { mma_scores<DT>(col_dp, sV, sO + nx * S::kStream); tc_commit(dp_full); }
        else tc_commit(acc_full);
      }
      __syncwarp();
    }
  } else {                                        // ---- values: thread = key row, 32 of the query columns
    const int c0 = (warp >> 2) * 32, key = k0 + (threadIdx.x & 127);
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = a.scale * kLog2e;
    bool ok = true;
    int q0 = first_q0;
    for (int it = 0; it < n_it; ++it) {
      const int st = it % S::kStages;
      const float* rows = row_values + st * 2 * BN + c0;
      ok = wait_for(row_full(st), (it / S::kStages) & 1, abort_flag, status, 59) && wait_for(s_full, it & 1, abort_flag, status, 60);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      float p[32];
      {
        uint32_t v[32], w[16];
        tmem_ld32(col_s + lanes + c0, v);
        tmem_ld_wait(v);
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float4 l = *reinterpret_cast<const float4*>(rows + i);
          const float2 x = fma_f32x2(make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), make_float2(c, c), make_float2(-l.x, -l.y));
          const float2 y = fma_f32x2(make_float2(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), make_float2(c, c), make_float2(-l.z, -l.w));
          p[i] = ex2(x.x); p[i + 1] = ex2(x.y); p[i + 2] = ex2(y.x); p[i + 3] = ex2(y.y);
        }
        if (!X && a.causal && q0 < k0 + TC_ROWS)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (q0 + c0 + i < key) p[i] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
        tmem_st16(col_s + lanes + c0, w);         // columns of this part, which are in registers
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full);
      ok = wait_for(dp_full, it & 1, abort_flag, status, 61);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      {
        uint32_t v[32], w[16];
        tmem_ld32(col_dp + lanes + c0, v);
        tmem_ld_wait(v);
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float4 d = *reinterpret_cast<const float4*>(rows + BN + i);
          const float2 x = add_f32x2(make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), make_float2(-d.x, -d.y));
          const float2 y = add_f32x2(make_float2(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), make_float2(-d.z, -d.w));
          w[i / 2] = pack_bf16(p[i] * x.x, p[i + 1] * x.y);
          w[i / 2 + 1] = pack_bf16(p[i + 2] * y.x, p[i + 3] * y.y);
        }
        tmem_st16(col_dp + lanes + c0, w);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(ds_full);
      q0 += BN;
      if (q0 >= qs.len) q0 = first;
    }
    if (ok && n_it > 0) ok = wait_for(acc_full, 0, abort_flag, status, 62);
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after();
    if (parts > 1) {                              // the tiles in shared memory have been read
      float* const dk = reinterpret_cast<float*>(sptr);
      float* const dv = dk + TC_ROWS * kSumLd<DT>;
      static_assert(2 * TC_ROWS * kSumLd<DT> * 4 <= 2 * S::kTile + 2 * S::kStages * S::kStream, "sums of a shared block");
      const int r = threadIdx.x & 127;
      leave_sums<DT>(dk + r * kSumLd<DT>, col_dk + lanes, c0, n_it > 0);
      leave_sums<DT>(dv + r * kSumLd<DT>, col_dv + lanes, c0, n_it > 0);
      if (!ok) dk[r * kSumLd<DT> + c0] = dv[r * kSumLd<DT> + c0] = NAN;
      __syncwarp();
      cluster_sync_all();
      finish_rows<DT>(a.dk, s, k0, hk, a.dim, dk, part, parts, S::kParts * 128, [&](int, int) { return a.scale; });
      finish_rows<DT>(a.dv, s, k0, hk, a.dim, dv, part, parts, S::kParts * 128, [&](int, int) { return 1.f; });
      __syncwarp();
      cluster_sync_all();                         // the others have read this block's sums
    } else if (X && n_it == 0) {                  // no queries: zeros
      if (key < s.len) {
        zero_columns(head_row_out<__nv_bfloat16>(a.dv, s.begin + key, hk), c0, a.dim);
        zero_columns(head_row_out<__nv_bfloat16>(a.dk, s.begin + key, hk), c0, a.dim);
      }
    } else {
      const int first_row = k0 + (warp & 3) * 32;
      uint8_t* const stage = sptr + (sQ - base) + warp * 2048;           // the streamed tiles have been read
      static_assert(DT == S::kParts * 32, "a part of the threads stores 32 columns of each gradient");
      static_assert(S::kParts * 4 * 2048 <= 2 * S::kStages * S::kStream, "staging");
      store_rows(head_row_out<__nv_bfloat16>(a.dv, s.begin + first_row, hk), a.dv.token, s.len - first_row, col_dv + lanes, c0, a.dim, 1.f, ok, stage);
      store_rows(head_row_out<__nv_bfloat16>(a.dk, s.begin + first_row, hk), a.dk.token, s.len - first_row, col_dk + lanes, c0, a.dim, a.scale, ok, stage);
    }
  }
  if (parts > 1 && warp >= kCopy) {
    __syncwarp();
    cluster_sync_all();
    cluster_sync_all();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssue) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kTmem);
  }
}

template <int DT, bool X> __device__ __forceinline__ void dq_block(const PackedArgs& a, const TcBwdMaps& maps, int block, int part, int parts) {
  using S = BwdShape<DT>;
  constexpr int BN = S::kCols, kCopy = S::kParts * 4, kIssue = kCopy + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = block % a.heads, hk = h / a.group;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const sptr = smem_raw + (base - raw);
  const uint32_t sQ = base, sO = sQ + S::kTile, sK = sO + S::kTile, sV = sK + S::kStages * S::kStream, bars = sV + S::kStages * S::kStream;
  const uint32_t q_full = bars;
  auto full = [&](int i) { return bars + 8 * (1 + i); };
  auto cleared = [&](int i) { return bars + 8 * (1 + S::kStages + i); };
  auto empty = [&](int i) { return bars + 8 * (1 + 2 * S::kStages + i); };
  const uint32_t s_full = bars + 8 * (1 + 3 * S::kStages), dp_full = s_full + 16, ds_full = s_full + 24, acc_full = s_full + 32;   // s_full: two
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(sptr + (bars - base) + 8 * S::kBars);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* const status = &g_attn_packed_status;

  if (warp == kCopy && lane == 0) {
    mbar_init(q_full, 1);
    for (int i = 0; i < S::kStages; ++i) { mbar_init(full(i), 1); mbar_init(cleared(i), 32); mbar_init(empty(i), 1); }
    mbar_init(s_full, 1); mbar_init(s_full + 8, 1); mbar_init(dp_full, 1); mbar_init(ds_full, S::kParts * 4); mbar_init(acc_full, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&maps.q); tma_prefetch_desc(&maps.d_o); tma_prefetch_desc(&maps.k); tma_prefetch_desc(&maps.v);
  }
  if (warp == kIssue) {
    tmem_alloc(smem_u32(tmem_slot), S::kTmem);
    tmem_relinquish();
  }
  SeqTile ks;
  SeqTile s;
  if constexpr (X) s = find_longest(a.cu, a.cu_kv, a.n_seqs, a.tokens, a.kv_tokens, block / a.heads, TC_LOG_ROWS, ks);
  else ks = s = find_tile(a.cu, a.n_seqs, a.tokens, block / a.heads, TC_LOG_ROWS);
  if (s.tile < 0) {
    __syncthreads();
    if (warp == kIssue) tmem_dealloc(*tmem_slot, S::kTmem);
    pdl_wait();
    return;
  }
  const int tile = (s.len + TC_ROWS - 1) / TC_ROWS - 1 - s.tile;                 // the tiles that see the most keys first
  const int q0 = tile * TC_ROWS, all = ((!X && a.causal ? min(s.len, q0 + TC_ROWS) : ks.len) + BN - 1) / BN;
  const int it0 = all * part / parts, n_it = all * (part + 1) / parts - it0;     // of the key tiles, this block's share
  auto copy_keys = [&](int it) {
    const int st = it % S::kStages;
    if (elect_one()) {
      mbar_arrive_expect_tx(full(st), 2 * S::kStream);
      copy_rows<DT, BN>(sK + st * S::kStream, &maps.k, full(st), hk, ks.begin + (it0 + it) * BN);
      copy_rows<DT, BN>(sV + st * S::kStream, &maps.v, full(st), hk, ks.begin + (it0 + it) * BN);
    }
    __syncwarp();
  };
  if (warp == kCopy && n_it > 0) {
    __syncwarp();
    if (elect_one()) {
      mbar_arrive_expect_tx(q_full, 2 * S::kTile);
      copy_rows<DT, TC_ROWS>(sQ, &maps.q, q_full, h, s.begin + q0);
      copy_rows<DT, TC_ROWS>(sO, &maps.d_o, q_full, h, s.begin + q0);
    }
    __syncwarp();
    copy_keys(0);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, col_s = tmem, col_dp = tmem + 2 * BN, col_dq = tmem + 3 * BN;

  if (warp == kCopy) {                            // ---- copies
    int armed = 1;
    bool ok = true;
    for (int it = 0; it < n_it; ++it) {
      const int st = it % S::kStages, k0 = (it0 + it) * BN;
      if (it >= S::kStages) ok = wait_for(empty(st), (it / S::kStages - 1) & 1, abort_flag, status, 71);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (it > 0) {
        copy_keys(it);
        ++armed;
      }
      if (k0 + BN > ks.len) {                      // keys of other sequences, or of none: zeros, where dS is zero
        ok = wait_for(full(st), (it / S::kStages) & 1, abort_flag, status, 72);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        clear_rows<DT>(sptr + (sK - base) + st * S::kStream, ks.len - k0);
        fence_async_smem();
      }
      mbar_arrive(cleared(st));
    }
    if (*abort_flag && n_it > 0) {                // nothing may be in flight when the block ends
      volatile int never = 0;
      wait_for(q_full, 0, &never, status, 73);
      for (int it = max(0, armed - S::kStages); it < armed; ++it) wait_for(full(it % S::kStages), (it / S::kStages) & 1, &never, status, 73);
    }
  } else if (warp == kIssue) {                    // ---- products
    auto ready = [&](int it) {
      const int st = it % S::kStages;
      return wait_for(full(st), (it / S::kStages) & 1, abort_flag, status, 74) && wait_for(cleared(st), (it / S::kStages) & 1, abort_flag, status, 75);
    };
    bool ok = n_it > 0 && wait_for(q_full, 0, abort_flag, status, 76) && ready(0) && (n_it < 2 || ready(1));
    if (ok) {
      tc_fence_after();
      if (elect_one()) {
        mma_scores<DT>(col_s, sQ, sK);
        tc_commit(s_full);
        mma_scores<DT>(col_dp, sO, sV);
        tc_commit(dp_full);
        if (n_it > 1) { mma_scores<DT>(col_s + BN, sQ, sK + S::kStream); tc_commit(s_full + 8); }
      }
      __syncwarp();
    }
    for (int it = 0; it < n_it && ok; ++it) {
      const int st = it % S::kStages, nx = (it + 1) % S::kStages, n2 = (it + 2) % S::kStages;
      ok = wait_for(ds_full, it & 1, abort_flag, status, 77);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        mma_gradient<DT>(col_dq, col_dp, sK + st * S::kStream, it > 0);
        tc_commit(empty(st));
        if (it + 1 < n_it) { mma_scores<DT>(col_dp, sO, sV + nx * S::kStream); tc_commit(dp_full); }
        else tc_commit(acc_full);
      }
      __syncwarp();
      if (it + 2 < n_it) {                        // the values of it have left this half of S
        ok = ready(it + 2);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) { mma_scores<DT>(col_s + (it & 1) * BN, sQ, sK + n2 * S::kStream); tc_commit(s_full + 8 * (it & 1)); }
        __syncwarp();
      }
    }
  } else {                                        // ---- values: thread = query row, 32 of the key columns
    const int c0 = (warp >> 2) * 32, row = q0 + (threadIdx.x & 127);
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float c = a.scale * kLog2e;
    const int64_t at = (int64_t)h * a.tokens + s.begin + row;
    pdl_wait();                                   // delta
    const float lse = row < s.len ? a.lse[at] * kLog2e : INFINITY, delta = row < s.len ? a.delta[at] : 0.f;
    const int limit = !X && a.causal ? min(s.len, row + 1) : ks.len;
    bool ok = true;
    for (int it = 0; it < n_it; ++it) {
      const int k0 = (it0 + it) * BN;
      ok = wait_for(s_full + 8 * (it & 1), (it >> 1) & 1, abort_flag, status, 78);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      float p[32];
      uint32_t v[32], w[16];
      tmem_ld32(col_s + lanes + (it & 1) * BN + c0, v);
      tmem_ld_wait(v);
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const float2 x = fma_f32x2(make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), make_float2(c, c), make_float2(-lse, -lse));
        p[i] = ex2(x.x); p[i + 1] = ex2(x.y);
      }
      ok = wait_for(dp_full, it & 1, abort_flag, status, 79);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      tmem_ld32(col_dp + lanes + c0, v);
      tmem_ld_wait(v);
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const float2 x = add_f32x2(make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), make_float2(-delta, -delta));
        p[i] *= x.x; p[i + 1] *= x.y;
      }
      if (k0 + BN > ks.len || (!X && a.causal && k0 + BN > q0 + 1))
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (k0 + c0 + i >= limit) p[i] = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
      tmem_st16(col_dp + lanes + c0, w);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(ds_full);
    }
    if (ok && n_it > 0) ok = wait_for(acc_full, 0, abort_flag, status, 80);
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after();
    if (parts > 1) {                              // the tiles in shared memory have been read
      float* const sums = reinterpret_cast<float*>(sptr);
      const int r = threadIdx.x & 127;
      leave_sums<DT>(sums + r * kSumLd<DT>, col_dq + lanes, c0, n_it > 0);
      if (!ok) sums[r * kSumLd<DT> + c0] = NAN;
      __syncwarp();
      cluster_sync_all();
      finish_rows<DT>(a.dq, s, q0, h, a.dim, sums, part, parts, S::kParts * 128, [&](int, int) { return a.scale; });
      __syncwarp();
      cluster_sync_all();                         // the others have read this block's sums
    } else if (X && n_it == 0) {                  // no keys: zeros
      if (row < s.len) zero_columns(head_row_out<__nv_bfloat16>(a.dq, s.begin + row, h), c0, a.dim);
    } else {
      const int first_row = q0 + (warp & 3) * 32;
      store_rows(head_row_out<__nv_bfloat16>(a.dq, s.begin + first_row, h), a.dq.token, s.len - first_row, col_dq + lanes, c0, a.dim, a.scale, ok,
                 sptr + (sK - base) + warp * 2048);                      // the streamed tiles have been read
    }
  }
  if (parts > 1 && warp >= kCopy) {
    __syncwarp();
    cluster_sync_all();
    cluster_sync_all();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssue) {
    tc_fence_after();
    tmem_dealloc(tmem, S::kTmem);
  }
}

// The blocks of dk and dv, and behind them, on the SMs that the longest of those leave free, the blocks of dq.
template <int DT, bool X>
__global__ void __launch_bounds__(BwdShape<DT>::kThreads, BwdShape<DT>::kBlocks)
attn_packed_bwd_tc_kernel(const __grid_constant__ PackedArgs a, const __grid_constant__ TcBwdMaps maps, int dkv_blocks) {
  const int parts = (int)cg::this_cluster().num_blocks(), part = (int)cg::this_cluster().block_rank(), block = blockIdx.x / parts;
  if (block < dkv_blocks) dkv_block<DT, X>(a, maps, block, part, parts);
  else dq_block<DT, X>(a, maps, block - dkv_blocks, part, parts);
}

// delta_i = do_i . o_i: eight lanes a row, two rows to each lane with all loads in flight; blockIdx.y is the head.  Rows outside the
// sequences get a value that nothing reads.
constexpr int DELTA_R = 2;
__global__ void __launch_bounds__(256) attn_packed_delta_tc_kernel(const __grid_constant__ PackedArgs a) {
  constexpr int R = DELTA_R;
  pdl_trigger();
  const int part = threadIdx.x & 7, h = blockIdx.y;
  const int64_t first = (int64_t)blockIdx.x * 32 * R + (threadIdx.x >> 3);
  uint4 x[R][2], y[R][2];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t token = min(first + r * 32, a.tokens - 1);
    const __nv_bfloat16 *o = head_row<__nv_bfloat16>(a.o, token, h), *g = head_row<__nv_bfloat16>(a.d_o, token, h);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = part * 8 + c * 64;
      x[r][c] = col < a.dim ? *reinterpret_cast<const uint4*>(o + col) : make_uint4(0u, 0u, 0u, 0u);
      y[r][c] = col < a.dim ? *reinterpret_cast<const uint4*>(g + col) : make_uint4(0u, 0u, 0u, 0u);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint32_t u[4] = {x[r][c].x, x[r][c].y, x[r][c].z, x[r][c].w}, w[4] = {y[r][c].x, y[r][c].y, y[r][c].z, y[r][c].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum = fmaf(__uint_as_float(u[e] << 16), __uint_as_float(w[e] << 16), sum);
        sum = fmaf(__uint_as_float(u[e] & 0xFFFF0000u), __uint_as_float(w[e] & 0xFFFF0000u), sum);
      }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (part == 0 && first + r * 32 < a.tokens) a.delta[(int64_t)h * a.tokens + first + r * 32] = sum;
  }
}

// ---- host side --------------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiledFn encode_fn() {
  static std::atomic<EncodeTiledFn> cached{nullptr};
  EncodeTiledFn fn = cached.load(std::memory_order_acquire);
  if (fn) return fn;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
  fn = reinterpret_cast<EncodeTiledFn>(p);
  cached.store(fn, std::memory_order_release);
  return fn;
}

// [dim, heads, tokens] map with boxes of 64 x 1 x rows; columns behind the head's width and rows behind the last token read as zeros
static cudaError_t encode_heads(CUtensorMap* map, const HeadView& x, int dim, int heads, int64_t tokens, int rows) {
  const EncodeTiledFn fn = encode_fn();
  if (!fn) return cudaErrorNotSupported;
  // a dimension of one entry may come with any stride: give it a valid one
  const cuuint64_t head = heads > 1 ? (cuuint64_t)x.head * 2 : 256, token = tokens > 1 ? (cuuint64_t)x.token * 2 : 256;
  const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens}, strides[2] = {head, token};
  const cuuint32_t box[3] = {64, 1, (cuuint32_t)rows}, step[3] = {1, 1, 1};
  const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(x.data), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// 16-byte rows and strides, none of them zero
static bool tc_view(const HeadView& x, int heads, int64_t tokens) {
  auto stride = [](int64_t s, int64_t n) { return n <= 1 || (s > 0 && s % 8 == 0 && s < ((int64_t)1 << 38)); };
  return aligned_to(x.data, 16) && stride(x.head, heads) && stride(x.token, tokens);
}

bool attn_packed_tc_takes(const PackedArgs& a, int dtype, bool backward) {
  const bool inputs = dtype == PM_BF16 && a.dim % 8 == 0 && tc_view(a.q, a.heads, a.tokens) && tc_view(a.k, a.kv_heads, a.kv_tokens) &&
                      tc_view(a.v, a.kv_heads, a.kv_tokens) && tc_view(a.o, a.heads, a.tokens);
  if (!inputs || !backward) return inputs;
  return tc_view(a.d_o, a.heads, a.tokens) && tc_view(a.dq, a.heads, a.tokens) && tc_view(a.dk, a.kv_heads, a.kv_tokens) &&
         tc_view(a.dv, a.kv_heads, a.kv_tokens);
}

template <typename K> static cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && (dev > 63 || !(done.load(std::memory_order_relaxed) >> dev & 1))) {
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev <= 63) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return e;
}

template <int DT, int NT, bool X> static cudaError_t fwd_launch(const PackedArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  using S = FwdShape<DT, NT>;
  TcMaps maps;
  const int pair = NT == 2 && a.group % 2 == 0, units = pair ? a.heads / 2 : a.heads;
  const int64_t blocks = most_tiles(a.tokens, a.n_seqs, pair ? TC_ROWS : NT * TC_ROWS) * units;
  if (!launchable(blocks)) return cudaErrorInvalidConfiguration;
  cudaError_t e = allow_smem(attn_packed_fwd_tc_kernel<DT, NT, X>, S::kSmem, done);
  if (e == cudaSuccess) e = encode_heads(&maps.q, a.q, a.dim, a.heads, a.tokens, TC_ROWS);
  if (e == cudaSuccess) e = encode_heads(&maps.k, a.k, a.dim, a.kv_heads, a.kv_tokens, TC_ROWS);
  if (e == cudaSuccess) e = encode_heads(&maps.v, a.v, a.dim, a.kv_heads, a.kv_tokens, TC_ROWS);
  if (e != cudaSuccess) return e;
  const int parts = NT == 1 ? forward_parts(blocks, a, TC_ROWS, 2 * kSms, 3) : 1;
  return launch_clusters(attn_packed_fwd_tc_kernel<DT, NT, X>, blocks, S::kThreads, S::kSmem, st, false, parts, a, maps, units, pair);
}

static cudaError_t stream_launch(const PackedArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  using S = StreamShape;
  TcMaps maps;
  cudaError_t e = allow_smem(attn_cross_stream_kernel, S::kSmem, done);
  if (e == cudaSuccess) e = encode_heads(&maps.q, a.q, a.dim, a.heads, a.tokens, TC_ROWS);
  if (e == cudaSuccess) e = encode_heads(&maps.k, a.k, a.dim, a.kv_heads, a.kv_tokens, TC_ROWS);
  if (e == cudaSuccess) e = encode_heads(&maps.v, a.v, a.dim, a.kv_heads, a.kv_tokens, TC_ROWS);
  if (e != cudaSuccess) return e;
  const int64_t all = most_tiles(a.tokens, a.n_seqs, TC_ROWS) * a.heads, blocks = std::max<int64_t>(2 * kSms, (all + S::kMost - 1) / S::kMost);
  if (!launchable(all)) return cudaErrorInvalidConfiguration;
  return launch_pdl(attn_cross_stream_kernel, dim3((unsigned)blocks), dim3(S::kThreads), S::kSmem, st, false, a, maps, a.heads);
}

// Two query tiles to a block read keys and values half as often and pay for heads of 128 once every SM has such a block.  8192 tokens,
// 16 heads of 128, us with two / one: 240 / 252; 4000 tokens, 4 heads of 128: 68 / 63; 8192 tokens, 16 heads of 64: 213 / 205.
template <bool X> static cudaError_t tc_forward(const PackedArgs& a, cudaStream_t st) {
  // blocks that stay where there are more tiles than run at a time
  if (X && a.dim <= 64 && most_tiles(a.tokens, a.n_seqs, TC_ROWS) * a.heads > 2 * kSms) return stream_launch(a, st);
  if (a.dim <= 64) return fwd_launch<64, 1, X>(a, st);
  const bool pair = a.group % 2 == 0;
  const int64_t blocks = most_tiles(a.tokens, a.n_seqs, pair ? TC_ROWS : 2 * TC_ROWS) * (pair ? a.heads / 2 : a.heads);
  return blocks >= kSms ? fwd_launch<128, 2, X>(a, st) : fwd_launch<128, 1, X>(a, st);
}
cudaError_t attn_packed_tc_forward(const PackedArgs& a, cudaStream_t st) { return a.cross ? tc_forward<true>(a, st) : tc_forward<false>(a, st); }

template <int DT, bool X> static cudaError_t bwd_launch(const PackedArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  using S = BwdShape<DT>;
  TcBwdMaps maps;
  const int64_t dkv = most_tiles(a.kv_tokens, a.n_seqs, TC_ROWS) * a.kv_heads, blocks = most_tiles(a.tokens, a.n_seqs, TC_ROWS) * a.heads + dkv;
  if (!launchable(blocks)) return cudaErrorInvalidConfiguration;
  cudaError_t e = allow_smem(attn_packed_bwd_tc_kernel<DT, X>, S::kSmem, done);
  if (e == cudaSuccess) e = encode_heads(&maps.q, a.q, a.dim, a.heads, a.tokens, S::kCols);
  if (e == cudaSuccess) e = encode_heads(&maps.k, a.k, a.dim, a.kv_heads, a.kv_tokens, S::kCols);
  if (e == cudaSuccess) e = encode_heads(&maps.v, a.v, a.dim, a.kv_heads, a.kv_tokens, S::kCols);
  if (e == cudaSuccess) e = encode_heads(&maps.d_o, a.d_o, a.dim, a.heads, a.tokens, S::kCols);
  if (e != cudaSuccess) return e;
  e = launch_pdl(attn_packed_delta_tc_kernel, dim3((unsigned)((a.tokens + 32 * DELTA_R - 1) / (32 * DELTA_R)), a.heads), dim3(256), 0, st, false, a);
  // starts beside the first's last blocks; its own wait for them before they read delta
  if (e == cudaSuccess)
    e = launch_clusters(attn_packed_bwd_tc_kernel<DT, X>, blocks, S::kThreads, S::kSmem, st, true,
                        backward_parts(blocks, a, S::kCols, 4 * kSms, 4), a, maps, (int)dkv);
  return e;
}
cudaError_t attn_packed_tc_backward(const PackedArgs& a, cudaStream_t st) {
  if (a.cross) return a.dim <= 64 ? bwd_launch<64, true>(a, st) : bwd_launch<128, true>(a, st);
  return a.dim <= 64 ? bwd_launch<64, false>(a, st) : bwd_launch<128, false>(a, st);
}

// Self-test of the bounded wait: one thread, no tensor memory, no copy in flight, a barrier on which nothing arrives.
__global__ void attn_packed_wait_probe_kernel(long long limit_cycles) {
  __shared__ __align__(8) uint64_t bar;
  __shared__ int abort_flag;
  const uint32_t b = smem_u32(&bar);
  mbar_init(b, 1);
  abort_flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  wait_for(b, 0, &abort_flag, &g_attn_packed_status, 99, limit_cycles);
}
cudaError_t attn_packed_wait_probe(int64_t limit_cycles, cudaStream_t st) {
  return launch_pdl(attn_packed_wait_probe_kernel, dim3(1), dim3(1), 0, st, false, (long long)limit_cycles);
}

// Reading and clearing are one step on the device, so that no record is lost or reported twice; what was taken passes through a word that
// one call uses at a time.
__device__ int g_attn_packed_taken;
__global__ void attn_packed_take_status_kernel() { g_attn_packed_taken = atomicExch(&g_attn_packed_status, 0); }

cudaError_t attn_packed_status(int* code, cudaStream_t st) {
  static std::mutex one_at_a_time;
  *code = 0;
  try {
    std::lock_guard<std::mutex> lock(one_at_a_time);
    cudaError_t e = launch_pdl(attn_packed_take_status_kernel, dim3(1), dim3(1), 0, st, false);
    if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(code, g_attn_packed_taken, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    return e;
  } catch (...) {                                 // from the mutex
    return cudaErrorOperatingSystem;
  }
}

}  // namespace pm
