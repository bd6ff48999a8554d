// Attention over packed sequences, of their own tokens or (cross attention) of the sequences of another tensor: arguments and the map
// from a block to its tile of a sequence.
#pragma once
#include "pm_ops.cuh"

namespace pm {

struct HeadView {
  const void* data;
  int64_t token, head;                            // strides in elements
};
struct PackedArgs {
  HeadView q, k, v, o, d_o, dq, dk, dv;           // o is written by the forward pass, dq, dk, dv by the backward pass
  const int32_t *cu, *cu_kv;                      // [n_seqs + 1], of the queries and of the keys: the same array without `cross`
  float *lse, *delta;                             // [heads][tokens]
  int64_t tokens, kv_tokens;                      // rows of q, o and of k, v
  int n_seqs, heads, kv_heads, group, dim, causal, cross;
  float scale;
};

template <typename T> __device__ __forceinline__ const T* head_row(const HeadView& x, int64_t token, int head) {
  return static_cast<const T*>(x.data) + token * x.token + (int64_t)head * x.head;
}
template <typename T> __device__ __forceinline__ T* head_row_out(const HeadView& x, int64_t token, int head) {
  return const_cast<T*>(head_row<T>(x, token, head));
}

struct SeqTile {
  int64_t begin;                                  // first token of the sequence
  int len, tile;                                  // its length; the tile's index inside it (-1: no such tile)
  int seq;                                        // which sequence it is
};

// The index-th tile of up to 32 PER sequences, PER consecutive ones to a lane: tiles counted through the sequences.
// With `other` the starts of the other side are loaded in the same round, and *there becomes its rows.
template <int PER>
__device__ __forceinline__ SeqTile find_counted(const int32_t* cu, int n_seqs, int tokens, int index, int log_rows, const int32_t* other = nullptr,
                                                int other_tokens = 0, SeqTile* there = nullptr) {
  const int lane = threadIdx.x & 31;
  int start[PER + 1], far[PER + 1], tiles[PER], mine = 0;
#pragma unroll
  for (int i = 0; i <= PER; ++i) {
    start[i] = min(max(cu[min(lane * PER + i, n_seqs)], 0), tokens);
    if (other) far[i] = min(max(other[min(lane * PER + i, n_seqs)], 0), other_tokens);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    tiles[i] = max(start[i + 1] - start[i] + (1 << log_rows) - 1, 0) >> log_rows;
    mine += tiles[i];
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) { const int v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
  int at = upto - mine;
  const unsigned has = __ballot_sync(0xffffffffu, index >= at && index < at + mine);
  if (!has) return SeqTile{0, 0, -1, 0};
  int tile = 0, len = 0, begin = 0, seq = 0, far_begin = 0, far_end = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (index >= at && index < at + tiles[i]) {
      tile = index - at; begin = start[i]; len = start[i + 1] - start[i]; seq = lane * PER + i;
      if (other) { far_begin = far[i]; far_end = far[i + 1]; }
    }
    at += tiles[i];
  }
  const int who = __ffs(has) - 1;
  if (other) {
    far_begin = __shfl_sync(0xffffffffu, far_begin, who);
    far_end = __shfl_sync(0xffffffffu, far_end, who);
    *there = SeqTile{far_begin, max(far_end - far_begin, 0), 0, 0};
  }
  return SeqTile{__shfl_sync(0xffffffffu, begin, who), __shfl_sync(0xffffffffu, len, who), __shfl_sync(0xffffffffu, tile, who),
                 __shfl_sync(0xffffffffu, seq, who)};
}

// The tile that has a slot: sequence b has the slots from (its start >> log_rows) + b to the next sequence's, at least as many as it has tiles
// and most_tiles() in all.  They ascend, so a slot's sequence is found by a search of 32 places at a time.  Out of line: it costs the kernels
// of few sequences nothing.
static __device__ __noinline__ SeqTile find_slot(const int32_t* cu, int n_seqs, int tokens, int slot, int log_rows) {
  const int lane = threadIdx.x & 31;
  auto start = [&](int b) { return min(max(cu[min(b, n_seqs)], 0), tokens); };
  const SeqTile none{0, 0, -1, 0};
  int first = 0, n = n_seqs;                      // the sequence is one of n from the first on
  while (n > 32) {
    const int step = (n + 31) / 32, b = first + lane * step;
    const int k = __popc(__ballot_sync(0xffffffffu, lane * step < n && (start(b) >> log_rows) + b <= slot));
    if (k == 0) return none;
    first += (k - 1) * step;
    n = min(step, n - (k - 1) * step);
  }
  const int mine = start(first + lane);
  const int k = __popc(__ballot_sync(0xffffffffu, lane < n && (mine >> log_rows) + first + lane <= slot));
  if (k == 0) return none;
  const int begin = __shfl_sync(0xffffffffu, mine, k - 1), next = __shfl_sync(0xffffffffu, mine, k & 31), end = k < 32 ? next : start(first + 32);
  const int len = end - begin, tile = slot - (begin >> log_rows) - (first + k - 1);
  if (tile < 0 || tile >= (len + (1 << log_rows) - 1) >> log_rows) return none;
  return SeqTile{begin, len, tile, first + k - 1};
}

// The tile of 2^log_rows rows of the index-th block; called by a whole warp, same result in every lane.  Up to 256 sequences are counted in one
// round of loads, and the blocks without a tile are the last.  Beyond, where counting would make every block walk through all sequences, the
// search takes two rounds for up to 1024 and a third for up to 32768; its blocks without a tile lie between the others (16 x 256 tokens, 16 heads
// of 64, forward: 16.6 us counted, 18.6 searched; 1000 x 32: 438 / 356; 4096 x 8: 2460 / 1330; 60000 of which one is not empty, 2 heads: 67800 /
// 740).  Starts are clipped to 0 .. tokens and a sequence that would end before it starts is empty: whatever the array holds, no tile
// reaches outside the tensors.
__device__ __forceinline__ SeqTile find_tile(const int32_t* cu, int n_seqs, int64_t tokens, int index, int log_rows) {
  if (n_seqs <= 32) return find_counted<1>(cu, n_seqs, (int)tokens, index, log_rows);
  if (n_seqs <= 256) return find_counted<8>(cu, n_seqs, (int)tokens, index, log_rows);
  return find_slot(cu, n_seqs, (int)tokens, index, log_rows);
}

// The rows of cross attention's other side that a tile's sequence meets.  Clipped as above.
__device__ __forceinline__ SeqTile other_side(const SeqTile& s, const int32_t* cu, int64_t tokens) {
  const int begin = min(max(cu[s.seq], 0), (int)tokens), end = min(max(cu[s.seq + 1], 0), (int)tokens);
  return SeqTile{begin, max(end - begin, 0), 0, s.seq};
}
// find_tile and other_side of cross attention, in one round of loads where the sequences are counted.  Where a warp holds all sequences the tiles
// of the one that has the longest other side come first.
__device__ __forceinline__ SeqTile find_longest(const int32_t* cu, const int32_t* cu_other, int n_seqs, int64_t tokens, int64_t other_tokens, int index, int log_rows,
                                                SeqTile& there) {
  if (n_seqs > 256) {
    const SeqTile s = find_slot(cu, n_seqs, (int)tokens, index, log_rows);
    if (s.tile >= 0) there = other_side(s, cu_other, other_tokens);
    return s;
  }
  if (n_seqs > 32) return find_counted<8>(cu, n_seqs, (int)tokens, index, log_rows, cu_other, (int)other_tokens, &there);
  const int lane = threadIdx.x & 31;
  auto start = [&](const int32_t* c, int64_t most, int b) { return min(max(c[min(b, n_seqs)], 0), (int)most); };
  const int begin = start(cu, tokens, lane), far = start(cu_other, other_tokens, lane);
  const int len = max(start(cu, tokens, lane + 1) - begin, 0), far_len = max(start(cu_other, other_tokens, lane + 1) - far, 0);
  const int tiles = (len + (1 << log_rows) - 1) >> log_rows;
  int at = 0;                                     // tiles of the sequences before this one
#pragma unroll 4
  for (int j = 0; j < n_seqs; ++j) {
    const int n = __shfl_sync(0xffffffffu, tiles, j), f = __shfl_sync(0xffffffffu, far_len, j);
    if (f > far_len || (f == far_len && j < lane)) at += n;
  }
  const unsigned has = __ballot_sync(0xffffffffu, index >= at && index < at + tiles);
  if (!has) return SeqTile{0, 0, -1, 0};
  const int who = __ffs(has) - 1;
  there = SeqTile{__shfl_sync(0xffffffffu, far, who), __shfl_sync(0xffffffffu, far_len, who), 0, 0};
  return SeqTile{__shfl_sync(0xffffffffu, begin, who), __shfl_sync(0xffffffffu, len, who), __shfl_sync(0xffffffffu, index - at, who), who};
}

// tiles of `rows` rows that sequences of `tokens` tokens in all can have at most, and their slots
inline int64_t most_tiles(int64_t tokens, int n_seqs, int rows) { return tokens / rows + n_seqs; }

// Whether one launch can have so many blocks; asked before anything is launched.
inline bool launchable(int64_t blocks) { return blocks <= 0x7fffffff; }

// `blocks` clusters of `parts` blocks
template <typename... K, typename... A>
inline cudaError_t launch_clusters(void (*kernel)(K...), int64_t blocks, int threads, int smem, cudaStream_t stream, bool pdl, int parts, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks * parts)); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (parts > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = parts; at[n].val.clusterDim.y = 1; at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (pdl) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<K>(args)...);
}

// Blocks that share the work of one: as many as leave no more than `most` in the launch (whose size is the most that the lengths can
// make), as long as each keeps `least` of the `streamed` tiles of a sequence of average length.  us shared /
// not: bf16, 2000 tokens, 2 heads of 64 on 1, forward 18 / 27, backward 35 / 76; 4000 tokens, 4 heads of 128, forward 45 / 63; 2 x 1000
// tokens, 8 heads of 128 on 2, backward 49 / 70; fp32, 700 + 300 + 13 tokens, 4 heads of 128 on 2, both 205 / 305; 493 tokens in 7, 4
// heads of 32 on 2, both 27 / 31.  Finer parts lose: the backward pass of the 2 x 1000 tokens in eight parts takes 80.
inline int packed_parts(int64_t blocks, int64_t streamed, int most, int least) {
  int parts = 1;
  while (parts < 8 && blocks * parts * 2 <= most && streamed >= parts * 2 * least) parts *= 2;
  return parts;
}
// tiles of `rows` rows of a sequence of average length
inline int64_t average_tiles(int64_t tokens, int n_seqs, int rows) { return ((tokens + n_seqs - 1) / n_seqs + rows - 1) / rows; }
// The forward pass streams keys alone, however many the queries (cross attention, us shared by the longer side / by the keys: 4000 tokens over
// 100, a head of 64 in bf16, 16.0 / 5.9; 2000 over 40, 2 heads of 64, bf16 10.5 / 5.9, fp32 21.6 / 6.2; 4000 over 600, 2 heads of 128, 19.2 / 13.9).
inline int forward_parts(int64_t blocks, const PackedArgs& a, int rows, int most, int least) {
  return packed_parts(blocks, average_tiles(a.kv_tokens, a.n_seqs, rows), most, least);
}
// The backward pass has blocks that stream keys and blocks that stream the queries of all heads that share them.  They share alike, by the
// longer of the two: a part that gets nothing of the shorter adds zeros.
inline int backward_parts(int64_t blocks, const PackedArgs& a, int rows, int most, int least) {
  return packed_parts(blocks, std::max(average_tiles(a.tokens, a.n_seqs, rows) * a.group, average_tiles(a.kv_tokens, a.n_seqs, rows)), most, least);
}

// launchers of the tensor-core kernels
bool attn_packed_tc_takes(const PackedArgs& a, int dtype, bool backward);
cudaError_t attn_packed_tc_forward(const PackedArgs& a, cudaStream_t st);
cudaError_t attn_packed_tc_backward(const PackedArgs& a, cudaStream_t st);
// the kernel of cross attention with few query rows, forward
bool attn_cross_step_takes(const PackedArgs& a, int dtype);
cudaError_t attn_cross_step(const PackedArgs& a, int dtype, cudaStream_t st);
// a wait of one thread that runs out after so many cycles, recorded as any other
cudaError_t attn_packed_wait_probe(int64_t limit_cycles, cudaStream_t st);
// the code of a device-side wait that ran out since the last call (0: none); synchronises the stream
cudaError_t attn_packed_status(int* code, cudaStream_t st);

}  // namespace pm
