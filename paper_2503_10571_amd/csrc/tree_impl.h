// Attention of drafted tokens over the cache: what the units of its kernel (tree.hip, one
// per element type and head dim) and its host side (draft.hip) share.
#pragma once

#include "attend_impl.h"

namespace radar_impl {

// A call is cut into blocks (b, kv head, split, row tile), one workgroup each: flash_rows
// of the pair's query rows i G + g (node i, head g of the group) against `tiles` steps of
// its cache rows. With one split a block leaves the outputs, with more a partial (max, sum,
// acc[d]) for each row.
struct TreeArgs {
  const void* q;             // [B][nodes][Hq][d], strides in elements
  void* out;
  int64_t q_seq, q_node, q_head, o_seq, o_node, o_head;
  int B, Hq, Hkv, G;
  float qscale;              // log2(e) / sqrt(d)
  const void *K, *V;
  const int64_t *lens, *counts;
  int64_t t, cap;
  int nodes;
  const int* parent;         // [B][nodes], or [nodes] if shared; null: a chain
  int parent_shared;
  int splits, mtiles, M;     // M = nodes G query rows of a pair
  int64_t tiles;
  float *acc, *ml;           // [B Hkv][splits][M][d], [..][M][2]
};

// a sequence's rows and nodes; rows < 0: its length or count is invalid
struct TreeSeq {
  int64_t rows;
  int nodes;
};
__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs& a, int64_t b) {
  const int64_t n = a.lens ? a.lens[b] : a.t, m = a.counts ? a.counts[b] : a.nodes;
  const bool ok = n >= 0 && n <= a.t && m >= 0 && m <= a.nodes && n + m <= a.cap;
  return {ok ? n : -1, ok ? (int)m : 0};
}
// the end of the rows that a tile's query rows, the last of them row1 - 1, attend
__device__ __forceinline__ int64_t tree_end(const TreeArgs& a, const TreeSeq& s, int row1) {
  return s.rows + (min(row1, s.nodes * a.G) - 1) / a.G + 1;
}

// tree.hip: rw in {1, 2, 4} row waves
void launch_tree_bf16_64(const TreeArgs& a, int rw, hipStream_t st);
void launch_tree_bf16_128(const TreeArgs& a, int rw, hipStream_t st);
void launch_tree_f32_64(const TreeArgs& a, int rw, hipStream_t st);
void launch_tree_f32_128(const TreeArgs& a, int rw, hipStream_t st);

}  // namespace radar_impl
