// Attention of drafted tokens over the cache: what the units of its kernel (tree.hip, one
// per element type and head dim) and its host side (draft.hip) share.
#pragma once

#include "attend_impl.h"

namespace radar_impl {

// Query rows i G + g (node i, head g of the group) of a pair (b, kv head) are taken
// flash_rows at a time, a row tile, over the pair's cache rows in steps of flash_tile. The
// steps of a pair are cut into parts, a workgroup for each and row tile: as many for each
// pair (parts > 0), or, for sequences of different lengths (parts = 0), parts of one number
// of steps, about 1 / units of all, which every workgroup finds by adding up the lengths. A
// pair of one part gets its outputs there, else each part leaves a partial (max, sum,
// acc[d]) for each row, in the place of the part among all.
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
  int parent_shared, zero;   // zero: outputs of nodes behind a sequence's own become 0
  int mtiles, M;             // M = nodes G query rows of a pair
  int parts, units, least, g_log2;     // least: steps of a part, at least
  int step_log2;             // rows of a step
  float *acc, *ml;           // [parts of all pairs][M][d], [..][M][2]
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
  return s.rows + ((min(row1, s.nodes * a.G) - 1) >> a.g_log2) + 1;
}

__device__ __forceinline__ int tree_steps(const TreeArgs& a, const TreeSeq& s) {
  return s.nodes > 0 ? (int)((s.rows + s.nodes - 1) >> a.step_log2) + 1 : 0;
}

// the sum of x over the lanes up to this one
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);     // row_shr:1 ..
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);     // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);     // row_bcast:31
  return x;
}

// Where a pair's parts are among all: `each` steps in one, and for one sequence the number
// of parts of a head, and how many come before its first. (All steps fit 31 bits.)
struct TreeCut {
  int each, parts, first;
};

// The sequences of a ragged batch as a wave sees them, 64 at a time; of up to 64 all at once,
// each in its lane, asked for once.
struct TreeBatch {
  const TreeArgs& a;
  TreeSeq own;
  __device__ __forceinline__ explicit TreeBatch(const TreeArgs& args) : a(args), own{-1, 0} {
    if (a.B <= kWave && lane() < a.B) own = tree_seq(a, lane());
  }
  __device__ __forceinline__ static int lane() { return threadIdx.x & 63; }
  // steps of sequence b0 + lane
  __device__ __forceinline__ int steps(int b0) const {
    if (a.B <= kWave) return tree_steps(a, own);
    return b0 + lane() < a.B ? tree_steps(a, tree_seq(a, b0 + lane())) : 0;
  }
  __device__ __forceinline__ TreeSeq seq(int b) const {            // b: uniform
    if (a.B > kWave) return tree_seq(a, b);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)own.rows, b);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(own.rows >> 32), b);
    return {(int64_t)((uint64_t)hi << 32 | lo), __builtin_amdgcn_readlane(own.nodes, b)};
  }
  // Steps of a part; the same in every wave. With 1 / units of all there are at most units
  // parts and a shorter one for each pair. (To look here for the fewest steps whose parts
  // just fill the chip gains nothing.)
  __device__ __forceinline__ int each() const {
    uint32_t all = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave)
      all += (uint32_t)__builtin_amdgcn_readlane(wave_scan(steps(b0)), kWave - 1);
    all *= a.Hkv;
    return max(a.least, (int)((all + a.units - 1) / (uint32_t)a.units));
  }
  // of sequence b; or, by_part, of the one that part x of all lies in, which becomes b (-1: none)
  __device__ __forceinline__ TreeCut cut(int each, bool by_part, int x, int* b) const {
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
      const int own_parts = (int)((uint32_t)(steps(b0) + each - 1) / (uint32_t)each);
      const int sum = wave_scan(own_parts * a.Hkv);
      const u64 hit = __ballot(by_part ? x < before + sum : b0 + lane() == *b);
      if (hit) {                           // uniform
        const int l = __ffsll(hit) - 1, parts = __builtin_amdgcn_readlane(own_parts, l);
        *b = b0 + l;
        return {each, parts, before + __builtin_amdgcn_readlane(sum, l) - parts * a.Hkv};
      }
      before += __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    *b = -1;
    return {each, 0, 0};
  }
};

// tree.hip: rw in {1, 2, 4} row waves, in workgroups of 4 waves or (bf16, d = 128, rw > 1) 8
void launch_tree_bf16_64(const TreeArgs& a, int rw, int waves, hipStream_t st);
void launch_tree_bf16_128(const TreeArgs& a, int rw, int waves, hipStream_t st);
void launch_tree_f32_64(const TreeArgs& a, int rw, int waves, hipStream_t st);
void launch_tree_f32_128(const TreeArgs& a, int rw, int waves, hipStream_t st);

}  // namespace radar_impl
