// The attention of the cache operators: what the units of its kernels
// (attend.hip, one per element type and head dim) and its host side
// (prefix.hip) share.
#pragma once

#include "cache_impl.h"

namespace radar_impl {

// A call's attention is cut into blocks, one workgroup each, that leave a
// partial (max, sum, acc[d]) for each of their query rows:
//  - of the shared prefix: (kv head, row tile, split), flash_rows query rows b G +
//    g against tiles_p tiles of prefix rows;
//  - of the sequences' own rows: (b, kv head, part), the G query rows of the
//    pair against tiles_o tiles.
struct FlashArgs {
  const void* q;             // [B][Hq][d]
  void* out;                 // the same (k_short)
  int B, Hq, Hkv, G;
  float qscale;              // log2(e) / sqrt(d)
  // prefix
  const void *Kp, *Vp;
  int64_t P, Pcap;
  int splits, tiles_p, mtiles, M;      // M = B G query rows of a kv head
  float *pacc, *pml;         // [Hkv][splits][M][d], [..][M][2]
  // own rows
  const void *K, *V;
  const int64_t* lens;
  int64_t t, cap;
  int parts, tiles_o;
  float *oacc, *oml;         // [B Hkv][parts][G][d], [..][G][2]
  float* logits;             // [B Hkv][G][tpad] q.k unscaled, or null
  int64_t tpad;
};

// cache rows of a workgroup's step, by element size and row waves
constexpr int flash_tile(int esz, int rw) {
  return rw == 1 ? (esz == 2 ? 128 : 64) : esz == 2 || rw == 2 ? 64 : 32;
}
// query rows of a workgroup
constexpr int flash_rows(int esz, int rw) { return rw == 1 && esz == 4 ? 16 : 32 * rw; }
// a sequence's own rows: its length, or -1 where lens holds none in [lo, t]
__device__ __forceinline__ int64_t own_len(const FlashArgs& a, int64_t b, int lo) {
  const int64_t n = a.lens ? a.lens[b] : a.t;
  return n >= lo && n <= a.t ? n : -1;
}

// attend.hip: rw in {1, 2, 4}: the prefix's blocks, then the own rows'; 0: k_short
void launch_flash_bf16_64(const FlashArgs& a, int rw, hipStream_t st);
void launch_flash_bf16_128(const FlashArgs& a, int rw, hipStream_t st);
void launch_flash_f32_64(const FlashArgs& a, int rw, hipStream_t st);
void launch_flash_f32_128(const FlashArgs& a, int rw, hipStream_t st);

}  // namespace radar_impl
