// Attention of drafted tokens, a tree or a chain, over the cache (compiled once per
// element type and head dim: -DRADAR_ATTEND_F32=0|1 -DRADAR_ATTEND_D=64|128). The pass
// over the rows is flash_impl.h's: a pair's query rows are those of all its nodes, and
// only the steps that hold drafted rows look at who attends which.
//
// Up to 64 query rows a pair memory bounds it, and at 128 nearly: at the margin 6.0 to 7.4 TB/s of the 7.2 that
// a pass of loads reaches (8, 16, 32 nodes of 32 / 8 heads of 128 over 131072 rows, bf16: 83, 85, 102
// us; one token 80); above, matrix cores, exponentials and LDS in turn, 0.94 PFLOP/s of the 1.35 of a large
// library product (64 nodes over 131072 rows: 161 us). A chunk of 1500 tokens behind 8000, 265 us, is 376
// row tiles for 256 CUs, of which 120 take two: 32% of the cycles are of matrix instructions, 43%
// where every CU has two (2048 tokens, 314 us; the clock is 2.08 and 1.94 GHz).
// Start and end are 5 to 14 us: the lengths, the parents and the first rows one after the
// other, 2 us each, the bits, and the partials of a full chip.
#include "flash_impl.h"
#include "tree_impl.h"

#ifndef RADAR_ATTEND_D
#define RADAR_ATTEND_D 128
#endif
#ifndef RADAR_ATTEND_F32
#define RADAR_ATTEND_F32 0
#endif

namespace radar_impl {
namespace {

constexpr int kTreeWords = RADAR_MAX_TREE / 32;
// a node's words in LDS: ones, its nodes' bits, zeros, zeros, whether its list of
// parents leaves the tree; an odd number, for the banks
constexpr int kNodeWords = (kTreeWords + 4) | 1;

struct TreeMask {
  static constexpr bool kOn = true;
  int64_t from, rows;        // the first row that not all attend; the sequence's rows
  const uint32_t* bits;      // of the tile's nodes; null: a chain
  int node0, g_log2;         // the tile's first node
  int* odd;                  // LDS
  bool direct;
  unsigned char* out;        // of the tile's first node, in bytes
  int64_t o_node, o_head;

  __device__ __forceinline__ uint32_t word(int i, int64_t x) const {
    const int n = i >> g_log2;
    if (!bits) {                           // uniform
      const int64_t last = rows + node0 + n - x;
      return last < 0 ? 0u : last >= 31 ? ~0u : (2u << last) - 1;
    }
    const int rel = (int)max(x - rows, (int64_t)-32);
    const uint32_t* w = bits + n * kNodeWords + min(rel >> 5, kTreeWords) + 1;
    return __builtin_amdgcn_alignbit(w[1], w[0], rel & 31);
  }
  __device__ __forceinline__ void found() const { *odd = 1; }
  __device__ __forceinline__ bool any_found() const {
    __syncthreads();
    return *odd != 0;
  }
  __device__ __forceinline__ float finish(int i, float l) const {
    return bits && bits[(i >> g_log2) * kNodeWords + kTreeWords + 3] ? __uint_as_float(0x7fc00000u) : l;
  }
  __device__ __forceinline__ void* out_row(int i) const {
    return out + (i >> g_log2) * o_node + (i & ((1 << g_log2) - 1)) * o_head;
  }
};

// The bits of nodes [node0, node0 + n): node i's are its own, its parent's, .. up to a
// root. A thread walks up from each, over a run of nodes that each follow the one before
// (up to 32, a word's) at once: of every node LDS holds where its run begins and the parent
// of that one, plus 2. own: this thread's parents, of nodes tid, tid + THREADS, ..
template <int THREADS>
__device__ __forceinline__ void tree_bits(const int (&own)[RADAR_MAX_TREE / THREADS], int nodes, int node0,
                                          int n, unsigned char* lds, uint32_t* bits) {
  constexpr int kOwn = RADAR_MAX_TREE / THREADS;
  int* up = reinterpret_cast<int*>(lds);           // parent + 2, then run begin << 16 | its parent + 2
  const int tid = threadIdx.x, lane = tid & 63;
  int begin[kOwn];
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    const int i = tid + THREADS * k;
    const bool good = i < nodes && own[k] >= -1 && own[k] < i;
    const u64 runs = __ballot(good && own[k] == i - 1);
    const uint32_t word = (uint32_t)(lane < 32 ? runs : runs >> 32);
    const uint32_t breaks = ~word & ((2u << (i & 31)) - 1);
    begin[k] = (i & ~31) + (breaks ? 31 - __clz(breaks) : 0);
    up[i] = good ? own[k] + 2 : 0;
  }
  __syncthreads();
  int jump[kOwn];
#pragma unroll
  for (int k = 0; k < kOwn; ++k) jump[k] = begin[k] << 16 | up[begin[k]];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kOwn; ++k) up[tid + THREADS * k] = jump[k];
  __syncthreads();
  for (int k = tid; k < n; k += THREADS) {
    uint32_t* o = bits + k * kNodeWords;
    o[0] = ~0u;
    for (int i = 1; i < kTreeWords + 3; ++i) o[i] = 0;
    uint32_t word = 0;
    int p = node0 + k, at = p >> 5;
    while (p >= 0) {                       // p descends
      const int j = up[p], s = j >> 16;
      if (p >> 5 != at) {
        o[1 + at] = word;
        word = 0;
        at = p >> 5;
      }
      word |= ((2u << (p & 31)) - 1) & ~((1u << (s & 31)) - 1);
      p = (j & 0xffff) - 2;
    }
    o[1 + at] = word;
    o[kTreeWords + 3] = p == -2;
  }
  __syncthreads();
}

// Workgroups i and i + 8 share an XCD and its L2. The units (the parts of all pairs) go round
// the XCDs, and a unit's row tiles, which read the same rows, follow one another on one, the
// last of them, which in a chain attends the most, first; the blocks of the last, not whole
// round are dealt out evenly. An XCD so gets parts of all sequences: each has about an eighth
// of the card's bandwidth, and one with the longest sequence for itself is waited for.
template <typename T, int D, int RW, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void k_tree(TreeArgs a) {
  using F = Flash<T, D, RW, WAVES>;
  constexpr int kRows = F::O::kRows * RW;
  using RowArray = float (*)[kRows];
  __shared__ __attribute__((aligned(16))) unsigned char lds[F::kLds];
  __shared__ float wm[F::TW * kRows], wl[F::TW * kRows];
  __shared__ uint32_t bits[kRows * kNodeWords];
  __shared__ int odd;
  const int units = a.parts ? a.B * a.Hkv * a.parts : a.units + a.B * a.Hkv, x = blockIdx.x % 8;
  int i = blockIdx.x / 8, unit = i / a.mtiles * 8 + x;
  if (i >= units / 8 * a.mtiles) {         // the last round
    const int rest = units % 8 * a.mtiles, each = (rest + 7) / 8;
    i -= units / 8 * a.mtiles;
    if (i >= each || x * each + i >= rest) return;
    i += x * each;
    unit = units / 8 * 8 + i / a.mtiles;
  }
  const int mt = a.mtiles - 1 - i % a.mtiles;
  int b, hk, part;
  TreeCut cut;
  TreeSeq s;
  if (a.parts) {                           // uniform
    const int pairs = a.B * a.Hkv, bh = unit % pairs;
    part = unit / pairs;
    unit = bh * a.parts + part;
    b = bh / a.Hkv;
    hk = bh % a.Hkv;
    const int steps = (int)((a.t + a.nodes - 1) >> a.step_log2) + 1;
    cut = {(steps + a.parts - 1) / a.parts, a.parts, 0};
    s = tree_seq(a, b);
  } else {
    const TreeBatch batch(a);
    cut = batch.cut(batch.each(), true, unit, &b);
    if (b < 0) return;
    s = batch.seq(b);
    hk = (unit - cut.first) / cut.parts;
    part = (unit - cut.first) % cut.parts;
  }
  constexpr int kOwn = RADAR_MAX_TREE / (WAVES * 64);
  int own[kOwn] = {};                      // (asked for ahead of what follows)
  if (a.parent)
#pragma unroll
    for (int k = 0; k < kOwn; ++k) {
      const int i = threadIdx.x + WAVES * 64 * k;
      if (i < a.nodes) own[k] = a.parent[(a.parent_shared ? 0 : (int64_t)b * a.nodes) + i];
    }
  const int row0 = mt * kRows, node0 = row0 >> a.g_log2;
  const bool direct = cut.parts == 1;
  TreeMask mask;
  mask.g_log2 = a.g_log2;
  mask.out = static_cast<unsigned char*>(a.out) +
             (b * a.o_seq + node0 * a.o_node + hk * a.G * a.o_head) * (int64_t)sizeof(T);
  mask.o_node = a.o_node * (int64_t)sizeof(T);
  mask.o_head = a.o_head * (int64_t)sizeof(T);
  if (s.rows < 0) {                        // (parts = 1: else the merge does it)
    for (int y = threadIdx.x; y < min(kRows, a.M - row0) * D; y += WAVES * 64)
      static_cast<T*>(mask.out_row(y / D))[y % D] = from_f32<T>(__uint_as_float(0x7fc00000u));
    return;
  }
  const int rows = min(kRows, s.nodes * a.G - row0);
  if (a.zero && a.parts == 1)              // uniform (parts = 0: the merge does it)
    for (int y = 4 * threadIdx.x + max(rows, 0) * D; y < min(kRows, a.M - row0) * D; y += 4 * WAVES * 64)
      store4(static_cast<T*>(mask.out_row(y / D)) + y % D, 0.f, 0.f, 0.f, 0.f);
  if (rows <= 0) return;
  const int64_t end = tree_end(a, s, row0 + rows), step = (int64_t)cut.each * F::NTG;
  const int64_t r0 = part * step, r1 = min(end, r0 + step);
  if (r0 >= end) return;
  mask.from = s.rows + (a.parent ? 0 : node0 + 1);
  mask.rows = s.rows;
  mask.bits = a.parent ? bits : nullptr;
  mask.node0 = node0;
  mask.odd = &odd;
  mask.direct = direct;
  if (r1 > mask.from) {                    // uniform
    if (threadIdx.x == 0) odd = 0;
    if (a.parent) tree_bits<WAVES * 64>(own, s.nodes, node0, (rows + a.G - 1) >> a.g_log2, lds, bits);
    else __syncthreads();
  }
  const T* q = static_cast<const T*>(a.q) + b * a.q_seq + node0 * a.q_node + hk * a.G * a.q_head;
  const int64_t bh = (int64_t)b * a.Hkv + hk, at = (int64_t)unit * a.M + row0;
  auto block = [&](auto once) {
    F::template block<false, false, decltype(once)::value>(
        static_cast<const T*>(a.K) + bh * a.cap * D, static_cast<const T*>(a.V) + bh * a.cap * D, r0, r1, rows,
        a.qscale,
        [&](int r) { return q + (r >> mask.g_log2) * a.q_node + (r & (a.G - 1)) * a.q_head; },
        a.acc + at * D, a.ml + at * 2, nullptr, 0, lds, reinterpret_cast<RowArray>(wm),
        reinterpret_cast<RowArray>(wl), nullptr, nullptr, 0, nullptr, mask);
  };
  // (past the caches where no other row tile reads the rows)
  if constexpr (RW == 4) {
    block(std::false_type{});
  } else {
    if (a.mtiles == 1) block(std::true_type{});
    else block(std::false_type{});
  }
}

template <typename T, int D>
void launch_tree(const TreeArgs& a, int rw, int waves, hipStream_t st) {
  const int64_t pairs = (int64_t)a.B * a.Hkv, units = a.parts ? pairs * a.parts : a.units + pairs;
  const dim3 grid((unsigned)(8 * (units / 8 * a.mtiles + ceil_div(units % 8 * a.mtiles, 8))));
  if constexpr (sizeof(T) == 2 && D == 128) {
    if (waves == 8) {
      if (rw == 2) launch(RADAR_K_ATTEND, k_tree<T, D, 2, 8>, grid, dim3(512), 0, st, a);
      else launch(RADAR_K_ATTEND, k_tree<T, D, 4, 8>, grid, dim3(512), 0, st, a);
      return;
    }
  }
  if (rw == 1) launch(RADAR_K_ATTEND, k_tree<T, D, 1, 4>, grid, dim3(256), 0, st, a);
  else if (rw == 2) launch(RADAR_K_ATTEND, k_tree<T, D, 2, 4>, grid, dim3(256), 0, st, a);
  else launch(RADAR_K_ATTEND, k_tree<T, D, 4, 4>, grid, dim3(256), 0, st, a);
}

}  // namespace

#if RADAR_ATTEND_F32 && RADAR_ATTEND_D == 64
void launch_tree_f32_64(const TreeArgs& a, int rw, int waves, hipStream_t st) { launch_tree<float, 64>(a, rw, waves, st); }
#elif RADAR_ATTEND_F32
void launch_tree_f32_128(const TreeArgs& a, int rw, int waves, hipStream_t st) { launch_tree<float, 128>(a, rw, waves, st); }
#elif RADAR_ATTEND_D == 64
void launch_tree_bf16_64(const TreeArgs& a, int rw, int waves, hipStream_t st) { launch_tree<bf16_t, 64>(a, rw, waves, st); }
#else
void launch_tree_bf16_128(const TreeArgs& a, int rw, int waves, hipStream_t st) { launch_tree<bf16_t, 128>(a, rw, waves, st); }
#endif

}  // namespace radar_impl
