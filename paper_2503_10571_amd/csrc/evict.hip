// Eviction by accumulated attention weight (include/radar_cache.h): which rows
// stay, and their move to the front of K, V and the masses, in place.
#include "cache_impl.h"
#include "evict_slices.h"

namespace radar_impl {
namespace {

struct EvictArgs {
  unsigned char *K, *V;
  float* mass;
  const int64_t* lens;
  int64_t* new_lens;
  int32_t* kept;
  int* cut;                // [B Hkv]: the length where it is cut, else -1
  int* turn;               // [B Hkv][2]: chunks of K and V taken so far
  int* arrived;            // [B Hkv][2][chunks]: the chunk is in registers
  int* src;                // [B Hkv][n]: the rows that stay, ascending
  int B, Hkv;
  int64_t t, cap;
  int sink, heavy, recent;
  int64_t n;               // sink + heavy + recent
  int n_kept;              // min(n, t): row length of kept
  int row_bytes, chunks;
  // caches of more than kStep rows: slices of slice_rows
  int slices, slice_rows;
  int* hist;               // [B Hkv][3][slices][kBins]
  int2* found;             // [B Hkv][2]: leading bits of the key, how many to take of them
  int* above;              // [B Hkv][2][slices]: of the slices before, keys above the bin
  float* moved;            // [B Hkv][n]: the masses of the rows that stay
};

// order-preserving key of a mass: larger is better; -0 as 0, a NaN above all
__device__ __forceinline__ uint32_t mass_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// ---------------------------------------------------------------------------
// which rows stay
// ---------------------------------------------------------------------------
// The heavy-th largest key of the rows between the sinks and the recent ones, by
// a radix search: a histogram of the keys' upper 11 bits gives its bin, two more of
// the bin's keys (11 and 10 bits) give the key. Then one ascending pass lists the
// rows.
//
// A cache of up to kStep rows takes one workgroup and one kernel that holds its
// masses in registers, lists the first bin's keys and ranks them if they are few.
// Longer ones are cut into slices, a workgroup each, with a kernel for each
// histogram, which adds up the one before over the slices, and one for the rows:
// one workgroup alone spends 2.2 us on a stage's 8192 rows (65600 rows of 64 pairs 86
// us, in slices 41; 200000 rows of 8 pairs 31; 16.8 MB of masses are read four times).
// Listing the first bin's keys instead of two more histograms is 2 us faster where
// they are few, and where most masses share a bin 1.5 ms slower (a million rows).
// bits of the key below each histogram's
__host__ __device__ constexpr int key_shift(int level) { return level == 0 ? 21 : level == 1 ? 10 : 0; }
constexpr int kBins = 2048, kRank = 256;   // (1024 keys: 25 us to rank, 6 by two histograms)
constexpr int kSelWaves = kSelThreads / kWave;

// Histograms in LDS are kept four times, by lane, side by side: a wave's keys
// share few bins (rows that were never met share one), and additions to one
// place follow one another.
constexpr int kCopies = 4;

// what the workgroup of a pair works on
struct Rows {
  int64_t bh;
  int len, lo, hi;         // rows [lo, hi) are candidates
  int begin, end;          // this workgroup's
  float* mass;
};

// Fills the rows of slice `slice` of pair bh; false where there are none. The
// first slice's workgroup also sets what the move needs, and what an uncut
// sequence gets.
__device__ __forceinline__ bool rows_of(const EvictArgs& a, int64_t bh, int slice, int slice_rows,
                                        bool first_kernel, Rows* r) {
  const int tid = threadIdx.x;
  const int64_t b = bh / a.Hkv;
  const int64_t len64 = a.lens ? a.lens[b] : a.t;
  const bool cut = len64 > a.n && len64 <= a.t;
  if (first_kernel && slice == 0) {
    if (tid == 0) a.cut[bh] = cut ? (int)len64 : -1;
    if (cut) {
      for (int i = tid; i < 2 * a.chunks; i += kSelThreads) a.arrived[bh * 2 * a.chunks + i] = 0;
      if (tid < 2) a.turn[bh * 2 + tid] = 0;
    } else if (a.kept) {
      for (int i = tid; i < a.n_kept; i += kSelThreads)
        a.kept[bh * a.n_kept + i] = len64 <= a.t && i < len64 ? i : -1;
    }
  }
  if (!cut) return false;
  r->bh = bh;
  r->len = (int)len64;
  r->lo = a.sink;
  r->hi = r->len - a.recent;
  r->begin = slice * slice_rows;
  r->end = slice_end(r->len, r->begin, slice_rows);
  r->mass = a.mass + bh * a.cap;
  return r->begin < r->len;
}

// a step's rows: i0 + 512 wave + 64 j + lane
__device__ __forceinline__ int step_row(int i0, int j) {
  return i0 + (int)(threadIdx.x & ~63u) * kPer + j * kWave + (int)(threadIdx.x & 63u);
}
__device__ __forceinline__ void load_step(const Rows& r, int i0, float (&x)[kPer]) {
#pragma unroll
  for (int j = 0; j < kPer; ++j) x[j] = r.mass[min(step_row(i0, j), r.len - 1)];
}
// f(first row of the step, its masses) over the workgroup's rows; x: the first
// step's, loaded ahead of whatever comes before; a step's loads are in flight
// together, and the next step's beside this one's work
template <typename F>
__device__ __forceinline__ void each_step(const Rows& r, float (&x)[kPer], F&& f) {
  float y[kPer];
#pragma unroll 1
  for (int i0 = r.begin; i0 < r.end; i0 += kStep) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) y[j] = x[j];
    if (i0 + kStep < r.end) load_step(r, i0 + kStep, x);
    f(i0, y);
  }
}

__device__ __forceinline__ void clear_bins(int* hist) {
  for (int i = threadIdx.x; i < kBins * kCopies; i += kSelThreads) hist[i] = 0;
  __syncthreads();
}
__device__ __forceinline__ void add_bin(int* hist, int bin) {
  atomicAdd(&hist[bin * kCopies + (threadIdx.x & (kCopies - 1))], 1);
}
__device__ __forceinline__ int bin_count(const int* hist, int bin) {
  const int4 v = *reinterpret_cast<const int4*>(hist + bin * kCopies);
  return (v.x + v.y) + (v.z + v.w);
}
__device__ __forceinline__ int2 two_bins(const int* hist, int bin) {
  return make_int2(bin_count(hist, bin), bin_count(hist, bin + 1));
}

// The bin, from the top, that holds the need-th key: x its number, y the keys
// above it, z its own; count(bin): the keys of the (even) bin and of the next.
// Thread x takes bins 2 x and 2 x + 1 from the top. A call of the whole workgroup.
template <typename Count>
__device__ __forceinline__ int3 pick_bin(int nb, int need, int* wsum, int* pick, Count&& count) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b0 = nb - 1 - 2 * tid, b1 = b0 - 1;
  const int2 both = b1 >= 0 ? count(b1) : make_int2(0, 0);
  const int c0 = both.y, c1 = both.x;
  const int incl = wave_incl_scan(c0 + c1, lane);
  if (lane == kWave - 1) wsum[wave] = incl;
  __syncthreads();
  int before = incl - (c0 + c1);
  for (int w = 0; w < wave; ++w) before += wsum[w];
  if (before < need && need <= before + c0) {
    pick[0] = b0; pick[1] = before; pick[2] = c0;
  } else if (before + c0 < need && need <= before + c0 + c1) {
    pick[0] = b1; pick[1] = before + c0; pick[2] = c1;
  }
  __syncthreads();
  const int3 got = make_int3(pick[0], pick[1], pick[2]);
  __syncthreads();
  return got;
}

// The need-th largest of n keys that share the bits of `prefix` under `mask`
// (the upper 11): the key, and how many equal to it are to be taken. key(i): the
// i-th. A call of the whole workgroup; ranks: kRank words of LDS.
struct Threshold {
  uint32_t key;
  int need;
};
template <typename Key>
__device__ __forceinline__ Threshold find_key(uint32_t prefix, int need, int n, Key&& key, int* hist,
                                              uint32_t* ranks, int* wsum, int* pick) {
  const int tid = threadIdx.x;
  if (n <= kRank) {
    if (tid < n) ranks[tid] = key(tid);
    __syncthreads();
    if (tid < n) {
      const uint32_t u = ranks[tid];
      int above = 0, equal = 0;
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        above += ranks[i] > u ? 1 : 0;
        equal += ranks[i] == u ? 1 : 0;
      }
      // (equal keys agree)
      if (above < need && need <= above + equal) { pick[0] = (int)u; pick[1] = above; }
    }
    __syncthreads();
    const Threshold got{(uint32_t)pick[0], need - pick[1]};
    __syncthreads();
    return got;
  }
  uint32_t mask = 0xffe00000u;
#pragma unroll 1
  for (int shift = 10; shift >= 0; shift -= 10) {
    const int nb = shift ? 2048 : 1024;
    clear_bins(hist);
    for (int i = tid; i < n; i += kSelThreads) {
      const uint32_t u = key(i);
      if ((u & mask) == prefix) add_bin(hist, (int)(u >> shift) & (nb - 1));
    }
    __syncthreads();
    const int3 b = pick_bin(nb, need, wsum, pick, [&](int x) { return two_bins(hist, x); });
    prefix |= (uint32_t)b.x << shift;
    mask |= (uint32_t)(nb - 1) << shift;
    need -= b.y;
  }
  return {prefix, need};
}

// A step's part of the last pass: keys above the threshold stay, and the first
// th.need of those equal to it. n_gt, n_eq: rows taken outright, and ties, before
// the step, moved on behind it. put(place, row, mass) of every row that stays.
// Every mass of the step is read before any is put: one barrier.
template <typename Put>
__device__ __forceinline__ void list_step(const EvictArgs& a, const Rows& r, const Threshold& th, int i0,
                                          const float (&y)[kPer], int& n_gt, int& n_eq,
                                          uint32_t* wcount, Put&& put) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t gt_bits = 0, eq_bits = 0;       // of this lane's rows
  uint32_t gt_all = 0, eq_all = 0;         // of the wave's
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = step_row(i0, j);
    const uint32_t u = mass_key(y[j]);
    const bool fixed = i < r.lo || i >= r.hi;
    const bool gt = i < r.len && (fixed || (a.heavy > 0 && u > th.key));
    const bool eq = i < r.len && !fixed && a.heavy > 0 && u == th.key;
    gt_bits |= (gt ? 1u : 0u) << j;
    eq_bits |= (eq ? 1u : 0u) << j;
    gt_all += (uint32_t)__popcll(__ballot(gt));
    eq_all += (uint32_t)__popcll(__ballot(eq));
  }
  if (lane == 0) wcount[wave] = gt_all | (eq_all << 16);   // (at most kStep each)
  __syncthreads();
  // the waves before this one, and all of them
  const uint32_t c = lane < kSelWaves ? wcount[lane] : 0u;
  const uint32_t incl = (uint32_t)wave_incl_scan((int)c, lane);
  const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)incl, kSelWaves - 1);
  const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)(incl - c), wave);
  int gt = n_gt + (int)(mine & 0xffffu), eq = n_eq + (int)(mine >> 16);
  const u64 below = (1ull << lane) - 1;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const u64 bg = __ballot((gt_bits >> j) & 1u), be = __ballot((eq_bits >> j) & 1u);
    const int eq_rank = eq + (int)__popcll(be & below);
    if (((gt_bits >> j) & 1u) || (((eq_bits >> j) & 1u) && eq_rank < th.need))
      put(gt + (int)__popcll(bg & below) + min(eq_rank, th.need), step_row(i0, j), y[j]);
    gt += (int)__popcll(bg);
    eq += (int)__popcll(be);
  }
  n_gt += (int)(all & 0xffffu);
  n_eq += (int)(all >> 16);
}

// Appends the step's keys in the bin to `list`, of which n_list counts the
// entries; returns this lane's rows above the bin (fixed rows too).
__device__ __forceinline__ int collect_step(const Rows& r, uint32_t prefix, int i0,
                                            const float (&y)[kPer], uint32_t* list, int* n_list) {
  constexpr uint32_t kTop = 0xffe00000u;
  const int lane = threadIdx.x & 63;
  uint32_t u[kPer];
  u64 in[kPer];
  int n = 0, above = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = step_row(i0, j);
    u[j] = mass_key(y[j]);
    const bool cand = i >= r.lo && i < r.hi;
    in[j] = __ballot(cand && (u[j] & kTop) == prefix);
    above += i < r.len && (!cand || (u[j] & kTop) > prefix) ? 1 : 0;
    n += (int)__popcll(in[j]);
  }
  if (n > 0) {                             // wave-uniform
    int at = 0;
    if (lane == 0) at = atomicAdd(n_list, n);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if ((in[j] >> lane) & 1ull) list[at + (int)__popcll(in[j] & ((1ull << lane) - 1))] = u[j];
      at += (int)__popcll(in[j]);
    }
  }
  return above;
}

// caches of up to kStep rows; the masses move in place (a place is at most the
// row itself)
__global__ __launch_bounds__(kSelThreads) void k_evict_select(EvictArgs a) {
  __shared__ __attribute__((aligned(16))) int hist[kBins * kCopies];
  __shared__ uint32_t list[kStep];
  __shared__ uint32_t ranks[kRank];
  __shared__ int wsum[kSelWaves], pick[3], n_list;
  __shared__ uint32_t wcount[kSelWaves];
  const int tid = threadIdx.x;
  Rows r;
  if (!rows_of(a, blockIdx.x, 0, kStep, true, &r)) return;
  float x[kPer];
  load_step(r, 0, x);
  Threshold th{0u, 0};
  if (a.heavy > 0) {
    if (tid == 0) n_list = 0;
    clear_bins(hist);
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (step_row(0, j) >= r.lo && step_row(0, j) < r.hi) add_bin(hist, (int)(mass_key(x[j]) >> 21));
    __syncthreads();
    const int3 b = pick_bin(kBins, a.heavy, wsum, pick, [&](int i) { return two_bins(hist, i); });
    const uint32_t prefix = (uint32_t)b.x << 21;
    collect_step(r, prefix, 0, x, list, &n_list);
    __syncthreads();
    th = find_key(prefix, a.heavy - b.y, b.z, [&](int i) { return list[i]; }, hist, ranks, wsum, pick);
  }
  int* src = a.src + r.bh * a.n;
  int32_t* kept = a.kept ? a.kept + r.bh * a.n_kept : nullptr;
  int n_gt = 0, n_eq = 0;
  list_step(a, r, th, 0, x, n_gt, n_eq, wcount, [&](int at, int i, float m) {
    src[at] = i;
    r.mass[at] = m;
    if (kept) kept[at] = i;
  });
  __syncthreads();
  for (int i = (int)a.n + tid; i < r.len; i += kSelThreads) r.mass[i] = 0.f;
}

// What the histograms of one level, added up over the slices, say about the need-th
// key: its bin, the keys above that, and of the slices before `mine` the keys above
// the bin and in it. A call of the whole workgroup.
struct Level {
  int bin, above, gt, eq;
};
__device__ __forceinline__ Level read_level(const EvictArgs& a, const Rows& r, int level, int need, int mine,
                                            int* wsum, int* pick, int* before) {
  const int slices = slices_of(r.len, a.slice_rows);
  const int* hist = a.hist + (r.bh * 3 + level) * a.slices * kBins;
  const int nb = level < 2 ? kBins : kBins / 2;
  int2 first = make_int2(0, 0);                // of the slices before
  if (threadIdx.x < 2) before[threadIdx.x] = 0;
  const int3 b = pick_bin(nb, need, wsum, pick, [&](int bin) {
    int2 all = make_int2(0, 0);
#pragma unroll 8
    for (int s = 0; s < slices; ++s) {
      const int2 v = *reinterpret_cast<const int2*>(hist + s * kBins + bin);
      all.x += v.x;
      all.y += v.y;
      first.x += s < mine ? v.x : 0;
      first.y += s < mine ? v.y : 0;
    }
    return all;
  });
  const int b0 = nb - 1 - 2 * (int)threadIdx.x, b1 = b0 - 1;   // as pick_bin has them
  const int gt = wave_sum_i32((b0 > b.x ? first.y : 0) + (b1 > b.x ? first.x : 0));
  if ((threadIdx.x & 63) == 0 && gt) atomicAdd(&before[0], gt);
  if (b0 == b.x) before[1] = first.y;
  if (b1 == b.x) before[1] = first.x;
  __syncthreads();
  return {b.x, b.y, before[0], before[1]};
}

// the histogram of each slice: of all its candidates, or of those in the bin that
// the last one gives
template <int LEVEL>
__global__ __launch_bounds__(kSelThreads) void k_evict_hist(EvictArgs a) {
  __shared__ __attribute__((aligned(16))) int hist[kBins * kCopies];
  __shared__ int wsum[kSelWaves], pick[3], before[2];
  const int mine = blockIdx.x;
  Rows r;
  if (!rows_of(a, blockIdx.y, mine, a.slice_rows, LEVEL == 0, &r) || a.heavy == 0) return;
  float x[kPer];
  load_step(r, r.begin, x);
  clear_bins(hist);
  uint32_t prefix = 0;
  if constexpr (LEVEL > 0) {
    constexpr int kLast = LEVEL > 0 ? LEVEL - 1 : 0;
    int need = a.heavy;
    if constexpr (LEVEL == 2) {
      const int2 f = a.found[r.bh * 2];
      prefix = (uint32_t)f.x;
      need = f.y;
    }
    const Level v = read_level(a, r, kLast, need, mine, wsum, pick, before);
    prefix |= (uint32_t)v.bin << key_shift(kLast);
    if (threadIdx.x == 0) {
      a.above[(r.bh * 2 + kLast) * a.slices + mine] = v.gt;
      if (mine == 0) a.found[r.bh * 2 + kLast] = make_int2((int)prefix, need - v.above);
    }
  }
  constexpr int kShift = key_shift(LEVEL), kAbove = LEVEL > 0 ? key_shift(LEVEL - 1) : 31;
  constexpr int nb = LEVEL < 2 ? kBins : kBins / 2;
  each_step(r, x, [&](int i0, const float (&y)[kPer]) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = step_row(i0, j);
      const uint32_t u = mass_key(y[j]);
      if (i >= r.lo && i < min(r.hi, r.end) && (LEVEL == 0 || u >> kAbove == prefix >> kAbove))
        add_bin(hist, (int)(u >> kShift) & (nb - 1));
    }
  });
  __syncthreads();
  int* out = a.hist + ((r.bh * 3 + LEVEL) * a.slices + mine) * kBins;
  for (int i = threadIdx.x; i < nb; i += kSelThreads) out[i] = bin_count(hist, i);
}

// and the rows that stay, each slice's behind those of the slices before it
__global__ __launch_bounds__(kSelThreads) void k_evict_list(EvictArgs a) {
  __shared__ int wsum[kSelWaves], pick[3], before[2];
  __shared__ uint32_t wcount[2][kSelWaves];
  const int mine = blockIdx.x;
  Rows r;
  if (!rows_of(a, blockIdx.y, mine, a.slice_rows, false, &r)) return;
  float x[kPer];
  load_step(r, r.begin, x);
  Threshold th{0u, 0};
  int n_gt = min(r.begin, r.lo) + max(r.begin - r.hi, 0), n_eq = 0, parity = 0;   // fixed rows
  if (a.heavy > 0) {
    const int2 f = a.found[r.bh * 2 + 1];
    const int* above = a.above + r.bh * 2 * a.slices + mine;
    n_gt += above[0] + above[a.slices];
    const Level v = read_level(a, r, 2, f.y, mine, wsum, pick, before);
    th = {(uint32_t)f.x | (uint32_t)v.bin, f.y - v.above};
    n_gt += v.gt;
    n_eq = v.eq;
  }
  int* src = a.src + r.bh * a.n;
  float* moved = a.moved + r.bh * a.n;
  int32_t* kept = a.kept ? a.kept + r.bh * a.n_kept : nullptr;
  each_step(r, x, [&](int i0, const float (&y)[kPer]) {
    list_step(a, r, th, i0, y, n_gt, n_eq, wcount[parity], [&](int at, int i, float m) {
      src[at] = i;
      moved[at] = m;
      if (kept) kept[at] = i;
    });
    parity ^= 1;
  });
}

// ---------------------------------------------------------------------------
// k_evict_move: row i of K and V takes row src[i] >= i, in place
// ---------------------------------------------------------------------------
// A workgroup moves a chunk of 128 KB of K or V (with 64 KB 5% slower): it
// loads the chunk's rows into registers, says so, and writes them once every chunk
// before it that reads rows at or behind its own first place has said so too (the
// chunks behind it read rows behind everything it writes). Chunks are handed out in
// ascending order, so the ones waited for have started, and none of them waits before
// it has loaded: every wait ends. What is waited for is that reads are over, no data
// goes from one workgroup to another, so nothing has to be flushed. Moving whole
// columns of a pair in order needs no waits but leaves few workgroups (315 us
// for 48 pairs of 16K rows of 256 bytes, 173 this way: 4.7 TB/s).
// The new lengths, which may replace the old ones, are written here, when nobody
// reads those any more.
template <int CPR, bool PAST>              // 16-byte chunks of a row; stores past the caches
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a) {
  constexpr int R = kMoveThreads * kMoveVecs / CPR;        // rows per chunk
  __shared__ int turn;
  __shared__ int from[R];
  const int tid = threadIdx.x;
  const int64_t bh = blockIdx.y;
  const bool cut = a.cut[bh] >= 0;                 // workgroup-uniform
  if (a.new_lens && bh % a.Hkv == 0 && blockIdx.x == 0 && blockIdx.z == 0 && tid == 0) {
    const int64_t b = bh / a.Hkv;
    a.new_lens[b] = cut ? a.n : a.lens ? a.lens[b] : a.t;
  }
  if (!cut) return;
  const int n = (int)a.n;
  if (blockIdx.z == 2) {                           // the masses, where slices listed them
    float* mass = a.mass + bh * a.cap;
    for (int64_t i = (int64_t)blockIdx.x * kMoveThreads + tid; i < a.cut[bh];
         i += (int64_t)gridDim.x * kMoveThreads)
      mass[i] = i < n ? a.moved[bh * a.n + i] : 0.f;
    return;
  }
  if (n == 0) return;
  const int64_t half = bh * 2 + blockIdx.z;
  if (tid == 0) turn = atomicAdd(&a.turn[half], 1);
  __syncthreads();
  const int c = turn, i0 = c * R;
  const int* src = a.src + bh * a.n;
  int* arrived = a.arrived + half * a.chunks;
  for (int i = tid; i < R; i += kMoveThreads) from[i] = src[min(i0 + i, n - 1)];
  __syncthreads();
  unsigned char* base = (blockIdx.z ? a.V : a.K) + bh * a.cap * a.row_bytes + (tid % CPR) * 16;
  uint4 x[kMoveVecs];
#pragma unroll
  for (int j = 0; j < kMoveVecs; ++j)
    x[j] = ld_stream(base + (int64_t)from[(j * kMoveThreads + tid) / CPR] * a.row_bytes);
  // every load of this thread has arrived, then of every thread
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (tid == 0) __hip_atomic_store(&arrived[c], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  for (int o = tid; o < c; o += kMoveThreads)
    if (src[(o + 1) * R - 1] >= i0)
      while (__hip_atomic_load(&arrived[o], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0)
        __builtin_amdgcn_s_sleep(2);
  __syncthreads();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int j = 0; j < kMoveVecs; ++j) {
    const int i = i0 + (j * kMoveThreads + tid) / CPR;
    if (i < n) put16<PAST>(base + (int64_t)i * a.row_bytes, x[j]);
  }
}

struct EvictWs {
  size_t turn, arrived, src, hist, found, above, moved, total;
  int64_t chunks;
};
EvictWs evict_ws(const Shape& s, int64_t t, int64_t n) {
  const size_t pairs = (size_t)s.B * s.Hkv;
  const int row_bytes = s.d * (s.dt == RADAR_BF16 ? 2 : 4);
  EvictWs w;
  w.chunks = move_chunks(n, row_bytes);
  w.turn = align256(pairs * 4);
  w.arrived = w.turn + align256(pairs * 8);
  w.src = w.arrived + align256(pairs * 2 * w.chunks * 4);
  w.total = w.src + align256(pairs * n * 4);
  w.hist = w.found = w.above = w.moved = w.total;
  if (t > kStep) {
    // (bounds for every smaller t too, whose slices may be more)
    const size_t slices = (size_t)std::min<int64_t>(kSlices, ceil_div(t, kStep));
    w.found = w.hist + align256(pairs * 3 * slices * kBins * 4);
    w.above = w.found + align256(pairs * 2 * sizeof(int2));
    w.moved = w.above + align256(pairs * 2 * slices * 4);
    w.total = w.moved + align256(pairs * n * 4);
  }
  return w;
}

}  // namespace
}  // namespace radar_impl

using namespace radar_impl;

extern "C" {

size_t radar_evict_workspace_bytes(const radar_config* cfg, int64_t t, int64_t heavy,
                                   int64_t recent) {
  Shape s;
  if (check_cache(cfg, &s) != RADAR_OK || t < 0 || t > s.cap || heavy < 0 || recent < 0 ||
      t > kMostRows || heavy > INT32_MAX || recent > INT32_MAX ||
      s.n_sink + heavy + recent > INT32_MAX)
    return 0;
  const EvictWs w = evict_ws(s, t, std::min<int64_t>(s.n_sink + heavy + recent, t));
  return w.chunks > kMostChunks ? 0 : w.total;
}

radar_status radar_evict(const radar_config* cfg, void* K, void* V, float* mass, int64_t t,
                         const int64_t* lens, int64_t heavy, int64_t recent, int64_t* new_lens,
                         int32_t* kept, void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  Shape s;
  radar_status r = check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  if (!K || !V || !mass || !aligned16(K) || !aligned16(V) || !aligned16(mass)) return RADAR_EINVAL;
  if ((lens && !aligned16(lens)) || (new_lens && !aligned16(new_lens)) ||
      (kept && !aligned16(kept)) || heavy < 0 || recent < 0)
    return RADAR_EINVAL;
  if (t < 0 || t > s.cap) return RADAR_ECAPACITY;
  const size_t need = radar_evict_workspace_bytes(cfg, t, heavy, recent);
  if (need == 0) return RADAR_EUNSUPPORTED;            // (the sizes are checked there)
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) return RADAR_EWORKSPACE;
  EvictArgs a{};
  a.K = static_cast<unsigned char*>(K);
  a.V = static_cast<unsigned char*>(V);
  a.mass = mass;
  a.lens = lens; a.new_lens = new_lens; a.kept = kept;
  const EvictWs w = evict_ws(s, t, std::min<int64_t>(s.n_sink + heavy + recent, t));
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.cut = reinterpret_cast<int*>(ws);
  a.turn = reinterpret_cast<int*>(ws + w.turn);
  a.arrived = reinterpret_cast<int*>(ws + w.arrived);
  a.src = reinterpret_cast<int*>(ws + w.src);
  a.chunks = (int)w.chunks;
  a.hist = reinterpret_cast<int*>(ws + w.hist);
  a.found = reinterpret_cast<int2*>(ws + w.found);
  a.above = reinterpret_cast<int*>(ws + w.above);
  a.moved = reinterpret_cast<float*>(ws + w.moved);
  a.slice_rows = (int)slice_rows_of(t);
  a.slices = t > 0 ? (int)ceil_div(t, a.slice_rows) : 1;
  a.B = s.B; a.Hkv = s.Hkv; a.t = t; a.cap = s.cap;
  a.sink = s.n_sink; a.heavy = (int)heavy; a.recent = (int)recent;
  a.n = s.n_sink + heavy + recent;
  a.n_kept = (int)std::min<int64_t>(a.n, t);
  a.row_bytes = s.d * (s.dt == RADAR_BF16 ? 2 : 4);
  const unsigned pairs = (unsigned)(s.B * s.Hkv);
  const bool sliced = t > kStep && a.n < t;
  if (sliced) {
    const dim3 grid((unsigned)a.slices, pairs), block(kSelThreads);
    launch(RADAR_K_TOPK, k_evict_hist<0>, grid, block, 0, stream, a);
    if (a.heavy > 0) {
      launch(RADAR_K_TOPK, k_evict_hist<1>, grid, block, 0, stream, a);
      launch(RADAR_K_TOPK, k_evict_hist<2>, grid, block, 0, stream, a);
    }
    launch(RADAR_K_TOPK, k_evict_list, grid, block, 0, stream, a);
  } else {
    launch(RADAR_K_TOPK, k_evict_select, dim3(pairs), dim3(kSelThreads), 0, stream, a);
  }
  r = launch_status();
  // (n = 0: the masses alone; n >= t: no sequence is longer)
  const bool moves = a.n > 0 && a.n < t;
  if (r != RADAR_OK || !(moves || sliced || new_lens)) return r;
  const dim3 grid(std::max(1u, moves ? (unsigned)w.chunks : 1u), pairs, sliced ? 3 : moves ? 2 : 1);
  // The stores pass the caches by where the rows that stay, K's and V's, read and
  // written, are more than 768 MB, three times what the caches hold; sequences that are
  // not cut, which only the GPU knows, count too. 64 pairs of 21004 rows of 256 bytes
  // (1376 MB): 265 us, 238 this way; 16384 (1074), a third of them uncut: 183, 173; but
  // 9004 (590): 105, 110.
  const bool past = 4 * a.n * pairs * a.row_bytes > ((int64_t)768 << 20);
  auto go = [&](auto cpr) {
    constexpr int kCpr = decltype(cpr)::value;
    if (past) launch(RADAR_K_APPEND, k_evict_move<kCpr, true>, grid, dim3(kMoveThreads), 0, stream, a);
    else launch(RADAR_K_APPEND, k_evict_move<kCpr, false>, grid, dim3(kMoveThreads), 0, stream, a);
  };
  if (a.row_bytes == 128) go(std::integral_constant<int, 8>{});
  else if (a.row_bytes == 256) go(std::integral_constant<int, 16>{});
  else go(std::integral_constant<int, 32>{});
  return launch_status();
}

}  // extern "C"
