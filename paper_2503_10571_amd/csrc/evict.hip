// Eviction by accumulated attention weight (include/radar_cache.h): which rows
// stay, and their move to the front of K, V and the masses, in place.
#include "cache_impl.h"

namespace radar_impl {
namespace {

struct EvictArgs {
  unsigned char *K, *V;
  float* mass;
  const int64_t* lens;
  int64_t* new_lens;
  int32_t* kept;
  int* src;                // [B Hkv][n]: the rows that stay, ascending
  int* cut;                // [B Hkv]: the length where it is cut, else -1
  int B, Hkv;
  int64_t t, cap;
  int sink, heavy, recent;
  int64_t n;               // sink + heavy + recent
  int n_kept;              // min(n, t): row length of kept
  int row_bytes;
};

// order-preserving key of a mass: larger is better; -0 as 0, a NaN above all
__device__ __forceinline__ uint32_t mass_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One workgroup per (b, kv head): the heavy-th largest key of the rows between
// the sinks and the recent ones by a radix search over 11, 11 and 10 bits, then
// one ascending pass that lists the rows and moves the masses.
constexpr int kSelThreads = 1024;
constexpr int kBins = 2048;

__global__ __launch_bounds__(kSelThreads) void k_evict_select(EvictArgs a) {
  __shared__ int hist[kBins];
  __shared__ int wsum[kSelThreads / kWave];
  __shared__ int pick[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t bh = blockIdx.x, b = bh / a.Hkv;
  const int64_t len64 = a.lens ? a.lens[b] : a.t;
  const int64_t cut = len64 > a.n && len64 <= a.t ? len64 : -1;
  if (tid == 0) a.cut[bh] = (int)cut;
  int32_t* kept = a.kept ? a.kept + bh * a.n_kept : nullptr;
  if (cut < 0) {
    if (kept)
      for (int i = tid; i < a.n_kept; i += kSelThreads)
        kept[i] = len64 <= a.t && i < len64 ? i : -1;
    return;
  }
  const int len = (int)cut, lo = a.sink, hi = len - a.recent;
  float* mass = a.mass + bh * a.cap;
  // (prefix, mask): the leading bits of the heavy-th largest key found so far,
  // of which `need` are still to be taken among the keys that match
  uint32_t prefix = 0, mask = 0;
  int need = a.heavy;
#pragma unroll 1
  for (int pass = 0; pass < 3 && need > 0; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const int bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int i0 = lo; i0 < hi; i0 += kSelThreads) {
      const int i = i0 + tid;
      const uint32_t u = i < hi ? mass_key(mass[i]) : 0;
      const bool in = i < hi && (u & mask) == prefix;
      const int bin = (int)(u >> shift) & ((1 << bits) - 1);
      // (rows that were never met share a bin: one addition for the wave)
      const u64 some = __ballot(in);
      if (some == 0) continue;
      const int first = __builtin_amdgcn_readlane(bin, (int)__builtin_ctzll(some));
      if (__ballot(in && bin != first) == 0) {
        if (lane == 0) atomicAdd(&hist[first], (int)__popcll(some));
      } else if (in) {
        atomicAdd(&hist[bin], 1);
      }
    }
    __syncthreads();
    // the bin, from the top, in which the need-th key lies: thread x takes bins
    // 2 x and 2 x + 1 from the top
    const int nb = 1 << bits;
    const int b0 = nb - 1 - 2 * tid, b1 = b0 - 1;
    const int c0 = b0 >= 0 ? hist[b0] : 0, c1 = b1 >= 0 ? hist[b1] : 0;
    const int incl = wave_incl_scan(c0 + c1, lane);
    if (lane == kWave - 1) wsum[wave] = incl;
    __syncthreads();
    int before = incl - (c0 + c1);
    for (int w = 0; w < wave; ++w) before += wsum[w];
    if (before < need && need <= before + c0) { pick[0] = b0; pick[1] = before; }
    else if (before + c0 < need && need <= before + c0 + c1) { pick[0] = b1; pick[1] = before + c0; }
    __syncthreads();
    prefix |= (uint32_t)pick[0] << shift;
    mask |= ((uint32_t)(nb - 1)) << shift;
    need -= pick[1];
    __syncthreads();
  }
  // keys above `prefix` stay, and the first `need` of those equal to it
  int* src = a.src + bh * a.n;
  int n_out = 0, n_eq = 0;                 // listed so far, equal keys so far
#pragma unroll 1
  for (int i0 = 0; i0 < len; i0 += kSelThreads) {
    const int i = i0 + tid;
    float x = 0.f;
    bool take = false, eq = false;
    if (i < len) {
      x = mass[i];
      if (i < lo || i >= hi) {
        take = true;
      } else if (a.heavy > 0) {
        const uint32_t u = mass_key(x);
        take = u > prefix;
        eq = u == prefix;
      }
    }
    // ranks among the equal keys, then among the rows taken
    const u64 be = __ballot(eq);
    const u64 below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
    if (lane == 0) wsum[wave] = (int)__popcll(be);
    __syncthreads();
    int eq_before = n_eq, eq_all = 0;
    for (int w = 0; w < kSelThreads / kWave; ++w) {
      eq_before += w < wave ? wsum[w] : 0;
      eq_all += wsum[w];
    }
    if (eq && eq_before + (int)__popcll(be & below) < need) take = true;
    n_eq += eq_all;
    __syncthreads();
    const u64 bt = __ballot(take);
    if (lane == 0) wsum[wave] = (int)__popcll(bt);
    __syncthreads();
    int at = n_out, all = 0;
    for (int w = 0; w < kSelThreads / kWave; ++w) {
      at += w < wave ? wsum[w] : 0;
      all += wsum[w];
    }
    // (every mass of this step is read: the place is at most the row itself)
    if (take) {
      at += (int)__popcll(bt & below);
      src[at] = i;
      mass[at] = x;
      if (kept) kept[at] = i;
    }
    n_out += all;
    __syncthreads();
  }
  for (int i = (int)a.n + tid; i < len; i += kSelThreads) mass[i] = 0.f;
}

// The rows' move: row i takes row src[i] >= i. A workgroup takes one 128-byte
// column of a (b, kv head)'s K or V and goes through the rows in ascending
// blocks: a block's rows are all in registers before any is written, and the
// rows of later blocks lie behind everything written so far, so the next block
// is loaded while this one is written. The new lengths, which may replace the old
// ones, are written here, when nobody reads those any more.
constexpr int kMoveThreads = 512, kMoveRows = 8;   // 16-byte chunks per thread

__global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a) {
  const int64_t bh = blockIdx.y;
  const bool cut = a.cut[bh] >= 0;                 // workgroup-uniform
  if (a.new_lens && bh % a.Hkv == 0 && blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0) {
    const int64_t b = bh / a.Hkv;
    a.new_lens[b] = cut ? a.n : a.lens ? a.lens[b] : a.t;
  }
  if (!cut || a.n == 0) return;
  constexpr int RPP = kMoveThreads / 8;            // rows per load instruction
  constexpr int R = RPP * kMoveRows;               // rows per block
  unsigned char* base = (blockIdx.z ? a.V : a.K) + bh * a.cap * a.row_bytes +
                        (int64_t)blockIdx.x * 128 + (threadIdx.x & 7) * 16;
  const int* src = a.src + bh * a.n;
  const int r = threadIdx.x >> 3;
  const int n = (int)a.n;
  uint4 x[kMoveRows], y[kMoveRows];
  auto load = [&](uint4 (&v)[kMoveRows], int i0) {
#pragma unroll
    for (int j = 0; j < kMoveRows; ++j) {
      const int i = min(i0 + j * RPP + r, n - 1);
      v[j] = *reinterpret_cast<const uint4*>(base + (int64_t)src[i] * a.row_bytes);
    }
  };
  auto store = [&](const uint4 (&v)[kMoveRows], int i0) {
#pragma unroll
    for (int j = 0; j < kMoveRows; ++j) {
      const int i = i0 + j * RPP + r;
      if (i < n) *reinterpret_cast<uint4*>(base + (int64_t)i * a.row_bytes) = v[j];
    }
  };
  // all loads of the block have arrived, for every thread of the workgroup
  auto arrived = [&] {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };
  load(x, 0);
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += 2 * R) {
    arrived();
    if (i0 + R < n) load(y, i0 + R);
    store(x, i0);
    if (i0 + R >= n) break;
    arrived();
    if (i0 + 2 * R < n) load(x, i0 + 2 * R);
    store(y, i0 + R);
  }
}

}  // namespace
}  // namespace radar_impl

using namespace radar_impl;

extern "C" {

size_t radar_evict_workspace_bytes(const radar_config* cfg, int64_t t, int64_t heavy,
                                   int64_t recent) {
  Shape s;
  if (check_cache(cfg, &s) != RADAR_OK || t < 0 || t > s.cap || heavy < 0 || recent < 0 ||
      heavy > INT32_MAX || recent > INT32_MAX || s.n_sink + heavy + recent > INT32_MAX)
    return 0;
  const int64_t n = std::min<int64_t>(s.n_sink + heavy + recent, t);
  return align256((size_t)s.B * s.Hkv * n * 4) + align256((size_t)s.B * s.Hkv * 4);
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
  if (need == 0) return RADAR_EUNSUPPORTED;
  if (!workspace || !aligned16(workspace) || workspace_bytes < need) return RADAR_EWORKSPACE;
  EvictArgs a{};
  a.K = static_cast<unsigned char*>(K);
  a.V = static_cast<unsigned char*>(V);
  a.mass = mass;
  a.lens = lens; a.new_lens = new_lens; a.kept = kept;
  a.cut = static_cast<int*>(workspace);
  a.src = a.cut + align256((size_t)s.B * s.Hkv * 4) / 4;
  a.B = s.B; a.Hkv = s.Hkv; a.t = t; a.cap = s.cap;
  a.sink = s.n_sink; a.heavy = (int)heavy; a.recent = (int)recent;
  a.n = s.n_sink + heavy + recent;
  a.n_kept = (int)std::min<int64_t>(a.n, t);
  a.row_bytes = s.d * (s.dt == RADAR_BF16 ? 2 : 4);
  const unsigned pairs = (unsigned)(s.B * s.Hkv);
  launch(RADAR_K_TOPK, k_evict_select, dim3(pairs), dim3(kSelThreads), 0, stream, a);
  r = launch_status();
  const bool moves = a.n > 0 && a.n < t;                   // else no row does
  if (r != RADAR_OK || !(moves || new_lens)) return r;
  launch(RADAR_K_APPEND, k_evict_move,
         moves ? dim3((unsigned)(a.row_bytes / 128), pairs, 2) : dim3(1, pairs, 1),
         dim3(kMoveThreads), 0, stream, a);
  return launch_status();
}

}  // extern "C"
