// What moves rows when a sequence branches (include/radar_cache.h): the
// acceptance of a path of drafted tokens, the index of the rows it added, and the
// forking of the cache's sequences.
#include "cache_impl.h"

namespace radar_impl {
namespace {

constexpr int kMaxTree = RADAR_MAX_TREE;

struct PathArgs {
  unsigned char *K, *V;
  const int64_t *lens, *counts;
  int64_t t, cap, nodes;   // keep: nodes is the row length of path
  int Hkv, row_bytes;
  const int* parent;
  int parent_shared;
  const int64_t *tokens, *first, *choice;
  const int* given;        // keep: the path
  int* path;
  int64_t *accepted, *next, *new_lens;
};

// Rows len + path(i) of a sequence's heads to len + i, i < n, in place: path(i) >= i
// ascends, so rows read later are not among those written, and of kPasses passes' rows at a
// time all are read before one is written. A wave per head, one after the other down the
// path: 8 rows of each of 8 heads 3.4 us, 512 rows 49, 4096 550; a row's 16-byte chunks on
// the lanes.
template <typename PathOf>
__device__ __forceinline__ void move_rows(const PathArgs& a, int64_t b, int64_t len, int n,
                                          PathOf&& path) {
  constexpr int kPasses = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int per = a.row_bytes / 16, rows = kWave / per;
  const int r = lane / per, c = lane % per;
  for (int h = wave; h < a.Hkv; h += waves) {
    const int64_t at = ((b * a.Hkv + h) * a.cap + len) * a.row_bytes + c * 16;
    for (int i0 = 0; i0 < n; i0 += kPasses * rows) {
      u32x4_t k[kPasses], v[kPasses];      // (arrays of uint4 go to scratch memory)
      int from[kPasses];
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int i = i0 + p * rows + r;
        from[p] = i < n ? path(i) : i;
        if (from[p] != i) {                // (a row that stays is not written)
          k[p] = *reinterpret_cast<const u32x4_t*>(a.K + at + (int64_t)from[p] * a.row_bytes);
          v[p] = *reinterpret_cast<const u32x4_t*>(a.V + at + (int64_t)from[p] * a.row_bytes);
        }
      }
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int i = i0 + p * rows + r;
        if (from[p] != i) {
          *reinterpret_cast<u32x4_t*>(a.K + at + (int64_t)i * a.row_bytes) = k[p];
          *reinterpret_cast<u32x4_t*>(a.V + at + (int64_t)i * a.row_bytes) = v[p];
        }
      }
    }
  }
}

// A workgroup per sequence. Its first wave holds the nodes, U to a lane, and walks
// down: of the nodes behind the current one whose parent it is and whose token is the
// one wanted, the lowest, by a ballot for each 64 (a step is some 100 cycles; the
// loads, all at once, are most of the kernel's time: 2.4 us for 26 nodes, 3.5 for 64
// sequences of 63). All waves then move the rows.
// The sequence's length is read by the first wave only and before anything is
// written, so that the new length may take its place.
template <int U>
__global__ __launch_bounds__(1024) void k_accept(PathArgs a) {
  __shared__ int path[kMaxTree];
  __shared__ int64_t at;
  __shared__ int n_path;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t b = blockIdx.x;
  if (tid < kWave) {
    const int64_t len = a.lens ? a.lens[b] : a.t;
    const int64_t cnt = a.counts ? a.counts[b] : a.nodes;
    const bool ok = len >= 0 && len <= a.t && cnt >= 0 && cnt <= a.nodes && len + cnt <= a.cap;
    const int nodes = ok ? (int)cnt : 0;
    int par[U];
    int64_t tok[U], pick[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = u * kWave + lane;
      par[u] = -2;                         // no node's
      tok[u] = pick[u] = 0;
      if (i < nodes) {
        par[u] = a.parent ? a.parent[(a.parent_shared ? 0 : b * a.nodes) + i] : i - 1;
        tok[u] = a.tokens[b * a.nodes + i];
        pick[u] = a.choice[b * a.nodes + i];
      }
    }
    int64_t want = a.first[b];
    int cur = -1, n = 0;
    for (;;) {                             // cur ascends
      int hit = -1;
      int64_t then = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (hit >= 0) continue;            // uniform
        const int i = u * kWave + lane;
        const u64 fits = __ballot(par[u] == cur && i > cur && tok[u] == want);
        if (fits) {
          const int l = __ffsll(fits) - 1;
          hit = u * kWave + l;
          const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)(u64)pick[u], l);
          const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)((u64)pick[u] >> 32), l);
          then = (int64_t)(((u64)hi << 32) | lo);
        }
      }
      if (hit < 0) break;
      if (lane == 0) path[n] = hit;
      ++n;
      cur = hit;
      want = then;
    }
    if (lane == 0) {
      at = ok ? len : -1;
      n_path = n;
      a.accepted[b] = n;
      a.next[b] = ok ? want : -1;
      if (a.new_lens) a.new_lens[b] = len + n;
    }
  }
  __syncthreads();
  const int n = n_path;
  for (int i = tid; i < a.nodes; i += blockDim.x) a.path[b * a.nodes + i] = i < n ? path[i] : -1;
  if (a.K) move_rows(a, b, at, n, [&](int i) { return path[i]; });
}

// The same move along a given path: the first wave looks it over.
__global__ __launch_bounds__(1024) void k_keep(PathArgs a) {
  __shared__ int64_t at;
  __shared__ int n_path;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t b = blockIdx.x;
  const int* given = a.given + b * a.nodes;
  if (tid < kWave) {
    const int64_t len = a.lens ? a.lens[b] : a.t;
    const int64_t cnt = a.counts ? a.counts[b] : a.nodes;
    bool ok = len >= 0 && len <= a.t && cnt >= 0 && cnt <= a.nodes;
    const int n = ok ? (int)cnt : 0;
    for (int i = lane; i < n; i += kWave) {
      const int x = given[i];
      if (x <= (i ? given[i - 1] : -1) || len + x >= a.cap) ok = false;
    }
    ok = __all(ok);
    if (lane == 0) {
      at = len;
      n_path = ok ? n : 0;
      if (a.new_lens) a.new_lens[b] = ok ? len + n : -1;
    }
  }
  __syncthreads();
  move_rows(a, b, at, n_path, [&](int i) { return given[i]; });
}

// Row j of pos: each sequence's j-th row of [lens0, lens) that ends a segment, -1 if
// there is none.
__global__ __launch_bounds__(256) void k_closings(const int64_t* lens0, const int64_t* lens, int64_t t,
                                                  int64_t most, int B, int c, int n_sink, int n,
                                                  int64_t* pos) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= B) return;
  const int64_t from = lens0[b], len = lens[b];
  const bool ok = from >= 0 && from <= len && len <= t;
  const int64_t end = min(len, from + most), x = max(from - n_sink, (int64_t)0);
  int64_t row = n_sink + (x / c + 1) * c - 1;
  for (int j = 0; j < n; ++j, row += c) pos[(int64_t)j * B + b] = ok && row < end ? row : -1;
}

// ---------------------------------------------------------------------------
// forking
// ---------------------------------------------------------------------------
struct ForkArgs {
  unsigned char *K, *V, *mass, *summ;
  const int64_t *src, *lens;
  int64_t* new_lens;       // written here, unless it is lens
  int B, Hkv;
  int64_t t, first, cap;
  int row_bytes;
  int c, n_sink, summ_bytes;         // of a summary
  int64_t summ_rows;
};

__device__ __forceinline__ int64_t fork_len(const ForkArgs& a, int64_t s) {
  return s == -1 ? 0 : s < -1 || s >= a.B ? -1 : a.lens ? a.lens[s] : a.t;
}

// A workgroup moves the same bytes of a head's rows in every sequence, so no other
// one meets the bytes that it overwrites, and the map needs an order within it only.
// Each workgroup makes the list of the moves once: those whose destination no move
// still has to read come first, then those that this sets free, and so on; what is
// left are cycles, whose first sequence is saved.
//
// Memory bounds it, by the streams that are open at once: one sequence to one 5.6 TB/s (268
// MB each way: 96 us), to seven 4.65 (16411 rows of 8 heads: 115 us), to 31 4.2; any map of 16
// 4.6 (12001 rows of 16 heads: 559 us). A workgroup's start, with the list, is some 5 us for up
// to 16 sequences (of 30 rows: 8 us). The list takes a round for each link of a chain and above
// 64 sequences, where a whole workgroup makes it, barriers in each; there every member of a
// cycle walks all of it (rows of one head, 16 a sequence, all moves: 64 sequences as pairs 37 us,
// a cycle 32, a chain 35; 65: 33, 38, 60; 256: 100, 119, 217; 2048: 741, 1600, 3330).
constexpr int kInFlight = 8, kForkThreads = 256;
// a move is dst << 16 | src; kNone as dst: src is saved; kSaved in src: src as it was saved;
// kZero as src: zeros
constexpr uint32_t kNone = 0xffffu, kSaved = 0x8000u, kZero = 0x7fffu;
static_assert(RADAR_MAX_FORK <= kZero, "sequences in 15 bits");
constexpr int kStay = -1, kFreed = -2;

struct ForkList {
  const uint32_t* moves;   // LDS
  const int* len;          // LDS
  int n;
};

// One kind of memory: a head's columns of V in a sequence, so many for its length
struct ForkPlane {
  unsigned char* base;     // of head 0 (v_off: of K, and V's lies v_off behind)
  int64_t v_off, head, seq;          // bytes
  int64_t units, lo;
  int sub, div, per;
  int64_t tiles;
  // columns of a sequence of m rows
  __device__ __forceinline__ int64_t columns(int m) const {
    return max((int64_t)0, (int64_t)((max(m, sub) - sub) / div) - lo) * per;
  }
};

// Up to kBatch moves of one tile, read together; what they read is written a step later,
// behind the next step's loads (a wait for loads is one for the stores before them too).
// The lanes hold 64 moves of the list, and how many of the tile's columns their sources
// have; moves of none are passed over. Moves from one sequence that follow one another
// read it once.
template <typename V, int COLS, bool MASS, bool NT>
struct ForkStep {
  static constexpr int kBatch = kInFlight / COLS, kTile = kForkThreads * COLS;
  V v[kBatch][COLS];
  unsigned char* at;       // this thread's first column in sequence 0
  int64_t seq;
  uint32_t lane_move;
  int lane_have, lane_old;
  u64 take;                // the lanes whose moves these are

  // the moves [e1, e1 + 64) of tile i: which of them do anything
  __device__ __forceinline__ u64 set(const ForkPlane& p, const ForkList& l, int64_t i, int e1) {
    const int64_t tile = i % p.tiles, plane = i / p.tiles, head = p.v_off ? plane >> 1 : plane;
    const int64_t x0 = tile * kTile;
    at = p.base + (p.v_off && (plane & 1) ? p.v_off : 0) + head * p.head +
         (x0 + threadIdx.x) * (int64_t)sizeof(V);
    seq = p.seq;
    const int e = e1 + (int)(threadIdx.x & 63);
    lane_move = l.moves[min(e, l.n - 1)];
    auto have = [&](uint32_t s) {
      return s < kZero ? (int)min(max(p.columns(l.len[s]) - x0, (int64_t)0), (int64_t)kTile) : 0;
    };
    lane_have = have(lane_move & 0x7fffu);
    lane_old = MASS ? have(lane_move >> 16) : 0;
    return __ballot(e < l.n && (lane_have > 0 || lane_old > 0));
  }
  // the first of them, and those that are left
  __device__ __forceinline__ u64 pick(u64 moves) {
    u64 rest = moves;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) rest &= rest - (rest != 0);
    take = moves ^ rest;
    return rest;
  }
  __device__ __forceinline__ void like(const ForkStep& o) {
    at = o.at;
    seq = o.seq;
    lane_move = o.lane_move;
    lane_have = o.lane_have;
    lane_old = o.lane_old;
  }
  __device__ __forceinline__ void load() {
    u64 t = take;
    uint32_t before = kNone;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (!t) continue;                    // uniform
      const int k = __ffsll(t) - 1;
      t &= t - 1;
      const uint32_t s = __builtin_amdgcn_readlane(lane_move, k) & 0xffffu;
      const bool again = s == before;
      before = s;
      if (again || s >= kZero) continue;
      const int have = __builtin_amdgcn_readlane(lane_have, k);
      const unsigned char* from = at + s * seq;
#pragma unroll
      for (int c = 0; c < COLS; ++c) {
        if (MASS) v[j][c] = V{};
        if ((int)threadIdx.x + c * kForkThreads < have) {
          const V* q = reinterpret_cast<const V*>(from + c * kForkThreads * sizeof(V));
          v[j][c] = NT ? __builtin_nontemporal_load(q) : *q;
        }
      }
    }
  }
  // MASS: zeros behind what the source has, up to the destination's length
  __device__ __forceinline__ void store(V (&saved)[COLS]) {
    u64 t = take;
    uint32_t before = kNone;
    V w[COLS];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (!t) continue;
      const int k = __ffsll(t) - 1;
      t &= t - 1;
      const uint32_t e = __builtin_amdgcn_readlane(lane_move, k), s = e & 0xffffu, dst = e >> 16;
      if (s != before) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) w[c] = s & kSaved ? saved[c] : s == kZero ? V{} : v[j][c];
        // (one of no columns here was passed over when it should have been saved)
        if (MASS && (s & kSaved) && __builtin_amdgcn_readlane(lane_have, k) == 0)
#pragma unroll
          for (int c = 0; c < COLS; ++c) w[c] = V{};
      }
      before = s;
      if (dst == kNone) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) saved[c] = w[c];
        continue;
      }
      int upto = __builtin_amdgcn_readlane(lane_have, k);
      if (MASS) upto = max(upto, __builtin_amdgcn_readlane(lane_old, k));
      unsigned char* to = at + dst * seq;
#pragma unroll
      for (int c = 0; c < COLS; ++c)
        if ((int)threadIdx.x + c * kForkThreads < upto) {
          V* q = reinterpret_cast<V*>(to + c * kForkThreads * sizeof(V));
          if (NT) __builtin_nontemporal_store(w[c], q);
          else *q = w[c];
        }
    }
  }
};

// Every tile of the planes of a kind, a step ahead. The workgroups take them in turn from
// number `turn` of all on, where the kind before has left off; returns the next turn.
template <typename V, int COLS, bool MASS, bool NT>
__device__ __forceinline__ int64_t fork_planes(ForkPlane p, const ForkList& l, int64_t planes, int64_t turn) {
  using Step = ForkStep<V, COLS, MASS, NT>;
  p.tiles = (p.units + Step::kTile - 1) / Step::kTile;
  const int64_t all = planes * p.tiles;
  const int late = (int)((blockIdx.x + gridDim.x - turn % gridDim.x) % gridDim.x);
  int64_t i = (int64_t)late - gridDim.x;
  int e1 = l.n;
  u64 rest = 0;
  V saved[COLS];
#pragma unroll
  for (int c = 0; c < COLS; ++c) saved[c] = V{};
  // the step behind `before`; false: there is none
  auto next = [&](Step& s, const Step& before) {
    if (rest) {
      s.like(before);
    } else {
      do {
        e1 += kWave;
        if (e1 >= l.n) {
          e1 = 0;
          i += gridDim.x;
          if (i >= all) return false;
        }
        rest = s.set(p, l, i, e1);
      } while (!rest);
    }
    rest = s.pick(rest);
    s.load();
    return true;
  };
  Step a, b;
  if (!next(a, b)) return turn + all;
  for (;;) {
    const bool more_b = next(b, a);
    a.store(saved);
    if (!more_b) break;
    const bool more_a = next(a, b);
    b.store(saved);
    if (!more_a) break;
  }
  return turn + all;
}

// (rows: of the longest sequence that a move reads; all: or writes)
template <int COLS, bool NT>
__device__ __forceinline__ void fork_all(const ForkArgs& a, const ForkList& l, int rows, int all) {
  ForkPlane kv{a.K + a.first * a.row_bytes, a.V - a.K, a.cap * a.row_bytes, a.Hkv * a.cap * a.row_bytes,
               0, a.first, 0, 1, a.row_bytes / 16, 0};
  kv.units = kv.columns(rows);
  int64_t turn = fork_planes<u32x4_t, COLS, false, NT>(kv, l, 2 * a.Hkv, 0);
  if (a.mass) {
    const ForkPlane mass{a.mass, 0, a.cap * 4, a.Hkv * a.cap * 4, all, 0, 0, 1, 1, 0};
    turn = fork_planes<uint32_t, COLS, true, false>(mass, l, a.Hkv, turn);
  }
  if (a.summ) {
    const int64_t seg0 = max((int64_t)0, a.first - a.n_sink) / a.c;
    ForkPlane summ{a.summ + seg0 * a.summ_bytes, 0, a.summ_rows * a.summ_bytes,
                   a.Hkv * a.summ_rows * a.summ_bytes, 0, seg0, a.n_sink, a.c, a.summ_bytes / 16, 0};
    summ.units = summ.columns(rows);
    fork_planes<u32x4_t, COLS, false, false>(summ, l, a.Hkv, turn);
  }
}

// The list of up to 64 sequences' moves by one wave, a sequence a lane: what a round's
// moves read is marked in LDS, by the round's number.
__device__ __forceinline__ int list_moves(const ForkArgs& a, int64_t s, int src, int* mark, uint32_t* list) {
  const int lane = threadIdx.x & 63;
  auto order = [] {                        // the wave's LDS operations, as written
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  bool open = src != kStay;
  int n = 0;
  for (int round = 1;; ++round) {
    mark[lane] = 0;
    order();
    if (open && src >= 0) mark[src] = round;
    order();
    const bool ready = open && mark[lane] != round;
    const u64 now = __ballot(ready);
    if (!now) break;
    if (ready) list[n + __popcll(now & ((1ull << lane) - 1))] = (uint32_t)lane << 16 | (src == kFreed ? kZero : src);
    n += __popcll(now);
    open = open && !ready;
  }
  u64 left = __ballot(open);               // cycles
  while (left) {
    const int b = __ffsll(left) - 1;
    if (lane == 0) list[n] = kNone << 16 | (uint32_t)b;
    ++n;
    for (int x = b;;) {
      const int y = __builtin_amdgcn_readlane(src, x);
      if (lane == 0) list[n] = (uint32_t)x << 16 | (uint32_t)y | (y == b ? kSaved : 0);
      ++n;
      left &= ~(1ull << x);
      if (y == b) break;
      x = y;
    }
  }
  return n;
}

__global__ __launch_bounds__(kForkThreads) void k_fork(ForkArgs a) {
  extern __shared__ int fork_lds[];
  const int lds_b = max(a.B, kWave);
  int* src = fork_lds;                     // or kStay, kFreed
  int* left = src + lds_b;                 // moves that still read it; -1: listed
  int* len = left + lds_b;
  uint32_t* list = reinterpret_cast<uint32_t*>(len + lds_b);   // dst << 16 | src
  __shared__ int n_list;
  __shared__ u64 moved;                    // rows of K
  __shared__ int longest[2];               // rows of a sequence that is read; or written
  const int tid = threadIdx.x;
  if (tid == 0) {
    n_list = 0;
    moved = 0;
    longest[0] = longest[1] = 0;
  }
  auto kind = [&](int64_t s, int b) {
    return s >= 0 && s < a.B && s != b && len[s] >= 0 ? (int)s : s == -1 ? kFreed : kStay;
  };
  if (a.B <= kWave) {
    if (tid < kWave) {
      const bool on = tid < a.B;
      const int64_t n = on && a.lens ? a.lens[tid] : a.t, s = on ? a.src[tid] : tid;
      len[tid] = on && n >= 0 && n <= a.t ? (int)n : -1;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const int m = list_moves(a, s, on ? kind(s, tid) : kStay, left, list);
      if (on && a.new_lens && blockIdx.x == 0) a.new_lens[tid] = fork_len(a, s);
      if (tid == 0) n_list = m;
    }
    __syncthreads();
  } else {
    for (int b = tid; b < a.B; b += kForkThreads) {
      const int64_t n = a.lens ? a.lens[b] : a.t;
      len[b] = n >= 0 && n <= a.t ? (int)n : -1;
      left[b] = 0;
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += kForkThreads) {
      const int64_t s = a.src[b];
      src[b] = kind(s, b);
      if (src[b] >= 0) atomicAdd(&left[src[b]], 1);
      if (a.new_lens && blockIdx.x == 0) a.new_lens[b] = fork_len(a, s);
    }
    // (a move takes its place in the list before it frees its source for others)
    for (bool more = true; more;) {
      __syncthreads();
      bool any = false;
      for (int b = tid; b < a.B; b += kForkThreads) {
        if (src[b] == kStay || __atomic_load_n(&left[b], __ATOMIC_RELAXED) != 0) continue;
        const uint32_t s = src[b] == kFreed ? kZero : (uint32_t)src[b];
        list[atomicAdd(&n_list, 1)] = (uint32_t)b << 16 | s;
        __threadfence_block();
        left[b] = -1;
        if (src[b] >= 0) atomicSub(&left[src[b]], 1);
        any = true;
      }
      more = __syncthreads_or(any);
    }
    // cycles: the lowest sequence of each writes it down
    for (int b = tid; b < a.B; b += kForkThreads) {
      if (src[b] == kStay || left[b] < 0) continue;
      int size = 1, low = b;
      for (int x = src[b]; x != b; x = src[x]) {
        low = min(low, x);
        ++size;
      }
      if (low != b) continue;
      uint32_t* out = list + atomicAdd(&n_list, size + 1);
      *out++ = kNone << 16 | (uint32_t)b;
      int x = b;
      for (; src[x] != b; x = src[x]) *out++ = (uint32_t)x << 16 | (uint32_t)src[x];
      *out = (uint32_t)x << 16 | (uint32_t)b | kSaved;
    }
    __syncthreads();
  }
  const int n = n_list;
  if (n == 0) return;
  // past the caches, of 256 MB, where the call moves more than they hold
  int64_t rows = 0;
  int most = 0, most_old = 0;
  for (int e = tid; e < n; e += kForkThreads) {
    const uint32_t from = list[e] & 0x7fffu, dst = list[e] >> 16;
    if (from != kZero) {
      rows += max((int64_t)0, len[from] - a.first);
      most = max(most, len[from]);
    }
    if (dst != kNone) most_old = max(most_old, len[dst]);
  }
  if (tid < n) {
    atomicAdd(&moved, (u64)rows);
    atomicMax(&longest[0], most);
    atomicMax(&longest[1], max(most, most_old));
  }
  __syncthreads();
  const bool past = 4 * a.Hkv * (int64_t)moved * a.row_bytes > (256 << 20);
  const ForkList l{list, len, n};
  // few moves: two columns of each in flight
  if (n <= 4) {
    if (past) fork_all<2, true>(a, l, longest[0], longest[1]);
    else fork_all<2, false>(a, l, longest[0], longest[1]);
  } else {
    if (past) fork_all<1, true>(a, l, longest[0], longest[1]);
    else fork_all<1, false>(a, l, longest[0], longest[1]);
  }
}

// the new lengths in the place of the old ones, once no workgroup reads those
__global__ __launch_bounds__(1024) void k_fork_lens(ForkArgs a) {
  constexpr int kPer = RADAR_MAX_FORK / 1024;
  int64_t n[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = i * 1024 + threadIdx.x;
    n[i] = b < a.B ? fork_len(a, a.src[b]) : 0;
  }
  __builtin_amdgcn_s_waitcnt(0);           // every load of this wave has returned
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = i * 1024 + threadIdx.x;
    if (b < a.B) a.new_lens[b] = n[i];
  }
}

bool bad16(const void* p) { return !p || !aligned16(p); }
bool odd16(const void* p) { return p && !aligned16(p); }
// lists of numbers, read one by one, lie on their elements' size: a row of one may
// begin anywhere
template <typename T>
bool off(const T* p) { return reinterpret_cast<uintptr_t>(p) % sizeof(T) != 0; }
template <typename... T>
bool any_off(const T*... p) { return (off(p) || ...); }
// two lists of n, given, share memory without being one
bool meet(const int64_t* p, const int64_t* q, int n) {
  return p && q && p != q && std::abs((intptr_t)p - (intptr_t)q) < (intptr_t)n * 8;
}
int esize(const Shape& s) { return s.dt == RADAR_BF16 ? 2 : 4; }
// what a call moves in place has its own memory
struct Plane {
  const void* p;
  int64_t bytes;
};
bool overlap(std::initializer_list<Plane> planes) {
  for (const Plane& x : planes)
    for (const Plane& y : planes)
      if (&x != &y && x.p && y.p && (uintptr_t)x.p <= (uintptr_t)y.p &&
          (uintptr_t)y.p - (uintptr_t)x.p < (uintptr_t)x.bytes)
        return true;
  return false;
}
int64_t cache_rows(const Shape& s) { return (int64_t)s.B * s.Hkv * s.cap; }
bool caches_overlap(const Shape& s, const void* K, const void* V) {
  const int64_t bytes = cache_rows(s) * s.d * esize(s);
  return overlap({{K, bytes}, {V, bytes}});
}

// the index's fields of the config, with radar.h's limits
radar_status check_index(const radar_config* cfg, Shape* s) {
  const radar_status r = check_cache(cfg, s);
  if (r != RADAR_OK) return r;
  const int n = cfg->n_features;
  if (cfg->seg_len < 1) return RADAR_EINVAL;
  if (n != 64 && n != 128 && n != 256 && n != 512 && n != 1024 && n != 2048) return RADAR_EUNSUPPORTED;
  s->n = n; s->c = cfg->seg_len; s->s_cap = cfg->capacity / cfg->seg_len;
  return RADAR_OK;
}

PathArgs path_args(const Shape& s, void* K, void* V, int64_t t, const int64_t* lens, int64_t nodes,
                   const int64_t* counts, int64_t* new_lens) {
  PathArgs a{};
  a.K = static_cast<unsigned char*>(K); a.V = static_cast<unsigned char*>(V);
  a.lens = lens; a.counts = counts; a.t = t; a.cap = s.cap; a.nodes = nodes;
  a.Hkv = s.Hkv; a.row_bytes = s.d * esize(s);
  a.new_lens = new_lens;
  return a;
}

int path_threads(const Shape& s) { return kWave * std::min(16, s.Hkv); }

int64_t closings(const Shape& s, int64_t most) { return ceil_div(most, s.c); }
int64_t closings_bytes(const Shape& s, int64_t most) {
  return (int64_t)align256((size_t)(closings(s, most) * s.B * 8));
}

}  // namespace
}  // namespace radar_impl

using namespace radar_impl;

extern "C" {

radar_status radar_accept_tree(const radar_config* cfg, void* K, void* V, int64_t t,
                               const int64_t* lens, int64_t nodes, const int64_t* counts,
                               const int32_t* parent, int32_t parent_shared,
                               const int64_t* tokens, const int64_t* first, const int64_t* choice,
                               int32_t* path, int64_t* accepted, int64_t* next, int64_t* new_lens,
                               hipStream_t stream) {
  Shape s;
  const radar_status r = check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  if (odd16(K) || odd16(V) || !K != !V || !tokens || !first || !choice || !path || !accepted || !next ||
      any_off(tokens, first, choice, path, accepted, next, lens, counts, parent, new_lens) || nodes < 1 ||
      meet(new_lens, lens, s.B) || meet(next, first, s.B))
    return RADAR_EINVAL;
  if (nodes > kMaxTree) return RADAR_EUNSUPPORTED;
  if (t < 0 || t > s.cap || (!lens && nodes > s.cap - t)) return RADAR_ECAPACITY;
  if (caches_overlap(s, K, V)) return RADAR_EINVAL;
  PathArgs a = path_args(s, K, V, t, lens, nodes, counts, new_lens);
  a.parent = parent; a.parent_shared = parent_shared != 0;
  a.tokens = tokens; a.first = first; a.choice = choice;
  a.path = path; a.accepted = accepted; a.next = next;
  const dim3 grid((unsigned)s.B), block((unsigned)path_threads(s));
  if (nodes <= kWave) launch(RADAR_K_APPEND, k_accept<1>, grid, block, 0, stream, a);
  else launch(RADAR_K_APPEND, k_accept<kMaxTree / kWave>, grid, block, 0, stream, a);
  return launch_status();
}

radar_status radar_keep_path(const radar_config* cfg, void* K, void* V, int64_t t,
                             const int64_t* lens, const int32_t* path, int64_t n,
                             const int64_t* counts, int64_t* new_lens, hipStream_t stream) {
  Shape s;
  const radar_status r = check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  if (bad16(K) || bad16(V) || n < 0 || (n > 0 && !path) || any_off(path, lens, counts, new_lens) ||
      meet(new_lens, lens, s.B))
    return RADAR_EINVAL;
  if (t < 0 || t > s.cap || n > s.cap) return RADAR_ECAPACITY;
  if (caches_overlap(s, K, V)) return RADAR_EINVAL;
  PathArgs a = path_args(s, K, V, t, lens, n, counts, new_lens);
  a.given = path;
  launch(RADAR_K_APPEND, k_keep, dim3((unsigned)s.B), dim3((unsigned)path_threads(s)), 0, stream, a);
  return launch_status();
}

size_t radar_extend_index_workspace_bytes(const radar_config* cfg, int64_t most) {
  Shape s;
  if (check_index(cfg, &s) != RADAR_OK || most < 0 || most > s.cap) return 0;
  return (size_t)std::max<int64_t>(256, closings_bytes(s, most));
}

radar_status radar_extend_index(const radar_config* cfg, const void* K, const void* omega,
                                int64_t t0, int64_t t, const int64_t* lens0, const int64_t* lens,
                                int64_t most, float* summaries, void* workspace,
                                size_t workspace_bytes, hipStream_t stream) {
  Shape s;
  radar_status r = check_index(cfg, &s);
  if (r != RADAR_OK) return r;
  if (cfg->omega_dtype != RADAR_F32 && cfg->omega_dtype != RADAR_BF16) return RADAR_EINVAL;
  if (cfg->omega_dtype == RADAR_BF16 && cfg->kv_dtype != RADAR_BF16) return RADAR_EINVAL;
  s.obf = cfg->omega_dtype == RADAR_BF16;
  if (bad16(K) || bad16(omega) || bad16(summaries) || any_off(lens0, lens) || !lens0 != !lens)
    return RADAR_EINVAL;
  if (t < 0 || t > s.cap) return RADAR_ECAPACITY;
  if (!lens) {
    if (t0 < 0 || t0 > t) return RADAR_ECAPACITY;
    const int64_t s0 = std::max<int64_t>(0, t0 - s.n_sink) / s.c;
    const int64_t s1 = std::max<int64_t>(0, t - s.n_sink) / s.c;
    if (s1 == s0) return RADAR_OK;
    return launch_build(s, after_sinks(s, K), omega, summaries, (int)s0, (int)(s1 - s0), nullptr, stream);
  }
  if (most < 0 || most > s.cap) return RADAR_ECAPACITY;
  if (bad16(workspace) || workspace_bytes < (size_t)std::max<int64_t>(256, closings_bytes(s, most)))
    return RADAR_EWORKSPACE;
  const int n = (int)closings(s, most);
  if (n == 0) return RADAR_OK;
  int64_t* pos = static_cast<int64_t*>(workspace);
  launch(RADAR_K_BUILD, k_closings, dim3((unsigned)ceil_div(s.B, 256)), dim3(256), 0, stream, lens0, lens, t,
         most, s.B, s.c, s.n_sink, n, pos);
  r = launch_status();
  for (int j = 0; j < n && r == RADAR_OK; ++j)
    r = launch_build(s, after_sinks(s, K), omega, summaries, 0, 1, pos + (int64_t)j * s.B, stream);
  return r;
}

radar_status radar_fork(const radar_config* cfg, void* K, void* V, float* mass, float* summaries,
                        const int64_t* src, int64_t first, int64_t t, const int64_t* lens,
                        int64_t* new_lens, hipStream_t stream) {
  Shape s;
  const radar_status r = summaries ? check_index(cfg, &s) : check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  if (bad16(K) || bad16(V) || odd16(mass) || odd16(summaries) || !src ||
      any_off(src, lens, new_lens) || src == new_lens || meet(new_lens, src, s.B) || meet(new_lens, lens, s.B) ||
      first < 0)
    return RADAR_EINVAL;
  if (t < 0 || t > s.cap) return RADAR_ECAPACITY;
  if (s.B > RADAR_MAX_FORK) return RADAR_EUNSUPPORTED;
  const int64_t kv_bytes = cache_rows(s) * s.d * esize(s);
  if (overlap({{K, kv_bytes},
               {V, kv_bytes},
               {mass, cache_rows(s) * 4},
               {summaries, (int64_t)s.B * s.Hkv * std::max<int64_t>(1, s.s_cap) * s.n * 4}}))
    return RADAR_EINVAL;
  const bool in_place = new_lens && new_lens == lens;
  ForkArgs a{};
  a.K = static_cast<unsigned char*>(K); a.V = static_cast<unsigned char*>(V);
  a.mass = reinterpret_cast<unsigned char*>(mass); a.summ = reinterpret_cast<unsigned char*>(summaries);
  a.src = src; a.lens = lens; a.new_lens = in_place ? nullptr : new_lens;
  a.B = s.B; a.Hkv = s.Hkv; a.t = t; a.first = std::min(first, t); a.cap = s.cap;
  a.row_bytes = s.d * esize(s);
  a.n_sink = s.n_sink;
  int64_t units[3] = {(t - a.first) * (a.row_bytes / 16), mass ? t : 0, 0};      // columns of a head, at most
  if (summaries) {
    a.c = s.c; a.summ_bytes = s.n * 4; a.summ_rows = std::max<int64_t>(1, s.s_cap);
    const int64_t seg0 = std::max<int64_t>(0, a.first - s.n_sink) / s.c;
    const int64_t seg1 = std::max<int64_t>(0, t - s.n_sink) / s.c;
    units[2] = (seg1 - seg0) * (a.summ_bytes / 16);
  }
  const int64_t items = s.Hkv * (2 * ceil_div(units[0], kForkThreads) + ceil_div(units[1], kForkThreads) +
                                 ceil_div(units[2], kForkThreads));
  // three words a sequence (of a wave's, at least), and up to 3/2 in the list
  const size_t lds = (size_t)std::max(s.B, kWave) * 18;
  const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(items, 4 * num_cu()));
  launch(RADAR_K_APPEND, k_fork, dim3(grid), dim3(kForkThreads), (lds + 15) / 16 * 16, stream, a);
  const radar_status st = launch_status();
  if (st != RADAR_OK || !in_place) return st;
  a.new_lens = new_lens;
  launch(RADAR_K_APPEND, k_fork_lens, dim3(1), dim3(1024), 0, stream, a);
  return launch_status();
}

}  // extern "C"
