// Attention of drafted tokens over the cache (include/radar_cache.h): how a call is cut
// into blocks and the merge of their partials. The blocks are tree.hip's.
#include "tree_impl.h"

namespace radar_impl {
namespace {

constexpr int kSlots = 512;                // workgroups that the chip holds at once
constexpr int kFew = 256;                  // partials of a row that one wave merges

// A query row's output from its partials by NW waves: D / 4 lanes on four dims each of one
// partial, the others on the next. One wave a row where there are enough rows to fill the
// chip (8192 rows of up to 13 partials, 29 MB: 10 us; 1024 of 63: 5.5 with four; 4671 of 10
// and up to 230, 27 sequences of one head: 8, with four 16.5).
//   out = sum_i acc_i 2^(m_i - m) / sum_i l_i 2^(m_i - m),  m = max_i m_i
template <typename T, int D, int NW>
__global__ __launch_bounds__(256) void k_tree_merge(TreeArgs a, int rows_per_tile) {
  constexpr int kThreads = NW * kWave, kTpp = D / 4, kGroups = kThreads / kTpp;
  constexpr int kPer = 4 / NW, kMost = NW == 1 ? kFew : kSlots + 1;
  __shared__ float f_lds[kPer][kMost], l_lds[kPer][kMost];
  __shared__ float red[8];
  __shared__ __attribute__((aligned(16))) f32x4_t acc_lds[256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int own = wave / NW, tid = threadIdx.x % kThreads;
  auto sync = [] {
    if constexpr (NW == 1) {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
      __syncthreads();
    }
  };
  const int n_rows = a.B * a.nodes * a.Hq;   // below 2^27
  const TreeBatch batch(a);
  const int each = a.parts ? ((int)((a.t + a.nodes - 1) >> a.step_log2) + a.parts) / a.parts : batch.each();
  for (int x = blockIdx.x * kPer + own; x < n_rows; x += gridDim.x * kPer) {
    const int hq = x % a.Hq, node = x / a.Hq % a.nodes, hk = hq >> a.g_log2;
    const int64_t b = x / a.Hq / a.nodes;
    const TreeSeq s = batch.seq(__builtin_amdgcn_readfirstlane((int)b));
    T* o = static_cast<T*>(a.out) + b * a.o_seq + node * a.o_node + hq * a.o_head;
    if (s.rows < 0 || (a.zero && node >= s.nodes)) {
      const T x = from_f32<T>(s.rows < 0 ? __uint_as_float(0x7fc00000u) : 0.f);
      for (int i = tid; i < D; i += kThreads) o[i] = x;
      continue;
    }
    if (node >= s.nodes) continue;
    const int row = node * a.G + (hq & (a.G - 1));
    int seq = (int)b;
    const TreeCut cut = a.parts ? TreeCut{each, a.parts, (int)b * a.Hkv * a.parts} : batch.cut(each, false, 0, &seq);
    if (cut.parts == 1) continue;          // written by its block
    // the parts that begin before the end of the row tile's rows
    const int64_t end = tree_end(a, s, (row / rows_per_tile + 1) * rows_per_tile);
    const int n = (int)((uint32_t)((int)((end - 1) >> a.step_log2) + each) / (uint32_t)each);
    const int64_t first = ((int64_t)cut.first + hk * cut.parts) * a.M + row;
    // the accumulators' first loads go out with those of m and l
    constexpr int kAhead = 4;
    const int grp = tid / kTpp, e = tid % kTpp;
    auto piece = [&](int i) {
      return *reinterpret_cast<const f32x4_t*>(a.acc + (first + (int64_t)i * a.M) * D + 4 * e);
    };
    f32x4_t ahead[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (grp + j * kGroups < n) ahead[j] = piece(grp + j * kGroups);
    float mx = -INFINITY;
    for (int i = tid; i < n; i += kThreads) {
      const float2 ml = *reinterpret_cast<const float2*>(a.ml + 2 * (first + (int64_t)i * a.M));
      f_lds[own][i] = ml.x;
      l_lds[own][i] = ml.y;
      mx = fmaxf(mx, ml.x);
    }
    mx = wave_max(mx);
    if constexpr (NW > 1) {
      if (lane == 0) red[wave] = mx;
      sync();
      mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    }
    float ls = 0.f;
    for (int i = tid; i < n; i += kThreads) {
      const float f = f_lds[own][i] == -INFINITY ? 0.f : fast_exp2(f_lds[own][i] - mx);
      f_lds[own][i] = f;
      ls = fmaf(l_lds[own][i], f, ls);
    }
    ls = wave_sum(ls);
    if constexpr (NW > 1) {
      if (lane == 0) red[4 + wave] = ls;
    }
    sync();
    if constexpr (NW > 1) ls = (red[4] + red[5]) + (red[6] + red[7]);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const f32x4_t& p, float f) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = fmaf(p[k], f, v[k]);
    };
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (grp + j * kGroups < n) add(ahead[j], f_lds[own][grp + j * kGroups]);
#pragma unroll 4
    for (int i = grp + kAhead * kGroups; i < n; i += kGroups) add(piece(i), f_lds[own][i]);
    acc_lds[threadIdx.x] = v;
    sync();
    const float* y = reinterpret_cast<const float*>(acc_lds + own * kThreads);
    for (int i = tid; i < D; i += kThreads) {
      float r = 0.f;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) r += y[g * D + i];
      o[i] = from_f32<T>(r / ls);
    }
    sync();                                // (the next row writes where this one reads)
  }
}

int log2_of(int n) { return n > 1 ? 1 + log2_of(n / 2) : 0; }
int esize(const Shape& s) { return s.dt == RADAR_BF16 ? 2 : 4; }
int slots() { return std::min(kSlots, 2 * num_cu()); }

// Row waves of M query rows a pair. Few: one, whose workgroups have the fewest rows and take
// the longest steps. More: two or four, so that fewer workgroups read the same rows; but one
// too where all row tiles are on the chip at once and a pair is short, for more workgroups
// without partials (32 / 8 heads, bf16: 64 nodes over 400 rows 19.2 us, 14.7, four sequences
// over 800 22.4, 19.2, 150 nodes over 800 21.8, 23.4; fp32: 64 nodes over 100 and 400 rows
// 22.2 and 23.0, 13.8 and 18.9, over 1500 33.2, 34.3; ragged, 121 over 377: 44, 32.5).
int tree_waves(const Shape& s, int64_t M, int64_t end, bool ragged) {
  const int64_t pairs = (int64_t)s.B * s.Hkv, tiles = pairs * ceil_div(M, flash_rows(esize(s), 1));
  if (esize(s) == 4) {
    if (M <= 48 || (tiles <= 512 && tiles * end <= (ragged ? 1 << 18 : 1 << 17))) return 1;
    return ceil_div(M, 64) * 64 < ceil_div(M, 128) * 128 ? 2 : 4;
  }
  if (M <= 32 || (tiles <= 256 && end <= 900)) return 1;
  return M <= 64 ? 2 : 4;
}

// How a call is cut: as many workgroups as the chip holds at once, or fewer, with at least
// 256 rows each in bf16 (fewer cost more in partials than they gain: four sequences of 2000
// rows and 16 nodes, 32 query heads: 21.1 us, with 128 rows 25.9; one of 4096 and 8 nodes:
// 15.5, with 512 rows 17.4) and 64 in fp32, whose products take eight times as long (16 nodes
// over 1000 rows: 19.7 us, with 256 rows 33; 121 over 400: 43, 52). Pairs of one length that
// nearly fill the chip, those of any that fill it twice and those of up to four steps (in
// fp32: of one) stay whole.
int least_rows(const Shape& s) { return esize(s) == 4 ? 64 : 256; }
int short_steps(const Shape& s) { return esize(s) == 4 ? 1 : 4; }

struct TreePlan {
  int rw, waves, mtiles, rows_per_tile, step, parts, units;
};

// Whether cutting the pairs, so that the longest has so many steps less in one part, saves
// more than the merge of so many parts takes: steps of 32, 64 and 128 query rows, of 1.3, 0.8
// and 1.1 us in bf16 at head dim 128 (fp32: 1.0 and 3.5), against 3 us and the partials there
// and back at 5 TB/s (chunks of 500 tokens, 32 / 8 heads: behind 250, whole 25 us, cut 32;
// behind 1000, 40.7 and 37.2). Not asked where memory bounds the steps.
bool worth(const Shape& s, const TreePlan& p, int64_t steps, int64_t parts, int64_t M) {
  if (M <= (esize(s) == 4 ? 48 : 32)) return true;
  double step_ns = (p.rw == 4 ? 1100. : p.rw == 2 ? 800. : 1300.) * s.d / 128 * (p.waves / 4);
  if (esize(s) == 4) step_ns = (p.rw == 1 ? 1000. : 3500.) * s.d / 128;
  return step_ns * (double)steps > 3000. + (double)(parts * M * s.d) * 4 * 2 / 5000;
}

TreePlan plan_tree(const Shape& s, int64_t nodes, int64_t t, bool ragged) {
  TreePlan p;
  const int64_t M = nodes * s.G, pairs = (int64_t)s.B * s.Hkv;
  p.rw = tree_waves(s, M, t + nodes, ragged);
  p.rows_per_tile = flash_rows(esize(s), p.rw);
  p.mtiles = (int)ceil_div(M, p.rows_per_tile);
  p.step = flash_tile(esize(s), p.rw);
  const int64_t blocks = pairs * p.mtiles;
  int room = slots();
  // Eight waves to a workgroup, whose accumulators meet in LDS: half as many workgroups and
  // partials, but all waves in step. For sequences of one length where each CU has four
  // steps and more to do and a pair at most two row tiles (16 nodes over 16K rows: 28.5 us,
  // 25.5, eight sequences of 9000: 62, 59.5; 32 nodes over 32K rows: 44.5, 41.8; four of 2000
  // and 64 nodes: 31.1, 29.1; but one of 4096 and 64: 21.7, 22.5, one of 64K and 128: 169,
  // 177), or is whole then (four of 4000 and 200 nodes: 97, 85); not at head dim 64, where
  // the vector ALUs bound (eight of 8000 and 64: 65, 69).
  p.waves = 4;
  if (p.rw > 1 && s.dt == RADAR_BF16 && s.d == 128 && !ragged && 2 * blocks <= room &&
      (p.mtiles <= 2 || 4 * blocks > room) && blocks * ceil_div(t + nodes, 2 * p.step) >= 4 * (room / 2)) {
    p.waves = 8;
    p.step *= 2;
    room /= 2;
  }
  // Up to 32 query rows a pair in bf16 (16 in fp32), whose waves have tiles of their own: one
  // workgroup a CU asks for as much as two, with half the partials (8 nodes over 64K rows: 56
  // us, 51; 32 sequences of 1000 rows, whole: 38, 29; in fp32 4 nodes over 16000: 33, 29.5;
  // but one token each, 16 sequences of 4000: 53.5, 56). And more than 48 in fp32, where the
  // matrix cores bound and one workgroup keeps them busy (32 nodes over 4000: 38.3, 34.5; 60
  // and 30 over 1500 and 750, 16 heads: 41.9, 35.4).
  const bool one = p.rw > 1 ? esize(s) == 4 : p.mtiles == 1;
  if (one) room /= 2;
  const int64_t steps = ceil_div(t + nodes, p.step);
  p.units = 0;
  const int64_t least = least_rows(s);
  if (ragged && steps > short_steps(s) && blocks <= 2 * room && pairs * steps < (1ll << 31)) {
    // (a pair's last part is shorter: as many more parts as there are pairs, at most)
    const int64_t units = std::max<int64_t>(1, room / p.mtiles);
    p.parts = 0;
    p.units = (int)std::max(units - (one ? pairs / 2 : pairs), (units + 1) / 2);
    // (as if all were of t rows)
    const int64_t each = std::max<int64_t>(std::max<int64_t>(1, least / p.step), ceil_div(steps * pairs, p.units));
    if (!worth(s, p, steps - each, std::min<int64_t>(p.units, pairs * ceil_div(steps, each)) + pairs, M)) p.parts = 1;
  } else {
    p.parts = ragged ? 1 : (int)std::max<int64_t>(1, std::min(room / blocks, ceil_div(t + nodes, least)));
    if (steps <= short_steps(s) || !worth(s, p, steps - ceil_div(steps, p.parts), pairs * p.parts, M)) p.parts = 1;
    // (as many of one length)
    p.parts = (int)ceil_div(steps, ceil_div(steps, p.parts));
  }
  return p;
}

// Partial rows of every call with at most these nodes and t: of slots / mtiles parts (or
// one), and where lengths differ one more for each of 2 slots / mtiles pairs at most, in
// mtiles tiles of min(M, 128) rows; and no more than one for each step of 32 rows, and one.
int64_t most_partials(const Shape& s, int64_t nodes, int64_t t) {
  const int64_t M = nodes * s.G, pairs = (int64_t)s.B * s.Hkv;
  return std::min(4ll * slots() * std::min<int64_t>(M, 128), (long long)(pairs * (ceil_div(t + nodes, 32) + 1) * M));
}
struct TreeWs {
  size_t acc, ml, total;
};
TreeWs tree_ws(const Shape& s, int64_t nodes, int64_t t) {
  TreeWs w;
  const size_t n = (size_t)most_partials(s, nodes, t);
  w.acc = 0;
  w.ml = align256(n * s.d * 4);
  w.total = std::max<size_t>(256, w.ml + align256(n * 8));
  return w;
}

radar_status check_nodes(const Shape& s, int64_t nodes, bool tree) {
  if (nodes < 1) return RADAR_EINVAL;
  if (tree && nodes > RADAR_MAX_TREE) return RADAR_EUNSUPPORTED;
  if (nodes > s.cap) return RADAR_ECAPACITY;
  return (int64_t)s.B * s.Hq * nodes < (1 << 27) ? RADAR_OK : RADAR_EUNSUPPORTED;
}

bool bad16(const void* p) { return !p || !aligned16(p); }
template <typename T>
bool off(const T* p) { return reinterpret_cast<uintptr_t>(p) % sizeof(T) != 0; }
bool good_rows(const radar_rows* r, int esz) {
  return r && r->data && aligned16(r->data) && r->seq * esz % 16 == 0 && r->token * esz % 16 == 0 &&
         r->head * esz % 16 == 0;
}

}  // namespace
}  // namespace radar_impl

using namespace radar_impl;

extern "C" {

size_t radar_attend_tree_workspace_bytes(const radar_config* cfg, int64_t nodes, int64_t t) {
  Shape s;
  if (check_cache(cfg, &s) != RADAR_OK || check_nodes(s, nodes, false) != RADAR_OK || t < 0 || t > s.cap)
    return 0;
  return tree_ws(s, nodes, t).total;
}

radar_status radar_attend_tree(const radar_config* cfg, const radar_rows* q, const void* K,
                               const void* V, int64_t t, const int64_t* lens, int64_t nodes,
                               const int64_t* counts, const int32_t* parent,
                               int32_t flags, const radar_rows* out, void* workspace,
                               size_t workspace_bytes, hipStream_t stream) {
  Shape s;
  radar_status r = check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  const int esz = esize(s);
  if (!good_rows(q, esz) || !good_rows(out, esz) || bad16(K) || bad16(V) || off(lens) || off(counts) ||
      off(parent) || (flags & ~(RADAR_TREE_SHARED | RADAR_TREE_ZERO)))
    return RADAR_EINVAL;
  r = check_nodes(s, nodes, parent != nullptr);
  if (r != RADAR_OK) return r;
  if (t < 0 || t > s.cap || (!lens && nodes > s.cap - t)) return RADAR_ECAPACITY;
  const TreeWs w = tree_ws(s, nodes, t);
  if (bad16(workspace) || workspace_bytes < w.total) return RADAR_EWORKSPACE;
  const TreePlan p = plan_tree(s, nodes, t, lens || counts);
  TreeArgs a{};
  a.q = q->data; a.q_seq = q->seq; a.q_node = q->token; a.q_head = q->head;
  a.out = out->data; a.o_seq = out->seq; a.o_node = out->token; a.o_head = out->head;
  a.B = s.B; a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
  a.qscale = kLog2e / std::sqrt((float)s.d);
  a.K = K; a.V = V; a.lens = lens; a.counts = counts; a.t = t; a.cap = s.cap;
  a.nodes = (int)nodes; a.parent = parent; a.parent_shared = flags & RADAR_TREE_SHARED; a.zero = (flags & RADAR_TREE_ZERO) && counts;
  a.mtiles = p.mtiles; a.M = (int)(nodes * s.G);
  a.parts = p.parts; a.units = p.units; a.least = std::max(1, least_rows(s) / p.step);
  a.g_log2 = log2_of(s.G); a.step_log2 = log2_of(p.step);
  a.acc = static_cast<float*>(workspace);
  a.ml = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + w.ml);
  if (s.dt == RADAR_BF16) {
    if (s.d == 64) launch_tree_bf16_64(a, p.rw, p.waves, stream);
    else launch_tree_bf16_128(a, p.rw, p.waves, stream);
  } else {
    if (s.d == 64) launch_tree_f32_64(a, p.rw, p.waves, stream);
    else launch_tree_f32_128(a, p.rw, p.waves, stream);
  }
  r = launch_status();
  if (r != RADAR_OK || p.parts == 1) return r;
  const int64_t rows = (int64_t)s.B * s.Hq * nodes;
  // (the heads of a sequence have as many each: 1 / Hkv of all, and one, at most)
  const bool few = (p.parts ? p.parts : p.units / s.Hkv + 1) <= kFew;
  auto merge = [&](auto tag, auto d) {
    typedef decltype(tag) T;
    constexpr int D = decltype(d)::value;
    if (few && rows > 4 * num_cu())
      launch(RADAR_K_COMBINE, k_tree_merge<T, D, 1>, dim3((unsigned)std::min<int64_t>(ceil_div(rows, 4), 1 << 16)),
             dim3(256), 0, stream, a, p.rows_per_tile);
    else
      launch(RADAR_K_COMBINE, k_tree_merge<T, D, 4>, dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(256), 0,
             stream, a, p.rows_per_tile);
  };
  if (s.dt == RADAR_BF16) {
    if (s.d == 64) merge(bf16_t{}, std::integral_constant<int, 64>{});
    else merge(bf16_t{}, std::integral_constant<int, 128>{});
  } else {
    if (s.d == 64) merge(float{}, std::integral_constant<int, 64>{});
    else merge(float{}, std::integral_constant<int, 128>{});
  }
  return launch_status();
}

}  // extern "C"
