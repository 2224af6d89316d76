// Attention over a shared prefix and attention that accumulates the rows'
// weights (include/radar_cache.h): how a call is cut into blocks, the merge of
// their partials, and the pass over the masses. The blocks are attend.hip's.
#include "attend_impl.h"

namespace radar_impl {
namespace {

// partials of a head: as many as there are workgroups, and two for roundings, of
// the prefix and, cut finer, of its own rows
constexpr int kSlots = 512, kFiner = 3;
constexpr int kMaxPartials = kSlots + 2 + kFiner * kSlots + 2;

// One head's output from its partials: 256 threads, D / 4 of them on four dims
// each of one partial, 1024 / D partials at once. The first of them are loaded with the
// maxima and sums, not behind them (26 partials: 6.3 us, 5.3). Few partials take a
// launch's 4 us, the 34 MB of 128 sequences of 32 heads 9.3.
//   out = sum_i acc_i 2^(m_i - m) / sum_i l_i 2^(m_i - m),  m = max_i m_i
template <typename T, int D>
__device__ __forceinline__ void merge_head(const FlashArgs& a, T* __restrict__ out, int64_t bhq,
                                           int lo, int64_t n_tile_o) {
  constexpr int TPP = D / 4, NG = 256 / TPP;
  __shared__ float f_lds[kMaxPartials], l_lds[kMaxPartials];
  __shared__ float red[8];
  __shared__ __attribute__((aligned(16))) f32x4_t acc_lds[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t b = bhq / a.Hq;
  const int hq = (int)(bhq % a.Hq), hk = hq / a.G, g = hq % a.G;
  const int64_t bh = b * a.Hkv + hk;
  const int64_t len = own_len(a, b, lo);
  T* o = out + bhq * D;
  const int n_own = len > 0 ? (int)((len + n_tile_o - 1) / n_tile_o) : 0;
  const int n = a.splits + n_own;
  if (len < 0 || n == 0) {                   // invalid length / nothing attended
    if (tid < D) o[tid] = from_f32<T>(len < 0 ? __uint_as_float(0x7fc00000u) : 0.f);
    return;
  }
  auto index = [&](int i) -> int64_t {       // of partial i: prefix, then own
    return i < a.splits ? ((int64_t)hk * a.splits + i) * a.M + b * a.G + g
                        : (bh * a.parts + i - a.splits) * a.G + g;
  };
  // the accumulators' first loads go out with those of m and l
  constexpr int kAhead = 4;
  const int grp = tid / TPP, e = tid % TPP;
  auto piece = [&](int i) {
    return *reinterpret_cast<const f32x4_t*>((i < a.splits ? a.pacc : a.oacc) + index(i) * D + 4 * e);
  };
  f32x4_t ahead[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
    if (grp + j * NG < n) ahead[j] = piece(grp + j * NG);
  float mx = -INFINITY;
  for (int i = tid; i < n; i += 256) {
    const float2 v = *reinterpret_cast<const float2*>((i < a.splits ? a.pml : a.oml) + 2 * index(i));
    f_lds[i] = v.x;
    l_lds[i] = v.y;
    mx = fmaxf(mx, v.x);
  }
  mx = wave_max(mx);
  if (lane == 0) red[wave] = mx;
  __syncthreads();
  const float M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  float ls = 0.f;
  for (int i = tid; i < n; i += 256) {
    const float f = f_lds[i] == -INFINITY ? 0.f : fast_exp2(f_lds[i] - M);
    f_lds[i] = f;
    ls = fmaf(l_lds[i], f, ls);
  }
  ls = wave_sum(ls);
  if (lane == 0) red[4 + wave] = ls;
  __syncthreads();
  const float L = (red[4] + red[5]) + (red[6] + red[7]);
  f32x4_t s = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](const f32x4_t& v, float f) {
#pragma unroll
    for (int x = 0; x < 4; ++x) s[x] = fmaf(v[x], f, s[x]);
  };
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
    if (grp + j * NG < n) add(ahead[j], f_lds[grp + j * NG]);
#pragma unroll 4
  for (int i = grp + kAhead * NG; i < n; i += NG) add(piece(i), f_lds[i]);
  acc_lds[tid] = s;
  __syncthreads();
  if (tid < D) {
    const float* x = reinterpret_cast<const float*>(acc_lds);
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) v += x[i * D + tid];
    o[tid] = from_f32<T>(v / L);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void k_merge(FlashArgs a, T* out, int64_t n_tile_o) {
  merge_head<T, D>(a, out, blockIdx.x, 0, n_tile_o);
}

// The end of an accumulating call: workgroups below B Hq merge a head's output,
// the others add the weights of kMassRows rows of a (b, kv head):
//   mass[i] += sum_g 2^(s_gi - m_g) / l_g.
// The logits were written by the attention pass, G words a row beside the 2 d
// elements that it read (at four heads of 128 in bf16 3% of the bytes, which cost
// the pass 15% and this one, with the masses, 10 us for 22 MB); reading K again
// instead would be half of the pass.
constexpr int kMassRows = 2048;

template <typename T, int D>
__global__ __launch_bounds__(256) void k_settle(FlashArgs a, T* out, float* __restrict__ mass,
                                                int64_t n_tile_o, int chunks) {
  const int n_head = a.B * a.Hq;
  if ((int)blockIdx.x < n_head) {
    merge_head<T, D>(a, out, blockIdx.x, 1, n_tile_o);
    return;
  }
  __shared__ float m_lds[kMaxG], r_lds[kMaxG];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t bh = (blockIdx.x - n_head) / chunks;
  const int64_t row0 = (int64_t)((blockIdx.x - n_head) % chunks) * kMassRows;
  const int64_t len = own_len(a, bh / a.Hkv, 1);
  if (row0 >= len) return;
  const int n_own = (int)((len + n_tile_o - 1) / n_tile_o);
  for (int g = wave; g < a.G; g += 4) {
    const float* ml = a.oml + 2 * (bh * a.parts * a.G + g);
    // (one pass: each lane's own maximum and sum, then the wave's)
    float m = -INFINITY, l = 0.f;
    for (int i = lane; i < n_own; i += kWave) {
      const float2 v = *reinterpret_cast<const float2*>(ml + 2 * (int64_t)i * a.G);
      const float top = fmaxf(m, v.x);
      // (no maximum yet: the sums so far are 0, or NaN where a part's logits are)
      l = top > -INFINITY ? l * fast_exp2(m - top) + v.y * fast_exp2(v.x - top) : l + v.y;
      m = top;
    }
    const float M = wave_max(m);
    l = wave_sum(m == -INFINITY ? l : l * fast_exp2(m - M));
    if (lane == 0) { m_lds[g] = M; r_lds[g] = 1.f / l; }
  }
  __syncthreads();
  const float* lg = a.logits + bh * a.G * a.tpad;
  float* ms = mass + bh * a.cap;
  const int64_t end = min(len, row0 + kMassRows);
  for (int64_t i = row0 + tid * 4; i < end; i += 1024) {
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < a.G; ++g) {
      const float4 s = *reinterpret_cast<const float4*>(lg + g * a.tpad + i);
      const float m = m_lds[g], r = r_lds[g];
      w[0] = fmaf(fast_exp2(fmaf(s.x, a.qscale, -m)), r, w[0]);
      w[1] = fmaf(fast_exp2(fmaf(s.y, a.qscale, -m)), r, w[1]);
      w[2] = fmaf(fast_exp2(fmaf(s.z, a.qscale, -m)), r, w[2]);
      w[3] = fmaf(fast_exp2(fmaf(s.w, a.qscale, -m)), r, w[3]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < end) ms[i + e] += w[e];
  }
}

// How a call is cut: about as many workgroups as the chip holds at once (two per
// CU), each with the same number of rows. Twice or three times as many only cost
// starts and partials (64K rows for 32 sequences of four heads, with the merge:
// 68 us, 84, 97). Blocks of the prefix of up to kShortBlock rows are twice as long, half
// as many starts, partials and parts to merge: 32 sequences over 8192 rows, 128 a block:
// 24.0 us, 19.9 this way; 16411, 257: 29.5, 26.4; 32768, 512: 38.4, 37.1; but 65536,
// 1024: 60.7, 62.5. With few query rows, whose partials are small, it is the starts (GPU
// time, eight kv heads, caches cold): four rows over 4096: 12.5, 11.3; over 16411: 22.1,
// 19.0; sixteen: 13.0, 12.5 and 23.2, 20.5; in fp32 four rows over 8192: 22.5, 18.9; but
// six sequences of 16 heads in fp32 over 8192 and 301 own rows 35.2, 40.0, and at head
// dim 64 four rows over 8192: 9.9, 10.4. Where the matrix cores bound (fp32, more than 16
// query rows) not: 64 rows over 4000: 28.3, 30.8; 30000: 98.8, 102.4.
//
// A sequence's own rows take as many blocks as come nearest to that length (32
// sequences of 700 rows over 16411, blocks of 607: one each 36, two 38 us). Of sequences
// of different lengths many blocks find nothing: they are cut three times finer (eight
// of up to 32K rows, weights accumulated: 129 us, 117 this way), but not to single tiles
// (eight of up to 2000: 20.1 us, 17.6 with two); beside a short prefix, whose blocks take
// longer, as long as those (eight of up to 3000 over 8192: 25.9 us, 23.2). Counting the
// own rows for less than the prefix's, as several are not there, gains nothing.
constexpr int kShortBlock = 512;

struct Plan {
  int rw, mtiles, splits, tiles_p, parts, tiles_o;
};

int esize(const Shape& s) { return s.dt == RADAR_BF16 ? 2 : 4; }
int slots() { return std::min(kSlots, 2 * num_cu()); }
// Row waves: the fewest that hold a kv head's query rows, at most four. In fp32, where
// the matrix cores bound even few rows, those that leave fewer rows of the last tile
// empty: tiles of 16 up to 48 rows (32 rows over a prefix of 30000: 64.7 us against
// 90.7; 48: 90.2, 95.6; 80: 164, 162), then of 64 or 128 (132 over 32768: 82, 104). In
// bf16 reading the prefix three times instead of two takes that back (132 rows: 134 us
// to 187 at 100000, 31.7 to 29.1 at 8192).
int row_waves(const Shape& s) {
  const int M = s.B * s.G;
  if (M <= (esize(s) == 4 ? 48 : flash_rows(esize(s), 1))) return 1;
  if (esize(s) == 4) return ceil_div(M, 64) * 64 < ceil_div(M, 128) * 128 ? 2 : 4;
  return M <= 64 ? 2 : 4;
}
int row_tiles(const Shape& s) {
  return (int)ceil_div(s.B * s.G, flash_rows(esize(s), row_waves(s)));
}

Plan plan_flash(const Shape& s, int64_t P, int64_t t, bool ragged) {
  Plan p{};
  const int pairs = s.B * s.Hkv;
  p.rw = row_waves(s);
  p.mtiles = row_tiles(s);
  const int ntp = flash_tile(esize(s), p.rw), nto = flash_tile(esize(s), 1);
  const int64_t rows = ceil_div((int64_t)s.Hkv * p.mtiles * P + pairs * t, slots());
  // a block of a short prefix spends as long on its start and its partials (64 KB at 128
  // query rows) as on its rows: one a CU then, twice as long
  const bool matrix_bound = esize(s) == 4 && s.B * s.G > flash_rows(4, 1);
  const bool is_long = rows > kShortBlock || matrix_bound;
  const int64_t rows_p = is_long ? rows : 2 * rows;
  const int64_t tp = ceil_div(P, ntp), to = ceil_div(t, nto);
  p.tiles_p = (int)std::max<int64_t>(1, ceil_div(rows_p, ntp));
  if (!ragged)
    p.tiles_o = (int)ceil_div(to, std::max<int64_t>(1, (t + rows / 2) / std::max<int64_t>(1, rows)));
  else if (P > 0 && !is_long)
    p.tiles_o = (int)ceil_div(rows_p, nto);
  else
    p.tiles_o = (int)std::max(std::min<int64_t>(2, ceil_div(rows, nto)), ceil_div(rows, kFiner * nto));
  p.tiles_o = std::max(1, p.tiles_o);
  // as many of each, of the same length (40 sequences of 2000 rows over 4096: 75 us, 70)
  p.splits = (int)ceil_div(tp, p.tiles_p);
  p.parts = (int)ceil_div(to, p.tiles_o);
  if (p.splits > 0) p.tiles_p = (int)ceil_div(tp, p.splits);
  if (p.parts > 0) p.tiles_o = (int)ceil_div(to, p.parts);
  return p;
}

// One launch where a workgroup of each (b, kv head) is through with the prefix and the
// own rows in five steps of 128 rows in bf16 or three of 64 in fp32, and all run at
// once: the GPU then takes as long as for the two kernels (bf16, head dim 128, 480 +
// 30 rows: 11.4 us, and 7.2 + 4.5; 64 sequences of eight heads over 300 + 200: 16.9,
// and 17.2 + 4.8; fp32, five steps: 13.2, and 6.5 + 3.8), and the host launches one
// less (2.8 us of 13).
bool is_short(const Shape& s, int64_t P, int64_t t) {
  const int n = flash_tile(esize(s), 1);
  return ceil_div(P, n) + ceil_div(t, n) <= (esize(s) == 2 ? 5 : 3) && s.B * s.Hkv <= slots();
}

// Bounds of splits and parts over all calls with at most these rows: tiles_p is
// at least Hkv mtiles P / (slots ntp), so there are at most slots / (Hkv mtiles)
// splits, and two for the roundings.
int most_splits(const Shape& s, int64_t P) {
  return (int)std::min(ceil_div(P, flash_tile(esize(s), row_waves(s))),
                       slots() / ((int64_t)s.Hkv * row_tiles(s)) + 2);
}
int most_parts(const Shape& s, int64_t t) {
  return (int)std::min(ceil_div(t, flash_tile(esize(s), 1)),
                       kFiner * slots() / ((int64_t)s.B * s.Hkv) + 2);
}

struct FlashWs {
  size_t pacc, pml, oacc, oml, logits, total;
};
FlashWs flash_ws(const Shape& s, int64_t splits, int64_t parts, int64_t logits) {
  FlashWs w;
  const size_t np = (size_t)s.Hkv * splits * s.B * s.G, no = (size_t)s.B * s.Hkv * parts * s.G;
  size_t off = 0;
  w.pacc = off; off += align256(np * s.d * 4);
  w.pml = off; off += align256(np * 8);
  w.oacc = off; off += align256(no * s.d * 4);
  w.oml = off; off += align256(no * 8);
  w.logits = off; off += align256((size_t)s.B * s.Hq * logits * 4);
  w.total = std::max<size_t>(off, 256);
  return w;
}

// a row's logits are written by whole steps
int64_t padded(const Shape& s, int64_t t) {
  const int n = flash_tile(esize(s), 1);
  return ceil_div(t, n) * n;
}

FlashArgs flash_args(const Shape& s, const Plan& p, const FlashWs& w, unsigned char* ws,
                     const void* q, const void* K, const void* V, int64_t t,
                     const int64_t* lens) {
  FlashArgs a{};
  a.q = q;
  a.B = s.B; a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
  a.qscale = kLog2e / std::sqrt((float)s.d);
  a.splits = p.splits; a.tiles_p = p.tiles_p; a.mtiles = p.mtiles; a.M = s.B * s.G;
  a.K = K; a.V = V; a.lens = lens; a.t = t; a.cap = s.cap;
  a.parts = p.parts; a.tiles_o = p.tiles_o;
  a.pacc = reinterpret_cast<float*>(ws + w.pacc);
  a.pml = reinterpret_cast<float*>(ws + w.pml);
  a.oacc = reinterpret_cast<float*>(ws + w.oacc);
  a.oml = reinterpret_cast<float*>(ws + w.oml);
  return a;
}

void launch_flash_any(const Shape& s, const FlashArgs& a, int rw, hipStream_t st) {
  if (s.dt == RADAR_BF16) {
    if (s.d == 64) launch_flash_bf16_64(a, rw, st);
    else launch_flash_bf16_128(a, rw, st);
  } else {
    if (s.d == 64) launch_flash_f32_64(a, rw, st);
    else launch_flash_f32_128(a, rw, st);
  }
}

// f(type tag, head dim tag) of the shape
template <typename F>
void by_type(const Shape& s, F&& f) {
  if (s.dt == RADAR_BF16) {
    if (s.d == 64) f(bf16_t{}, std::integral_constant<int, 64>{});
    else f(bf16_t{}, std::integral_constant<int, 128>{});
  } else {
    if (s.d == 64) f(float{}, std::integral_constant<int, 64>{});
    else f(float{}, std::integral_constant<int, 128>{});
  }
}

bool bad16(const void* p) { return !p || !aligned16(p); }

}  // namespace
}  // namespace radar_impl

using namespace radar_impl;

extern "C" {

size_t radar_attend_prefix_workspace_bytes(const radar_config* cfg, int64_t prefix_len,
                                           int64_t t) {
  Shape s;
  if (check_cache(cfg, &s) != RADAR_OK || prefix_len < 0 || prefix_len > INT32_MAX || t < 0 ||
      t > s.cap)
    return 0;
  return flash_ws(s, most_splits(s, prefix_len), most_parts(s, t), 0).total;
}

radar_status radar_attend_prefix(const radar_config* cfg, const void* q, const void* Kp,
                                 const void* Vp, int64_t prefix_len, int64_t prefix_capacity,
                                 const void* K, const void* V, int64_t t, const int64_t* lens,
                                 void* out, void* workspace, size_t workspace_bytes,
                                 hipStream_t stream) {
  Shape s;
  radar_status r = check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  if (bad16(q) || bad16(out) || (lens && !aligned16(lens))) return RADAR_EINVAL;
  if (prefix_len < 0 || prefix_len > prefix_capacity || t < 0 || t > s.cap)
    return RADAR_ECAPACITY;
  if (prefix_capacity > INT32_MAX) return RADAR_EUNSUPPORTED;
  if ((prefix_len > 0 && (bad16(Kp) || bad16(Vp))) || (t > 0 && (bad16(K) || bad16(V))))
    return RADAR_EINVAL;
  const Plan p = plan_flash(s, prefix_len, t, lens != nullptr);
  const FlashWs w = flash_ws(s, most_splits(s, prefix_len), most_parts(s, t), 0);
  if (bad16(workspace) || workspace_bytes < w.total) return RADAR_EWORKSPACE;
  FlashArgs a = flash_args(s, p, w, static_cast<unsigned char*>(workspace), q, K, V, t, lens);
  a.Kp = Kp; a.Vp = Vp; a.P = prefix_len; a.Pcap = prefix_capacity;
  a.out = out;
  if (is_short(s, prefix_len, t)) {
    launch_flash_any(s, a, 0, stream);
    return launch_status();
  }
  if (p.splits + p.parts > 0) {
    launch_flash_any(s, a, p.rw, stream);
    r = launch_status();
    if (r != RADAR_OK) return r;
  }
  const int64_t n_tile_o = (int64_t)p.tiles_o * flash_tile(esize(s), 1);
  by_type(s, [&](auto tag, auto d) {
    typedef decltype(tag) T;
    launch(RADAR_K_COMBINE, k_merge<T, decltype(d)::value>, dim3((unsigned)(s.B * s.Hq)),
           dim3(256), 0, stream, a, static_cast<T*>(out), n_tile_o);
  });
  return launch_status();
}

size_t radar_attend_accumulate_workspace_bytes(const radar_config* cfg, int64_t t) {
  Shape s;
  if (check_cache(cfg, &s) != RADAR_OK || t < 1 || t > s.cap) return 0;
  return flash_ws(s, 0, most_parts(s, t), padded(s, t)).total;
}

radar_status radar_attend_accumulate(const radar_config* cfg, const void* q, const void* K,
                                     const void* V, float* mass, int64_t t, const int64_t* lens,
                                     void* out, void* workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
  Shape s;
  radar_status r = check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  if (bad16(q) || bad16(K) || bad16(V) || bad16(mass) || bad16(out) ||
      (lens && !aligned16(lens)))
    return RADAR_EINVAL;
  if (t < 1 || t > s.cap) return RADAR_ECAPACITY;
  const Plan p = plan_flash(s, 0, t, lens != nullptr);
  const FlashWs w = flash_ws(s, 0, most_parts(s, t), padded(s, t));
  if (bad16(workspace) || workspace_bytes < w.total) return RADAR_EWORKSPACE;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  FlashArgs a = flash_args(s, p, w, ws, q, K, V, t, lens);
  a.logits = reinterpret_cast<float*>(ws + w.logits);
  a.tpad = padded(s, t);
  launch_flash_any(s, a, 1, stream);
  r = launch_status();
  if (r != RADAR_OK) return r;
  const int64_t n_tile_o = (int64_t)p.tiles_o * flash_tile(esize(s), 1);
  const int chunks = (int)ceil_div(t, kMassRows);
  const unsigned grid = (unsigned)(s.B * s.Hq) + (unsigned)(s.B * s.Hkv) * chunks;
  by_type(s, [&](auto tag, auto d) {
    typedef decltype(tag) T;
    launch(RADAR_K_COMBINE, k_settle<T, decltype(d)::value>, dim3(grid), dim3(256), 0, stream, a,
           static_cast<T*>(out), mass, n_tile_o, chunks);
  });
  return launch_status();
}

}  // extern "C"
