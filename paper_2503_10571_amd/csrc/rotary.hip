// Rotary positions: the rotation of q and k rows, and the same on the way into
// the cache (include/radar_cache.h).
//
//   a' = m (a cos - b sin),  b' = m (b cos + a sin),  angle = p f_i
//
// Every element is read once and written once, so memory bounds it. The angle
// is taken as turns, p f_i / 2 pi, in 64 bits (at position 2^20 a 32-bit angle
// is off by 0.06 rad), its fraction then in 32 bits. Measured: 16384 tokens of 32 + 8
// + 8 heads of 128 in bf16 into the cache 71 us, 5.7 TB/s, where a copy reaches 6.4;
// one token of 32 + 8 heads 4 us, which the launch and the binding's 11 us hide.
#include "cache_impl.h"

namespace radar_impl {
namespace {

constexpr int kRopeMaxDim = 256;

// one operand: its rows, where they go, and how (strides in bytes)
struct RotSide {
  const unsigned char* src;
  unsigned char* dst;
  int64_t ss_seq, ss_tok, ss_head, ds_seq, ds_tok, ds_head;
  int heads;
  int rotate;              // 0: copied (v)
  int cached;              // the destination's token axis is the cache's rows
};

struct RotArgs {
  RotSide side[3];
  int n_side, heads;       // heads of all sides
  int T;
  int64_t n_tok;           // B * T
  const double* freq;
  int pairs;               // rot_dim / 2
  float mscale;
  int64_t pos0;
  const int64_t* pos;
  int per_token, inverse;
  const int64_t* lens;
  int64_t row0;
  const int64_t* rows;
  int64_t cap;
  int d;
};

// The place of one token, wave-uniform: its sequence and index, position and
// cache row; false where it is not to be touched.
struct TokenAt {
  int64_t b, t, pos, row;
};
__device__ __forceinline__ bool token_at(const RotArgs& a, int64_t i, TokenAt* o) {
  if (i >= a.n_tok) return false;
  o->b = (int)i / a.T;
  o->t = (int)i - o->b * a.T;
  if (a.lens && o->t >= a.lens[o->b]) return false;
  o->pos = a.pos ? (a.per_token ? a.pos[i] : a.pos[o->b] + o->t) : a.pos0 + o->t;
  o->row = (a.rows ? a.rows[o->b] : a.row0) + o->t;
  return true;
}

// the first of a workgroup's four tokens: a launch has fewer than 2^32 threads along
// x, so more than kRotWgs workgroups go on along z
constexpr int64_t kRotWgs = 1 << 23;
__device__ __forceinline__ int64_t first_token() {
  return ((int64_t)blockIdx.z * kRotWgs + blockIdx.x) * 4;
}

// (cos, sin) of a pair, times mscale; the sign of the direction in sin
__device__ __forceinline__ float2 turn_of(const RotArgs& a, int pair, int64_t pos) {
  constexpr double kInv2Pi = 0.15915494309189533577;
  const double turns = (double)pos * a.freq[pair] * kInv2Pi;
  float s, c;
  sincospif(2.f * (float)(turns - __builtin_rint(turns)), &s, &c);
  s *= a.mscale;
  return make_float2(c * a.mscale, a.inverse ? -s : s);
}

// the side that head h of all sides belongs to, and its rows' addresses for one
// token; false: nothing to write
__device__ __forceinline__ bool side_rows(const RotArgs& a, const TokenAt& at, int h,
                                          const unsigned char** src, unsigned char** dst,
                                          bool* rotate) {
  // (selects of uniform values: an index that differs by lane would make a load
  // of each field)
  const unsigned char* from[3];
  unsigned char* to[3];
  int64_t from_head[3], to_head[3];
  bool on[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const RotSide& s = a.side[i];
    on[i] = !s.cached || (at.row >= 0 && at.row < a.cap);
    from[i] = s.src + at.b * s.ss_seq + at.t * s.ss_tok;
    to[i] = s.dst + at.b * s.ds_seq + (s.cached ? at.row : at.t) * s.ds_tok;
    from_head[i] = s.ss_head;
    to_head[i] = s.ds_head;
  }
  const int h1 = a.side[0].heads, h2 = h1 + a.side[1].heads;
  const int i = h < h1 ? 0 : h < h2 ? 1 : 2;
  const int64_t head = h - (i == 0 ? 0 : i == 1 ? h1 : h2);
  *src = (i == 0 ? from[0] : i == 1 ? from[1] : from[2]) +
         head * (i == 0 ? from_head[0] : i == 1 ? from_head[1] : from_head[2]);
  *dst = (i == 0 ? to[0] : i == 1 ? to[1] : to[2]) +
         head * (i == 0 ? to_head[0] : i == 1 ? to_head[1] : to_head[2]);
  *rotate = i == 0 ? a.side[0].rotate : i == 1 ? a.side[1].rotate : a.side[2].rotate;
  return i == 0 ? on[0] : i == 1 ? on[1] : on[2];
}

template <typename T>
__device__ __forceinline__ uint4 pack16(const float* f);
template <>
__device__ __forceinline__ uint4 pack16<float>(const float* f) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                    __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ uint4 pack16<bf16_t>(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf16x2v_t p;                           // one conversion instruction, to nearest even
    p[0] = (__bf16)f[2 * i];
    p[1] = (__bf16)f[2 * i + 1];
    w[i] = __builtin_bit_cast(uint32_t, p);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One wave per token and group of heads. The wave's lanes take the sines of the
// token's pairs once, into LDS (one per lane at rot_dim 128, where every lane of
// a row computing its own would take eight); then every lane moves two 16-byte
// chunks of a row: for half pairs a chunk of first dims and the matching chunk
// of second dims, otherwise chunks u and u + U of the row's 2 U. kRotPasses heads
// (of 1, 2 and 4 the best for large calls: 1 GB 208, 178, 182 us)
// per lane are loaded before any is written, which also makes an output that
// is its own input safe: nobody else reads a lane's chunks.
constexpr int kRotPasses = 2;

template <typename T, bool INTER, bool PAST>
__global__ __launch_bounds__(256) void k_rotary(RotArgs a, int lpr_log2) {
  constexpr int EPL = Elem<T>::kPer16;
  __shared__ float2 turn_lds[4][kRopeMaxDim / 2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TokenAt at;
  if (!token_at(a, first_token() + wave, &at)) return;   // wave-uniform
  float2* turn = turn_lds[wave];
  for (int i = lane; i < a.pairs; i += kWave) turn[i] = turn_of(a, i, at.pos);
  // (the wave reads what it wrote)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

  const int U = a.d / EPL / 2;
  const int u = lane & ((1 << lpr_log2) - 1);
  if (u >= U) return;
  const int hpp = kWave >> lpr_log2;       // heads per pass
  const int h0 = blockIdx.y * hpp * kRotPasses + (lane >> lpr_log2);
  // chunks of this lane in a rotated row, and where its pairs begin in the table
  const int hp = a.pairs / EPL;            // chunks of first dims (half pairs)
  int ca, cb;
  if (INTER || u >= hp) {
    const int first = INTER ? 0 : 2 * hp;
    ca = INTER ? u : first + u - hp;
    cb = ca + (INTER ? U : U - hp);
  } else {
    ca = u;
    cb = u + hp;
  }
  uint4 x[kRotPasses], y[kRotPasses];
  unsigned char* dst[kRotPasses];
  bool rot[kRotPasses], on[kRotPasses];
#pragma unroll
  for (int p = 0; p < kRotPasses; ++p) {
    const unsigned char* src = nullptr;
    const int h = h0 + p * hpp;
    on[p] = h < a.heads && side_rows(a, at, h, &src, &dst[p], &rot[p]);
    if (on[p]) {
      x[p] = PAST ? ld_stream(src + ca * 16) : *reinterpret_cast<const uint4*>(src + ca * 16);
      y[p] = PAST ? ld_stream(src + cb * 16) : *reinterpret_cast<const uint4*>(src + cb * 16);
    }
  }
#pragma unroll
  for (int p = 0; p < kRotPasses; ++p) {
    if (!on[p]) continue;
    if (rot[p]) {
      float f[EPL], g[EPL];
      if constexpr (INTER) {
        const int rc = 2 * a.pairs / EPL;  // rotated chunks
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          uint4& v = z ? y[p] : x[p];
          const int c = z ? cb : ca;
          if (c >= rc) continue;
          unpack16<T>(v, f);
#pragma unroll
          for (int e = 0; e < EPL; e += 2) {
            const float2 t = turn[(c * EPL + e) / 2];
            g[e] = f[e] * t.x - f[e + 1] * t.y;
            g[e + 1] = f[e + 1] * t.x + f[e] * t.y;
          }
          v = pack16<T>(g);
        }
      } else if (u < hp) {
        unpack16<T>(x[p], f);
        unpack16<T>(y[p], g);
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float2 t = turn[u * EPL + e];
          const float b = g[e];
          g[e] = b * t.x + f[e] * t.y;
          f[e] = f[e] * t.x - b * t.y;
        }
        x[p] = pack16<T>(f);
        y[p] = pack16<T>(g);
      }
    }
    put16<PAST>(dst[p] + ca * 16, x[p]);
    put16<PAST>(dst[p] + cb * 16, y[p]);
  }
}

// Rotated parts whose halves do not end on 16 bytes: a pair (or two copied
// dims) per lane, element by element.
template <typename T>
__global__ __launch_bounds__(256) void k_rotary_any(RotArgs a, int inter) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TokenAt at;
  if (!token_at(a, first_token() + wave, &at)) return;
  for (int i = lane; i < a.d / 2; i += kWave) {
    const bool turned = i < a.pairs;
    float2 t = make_float2(1.f, 0.f);
    if (turned) t = turn_of(a, i, at.pos);
    const int lo = turned && !inter ? i : 2 * i;
    const int hi = turned && !inter ? i + a.pairs : 2 * i + 1;
    for (int h = blockIdx.y * 8; h < min(a.heads, (int)blockIdx.y * 8 + 8); ++h) {
      const unsigned char* src;
      unsigned char* dst;
      bool rot;
      if (!side_rows(a, at, h, &src, &dst, &rot)) continue;
      const T* s = reinterpret_cast<const T*>(src);
      T* o = reinterpret_cast<T*>(dst);
      const T xa = s[lo], xb = s[hi];
      if (turned && rot) {
        const float fa = to_f32<T>(xa), fb = to_f32<T>(xb);
        o[lo] = from_f32<T>(fa * t.x - fb * t.y);
        o[hi] = from_f32<T>(fb * t.x + fa * t.y);
      } else {
        o[lo] = xa;
        o[hi] = xb;
      }
    }
  }
}

bool good_rows(const radar_rows* r, int esz) {
  return r && r->data && aligned16(r->data) && r->seq * esz % 16 == 0 &&
         r->token * esz % 16 == 0 && r->head * esz % 16 == 0;
}

RotSide side_of(const radar_rows& src, const radar_rows& dst, int heads, int esz, bool rotate,
                bool cached) {
  return {static_cast<const unsigned char*>(src.data), static_cast<unsigned char*>(dst.data),
          src.seq * esz, src.token * esz, src.head * esz, dst.seq * esz, dst.token * esz,
          dst.head * esz, heads, rotate ? 1 : 0, cached ? 1 : 0};
}

radar_status check_rope(const radar_rope* rope, int head_dim, radar_dtype dt) {
  if (!rope || !rope->inv_freq || !aligned16(rope->inv_freq)) return RADAR_EINVAL;
  if (rope->interleaved != 0 && rope->interleaved != 1) return RADAR_EINVAL;
  if (dt != RADAR_F32 && dt != RADAR_BF16) return RADAR_EINVAL;
  if (head_dim < 1 || rope->rot_dim < 2 || rope->rot_dim % 2 != 0 || rope->rot_dim > head_dim)
    return RADAR_EINVAL;
  if (head_dim % 16 != 0 || head_dim > kRopeMaxDim) return RADAR_EUNSUPPORTED;
  return RADAR_OK;
}

// Loads and stores pass the caches (256 MB) by where a call moves more than they hold
// (three calls of 400 MB in turn: 82.7 us, 72.2; of 1 GB: 194, 178) and its stores are
// of whole 128-byte lines (383 MB of rows with 16 rotated dims of 64 in fp32, whose lines
// two stores share: 83 us, 127). Where both sides fit, the stores cost nothing now and
// the next kernel's reads little (84 MB: 17.2 us, 27.3).
bool past_caches(const RotArgs& a, bool inter, int epl) {
  const int U = a.d / epl / 2, hp = a.pairs / epl;
  return 2 * a.n_tok * a.heads * a.d * (16 / epl) > (256 << 20) && U % 8 == 0 &&
         (inter || hp % 8 == 0);
}

template <typename T>
void launch_rotary(const RotArgs& a, const radar_rope& rope, hipStream_t st) {
  constexpr int EPL = Elem<T>::kPer16;
  const int64_t wgs = ceil_div(a.n_tok, 4);
  const unsigned gx = (unsigned)std::min(wgs, kRotWgs), gz = (unsigned)ceil_div(wgs, kRotWgs);
  // vectors where the pairs of a 16-byte chunk are whole chunks (or lie in it)
  const bool whole = rope.interleaved ? rope.rot_dim % EPL == 0 : a.pairs % EPL == 0;
  if (!whole) {
    launch(RADAR_K_APPEND, k_rotary_any<T>, dim3(gx, (unsigned)ceil_div(a.heads, 8), gz),
           dim3(256), 0, st, a, (int)rope.interleaved);
    return;
  }
  int lpr_log2 = 0;
  while ((1 << lpr_log2) < a.d / EPL / 2) ++lpr_log2;
  const int per_wave = (kWave >> lpr_log2) * kRotPasses;
  const dim3 grid(gx, (unsigned)ceil_div(a.heads, per_wave), gz);
  const bool past = past_caches(a, rope.interleaved, EPL);
  auto go = [&](auto inter) {
    constexpr bool kInter = decltype(inter)::value;
    if (past) launch(RADAR_K_APPEND, k_rotary<T, kInter, true>, grid, dim3(256), 0, st, a, lpr_log2);
    else launch(RADAR_K_APPEND, k_rotary<T, kInter, false>, grid, dim3(256), 0, st, a, lpr_log2);
  };
  if (rope.interleaved) go(std::true_type{});
  else go(std::false_type{});
}

radar_status run_rotary(RotArgs& a, const radar_rope& rope, radar_dtype dt, hipStream_t st) {
  a.freq = rope.inv_freq;
  a.pairs = rope.rot_dim / 2;
  a.mscale = rope.mscale;
  a.heads = 0;
  for (int i = 0; i < a.n_side; ++i) a.heads += a.side[i].heads;
  if (dt == RADAR_BF16) launch_rotary<bf16_t>(a, rope, st);
  else launch_rotary<float>(a, rope, st);
  return launch_status();
}

// the tokens of a call: B * T rows, fewer than 2^31
radar_status check_tokens(int64_t batch, int64_t tokens) {
  if (batch < 1 || tokens < 0) return RADAR_EINVAL;
  if (tokens > INT32_MAX || batch * tokens > INT32_MAX) return RADAR_EUNSUPPORTED;
  return RADAR_OK;
}

}  // namespace
}  // namespace radar_impl

using namespace radar_impl;

extern "C" {

radar_status radar_rotary(const radar_rope* rope, int32_t batch, int64_t tokens,
                          int32_t head_dim, radar_dtype dtype, int32_t n_q_heads,
                          const radar_rows* q, const radar_rows* q_out, int32_t n_k_heads,
                          const radar_rows* k, const radar_rows* k_out, int64_t pos0,
                          const int64_t* pos, int32_t pos_per_token, const int64_t* lens,
                          int32_t inverse, hipStream_t stream) {
  radar_status r = check_rope(rope, head_dim, dtype);
  if (r != RADAR_OK) return r;
  const int esz = dtype == RADAR_BF16 ? 2 : 4;
  if (n_q_heads < 1 || n_k_heads < 0 || !good_rows(q, esz) || !good_rows(q_out, esz))
    return RADAR_EINVAL;
  if (n_k_heads > 0 && (!good_rows(k, esz) || !good_rows(k_out, esz))) return RADAR_EINVAL;
  if ((int64_t)n_q_heads + n_k_heads > 65535) return RADAR_EUNSUPPORTED;
  if ((pos && !aligned16(pos)) || (lens && !aligned16(lens))) return RADAR_EINVAL;
  r = check_tokens(batch, tokens);
  if (r != RADAR_OK || tokens == 0) return r;
  RotArgs a{};
  a.side[0] = side_of(*q, *q_out, n_q_heads, esz, true, false);
  a.n_side = 1;
  if (n_k_heads > 0) a.side[a.n_side++] = side_of(*k, *k_out, n_k_heads, esz, true, false);
  a.T = (int)tokens;
  a.n_tok = batch * tokens;
  a.pos0 = pos0; a.pos = pos; a.per_token = pos_per_token != 0; a.lens = lens;
  a.inverse = inverse != 0;
  a.d = head_dim;
  return run_rotary(a, *rope, dtype, stream);
}

radar_status radar_rotary_fill(const radar_config* cfg, const radar_rope* rope, int64_t tokens,
                               const radar_rows* q, const radar_rows* q_out, const radar_rows* k,
                               const radar_rows* v, void* K, void* V, int64_t row0,
                               const int64_t* rows, int64_t pos0, const int64_t* pos,
                               int32_t pos_per_token, const int64_t* lens, hipStream_t stream) {
  Shape s;
  radar_status r = check_cache(cfg, &s);
  if (r != RADAR_OK) return r;
  r = check_rope(rope, s.d, s.dt);
  if (r != RADAR_OK) return r;
  const int esz = s.dt == RADAR_BF16 ? 2 : 4;
  if (!good_rows(k, esz) || !good_rows(v, esz) || !K || !V || !aligned16(K) || !aligned16(V))
    return RADAR_EINVAL;
  if (q && (!good_rows(q, esz) || !good_rows(q_out, esz))) return RADAR_EINVAL;
  if ((pos && !aligned16(pos)) || (lens && !aligned16(lens)) || (rows && !aligned16(rows)))
    return RADAR_EINVAL;
  if (s.Hq + 2 * s.Hkv > 65535) return RADAR_EUNSUPPORTED;
  r = check_tokens(s.B, tokens);
  if (r != RADAR_OK) return r;
  if (!rows && (row0 < 0 || row0 > s.cap - tokens)) return RADAR_ECAPACITY;
  if (tokens == 0) return RADAR_OK;
  // the cache as rows [B][capacity][Hkv][d]: a head's rows are contiguous
  const radar_rows Kr{K, s.Hkv * s.cap * s.d, s.d, s.cap * s.d};
  const radar_rows Vr{V, s.Hkv * s.cap * s.d, s.d, s.cap * s.d};
  RotArgs a{};
  a.side[a.n_side++] = side_of(*k, Kr, s.Hkv, esz, true, true);
  a.side[a.n_side++] = side_of(*v, Vr, s.Hkv, esz, false, true);
  if (q) a.side[a.n_side++] = side_of(*q, *q_out, s.Hq, esz, true, false);
  a.T = (int)tokens;
  a.n_tok = s.B * tokens;
  a.pos0 = pos0; a.pos = pos; a.per_token = pos_per_token != 0; a.lens = lens;
  a.row0 = row0; a.rows = rows; a.cap = s.cap;
  a.d = s.d;
  return run_rotary(a, *rope, s.dt, stream);
}

}  // extern "C"
