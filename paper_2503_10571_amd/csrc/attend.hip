// Exact attention of few query rows over long runs of cache rows, for the
// shared prefix and for the rows of each sequence (compiled once per element
// type and head dim: -DRADAR_ATTEND_F32=0|1 -DRADAR_ATTEND_D=64|128).
//
// One pass over K and V with a running maximum m and sum l per query row, in 32
// bits (m in units of log2). A workgroup of four waves takes 32 RW query rows:
// RW waves with 32 rows each, and 4 / RW such groups that share the tokens of a
// tile. Both products are 32x32 MFMAs that put the query rows on the lanes,
//   S[token][row] = K Q^T,    O^T[dim][row] += V^T P^T,
// so m, l and every scale are one value per lane, and the logits that a lane
// ends with (tokens 8 (i / 4) + 4 (lane / 32) + i % 4) are its k-slots of P^T if
// the rows of V are taken in the same order: no value of P crosses lanes.
//
// K and V come to LDS through registers, the next tile's loads in flight while
// this one is computed. Rows are stored whole, their 16-byte chunks at places
// XORed with the row, so that neither the operand reads nor the writes meet on
// a bank.
#include "attend_impl.h"

#ifndef RADAR_ATTEND_D
#define RADAR_ATTEND_D 128
#endif
#ifndef RADAR_ATTEND_F32
#define RADAR_ATTEND_F32 0
#endif

namespace radar_impl {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8v_t __attribute__((ext_vector_type(8)));

// token (of 32) of a lane's i-th logit
__device__ __forceinline__ int token_of(int i, int half) {
  return 8 * (i / 4) + 4 * half + (i % 4);
}

// The operands of one wave: 32 query rows (a lane's row is lane % 32) against
// tiles of rows of D elements in LDS.
template <typename T, int D> struct Ops;

template <int D> struct Ops<bf16_t, D> {
  static constexpr int CPR = D / 8;              // 16-byte chunks per row
  static constexpr int NDB = D / 32;             // 32-dim blocks
  bf16x8v_t q[D / 16];

  __device__ static __forceinline__ int k_place(int row, int c) {
    return c ^ (D == 128 ? row & 15 : (row >> 1) & 7);
  }
  // four consecutive rows are read together, 32 bytes of each twice
  __device__ static __forceinline__ int v_place(int row, int c) {
    return c ^ (D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2);
  }
  __device__ __forceinline__ void load_q(const bf16_t* row, int lane) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      q[ks] = *reinterpret_cast<const bf16x8v_t*>(row + ks * 16 + (lane >> 5) * 8);
  }
  // logits of tokens tok0 .. tok0 + 31 of the tile
  __device__ __forceinline__ f32x16_t logits(const unsigned char* k, int tok0, int lane) const {
    const int row = tok0 + (lane & 31), h = lane >> 5;
    f32x16_t s = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const bf16x8v_t a =
          *reinterpret_cast<const bf16x8v_t*>(k + row * (D * 2) + k_place(row, 2 * ks + h) * 16);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[ks], s, 0, 0, 0);
    }
    return s;
  }
  // acc += V^T P^T. The matrix cores take p in bf16. Where the 32 columns hold
  // 16 rows twice (`low` set in the second copy), the first takes p's upper 8
  // bits and the second the next 8, and their accumulators are added at the end:
  // p to 16 bits at no cost. Otherwise p is rounded to bf16, half a step of 2^-8
  // each, of the size of the output's own rounding; the second product that
  // more bits would take is half of the kernel's matrix work again.
  __device__ __forceinline__ void pv(const unsigned char* v, int tok0, const f32x16_t& p, bool twice,
                                     bool low, f32x16_t (&acc)[NDB], int lane) const {
    constexpr float kTiny = 1.17549435e-38f;     // smallest normal number
    const int h = lane >> 5, l16 = lane & 15, hf = (lane >> 4) & 1;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8v_t b;
      if (twice) {                         // uniform
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t x[2];
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const float pz = p[8 * ks + 2 * i + z];
            const float rest = pz - __uint_as_float(__float_as_uint(pz) & 0xffff0000u);
            // (never 0 where p is not: an infinite V times 0 would be NaN)
            x[z] = __float_as_uint(low ? __builtin_amdgcn_fmed3f(rest, pz, kTiny) : pz);
          }
          w[i] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);   // upper halves
        }
        b = __builtin_bit_cast(bf16x8v_t, make_uint4(w[0], w[1], w[2], w[3]));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = (__bf16)p[8 * ks + i];
      }
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        // lane (hf, l16) of a half ends with dim 32 db + 16 hf + l16 of the
        // tokens 16 ks + 4 h .. + 3 and 16 ks + 8 + 4 h .. + 3: transposed reads
        // of four rows by 16 dims, of which it supplies row l16 / 4, dims
        // 4 (l16 % 4) .. + 3
        s16x4_t part[2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int row = tok0 + 16 * ks + 8 * z + 4 * h + (l16 >> 2);
          const int c = (32 * db + 16 * hf) / 8 + ((l16 & 3) >> 1);
          const unsigned char* src = v + row * (D * 2) + v_place(row, c) * 16 + (l16 & 1) * 8;
          part[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4_t*)(src));
        }
        typedef short s16x8_t __attribute__((ext_vector_type(8)));
        const s16x8_t av = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8v_t, av), b,
                                                          acc[db], 0, 0, 0);
      }
    }
  }
};

template <int D> struct Ops<float, D> {
  static constexpr int CPR = D / 4;
  static constexpr int NDB = D / 32;
  float q[D / 2];

  __device__ static __forceinline__ int k_place(int row, int c) { return c ^ (row & 15); }
  // the two halves of a wave read rows four apart
  __device__ static __forceinline__ int v_place(int row, int c) { return c ^ (((row >> 2) & 1) << 3); }
  // (dims in the order that logits() takes them: 8 j + 4 half + e)
  __device__ __forceinline__ void load_q(const float* row, int lane) {
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      const float4 x = *reinterpret_cast<const float4*>(row + 8 * j + 4 * (lane >> 5));
      q[4 * j] = x.x; q[4 * j + 1] = x.y; q[4 * j + 2] = x.z; q[4 * j + 3] = x.w;
    }
  }
  __device__ __forceinline__ f32x16_t logits(const unsigned char* k, int tok0, int lane) const {
    const int row = tok0 + (lane & 31), h = lane >> 5;
    f32x16_t s = {};
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
      const float4 x =
          *reinterpret_cast<const float4*>(k + row * (D * 4) + k_place(row, 2 * j + h) * 16);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x, q[4 * j], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y, q[4 * j + 1], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(x.z, q[4 * j + 2], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(x.w, q[4 * j + 3], s, 0, 0, 0);
    }
    return s;
  }
  __device__ __forceinline__ void pv(const unsigned char* v, int tok0, const f32x16_t& p, bool, bool,
                                     f32x16_t (&acc)[NDB], int lane) const {
    const int h = lane >> 5, dim = lane & 31;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = tok0 + token_of(i, h);
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        const float x = *reinterpret_cast<const float*>(
            v + row * (D * 4) + v_place(row, 8 * db + (dim >> 2)) * 16 + (dim & 3) * 4);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p[i], acc[db], 0, 0, 0);
      }
    }
  }
};

template <typename T, int D, int RW>
struct Flash {
  static constexpr int TW = 4 / RW;              // groups that share a tile's tokens
  static constexpr int NT = flash_tile(sizeof(T), RW);
  static constexpr int kSub = NT / TW / 32;      // 32-token steps of a wave in a tile
  static constexpr int kBytes = NT * D * (int)sizeof(T);   // of K, and of V
  static constexpr int NCH = kBytes / 16 / 256;  // chunks of each per thread
  static constexpr int NDB = D / 32;
  // the groups' accumulators are added in LDS
  static constexpr int kMerge = TW > 1 ? 4 * 32 * D * 4 : 0;
  static constexpr int kLds = 2 * kBytes > kMerge ? 2 * kBytes : kMerge;
  using O = Ops<T, D>;

  // Rows [r0, r1) of K and V (r1 > r0) for the query rows of this workgroup:
  // row_q(i) points to row i < rows; the partials go to acc_out [rows][D] and
  // ml_out [rows][2]. With LOG the logits of row i go to log_out + i * log_stride,
  // by token.
  template <bool LOG, typename RowQ>
  __device__ static __forceinline__ void block(const T* __restrict__ K, const T* __restrict__ V,
                                               int64_t r0, int64_t r1, int rows, float qscale,
                                               RowQ&& row_q, float* acc_out, float* ml_out,
                                               float* log_out, int64_t log_stride,
                                               unsigned char* lds, float (*wm)[32 * RW],
                                               float (*wl)[32 * RW]) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, tw = wave / RW;
    const int h = lane >> 5, col = lane & 31;
    const bool twice = RW == 1 && sizeof(T) == 2 && rows <= 16;
    const bool low = twice && col >= 16;
    const int row = rw * 32 + (twice ? col & 15 : col);    // this lane's query row
    unsigned char* kl = lds;
    unsigned char* vl = lds + kBytes;

    O ops;
    ops.load_q(row_q(min(row, rows - 1)), lane);
    f32x16_t acc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) acc[db] = f32x16_t{};
    float m = -INFINITY, l = 0.f;

    uint4 kr[NCH], vr[NCH];
    // rows behind the last are read as the last, and zeroed on the way to LDS
    // (their weight is 0, which an infinity there would turn into NaN)
    auto load = [&](int64_t at) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int x = i * 256 + tid;
        const int64_t r = min(at + x / O::CPR, r1 - 1);
        const int64_t off = r * D + (x % O::CPR) * (16 / (int)sizeof(T));
        kr[i] = RW < 4 ? ld_stream(K + off) : *reinterpret_cast<const uint4*>(K + off);
        vr[i] = RW < 4 ? ld_stream(V + off) : *reinterpret_cast<const uint4*>(V + off);
      }
    };
    load(r0);
    for (int64_t at = r0; at < r1; at += NT) {
      const int len = (int)min<int64_t>(NT, r1 - at);
      if (at > r0) __syncthreads();              // the last tile is read
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int x = i * 256 + tid, r = x / O::CPR, c = x % O::CPR;
        if (len < NT && r >= len) vr[i] = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(kl + (r * O::CPR + O::k_place(r, c)) * 16) = kr[i];
        *reinterpret_cast<uint4*>(vl + (r * O::CPR + O::v_place(r, c)) * 16) = vr[i];
      }
      __syncthreads();
      if (at + NT < r1) load(at + NT);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub) {
        const int tok0 = (tw * kSub + sub) * 32;
        if (tok0 >= len) break;                  // wave-uniform
        f32x16_t s = ops.logits(kl, tok0, lane);
        if constexpr (LOG) {
          if (row < rows && !low) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const int tok = tok0 + token_of(i, h);
              if (tok < len)                     // (rows come in fours, padded)
                *reinterpret_cast<float4*>(log_out + row * log_stride + at + tok) =
                    make_float4(s[i], s[i + 1], s[i + 2], s[i + 3]);
            }
          }
        }
        if (tok0 + 32 > len) {                   // uniform
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = tok0 + token_of(i, h) < len ? s[i] : -INFINITY;
        }
        float mt = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
        float lo, hi;
        xor_pair<32>(mt, lo, hi);
        const float mn = fmaxf(m, fmaxf(lo, hi) * qscale);
        const float mref = mn == -INFINITY ? 0.f : mn;
        if (__ballot(mn != m)) {                 // some row's maximum grew
          const float scale = fast_exp2(m - mref);   // 0 on the row's first tile
          l *= scale;
#pragma unroll
          for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] *= scale;
          m = mn;
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] = fast_exp2(fmaf(s[i], qscale, -mref));
          sum += s[i];
        }
        l += sum;
        ops.pv(vl, tok0, s, twice, low, acc, lane);
      }
    }
    l = xor_sum<32>(l);
    if (twice) {                                 // the two parts of p
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = xor_sum<16>(acc[db][i]);
    }
    const bool mine = row < rows && !low;
    if constexpr (TW == 1) {
      if (!mine) return;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(acc_out + (int64_t)row * D + 32 * db + token_of(i, h)) =
              make_float4(acc[db][i], acc[db][i + 1], acc[db][i + 2], acc[db][i + 3]);
      if (h == 0) *reinterpret_cast<float2*>(ml_out + 2 * row) = make_float2(m, l);
    } else {
      constexpr int RS = 32 * RW;
      float* wacc = reinterpret_cast<float*>(lds);
      // 16-byte pieces of a row at places XORed with the row
      auto place = [](int r, int piece) { return piece ^ (r & (D / 4 - 1)); };
      __syncthreads();                           // no wave reads its tile any more
      if (mine) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<float4*>(wacc + (tw * RS + row) * D +
                                       4 * place(row, 8 * db + token_of(i, h) / 4)) =
                make_float4(acc[db][i], acc[db][i + 1], acc[db][i + 2], acc[db][i + 3]);
        if (h == 0) { wm[tw][row] = m; wl[tw][row] = l; }
      }
      __syncthreads();
      for (int x = tid; x < rows * (D / 4); x += 256) {
        const int r = x / (D / 4), c = x % (D / 4);
        float M = wm[0][r];
#pragma unroll
        for (int w = 1; w < TW; ++w) M = fmaxf(M, wm[w][r]);
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        float L = 0.f;
#pragma unroll
        for (int w = 0; w < TW; ++w) {
          const float f = wm[w][r] == -INFINITY ? 0.f : fast_exp2(wm[w][r] - M);
          const float4 v = *reinterpret_cast<const float4*>(wacc + (w * RS + r) * D + 4 * place(r, c));
          a.x = fmaf(v.x, f, a.x); a.y = fmaf(v.y, f, a.y);
          a.z = fmaf(v.z, f, a.z); a.w = fmaf(v.w, f, a.w);
          L = fmaf(wl[w][r], f, L);
        }
        *reinterpret_cast<float4*>(acc_out + (int64_t)r * D + 4 * c) = a;
        if (c == 0) *reinterpret_cast<float2*>(ml_out + 2 * r) = make_float2(M, L);
      }
    }
  }
};

// Blocks of the prefix first, then of the sequences' own rows. Workgroups i and
// i + 8 share an XCD and its L2: the row tiles of one (kv head, split) read the
// same rows and lie 8 apart.
template <typename T, int D, int RW, bool LOG>
__global__ __launch_bounds__(256, flash_wgs(sizeof(T), D)) void k_flash(FlashArgs a) {
  using F = Flash<T, D, RW>;
  using F1 = Flash<T, D, 1>;
  constexpr int kLds = F::kLds > F1::kLds ? F::kLds : F1::kLds;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kLds];
  __shared__ float wm[4][32], wl[4][32];         // [TW][32 RW]
  const int n_units = a.Hkv * a.splits;          // (kv head, split)
  const int n_prefix = (n_units + 7) / 8 * 8 * a.mtiles;
  int i = blockIdx.x;
  if constexpr (!LOG) {
    if (i < n_prefix) {
      const int unit = i / (8 * a.mtiles) * 8 + i % 8, mt = i / 8 % a.mtiles;
      if (unit >= n_units) return;
      const int hk = unit / a.splits, sp = unit % a.splits;
      const int64_t r0 = (int64_t)sp * a.tiles_p * F::NT;
      const int64_t r1 = min(a.P, r0 + (int64_t)a.tiles_p * F::NT);
      const int row0 = mt * 32 * RW;
      const int64_t at = (int64_t)unit * a.M + row0;
      F::template block<false>(
          static_cast<const T*>(a.Kp) + hk * a.Pcap * D, static_cast<const T*>(a.Vp) + hk * a.Pcap * D,
          r0, r1, min(a.M - row0, 32 * RW), a.qscale,
          [&](int r) {
            const int x = row0 + r;              // b G + g
            return static_cast<const T*>(a.q) + ((int64_t)(x / a.G) * a.Hq + hk * a.G + x % a.G) * D;
          },
          a.pacc + at * D, a.pml + at * 2, nullptr, 0, lds,
          reinterpret_cast<float (*)[32 * RW]>(wm), reinterpret_cast<float (*)[32 * RW]>(wl));
      return;
    }
    i -= n_prefix;
  }
  const int64_t bh = i / a.parts, part = i % a.parts;
  const int64_t b = bh / a.Hkv, hk = bh % a.Hkv;
  const int64_t len = own_len(a, b, LOG ? 1 : 0);
  const int64_t r0 = part * a.tiles_o * F1::NT;
  if (r0 >= len) return;
  const int64_t r1 = min(len, r0 + (int64_t)a.tiles_o * F1::NT);
  const int64_t at = (bh * a.parts + part) * a.G;
  F1::template block<LOG>(
      static_cast<const T*>(a.K) + bh * a.cap * D, static_cast<const T*>(a.V) + bh * a.cap * D, r0, r1,
      a.G, a.qscale,
      [&](int r) { return static_cast<const T*>(a.q) + (b * a.Hq + hk * a.G + r) * D; },
      a.oacc + at * D, a.oml + at * 2, a.logits + bh * a.G * a.tpad, a.tpad, lds, wm, wl);
}

template <typename T, int D>
void launch_flash(const FlashArgs& a, int rw, hipStream_t st) {
  const unsigned n = (unsigned)(ceil_div(a.Hkv * a.splits, 8) * 8 * a.mtiles + a.B * a.Hkv * a.parts);
  if (a.logits)
    launch(RADAR_K_ATTEND, k_flash<T, D, 1, true>, dim3(n), dim3(256), 0, st, a);
  else if (rw == 1)
    launch(RADAR_K_ATTEND, k_flash<T, D, 1, false>, dim3(n), dim3(256), 0, st, a);
  else if (rw == 2)
    launch(RADAR_K_ATTEND, k_flash<T, D, 2, false>, dim3(n), dim3(256), 0, st, a);
  else
    launch(RADAR_K_ATTEND, k_flash<T, D, 4, false>, dim3(n), dim3(256), 0, st, a);
}

}  // namespace

#if RADAR_ATTEND_F32 && RADAR_ATTEND_D == 64
void launch_flash_f32_64(const FlashArgs& a, int rw, hipStream_t st) { launch_flash<float, 64>(a, rw, st); }
#elif RADAR_ATTEND_F32
void launch_flash_f32_128(const FlashArgs& a, int rw, hipStream_t st) { launch_flash<float, 128>(a, rw, st); }
#elif RADAR_ATTEND_D == 64
void launch_flash_bf16_64(const FlashArgs& a, int rw, hipStream_t st) { launch_flash<bf16_t, 64>(a, rw, st); }
#else
void launch_flash_bf16_128(const FlashArgs& a, int rw, hipStream_t st) { launch_flash<bf16_t, 128>(a, rw, st); }
#endif

}  // namespace radar_impl
