// Exact attention of few query rows over long runs of cache rows, for the
// shared prefix and for the rows of each sequence (compiled once per element
// type and head dim: -DRADAR_ATTEND_F32=0|1 -DRADAR_ATTEND_D=64|128).
//
// One pass over K and V with a running maximum m and sum l per query row, in 32
// bits (m in units of log2). Both products are MFMAs that put the query rows on
// the lanes,
//   S[token][row] = K Q^T,    O^T[dim][row] += V^T P^T,
// so m, l and every scale are one value per lane; and a lane's logits are of
// four consecutive tokens at a time, which are its k-slots of P^T if the rows of
// V are taken in the same order: no value of P crosses lanes.
//
// Up to 32 query rows per kv head (16 in fp32) memory bounds it: 6.4 TB/s of the
// 7.2 that one pass of loads over 2 GiB and more reaches (32000 own rows of 8 x 8 pairs, head dim 128: 162 us). Above,
// the matrix cores, the exponentials and the LDS reads of their operands share
// the time: 0.8 PFLOP/s of the 1.28 that a large library product reaches (512
// rows per kv head over a prefix of 100000: 265 us, at a clock of 1.8 GHz). In fp32 the matrix cores' 32-bit
// rate.
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

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8v_t __attribute__((ext_vector_type(8)));

// The operands of one wave: kRows query rows (a lane's row is lane % kRows)
// against steps of kTok tokens, of which a lane gets kVals logits: token
// token_of(i) is its i-th. acc[block][i] is dim block * kDims + dim_of(i).

// 32 rows: 32x32 products; a lane's half takes four of every eight tokens (dims)
struct Wide {
  static constexpr int kRows = 32, kTok = 32, kVals = 16, kDims = 32;
  typedef f32x16_t Vec;
  __device__ static __forceinline__ int token_of(int i, int lane) {
    return 8 * (i / 4) + 4 * (lane >> 5) + (i % 4);
  }
  __device__ static __forceinline__ int dim_of(int i, int lane) { return token_of(i, lane); }
  // over the lanes of a row
  __device__ static __forceinline__ float row_maximum(float v) {
    float lo, hi;
    xor_pair<32>(v, lo, hi);
    return fmaxf(lo, hi);
  }
  __device__ static __forceinline__ float row_total(float v) { return xor_sum<32>(v); }
};

// 16 rows: 16x16 products; a lane's quarter takes four of sixteen
struct Narrow {
  static constexpr int kRows = 16, kTok = 16, kVals = 4, kDims = 16;
  typedef f32x4_t Vec;
  __device__ static __forceinline__ int token_of(int i, int lane) { return 4 * (lane >> 4) + i; }
  __device__ static __forceinline__ int dim_of(int i, int lane) { return token_of(i, lane); }
  __device__ static __forceinline__ float row_maximum(float v) {
    float lo, hi;
    xor_pair<16>(v, lo, hi);
    xor_pair<32>(fmaxf(lo, hi), lo, hi);
    return fmaxf(lo, hi);
  }
  __device__ static __forceinline__ float row_total(float v) { return xor_sum<32>(xor_sum<16>(v)); }
};

template <typename T, int D, int RW> struct Ops;

template <int D, int RW> struct Ops<bf16_t, D, RW> : Wide {
  static constexpr int CPR = D / 8;              // 16-byte chunks per row
  static constexpr int NDB = D / kDims;
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
  __device__ __forceinline__ Vec logits(const unsigned char* k, int tok0, int lane) const {
    const int row = tok0 + (lane & 31), h = lane >> 5;
    bf16x8v_t a[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      a[ks] = *reinterpret_cast<const bf16x8v_t*>(k + row * (D * 2) + k_place(row, 2 * ks + h) * 16);
    Vec s = {};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[ks], q[ks], s, 0, 0, 0);
    return s;
  }
  // The matrix cores take p in bf16. Where the 32 columns hold 16 rows twice
  // (RW = 1; `low` set in the second copy), the first takes p's upper 8 bits and
  // the second the next 8, and their accumulators are added at the end: p to 16
  // bits at no cost, and the output's error (of its norm, over 8192 rows) is that of its
  // own rounding, 1.62e-3. Otherwise p is rounded to bf16, half a step of 2^-8 each, and
  // both roundings together are 1.93e-3 at 20 query rows, 2.17e-3 at 64, 2.27e-3 at 512,
  // where the output's alone is 1.66e-3; the second product that more bits would take is
  // half of the kernel's matrix work again.
  __device__ static __forceinline__ bf16x8v_t p_operand(const Vec& p, int ks, bool twice, bool low) {
    constexpr float kTiny = 1.17549435e-38f;     // smallest normal number
    bf16x8v_t b;
    if (RW == 1 && twice) {                // uniform
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
    return b;
  }
  // Lane (hf, l16) of a half gets dim 32 db + 16 hf + l16 of the tokens
  // t0 + 4 h .. + 3 and t0 + 8 + 4 h .. + 3: transposed reads of four rows by 16
  // dims, of which it supplies row l16 / 4, dims 4 (l16 % 4) .. + 3.
  __device__ static __forceinline__ void v_operands(const unsigned char* v, int t0, int lane,
                                                    bf16x8v_t (&a)[NDB]) {
    const int h = lane >> 5, l16 = lane & 15, hf = (lane >> 4) & 1;
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      s16x4_t part[2];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int row = t0 + 8 * z + 4 * h + (l16 >> 2);
        const int c = (32 * db + 16 * hf) / 8 + ((l16 & 3) >> 1);
        const unsigned char* src = v + row * (D * 2) + v_place(row, c) * 16 + (l16 & 1) * 8;
        part[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4_t*)(src));
      }
      a[db] = __builtin_bit_cast(bf16x8v_t,
                                 __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
  // acc += V^T P^T over N steps of 32 tokens; with RW > 1, where the products
  // bound the loop, the operands of the next 16 tokens are read before the
  // products of these
  template <int N>
  __device__ static __forceinline__ void pv(const unsigned char* v, int tok0, const Vec (&p)[N],
                                            bool twice, bool low, Vec (&acc)[NDB], int lane) {
    constexpr int kPin = 0x6;              // vector and scalar ALU may pass
    constexpr int kAhead = RW > 1 ? 1 : 0;
    bf16x8v_t a[1 + kAhead][NDB];
    if constexpr (kAhead) v_operands(v, tok0, lane, a[0]);
    static_for<0, 2 * N>([&](auto kc) {
      constexpr int ks = decltype(kc)::value, next = ks + kAhead;
      if constexpr (kAhead) __builtin_amdgcn_sched_barrier(kPin);
      if constexpr (next < 2 * N) v_operands(v, tok0 + 16 * next, lane, a[next & kAhead]);
      const bf16x8v_t b = p_operand(p[ks / 2], ks % 2, twice, low);
      if constexpr (kAhead) __builtin_amdgcn_sched_barrier(kPin);
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[ks & kAhead][db], b, acc[db], 0, 0, 0);
    });
  }
};

// 32-bit operands for more than 16 rows
template <int D, int RW> struct Ops<float, D, RW> : Wide {
  static constexpr int CPR = D / 4;
  static constexpr int NDB = D / kDims;
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
  __device__ __forceinline__ Vec logits(const unsigned char* k, int tok0, int lane) const {
    const int row = tok0 + (lane & 31), h = lane >> 5;
    Vec s = {};
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
  template <int N>
  __device__ static __forceinline__ void pv(const unsigned char* v, int tok0, const Vec (&p)[N],
                                            bool, bool, Vec (&acc)[NDB], int lane) {
    const int dim = lane & 31;
#pragma unroll
    for (int i = 0; i < N * kVals; ++i) {
      const int row = tok0 + i / kVals * kTok + token_of(i % kVals, lane);
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        const float x = *reinterpret_cast<const float*>(
            v + row * (D * 4) + v_place(row, 8 * db + (dim >> 2)) * 16 + (dim & 3) * 4);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p[i / kVals][i % kVals], acc[db], 0, 0, 0);
      }
    }
  }
};

// 32-bit operands for up to 16 rows, at half the matrix work of 32
template <int D> struct Ops<float, D, 1> : Narrow {
  static constexpr int CPR = D / 4;
  static constexpr int NDB = D / kDims;
  float q[D / 4];

  __device__ static __forceinline__ int k_place(int row, int c) { return c ^ (row & 15); }
  // the four quarters of a wave read rows four apart, 64 bytes of each
  __device__ static __forceinline__ int v_place(int row, int c) { return c ^ (((row >> 2) & 3) << 2); }
  // (dims in the order that logits() takes them: 16 j + 4 quarter + e)
  __device__ __forceinline__ void load_q(const float* row, int lane) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      const float4 x = *reinterpret_cast<const float4*>(row + 16 * j + 4 * (lane >> 4));
      q[4 * j] = x.x; q[4 * j + 1] = x.y; q[4 * j + 2] = x.z; q[4 * j + 3] = x.w;
    }
  }
  __device__ __forceinline__ Vec logits(const unsigned char* k, int tok0, int lane) const {
    const int row = tok0 + (lane & 15), g = lane >> 4;
    Vec s = {};
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      const float4 x =
          *reinterpret_cast<const float4*>(k + row * (D * 4) + k_place(row, 4 * j + g) * 16);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, q[4 * j], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, q[4 * j + 1], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, q[4 * j + 2], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, q[4 * j + 3], s, 0, 0, 0);
    }
    return s;
  }
  template <int N>
  __device__ static __forceinline__ void pv(const unsigned char* v, int tok0, const Vec (&p)[N],
                                            bool, bool, Vec (&acc)[NDB], int lane) {
    const int dim = lane & 15;
#pragma unroll
    for (int i = 0; i < N * kVals; ++i) {
      const int row = tok0 + i / kVals * kTok + token_of(i % kVals, lane);
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        const float x = *reinterpret_cast<const float*>(
            v + row * (D * 4) + v_place(row, 4 * db + (dim >> 2)) * 16 + (dim & 3) * 4);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, p[i / kVals][i % kVals], acc[db], 0, 0, 0);
      }
    }
  }
};

// Orders the scheduler's region: AHEAD operand reads from LDS, then one more for
// each of the N matrix instructions. (Left alone the compiler puts every read
// right before its use, and the matrix instructions wait for LDS one by one.)
template <int N, int AHEAD>
__device__ __forceinline__ void interleave() {
  constexpr int kMfma = 0x8, kRead = 0x100;
  __builtin_amdgcn_sched_group_barrier(kRead, AHEAD, 0);
  static_for<0, N - AHEAD>([](auto) {
    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
  });
  __builtin_amdgcn_sched_group_barrier(kMfma, AHEAD, 0);
}

// x, of which the compiler computes nothing ahead of this place: what only a last,
// partial tile needs would take registers through the whole loop
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A workgroup of four waves. RW = 1: every wave takes the same query rows (up to
// kRows) and tiles of its own, in its own part of the LDS, with no barrier in the
// loop: what memory bounds. RW = 2 or 4: RW waves with 32 rows each, and 4 / RW
// such groups that share the tokens of a tile.
template <typename T, int D, int RW>
struct Flash {
  using O = Ops<T, D, RW>;
  using Vec = typename O::Vec;
  static constexpr int TW = 4 / RW;              // groups with tokens of their own
  static constexpr int NTG = flash_tile(sizeof(T), RW);   // tokens of a workgroup's step
  static constexpr int NT = RW == 1 ? NTG / 4 : NTG;      // of one tile in LDS
  static constexpr int NTHR = RW == 1 ? 64 : 256;         // threads that load it
  static constexpr int kSub = NTG / TW / O::kTok;         // steps of a wave in it
  static constexpr int kBytes = NT * D * (int)sizeof(T);  // of K, and of V
  static constexpr int NCH = kBytes / 16 / NTHR; // chunks of each per thread
  static constexpr int NDB = O::NDB;
  // two buffers save the barrier before a tile is written
  static constexpr int kBuf = RW > 1 && 4 * kBytes <= (64 << 10) ? 2 : 1;
  static constexpr int kTiles = (RW == 1 ? 4 : kBuf) * 2 * kBytes;
  // the groups' accumulators are added in LDS
  static constexpr int kMerge = TW > 1 ? 4 * O::kRows * D * 4 : 0;
  static constexpr int kLds = kTiles > kMerge ? kTiles : kMerge;

  // Rows [r0, r1) of K and V (r1 > r0) for the query rows of this workgroup:
  // row_q(i) points to row i < rows; the partials go to acc_out [rows][D] and
  // ml_out [rows][2]. With LOG the logits of row i go to log_out + i * log_stride,
  // by token, a whole step's; rows is a power of two then, at most 8. With BOTH (RW =
  // 1) the rows [0, own_r1) of own_K and own_V follow, and the outputs, not the
  // partials, go to out [rows][D]. ONCE: no other workgroup reads these rows, and they
  // pass the caches by: kept there, they make the next call over the same 200 MB up to
  // 10% faster, but one over another layer's 14% slower (eight sequences of 6000 rows:
  // 36.1 us against 36.7, and 43.3 against 37.9).
  template <bool LOG, bool BOTH, bool ONCE, typename RowQ>
  __device__ static __forceinline__ void block(const T* __restrict__ K, const T* __restrict__ V,
                                               int64_t r0, int64_t r1, int rows, float qscale,
                                               RowQ&& row_q, float* acc_out, float* ml_out,
                                               float* log_out, int64_t log_stride,
                                               unsigned char* lds, float (*wm)[O::kRows * RW],
                                               float (*wl)[O::kRows * RW], const T* __restrict__ own_K = nullptr,
                                               const T* __restrict__ own_V = nullptr, int64_t own_r1 = 0,
                                               T* out = nullptr) {
    // The running maximum may lag the true one by this much (in log2): p grows
    // to 256 at most, which no sum minds, and the accumulators are rescaled once
    // or twice a run instead of whenever one of a wave's rows meets a new
    // maximum.
    constexpr float kSlack = 8.f;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rw = wave % RW, tw = wave / RW;
    const int col = lane % O::kRows;
    const bool twice = RW == 1 && sizeof(T) == 2 && rows <= 16;
    const bool low = twice && col >= 16;
    // this lane's query row (rows < 16 with logits: over and over)
    const int row = rw * O::kRows + (twice ? col & 15 : col);
    const int row_in = LOG ? col & (rows - 1) : min(row, rows - 1);
    const int ltid = RW == 1 ? lane : tid;
    unsigned char* tile0 = lds + (RW == 1 ? wave * 2 * kBytes : 0);

    O ops;
    ops.load_q(row_q(row_in), lane);
    Vec acc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) acc[db] = Vec{};
    float m = -INFINITY, l = 0.f;

    u32x4_t kr[NCH], vr[NCH];
    constexpr int kRowBytes = D * (int)sizeof(T);
    // rows behind the last are read as the last; with BOTH the own rows begin behind
    // the prefix's last step
    const int64_t own_at = BOTH ? (r1 + NTG - 1) / NTG * NTG : 0;
    const int64_t end = BOTH ? own_at + own_r1 : r1;
    auto rows_left = [&](int64_t at) { return (BOTH && at < own_at ? r1 : end) - at; };
    auto load = [&](int64_t at) {
      const bool own = BOTH && at >= own_at;
      const int64_t row = own ? at - own_at : at;
      const unsigned char* kb = reinterpret_cast<const unsigned char*>((own ? own_K : K) + row * D);
      const unsigned char* vb = reinterpret_cast<const unsigned char*>((own ? own_V : V) + row * D);
      auto get = [](const unsigned char* p) {
        const u32x4_t* v = reinterpret_cast<const u32x4_t*>(p);
        return ONCE ? __builtin_nontemporal_load(v) : *v;
      };
      const int last = (int)min<int64_t>(NT, rows_left(at)) - 1, lt = here(ltid);
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int x = i * NTHR + lt, r = x / O::CPR;
        const uint32_t off = min(r, last) * kRowBytes + x % O::CPR * 16;
        kr[i] = get(kb + off);
        vr[i] = get(vb + off);
      }
    };
    auto sync = [] {
      if constexpr (RW == 1) {                   // (the wave reads what it wrote)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      } else {
        __syncthreads();
      }
    };
    // this wave's next tile: of the prefix one may lie behind its rows
    auto there_is = [&](int64_t& at) {
      if (BOTH && at < own_at && at >= r1) at += NTG;
      return at < end;
    };
    int64_t at = r0 + (RW == 1 ? wave * NT : 0);
    if (there_is(at)) load(at);
    int buf = 0;
#pragma unroll 1
    for (int64_t next; at < end; at = next) {
      next = at + NTG;
      const bool more = there_is(next);
      unsigned char* kl = tile0 + buf * 2 * kBytes;
      unsigned char* vl = kl + kBytes;
      const int len = (int)min<int64_t>(NT, rows_left(at));
      if (kBuf == 1) sync();                     // the last tile is read
      // (32 rows in fp32 leave no register free: kept through the loop, the places in
      // LDS spill; 5%)
      const int pt = RW == 2 && sizeof(T) == 4 ? here(ltid) : ltid;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int x = i * NTHR + pt, r = x / O::CPR, c = x % O::CPR;
        *reinterpret_cast<u32x4_t*>(kl + (r * O::CPR + O::k_place(r, c)) * 16) = kr[i];
        *reinterpret_cast<u32x4_t*>(vl + (r * O::CPR + O::v_place(r, c)) * 16) = vr[i];
      }
      // V's rows behind the last become zeros here (their weight is 0, which an
      // infinity would turn into NaN); done where they are loaded, it would wait
      // for one load after the other
      if (len < NT) {                            // uniform
        const int lt = here(ltid);
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
          const int x = i * NTHR + lt, r = x / O::CPR, c = x % O::CPR;
          if (r >= len)
            *reinterpret_cast<u32x4_t*>(vl + (r * O::CPR + O::v_place(r, c)) * 16) = u32x4_t{0, 0, 0, 0};
        }
      }
      sync();
      if constexpr (!LOG) {
        if (more) load(next);
        __builtin_amdgcn_sched_barrier(0);
      }
      buf = kBuf == 2 ? buf ^ 1 : 0;
      const int tok0 = RW == 1 ? 0 : tw * kSub * O::kTok;
      Vec s[kSub];
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub) s[sub] = ops.logits(kl, tok0 + sub * O::kTok, lane);
      if constexpr (sizeof(T) == 2) interleave<kSub * D / 16, D / 32>();
      if constexpr (LOG) {
        // Row r's logits are in the columns r, r + rows, ...: copy u writes the
        // u-th four of the lane's tokens, so that a step's logits of a row leave
        // as whole lines by one store. (Ahead of the next tile's loads: behind
        // them, the wait for those would be one for the store too; 123 -> 118 us
        // for eight ragged sequences of 32K rows, 102 with no store at all.)
        static_assert(kSub == 1, "one step per tile");
        const int u = col / rows;
        float x[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
        int tok = O::token_of(0, lane);
#pragma unroll
        for (int i = 4; i < O::kVals; i += 4) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = 4 * u == i ? s[0][i + e] : x[e];
          tok = 4 * u == i ? O::token_of(i, lane) : tok;
        }
        if (4 * u < O::kVals)
          *reinterpret_cast<float4*>(log_out + row_in * log_stride + at + tok) =
              make_float4(x[0], x[1], x[2], x[3]);
        __builtin_amdgcn_sched_barrier(0);
        if (more) load(next);
        __builtin_amdgcn_sched_barrier(0);
      }
      // Of a SIMD's two waves the one with products to issue goes first: the other's
      // vector instructions fit between them (512 rows over 32768: 105.6 us, 100.5).
      if constexpr (RW == 4) __builtin_amdgcn_s_setprio(0);
      if (len < NT) {                            // uniform
#pragma unroll
        for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
          for (int i = 0; i < O::kVals; ++i)
            s[sub][i] = tok0 + sub * O::kTok + O::token_of(i, lane) < len ? s[sub][i] : -INFINITY;
      }
      float mt = s[0][0];
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
        for (int i = 0; i < O::kVals; ++i) mt = fmaxf(mt, s[sub][i]);
      const float mn = O::row_maximum(mt) * qscale;
      if (__ballot(mn > m + kSlack)) {
        const float top = fmaxf(m, mn);
        const float scale = top == -INFINITY ? 1.f : fast_exp2(m - top);   // 0 at first
        l *= scale;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int i = 0; i < (int)(sizeof(Vec) / 4); ++i) acc[db][i] *= scale;
        m = top;
      }
      const float mref = m == -INFINITY ? 0.f : m;
      float sum = 0.f;
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
        for (int i = 0; i < O::kVals; ++i) {
          s[sub][i] = fast_exp2(fmaf(s[sub][i], qscale, -mref));
          sum += s[sub][i];
        }
      l += sum;
      if constexpr (RW == 4) __builtin_amdgcn_s_setprio(2);
      O::pv(vl, tok0, s, twice, low, acc, lane);
    }
    l = O::row_total(l);
    constexpr int kAccVals = (int)(sizeof(Vec) / 4);
    if (twice) {                                 // the two parts of p
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < kAccVals; ++i) acc[db][i] = xor_sum<16>(acc[db][i]);
    }
    const bool mine = row < rows && !low;
    const bool first = lane < O::kRows;          // one lane of a row
    if constexpr (TW == 1) {
      if (!mine) return;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < kAccVals; i += 4)
          *reinterpret_cast<float4*>(acc_out + (int64_t)row * D + O::kDims * db + O::dim_of(i, lane)) =
              make_float4(acc[db][i], acc[db][i + 1], acc[db][i + 2], acc[db][i + 3]);
      if (first) *reinterpret_cast<float2*>(ml_out + 2 * row) = make_float2(m, l);
    } else {
      constexpr int RS = O::kRows * RW;
      float* wacc = reinterpret_cast<float*>(lds);
      // 16-byte pieces of a row at places XORed with the row
      auto place = [](int r, int piece) { return piece ^ (r & (D / 4 - 1)); };
      __syncthreads();                           // no wave reads its tile any more
      if (mine) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int i = 0; i < kAccVals; i += 4)
            *reinterpret_cast<float4*>(
                wacc + (tw * RS + row) * D +
                4 * place(row, (O::kDims * db + O::dim_of(i, lane)) / 4)) =
                make_float4(acc[db][i], acc[db][i + 1], acc[db][i + 2], acc[db][i + 3]);
        if (first) { wm[tw][row] = m; wl[tw][row] = l; }
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
        if constexpr (BOTH) {
          T* o = out + (int64_t)r * D + 4 * c;
          const float x[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = from_f32<T>(end > 0 ? x[e] / L : 0.f);
        } else {
          *reinterpret_cast<float4*>(acc_out + (int64_t)r * D + 4 * c) = a;
          if (c == 0) *reinterpret_cast<float2*>(ml_out + 2 * r) = make_float2(M, L);
        }
      }
    }
  }
};

// Blocks of the prefix first, then of the sequences' own rows. Workgroups i and
// i + 8 share an XCD and its L2: the row tiles of one (kv head, split) read the
// same rows and lie 8 apart.
template <typename T, int D, int RW, bool LOG>
__global__ __launch_bounds__(256, 2) void k_flash(FlashArgs a) {
  using F = Flash<T, D, RW>;
  using F1 = Flash<T, D, 1>;
  constexpr int kLds = F::kLds > F1::kLds ? F::kLds : F1::kLds;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kLds];
  __shared__ float wm[4 * 32], wl[4 * 32];       // [TW][rows]
  const int n_units = a.Hkv * a.splits;          // (kv head, split)
  const int n_prefix = (n_units + 7) / 8 * 8 * a.mtiles;
  int i = blockIdx.x;
  if constexpr (!LOG) {
    if (i < n_prefix) {
      using RowArray = float (*)[F::O::kRows * RW];
      const int unit = i / (8 * a.mtiles) * 8 + i % 8, mt = i / 8 % a.mtiles;
      if (unit >= n_units) return;
      const int hk = unit / a.splits, sp = unit % a.splits;
      const int64_t r0 = (int64_t)sp * a.tiles_p * F::NTG;
      const int64_t r1 = min(a.P, r0 + (int64_t)a.tiles_p * F::NTG);
      const int row0 = mt * F::O::kRows * RW;
      const int64_t at = (int64_t)unit * a.M + row0;
      auto block = [&](auto once) {
        F::template block<false, false, decltype(once)::value>(
            static_cast<const T*>(a.Kp) + hk * a.Pcap * D, static_cast<const T*>(a.Vp) + hk * a.Pcap * D,
            r0, r1, min(a.M - row0, F::O::kRows * RW), a.qscale,
            [&](int r) {
              const int x = row0 + r;              // b G + g
              return static_cast<const T*>(a.q) + ((int64_t)(x / a.G) * a.Hq + hk * a.G + x % a.G) * D;
            },
            a.pacc + at * D, a.pml + at * 2, nullptr, 0, lds, reinterpret_cast<RowArray>(wm),
            reinterpret_cast<RowArray>(wl));
      };
      // (once: where there is one row tile)
      if constexpr (sizeof(T) == 2) {
        block(std::bool_constant<(RW < 4)>{});
      } else if constexpr (RW == 1) {
        if (a.mtiles == 1) block(std::true_type{});
        else block(std::false_type{});
      } else {
        block(std::false_type{});
      }
      return;
    }
    i -= n_prefix;
  }
  using RowArray = float (*)[F1::O::kRows];
  // (the parts of a pair on different XCDs, and an XCD's parts of different pairs:
  // pairs of a ragged batch have different numbers of them)
  const int pairs = a.B * a.Hkv, part = i / pairs;
  const int64_t bh = (i + part) % pairs;
  const int64_t b = bh / a.Hkv, hk = bh % a.Hkv;
  const int64_t len = own_len(a, b, LOG ? 1 : 0);
  const int64_t r0 = (int64_t)part * a.tiles_o * F1::NTG;
  if (r0 >= len) return;
  const int64_t r1 = min(len, r0 + (int64_t)a.tiles_o * F1::NTG);
  const int64_t at = (bh * a.parts + part) * a.G;
  F1::template block<LOG, false, true>(
      static_cast<const T*>(a.K) + bh * a.cap * D, static_cast<const T*>(a.V) + bh * a.cap * D, r0, r1,
      a.G, a.qscale,
      [&](int r) { return static_cast<const T*>(a.q) + (b * a.Hq + hk * a.G + r) * D; },
      a.oacc + at * D, a.oml + at * 2, a.logits + bh * a.G * a.tpad, a.tpad, lds,
      reinterpret_cast<RowArray>(wm), reinterpret_cast<RowArray>(wl));
}

// A short prefix and few own rows: a workgroup of each (b, kv head) attends both
// and leaves the outputs.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void k_short(FlashArgs a) {
  using F = Flash<T, D, 1>;
  using RowArray = float (*)[F::O::kRows];
  __shared__ __attribute__((aligned(16))) unsigned char lds[F::kLds];
  __shared__ float wm[4 * 32], wl[4 * 32];
  const int64_t bh = blockIdx.x, b = bh / a.Hkv, hk = bh % a.Hkv;
  const int64_t len = own_len(a, b, 0), row0 = b * a.Hq + hk * a.G;
  T* out = static_cast<T*>(a.out) + row0 * D;
  if (len < 0) {
    for (int x = threadIdx.x; x < a.G * D; x += 256) out[x] = from_f32<T>(__uint_as_float(0x7fc00000u));
    return;
  }
  F::template block<false, true, true>(
      static_cast<const T*>(a.Kp) + hk * a.Pcap * D, static_cast<const T*>(a.Vp) + hk * a.Pcap * D, 0, a.P,
      a.G, a.qscale, [&](int r) { return static_cast<const T*>(a.q) + (row0 + r) * D; }, nullptr, nullptr,
      nullptr, 0, lds, reinterpret_cast<RowArray>(wm), reinterpret_cast<RowArray>(wl),
      static_cast<const T*>(a.K) + bh * a.cap * D, static_cast<const T*>(a.V) + bh * a.cap * D, len, out);
}

template <typename T, int D>
void launch_flash(const FlashArgs& a, int rw, hipStream_t st) {
  const unsigned n = (unsigned)(ceil_div(a.Hkv * a.splits, 8) * 8 * a.mtiles + a.B * a.Hkv * a.parts);
  if (rw == 0)
    launch(RADAR_K_ATTEND, k_short<T, D>, dim3((unsigned)(a.B * a.Hkv)), dim3(256), 0, st, a);
  else if (a.logits)
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
