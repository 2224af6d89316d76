// Exact attention of few query rows over long runs of cache rows, for the
// shared prefix and for the rows of each sequence (compiled once per element
// type and head dim: -DRADAR_ATTEND_F32=0|1 -DRADAR_ATTEND_D=64|128). The pass over
// the rows is flash_impl.h's.
#include "flash_impl.h"

#ifndef RADAR_ATTEND_D
#define RADAR_ATTEND_D 128
#endif
#ifndef RADAR_ATTEND_F32
#define RADAR_ATTEND_F32 0
#endif

namespace radar_impl {
namespace {

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
