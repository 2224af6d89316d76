// Shared by the units of the cache operators (rotary.hip, attend.hip,
// evict.hip): the config checks and launch limits of include/radar_cache.h.
#pragma once

#include "radar_cache.h"
#include "radar_impl.h"

namespace radar_impl {

// The config fields that the cache operators read, with radar.h's limits.
// Fills B, Hq, Hkv, G, d, cap, dt and n_sink of the shape.
inline radar_status check_cache(const radar_config* cfg, Shape* s) {
  if (!cfg) return RADAR_EINVAL;
  if (cfg->batch < 1 || cfg->n_q_heads < 1 || cfg->n_kv_heads < 1 || cfg->capacity < 1 ||
      cfg->n_q_heads % cfg->n_kv_heads != 0 || cfg->n_sink < 0 || cfg->n_sink > cfg->capacity)
    return RADAR_EINVAL;
  if (cfg->kv_dtype != RADAR_F32 && cfg->kv_dtype != RADAR_BF16) return RADAR_EINVAL;
  const int G = cfg->n_q_heads / cfg->n_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8) return RADAR_EUNSUPPORTED;
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return RADAR_EUNSUPPORTED;
  if (cfg->capacity > INT32_MAX) return RADAR_EUNSUPPORTED;
  if ((int64_t)cfg->batch * cfg->n_kv_heads > 65535) return RADAR_EUNSUPPORTED;
  *s = Shape{};
  s->B = cfg->batch; s->Hq = cfg->n_q_heads; s->Hkv = cfg->n_kv_heads; s->G = G;
  s->d = cfg->head_dim; s->cap = cfg->capacity; s->dt = cfg->kv_dtype;
  s->n_sink = cfg->n_sink;
  return RADAR_OK;
}

// 16 bytes to dst, past the caches or not
template <bool PAST>
__device__ __forceinline__ void put16(unsigned char* dst, const uint4& v) {
  if constexpr (PAST)
    __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_t*>(dst));
  else
    *reinterpret_cast<uint4*>(dst) = v;
}

}  // namespace radar_impl
