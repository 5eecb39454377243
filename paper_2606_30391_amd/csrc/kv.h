// kv.h -- what the kernels that write the 8-bit key/value cache and those that read it share.
#ifndef FESTINA_KV_H
#define FESTINA_KV_H

#include <climits>
#include <cstdint>

#include "festina.h"

namespace festina_kv {

constexpr float kScaleMin = 0x1p-32f, kScaleMax = 0x1p32f;   // range of the cache's scales

inline bool power_of_two(int x) { return x > 0 && (x & (x - 1)) == 0; }

// Sizes and pointers of a cache: FESTINA_OK, or what is wrong with them.
inline festina_status check_cache(const festina_kv_cache *c) {
  if (!c || c->n_blocks < 1 || c->block_tokens < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return FESTINA_ERR_INVALID;
  const int bt = c->block_tokens, d = c->head_dim;
  if (bt < 16 || bt > 256 || !power_of_two(bt)) return FESTINA_ERR_UNSUPPORTED;
  if (d != 64 && d != 96 && d != 128 && d != 256) return FESTINA_ERR_UNSUPPORTED;
  if ((long long)c->n_blocks * bt > INT_MAX || c->n_kv_heads > 1024) return FESTINA_ERR_UNSUPPORTED;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return FESTINA_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15) return FESTINA_ERR_INVALID;
  return FESTINA_OK;
}

}  // namespace festina_kv

#endif
