// Argument checks that the entry points share.
#pragma once

#include <stdint.h>

#include "cronus_internal.h"

namespace cronus {

inline int check_cache(const cronus_kv_cache* c) {
  if (!c || !c->k_cache || !c->v_cache || c->num_blocks <= 0) return CRONUS_ERR_INVALID_ARG;
  if (c->num_q_heads <= 0 || c->num_kv_heads <= 0) return CRONUS_ERR_INVALID_ARG;
  if (c->block_size != kBlock) return CRONUS_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return CRONUS_ERR_UNSUPPORTED;
  if (c->num_q_heads % c->num_kv_heads) return CRONUS_ERR_UNSUPPORTED;
  if (c->kv_dtype == CRONUS_KV_BF16) {
    if (c->k_scale || c->v_scale) return CRONUS_ERR_INVALID_ARG;
  } else if (c->kv_dtype == CRONUS_KV_FP8_E4M3) {
    if (!c->k_scale || !c->v_scale) return CRONUS_ERR_INVALID_ARG;
  } else {
    return CRONUS_ERR_UNSUPPORTED;
  }
  return CRONUS_OK;
}

// Shape-only variant for the size queries, which need no device pointers.
inline int check_shape(const cronus_kv_cache* c) {
  if (!c || c->num_q_heads <= 0 || c->num_kv_heads <= 0) return CRONUS_ERR_INVALID_ARG;
  if (c->block_size != kBlock) return CRONUS_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return CRONUS_ERR_UNSUPPORTED;
  if (c->num_q_heads % c->num_kv_heads) return CRONUS_ERR_UNSUPPORTED;
  if (c->kv_dtype != CRONUS_KV_BF16 && c->kv_dtype != CRONUS_KV_FP8_E4M3) return CRONUS_ERR_UNSUPPORTED;
  return CRONUS_OK;
}

inline bool workspace_refused(const void* workspace) { return !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u); }

}  // namespace cronus
