// Host-side argument checks shared by the entry points.
#pragma once

#include "saw_common.h"

namespace saw {

inline bool aligned16(const void* p) { return (((uintptr_t)p) & 15u) == 0; }

inline bool shape_ok(const saw_cache_t* c) {
  if (c->page_size != 16) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->n_kv_heads < 1 || c->num_pages < 1) return false;
  return true;
}

inline bool block_ok(const saw_cache_t* c) {
  const int h = c->had_block;
  if (!(h == 1 || h == 16 || h == 32 || h == 64 || h == 128)) return false;
  if (h > c->head_dim) return false;
  if (c->rotate_mask & ~(SAW_ROT_K | SAW_ROT_V)) return false;
  // sign bits exist for the head's channels only
  if (c->head_dim == 64 && (c->sign_bits[2] | c->sign_bits[3])) return false;
  // the learned rotation is built for head_dim 128, its prepared buffer read with 16-byte loads
  if (c->dense_rot && (c->head_dim != kDenseD || !aligned16(c->dense_rot))) return false;
  return true;
}

}  // namespace saw
