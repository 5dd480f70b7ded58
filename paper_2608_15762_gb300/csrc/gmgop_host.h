// Host-side checks that the decoder-layer operators share.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/gmgop.h"

namespace gop {

inline bool cache_ok(const op_cache_t* c) {
  if (!c || !c->pool || !c->table || !c->lens || !c->refs || !c->status) return false;
  if (c->dtype != GMG_OP_BF16 && c->dtype != GMG_OP_F16) return false;
  if (c->n_pages < 1 || c->n_layers < 1 || c->n_kv_heads < 1 || c->n_seq < 1 || c->max_pages < 1 ||
      c->max_pages > (1 << 22))
    return false;
  if (c->page_tokens < 8 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return false;
  if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return false;
  return (reinterpret_cast<uintptr_t>(c->pool) & 15) == 0;
}

// Whether every row of a tensor with these strides (in elements of e bytes) starts on 16 bytes.
inline bool aligned(const void* p, int64_t s0, int64_t s1, int e) {
  return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(s0 * e) | uintptr_t(s1 * e)) & 15) == 0;
}

}  // namespace gop
