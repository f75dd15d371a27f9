// What the operators beside the products share: answers of the entry points, checks of arguments.
#ifndef EGT_SERVE_H
#define EGT_SERVE_H

#include "egt_device.h"

namespace egt {

inline bool whole16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
// strides (elements of two bytes) that keep 16-byte pieces whole
inline bool whole8(int64_t a) { return a >= 0 && a % 8 == 0; }
template <typename... T>
inline bool whole8(int64_t a, T... rest) { return whole8(a) && whole8(rest...); }

inline egt_status answer(hipError_t e) {
  if (e == hipSuccess) return EGT_OK;
  note_hip_error(e);
  return EGT_ERR_HIP;
}

// A cache's sizes, and its pointers and strides where `pointers` is set.
inline egt_status check_cache(const egt_kv_cache *c, bool pointers) {
  if (!c) return EGT_ERR_NULL;
  if (c->blocks < 0 || c->heads < 1 || c->dim < 8 || c->dim % 8 != 0 || c->dim > 256 || c->page < 1 || (c->page & (c->page - 1)) != 0 ||
      (int64_t)c->blocks * c->page >= (1ll << 31))
    return EGT_ERR_SHAPE;
  if (!pointers) return EGT_OK;
  if (c->blocks > 0 && (!c->k || !c->v)) return EGT_ERR_NULL;
  if (!whole8(c->k_block, c->k_head, c->k_token, c->v_block, c->v_head, c->v_token) || !whole16(c->k) || !whole16(c->v)) return EGT_ERR_BUFFER;
  return EGT_OK;
}

inline int log2_of(int page) {
  int s = 0;
  while ((1 << s) < page) ++s;
  return s;
}

}  // namespace egt
#endif
