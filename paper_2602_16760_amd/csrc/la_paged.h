// Host-side checks of the shared cache's entry points.
#pragma once
#include <initializer_list>

#include "la_device.h"
#include "la_internal.h"

namespace la {

inline bool aligned16(std::initializer_list<const void *> ps) {
  uintptr_t all = 0;
  for (const void *p : ps) all |= (uintptr_t)p;
  return all % 16 == 0;
}
inline size_t esize(const la_pages_desc *p) { return p->dtype == LA_F32 ? 4 : 2; }
inline size_t layer_bytes(const la_pages_desc *p) { return (size_t)p->n_pages * p->n_kv_heads * p->page_size * p->head_dim * esize(p); }
int check_pages(const la_pages_desc *p, int layer);

}  // namespace la
