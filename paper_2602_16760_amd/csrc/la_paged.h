// The shared cache: host-side checks of its entry points, and the attention as la_forward_paged launches it.
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

// Bytes of workspace that the attention of up to B rows of Hq heads takes at any length of the table.
size_t paged_attend_bytes(const la_pages_desc &p, int Hq, int B);
// The attention of a model's rows.  q_tiles > 0: q in the prompt pass's operand fragments for that many row tiles, scaled already (scale 1); otherwise rows of the pages'
// type.  out: AT_OUT_FLOAT: float rows, AT_OUT_FRAGMENTS: half-precision operand fragments for q_tiles row tiles.
enum PagedOut { AT_OUT_ROWS = 0, AT_OUT_FLOAT = 1, AT_OUT_FRAGMENTS = 2 };
struct PagedRows {
  const int32_t *table;
  int64_t ldt;
  int n_req, max_blocks;
  const int32_t *req, *pos, *slot;
  int B;
  // trees (first != NULL): as la_paged_tree_attend takes them
  const int32_t *first, *len;
  const uint64_t *vis;
  int max_rows;
};
int paged_attend_rows(const la_pages_desc &p, int layer, const void *q, int q_tiles, int Hq, float scale, const PagedRows &r, PagedOut kind, void *out, void *workspace,
                      hipStream_t s);
// The same of trees of up to LA_MAX_ROWS rows of as many requests together (workspace: tree_attend_bytes).
int tree_attend_rows(const la_pages_desc &p, int layer, const void *q, int q_tiles, int Hq, float scale, const PagedRows &r, PagedOut kind, void *out, void *workspace, hipStream_t s);

}  // namespace la
