// The paged cache as the kernels see it, and what they share: a slot's place in memory, a
// sequence's lengths.  Every index that comes from device memory is checked before it is used.
#pragma once
#include "common.h"
#include "kernels.h"

namespace dk {

enum : int32_t { DEV_BAD_PAGE = 32 };

// the page of a sequence's slot, -1 where the table names none of the cache's
DEVI int page_of(const PagedView &c, int b, int slot) {
  const int page = c.table[(int64_t)b * c.max_pages + (slot >> c.page_shift)];
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}
// element offset of a slot's rows in k and v (layer 0, head 0)
DEVI int64_t slot_offset(const PagedView &c, int page, int slot) {
  return page * c.page_stride + (slot & ((1 << c.page_shift) - 1)) * c.slot_stride;
}
// element offset of a slot's accumulated weight: [layer][page][head][slot]
DEVI int64_t weight_offset(const PagedView &c, int layer, int page, int head, int slot) {
  return ((((int64_t)layer * c.n_pages + page) * c.n_kv + head) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
}

// Tokens [start, start + n) of the packed rows are sequence b's new ones, the last n of its len slots.
struct SeqRange {
  int start, n, len;
};
// false: nothing to do for the sequence (no new tokens, or lengths that disagree, which sets the error word)
DEVI bool seq_range(const int32_t *starts, const int32_t *lens, int b, int tokens, int max_new, int max_len, int32_t *err,
                    SeqRange &s) {
  const int lo = starts[b], hi = starts[b + 1];
  s.start = lo;
  s.n = 0;
  s.len = 0;
  if (lo == hi) return false;
  const int len = lens[b];
  // (hi - lo fits: both are in [0, tokens] once the first two hold)
  if (lo < 0 || hi > tokens || hi < lo || hi - lo > max_new || len < hi - lo || len > max_len) {
    if (err) raise_error(err, DEV_BAD_CTX_LEN);
    return false;
  }
  s.n = hi - lo;
  s.len = len;
  return true;
}

}  // namespace dk
