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
DEVI bool check_range(int lo, int hi, int len, int tokens, int max_new, int max_len, int32_t *err, SeqRange &s) {
  s.start = lo;
  s.n = 0;
  s.len = 0;
  if (lo == hi) return false;
  // (hi - lo fits: both are in [0, tokens] once the first two hold)
  if (lo < 0 || hi > tokens || hi < lo || hi - lo > max_new || len < hi - lo || len > max_len) {
    if (err) raise_error(err, DEV_BAD_CTX_LEN);
    return false;
  }
  s.n = hi - lo;
  s.len = len;
  return true;
}
DEVI bool seq_range(const int32_t *starts, const int32_t *lens, int b, int tokens, int max_new, int max_len, int32_t *err,
                    SeqRange &s) {
  const int lo = starts[b], hi = starts[b + 1], len = lens[b];  // one round trip
  return check_range(lo, hi, len, tokens, max_new, max_len, err, s);
}

// Starts that go down put rows into two sequences, and more rows into all of them than a launch has tiles for: the first sequence
// whose starts do and all behind it are left out, in every kernel.  True for a sequence before those (found by a whole wave, the same b in every lane).
// Costs the weights of 512 sequences' next tokens 6 us of 506, of 64 1 us of 615 (a barrier and all four waves 4).
DEVI bool starts_ascend(const int32_t *starts, int b) {
  constexpr int U = 8;  // loads on their way at a time, where there are many sequences
  const int lane = threadIdx.x & 63;
  bool down = starts[min(lane, b) + 1] < starts[min(lane, b)];
  for (int s0 = 64; s0 <= b; s0 += 64 * U) {
    int at[U], next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(s0 + 64 * u + lane, b);
      at[u] = starts[i];
      next[u] = starts[i + 1];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) down |= next[u] < at[u];
  }
  return __ballot(down) == 0;
}

// The sequence of packed row t, found by a whole wave (the same t in every lane): a lane loads a sequence's starts and length.  False for
// rows before the first sequence or behind the last, and in sequences that are left out.
DEVI bool seq_of_token(const int32_t *starts, const int32_t *lens, int batch, int t, int tokens, int max_new, int max_len, int &b,
                       SeqRange &s) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < batch; s0 += 64) {
    const int i = min(s0 + lane, batch - 1);
    const int lo = starts[i], hi = starts[i + 1], len = lens[i];
    // (lanes behind the last sequence repeat it: the first of a run of equal lanes is the one that counts)
    const uint64_t down = __ballot(hi < lo), past = __ballot(hi > t);
    if (!(down | past)) continue;
    const int l = __ffsll((unsigned long long)(down | past)) - 1;
    b = s0 + l;
    return !(down >> l & 1) && check_range(__builtin_amdgcn_readlane(lo, l), __builtin_amdgcn_readlane(hi, l),
                                           __builtin_amdgcn_readlane(len, l), tokens, max_new, max_len, nullptr, s) && t >= s.start;
  }
  return false;
}

// two fp32 values as neighbouring bf16 values, rounded to the nearest (even) by the conversion instruction
DEVI uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// Running sum over the lanes of a wave, by lane moves alone.
DEVI int wave_running_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast 31 into rows 2 and 3
  return v;
}

}  // namespace dk
