// A cache of pages: the append of new tokens with their rotary positions, the commit of an
// accepted path, and eviction by accumulated attention weight.
#include "paged.h"

namespace dk {

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------
// Eight elements of a head a lane: 16 (d_h 128) or 8 lanes a head.  A lane reads its own eight and, with rotated
// halves, the eight that they are paired with, so nothing passes between lanes but a head's sum of squares.
// Per pair (x, y) at angle a = position * frequency: (x cos a - y sin a, y cos a + x sin a).  The angle is a number of
// turns in fp64, taken modulo one before it is rounded: positions in the millions keep fp32's accuracy.
// Bound by the rows' bytes, each read and written once: 9384 tokens of 32 + 2 x 8 heads of 128 bf16 values 56 us, 4.1 TB/s; one token 4.9.
constexpr int kAppendThreads = 256;

template <typename T>
DEVI void load8(const T *p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 w = *(const u32x4 *)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  } else {
    const floatx4 a = *(const floatx4 *)p, b = *(const floatx4 *)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = a[e];
      x[4 + e] = b[e];
    }
  }
}
template <typename T>
DEVI void store8(T *p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
    *(u32x4 *)p = w;
  } else {
    *(floatx4 *)p = floatx4{x[0], x[1], x[2], x[3]};
    *(floatx4 *)(p + 4) = floatx4{x[4], x[5], x[6], x[7]};
  }
}

template <typename T, int DH>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int LPH = DH / 8, GROUPS = kAppendThreads / LPH;
  const int t = blockIdx.x, j = threadIdx.x % LPH, grp = threadIdx.x / LPH;
  const int room = a.c.max_pages << a.c.page_shift;
  if (t == a.tokens) {  // one workgroup more than there are rows looks at all sequences, also those that have no row
    SeqRange all;
    for (int i = threadIdx.x; i < a.c.batch; i += kAppendThreads) seq_range(a.starts, a.lens, i, a.tokens, a.tokens, room, a.err, all);
    return;
  }
  int b;
  SeqRange s;
  if (!seq_of_token(a.starts, a.lens, a.c.batch, t, a.tokens, a.tokens, room, b, s)) return;
  const int slot = s.len - s.n + (t - s.start);
  const int page = page_of(a.c, b, slot);
  if (page < 0) raise_error(a.err, DEV_BAD_PAGE);
  const int64_t off = slot_offset(a.c, max(page, 0), slot);

  // factors of this lane's elements: out = own * cs + partner * sn
  float cs[8], sn[8];
  const int half = a.rot / 2, e0 = 8 * j;
  const bool turned = e0 < a.rot;
  int partner = e0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  if (turned) {
    const double pos = a.positions ? a.positions[t] : slot;
    const bool second = !a.interleaved && e0 >= half;
    const int f0 = a.interleaved ? e0 / 2 : (second ? e0 - half : e0);
    if (!a.interleaved) partner = second ? e0 - half : e0 + half;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (a.interleaved && (e & 1)) continue;
      const double turns = pos * a.freq[f0 + (a.interleaved ? e / 2 : e)] * 0.15915494309189535;  // 1 / (2 pi)
      float c, d;
      sincospif(2.f * (float)(turns - rint(turns)), &d, &c);
      c *= a.rope_scale;
      d *= a.rope_scale;
      if (a.interleaved) {
        cs[e] = cs[e + 1] = c;
        sn[e] = -d;
        sn[e + 1] = d;
      } else {
        cs[e] = c;
        sn[e] = second ? d : -d;
      }
    }
  }

  const int heads = a.nq + 2 * a.c.n_kv;
  for (int h = blockIdx.y * GROUPS + grp; h < heads; h += gridDim.y * GROUPS) {
    const bool is_q = h < a.nq, is_v = h >= a.nq + a.c.n_kv;
    const int hk = is_q ? h : (is_v ? h - a.nq - a.c.n_kv : h - a.nq);
    const T *src = is_q ? (const T *)a.q + (int64_t)t * a.q_stride + (int64_t)hk * DH
                        : (is_v ? (const T *)a.vn + (int64_t)t * a.v_stride + (int64_t)hk * DH
                                : (const T *)a.kn + (int64_t)t * a.k_stride + (int64_t)hk * DH);
    T *dst = is_q ? (T *)a.q_out + (int64_t)t * a.o_stride + (int64_t)hk * DH
                  : (T *)(is_v ? a.c.v : a.c.k) + a.layer * a.c.layer_stride + off + hk * a.c.head_stride;
    float x[8], y[8];
    load8(src + e0, x);
    if (!is_v) {
      const T *gain = (const T *)(is_q ? a.q_norm : a.k_norm);
      float g[8], gp[8], r = 1.f;
      const bool pair = turned && !a.interleaved;
      if (pair) load8(src + partner, y);
      if (gain) {
        load8(gain + e0, g);
        if (pair) load8(gain + partner, gp);
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
#pragma unroll
        for (int o = LPH / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
        r = 1.f / sqrtf(ss * (1.f / DH) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * r * g[e];
        if (pair) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = y[e] * r * gp[e];
        }
      }
      if (turned) {
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = x[e ^ 1];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * cs[e] + y[e] * sn[e];
      }
    }
    if (is_q || page >= 0) store8(dst + e0, x);
    if (!is_q && !is_v && page >= 0 && a.c.weights && j == 0) a.c.weights[weight_offset(a.c, a.layer, page, hk, slot)] = 0.f;
  }
}

// ---------------------------------------------------------------------------
// commit: rows n + node(d) move to n + d.  A workgroup has one head of one layer and sequence:
// every source is in registers before the first row is written.
// ---------------------------------------------------------------------------
constexpr int kMoveThreads = 256;

// PER items of 16 bytes a thread: what bounds it is how many workgroups a CU holds, so the usual few rows take few registers (32 trees
// of depth 15, 36 layers: 19.6 us with 4, 26.9 with the 16 that 63 rows of 128 fp32 values need).
template <int PER>
__global__ __launch_bounds__(kMoveThreads) void paged_commit_kernel(PagedView c, int nn, int max_depth,
                                                                    const int32_t *__restrict__ ctx_lens,
                                                                    const int32_t *__restrict__ accept_len,
                                                                    const int32_t *__restrict__ accepted,
                                                                    int32_t *__restrict__ new_lens, int32_t *err) {
  const int head = blockIdx.x % c.n_kv, b = (blockIdx.x / c.n_kv) % c.batch, layer = blockIdx.x / c.n_kv / c.batch;
  const int tid = threadIdx.x, n = ctx_lens[b], a = accept_len[b];
  const bool lead = layer == 0 && head == 0 && tid == 0;
  __shared__ int64_t from[64], to[64], w_from[64], w_to[64];
  __shared__ int bad;
  if (tid == 0) bad = 0;
  __syncthreads();
  if (n < 0 || a < 0 || a > max_depth || n > (c.max_pages << c.page_shift) - nn) {
    if (lead) {
      raise_error(err, DEV_BAD_CTX_LEN);
      new_lens[b] = n;
    }
    return;
  }
  if (tid < a) {  // a <= 63
    const int d = tid + 1, x = accepted[(size_t)b * max_depth + tid];
    from[tid] = -1;  // stays
    if (x < d || x >= nn) {
      atomicOr(&bad, DEV_BAD_TREE);
    } else if (x != d) {
      const int pf = page_of(c, b, n + x), pt = page_of(c, b, n + d);
      if (pf < 0 || pt < 0) atomicOr(&bad, DEV_BAD_PAGE);
      from[tid] = slot_offset(c, max(pf, 0), n + x);
      to[tid] = slot_offset(c, max(pt, 0), n + d);
      w_from[tid] = weight_offset(c, layer, max(pf, 0), head, n + x);
      w_to[tid] = weight_offset(c, layer, max(pt, 0), head, n + d);
    }
  }
  __syncthreads();
  if (bad) {
    if (lead) {
      raise_error(err, bad);
      new_lens[b] = n;
    }
    return;
  }
  if (lead) new_lens[b] = n + 1 + a;
  if (a == 0) return;
  const int esz = c.bf16 ? 2 : 4, shift = __builtin_ctz(c.dh * esz / 16), half = a << shift, items = 2 * half;  // (8, 16 or 32 items a row)
  const int64_t base = (layer * c.layer_stride + head * c.head_stride) * esz;
  // item `it`: 16 bytes of a row of k, then of v; its place from `rows`' offset of the row
  auto place = [&](int it, const int64_t *rows) {
    const int rem = it < half ? it : it - half;
    return (it < half ? c.k : c.v) + base + rows[rem >> shift] * esz + (rem & ((1 << shift) - 1)) * 16;
  };
  auto moves = [&](int it) { return it < items && from[(it < half ? it : it - half) >> shift] >= 0; };
  u32x4 v[PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const int it = tid + q * kMoveThreads;
    v[q] = u32x4{0, 0, 0, 0};
    if (q * kMoveThreads < items && moves(it)) v[q] = *(const u32x4 *)place(it, from);
  }
  float w = 0.f;
  if (c.weights && tid < a && from[tid] >= 0) w = c.weights[w_from[tid]];
#pragma unroll
  for (int q = 0; q < PER; ++q) __asm__ volatile("" ::"v"(v[q]));  // every load has arrived before the barrier
  __asm__ volatile("" ::"v"(w));
  __syncthreads();
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const int it = tid + q * kMoveThreads;
    if (q * kMoveThreads < items && moves(it)) *(u32x4 *)place(it, to) = v[q];
  }
  if (c.weights && tid < a && from[tid] >= 0) c.weights[w_to[tid]] = w;
}

// ---------------------------------------------------------------------------
// eviction
// ---------------------------------------------------------------------------
// Unsigned order of a weight: NaN and anything below zero as it compares, NaN lowest.
DEVI uint32_t weight_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Which slots of one (layer, sequence, head) stay, in order: the first `sink`, the last `recent`, and the m of greatest weight
// between them.  A workgroup has a slice of 16384 slots, a wave 1024 of them, whose keys it keeps in registers (16 a lane).  The m-th
// greatest key is found by three counts over its digits (11, 11 and 10 bits): kept are the keys above it and the first `need` that
// equal it.  Then every wave counts the kept slots of its stretch, and writes them behind those of the waves before it.
//   one slice    one launch: bound by the chain of its steps (1100 slots 8.7 us, 384 heads of up to 16384 36)
//   more slices  a launch for each count and one that writes; a slice's counts are its own, and the next launch adds them up.
//                (100003 slots of 16 heads in one workgroup each took 125 us: bound by its instructions)
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kSelStep = 256, kSelSteps = 4;  // slots of a wave's step (four neighbours a lane), steps of a wave's stretch
constexpr int kSelWave = kSelStep * kSelSteps;
static_assert(kSelWaves * kSelWave == kEvictSlice, "a slice is what a workgroup's registers hold");

// A workgroup's slice of one head: its wave's stretch [w0, w1) of the n slots, those of [first, last) with a choice.
struct Slice {
  int n, first, last, m, w0, w1;
  bool lost;
  uint32_t key[kSelSteps][4];  // of slots w0 + x * kSelStep + lane * 4 + e
};

template <bool TINY_PAGES>
DEVI void slice_load(const PagedEvictArgs &a, int b, int layer, int head, int slice, int n, Slice &s) {
  const PagedView &c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  s.n = n;
  s.first = a.sink;
  s.last = n - a.recent;
  s.m = a.budget - a.sink - a.recent;
  // (a sequence that one workgroup has alone is spread over its waves)
  const int per = n > kEvictSlice ? kSelWave : (n + kSelWaves * kSelStep - 1) / (kSelWaves * kSelStep) * kSelStep;
  s.w0 = min(n, slice * kEvictSlice + wave * per);
  s.w1 = min(n, s.w0 + per);
  s.lost = false;
  if (s.w0 == s.w1) return;
  const float *weights = c.weights + (((int64_t)layer * c.n_pages * c.n_kv + head) << c.page_shift);
  const int64_t page_step = (int64_t)c.n_kv << c.page_shift;
  const int in_page = (1 << c.page_shift) - 1;
  constexpr int PE = TINY_PAGES ? 4 : 1;  // four neighbours lie in one page of four slots or more
  int page[kSelSteps][PE];
#pragma unroll
  for (int x = 0; x < kSelSteps; ++x)
#pragma unroll
    for (int e = 0; e < PE; ++e) page[x][e] = page_of(c, b, min(s.w0 + x * kSelStep + lane * 4 + e, n - 1));
  floatx4 w[kSelSteps];
#pragma unroll
  for (int x = 0; x < kSelSteps; ++x) {
    const int slot = s.w0 + x * kSelStep + lane * 4;
#pragma unroll
    for (int e = 0; e < PE; ++e) {
      const float *at = weights + max(page[x][e], 0) * page_step;
      if (TINY_PAGES) w[x][e] = at[min(slot + e, n - 1) & in_page];
      else w[x] = *(const floatx4 *)(at + (min(slot, (n - 1) & ~3) & in_page));
    }
  }
#pragma unroll
  for (int x = 0; x < kSelSteps; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool known = page[x][TINY_PAGES ? e : 0] >= 0;
      s.lost |= !known;
      s.key[x][e] = known ? weight_key(w[x][e]) : 0;
    }
}

constexpr int digit_shift(int pass) { return pass == 0 ? 21 : (pass == 1 ? 10 : 0); }
constexpr int digit_bits(int pass) { return pass == 2 ? 10 : 11; }

// hist[d] = how many keys of the slice with a choice share `prefix` and have d for the next digit
DEVI void slice_count(const Slice &s, int pass, uint32_t prefix, uint32_t *hist) {
  const int lane = threadIdx.x & 63, shift = digit_shift(pass), bits = digit_bits(pass);
  for (int i = threadIdx.x; i < 2048; i += kSelThreads) hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kSelSteps; ++x) {
    const int s0 = s.w0 + x * kSelStep;
    if (s0 >= s.w1) break;
    const bool inner = s0 >= s.first && s0 + kSelStep <= min(s.last, s.w1);  // wave-uniform
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int slot = s0 + lane * 4 + e;
      bool in = pass == 0 || (s.key[x][e] >> (shift + bits)) == prefix;
      if (!inner) in = in && slot >= s.first && slot < min(s.last, s.w1);
      if (in) {
        // slots that all share one digit are counted at once: most may hold one value
        const uint32_t bin = (s.key[x][e] >> shift) & ((1u << bits) - 1), b0 = __builtin_amdgcn_readfirstlane(bin);
        const uint64_t all = __ballot(true);
        if (__ballot(bin == b0) == all) {
          if (lane == __ffsll((unsigned long long)all) - 1) atomicAdd(&hist[b0], (uint32_t)__popcll(all));
        } else {
          atomicAdd(&hist[bin], 1u);
        }
      }
    }
  }
  __syncthreads();
}

// From the top digit down: the one where the running count reaches `need`; it joins the prefix, and what lies above it leaves `need`.
// A thread has two digits, and the waves' sums meet in LDS.  (All counts together are over `need`: more slots have a choice than stay.)
DEVI void next_digit(const uint32_t *hist, int pass, uint32_t &prefix, uint32_t &need) {
  static_assert(kSelThreads * 2 == 2048, "two digits a thread");
  __shared__ uint32_t s_sum[kSelWaves], s_bin, s_above;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, low = 2046 - 2 * (int)threadIdx.x;
  const uint2 two = *(const uint2 *)(hist + low);
  const uint32_t mine = two.x + two.y, incl = wave_running_sum(mine);
  if (lane == 63) s_sum[wave] = incl;
  __syncthreads();
  const uint32_t before = __builtin_amdgcn_readlane(wave_running_sum(lane < wave ? s_sum[lane] : 0), 63);
  const uint32_t upto = before + incl, above = upto - mine;
  if ((above < need && upto >= need) || (low == 0 && upto < need)) {
    const bool high = above + two.y >= need;
    s_bin = low + high;
    s_above = high ? above : above + two.y;
  }
  __syncthreads();
  prefix = (prefix << digit_bits(pass)) | s_bin;
  need -= s_above;
}

// bit masks over the lanes of a step's slots that stay for sure, and of those that equal the last key that does
DEVI void slice_marks(const Slice &s, int x, uint32_t prefix, uint64_t (&sure)[4], uint64_t (&tie)[4]) {
  const int lane = threadIdx.x & 63, s0 = s.w0 + x * kSelStep;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int slot = s0 + lane * 4 + e;
    const bool in = slot >= s.first && slot < s.last;
    sure[e] = __ballot(slot < s.w1 && (!in || (s.m > 0 && s.key[x][e] > prefix)));
    tie[e] = __ballot(slot < s.w1 && in && s.m > 0 && s.key[x][e] == prefix);
  }
}
// what the wave's stretch holds of both
DEVI uint2 slice_sum(const Slice &s, uint32_t prefix) {
  uint2 sum = make_uint2(0, 0);
#pragma unroll
  for (int x = 0; x < kSelSteps; ++x) {
    if (s.w0 + x * kSelStep >= s.w1) break;
    uint64_t sure[4], tie[4];
    slice_marks(s, x, prefix, sure, tie);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum.x += __popcll(sure[e]);
      sum.y += __popcll(tie[e]);
    }
  }
  return sum;
}
// writes the wave's kept slots; `before`: what the stretches before it hold of both
DEVI void slice_write(const Slice &s, uint32_t prefix, uint32_t need, uint2 before, int32_t *kept, int budget) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int x = 0; x < kSelSteps; ++x) {
    const int s0 = s.w0 + x * kSelStep;
    if (s0 >= s.w1) break;
    uint64_t sure[4], tie[4];
    slice_marks(s, x, prefix, sure, tie);
    uint32_t bs = before.x, bt = before.y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bs += __popcll(sure[e] & below);
      bt += __popcll(tie[e] & below);
      before.x += __popcll(sure[e]);
      before.y += __popcll(tie[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = sure[e] >> lane & 1, t = tie[e] >> lane & 1;
      const uint32_t to = bs + min(bt, need);
      if ((in || (t && bt < need)) && to < (uint32_t)budget) kept[to] = s0 + lane * 4 + e;
      bs += in;
      bt += t;
    }
  }
}
// the waves' sums of the workgroup added up before this one's
DEVI uint2 sums_before(uint2 mine) {
  __shared__ uint2 s_sum[kSelWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) s_sum[wave] = mine;
  __syncthreads();
  const uint2 s = lane < wave ? s_sum[lane] : make_uint2(0, 0);
  return make_uint2(__builtin_amdgcn_readlane(wave_running_sum(s.x), 63), __builtin_amdgcn_readlane(wave_running_sum(s.y), 63));
}

// Sequences with nothing to choose: new length and kept slots.  True for those.
DEVI bool evict_trivial(const PagedEvictArgs &a, int b, bool lead, int n, int32_t *kept) {
  const bool bad = n < 0 || n > a.max_len;
  if (lead && threadIdx.x == 0) {
    if (bad) raise_error(a.err, DEV_BAD_CTX_LEN);
    a.new_lens[b] = bad ? n : min(n, a.budget);
  }
  if (!bad && n > a.budget) return false;
  for (int i = threadIdx.x; i < a.budget; i += kSelThreads) kept[i] = !bad && i < n ? i : -1;
  return true;
}

template <bool TINY_PAGES>
__global__ __launch_bounds__(kSelThreads) void paged_evict_select_kernel(PagedEvictArgs a) {
  const PagedView &c = a.c;
  const int head = blockIdx.x % c.n_kv, b = (blockIdx.x / c.n_kv) % c.batch, layer = blockIdx.x / c.n_kv / c.batch;
  int32_t *kept = a.kept + (size_t)blockIdx.x * a.budget;
  const int n = a.lens[b];
  if (evict_trivial(a, b, layer == 0 && head == 0, n, kept)) return;
  __shared__ __align__(8) uint32_t hist[2048];
  Slice s;
  slice_load<TINY_PAGES>(a, b, layer, head, 0, n, s);
  uint32_t prefix = 0, need = s.m;
  for (int pass = 0; pass < 3 && s.m > 0; ++pass) {
    slice_count(s, pass, prefix, hist);
    next_digit(hist, pass, prefix, need);
  }
  const uint2 before = sums_before(slice_sum(s, prefix));
  slice_write(s, prefix, need, before, kept, a.budget);
  if (s.lost) raise_error(a.err, DEV_BAD_PAGE);
}

// The sum of `v` over a workgroup's threads.
DEVI uint32_t block_sum(uint32_t v) {
  __shared__ uint32_t s_v[kSelWaves];
  const int lane = threadIdx.x & 63;
  v = wave_running_sum(v);
  __syncthreads();
  if (lane == 63) s_v[threadIdx.x >> 6] = v;
  __syncthreads();
  return __builtin_amdgcn_readlane(wave_running_sum(lane < kSelWaves ? s_v[lane] : 0), 63);
}

// The same over several slices, phase by phase: 0 to 2 count a digit, 3 writes.  Between them a head's slices leave `parts`
// [2][head][slices][2048], a phase's counts beside those that it reads; `state` [head][2], (prefix, need) after the first two digits; and
// `sums` [head][slices], the slice's keys above those digits.  So the last phase knows how many slots stay in the slices before its own.
template <bool TINY_PAGES>
__global__ __launch_bounds__(kSelThreads) void paged_evict_phase_kernel(PagedEvictArgs a, int phase, int slices) {
  const PagedView &c = a.c;
  const int slice = blockIdx.x % slices, at = blockIdx.x / slices;
  const int head = at % c.n_kv, b = (at / c.n_kv) % c.batch, layer = at / c.n_kv / c.batch;
  int32_t *kept = a.kept + (size_t)at * a.budget;
  const size_t half = (size_t)gridDim.x * 2048, mine = (size_t)at * slices * 2048;
  const uint32_t *counted = a.parts + ((phase & 1) ^ 1) * half + mine;
  uint2 *state = a.state + (size_t)at * 2;
  uint32_t *sums = a.sums + (size_t)at * slices;
  const int n = a.lens[b];
  if (phase == 0 && slice == 0 && evict_trivial(a, b, layer == 0 && head == 0, n, kept)) return;
  if (n <= a.budget || n > a.max_len || slice * kEvictSlice >= n) return;
  __shared__ __align__(8) uint32_t hist[2048];
  const int used = (n + kEvictSlice - 1) / kEvictSlice;
  Slice s;
  slice_load<TINY_PAGES>(a, b, layer, head, slice, n, s);
  uint32_t prefix = 0, need = s.m;
  uint2 before = make_uint2(0, 0);
  if (s.m > 0 && phase > 0) {
    if (phase > 1) {
      prefix = state[phase - 2].x;
      need = state[phase - 2].y;
    }
    // the digit that the last phase counted: all slices' counts, and of them this slice's, or in the end those of the slices before.
    // (Eight slices' loads at a time, of both digits: one by one they took 5 us of a phase's 12.5, 11 of the last one's 19.)
    constexpr int PER = 2048 / kSelThreads, U = 8;
    uint32_t all[PER] = {}, part[PER] = {};
    for (int x0 = 0; x0 < used; x0 += U) {
      uint32_t v[U][PER];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < PER; ++k) v[u][k] = counted[(size_t)min(x0 + u, used - 1) * 2048 + k * kSelThreads + threadIdx.x];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = x0 + u;
        const bool mine = phase < 3 ? x == slice : x < slice;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          all[k] += x < used ? v[u][k] : 0;
          part[k] += x < used && mine ? v[u][k] : 0;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) hist[k * kSelThreads + threadIdx.x] = all[k];
    __syncthreads();
    next_digit(hist, phase - 1, prefix, need);
    if (slice == 0 && threadIdx.x == 0 && phase < 3) state[phase - 1] = make_uint2(prefix, need);
    const int bin = prefix & ((1u << digit_bits(phase - 1)) - 1);
    __shared__ uint32_t s_equal;
    uint32_t above = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = k * kSelThreads + threadIdx.x;
      above += i > bin ? part[k] : 0;
      if (i == bin) s_equal = part[k];
    }
    if (phase == 3)
      for (int x = threadIdx.x; x < slice; x += kSelThreads) above += sums[x];
    above = block_sum(above);
    if (phase < 3) {
      if (threadIdx.x == 0) sums[slice] = (phase == 1 ? 0 : sums[slice]) + above;
    } else {
      before = make_uint2(above, s_equal);
    }
  }
  if (phase < 3) {
    if (s.m > 0) {
      slice_count(s, phase, prefix, hist);
      uint32_t *to = a.parts + (phase & 1) * half + mine + (size_t)slice * 2048;
      for (int i = threadIdx.x; i < 2048; i += kSelThreads) to[i] = hist[i];
    }
  } else {
    const int past = slice * kEvictSlice;  // slots of the slices before, some of them without a choice
    before.x += min(past, s.first) + max(0, past - s.last);
    const uint2 waves = sums_before(slice_sum(s, prefix));
    slice_write(s, prefix, need, make_uint2(before.x + waves.x, before.y + waves.y), kept, a.budget);
    if (s.lost) raise_error(a.err, DEV_BAD_PAGE);
  }
}

// Rows kept[i] move to slot i.  In place, a workgroup has one column slice of one head's keys or values (or the head's
// weights) and goes up the slots in rounds: kept[i] >= i, so a round writes no slot that a later one reads, and reads all of its own
// before it writes.  To new pages there is no such order: a workgroup has a stretch of rows (1.97 GB read and written 403 us, 4.9 TB/s).
template <bool WEIGHTS, int SLICE>  // SLICE: 16-byte items of a row's slice
DEVI void evict_in_place(const PagedEvictArgs &a, int b, int layer, int head, const int32_t *kept, int count, char *data,
                         int64_t base, int esz, int slice) {
  constexpr int PER = 8, ITEMS = WEIGHTS ? 1 : SLICE, ROWS = kMoveThreads * PER / ITEMS;
  const PagedView &c = a.c;
  const int tid = threadIdx.x;
  bool lost = false;
  // where this thread's items of a round are (bytes, or elements of the weights), and go to; -1: they stay.  A round's places are found while
  // the rows of the one before are on their way: nothing that they follow from is moved.
  int64_t from[PER], to[PER];
  auto find = [&](int r0) {
    int s[PER];
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      s[q] = 0;
      if (r0 + q * (kMoveThreads / ITEMS) < count) s[q] = kept[min(r0 + (tid + q * kMoveThreads) / ITEMS, count - 1)];
    }
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int it = tid + q * kMoveThreads, i = r0 + it / ITEMS;
      to[q] = from[q] = -1;
      if (i >= count || s[q] <= i) continue;  // (its own place: it stays)
      const int pf = page_of(c, b, s[q]), pt = page_of(c, b, i);
      if (pf < 0 || pt < 0) {
        lost = true;
        continue;
      }
      if (WEIGHTS) {
        from[q] = weight_offset(c, layer, pf, head, s[q]);
        to[q] = weight_offset(c, layer, pt, head, i);
      } else {
        const int64_t col = (slice * SLICE + it % ITEMS) * 16;
        from[q] = base + slot_offset(c, pf, s[q]) * esz + col;
        to[q] = base + slot_offset(c, pt, i) * esz + col;
      }
    }
  };
  find(0);
  for (int r0 = 0; r0 < count; r0 += ROWS) {
    u32x4 v[PER];
    float w[PER];
    int64_t at[PER];
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      v[q] = u32x4{0, 0, 0, 0};
      w[q] = 0.f;
      at[q] = to[q];
      if (at[q] < 0) continue;
      if (WEIGHTS) w[q] = c.weights[from[q]];
      else v[q] = *(const u32x4 *)(data + from[q]);
    }
    if (r0 + ROWS < count) find(r0 + ROWS);
#pragma unroll
    for (int q = 0; q < PER; ++q) __asm__ volatile("" ::"v"(v[q]), "v"(w[q]));  // every load has arrived
    __syncthreads();
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      if (at[q] < 0) continue;
      if (WEIGHTS) c.weights[at[q]] = w[q];
      else *(u32x4 *)(data + at[q]) = v[q];
    }
    __syncthreads();
  }
  if (lost) raise_error(a.err, DEV_BAD_PAGE);
}

template <int SLICE>
__global__ __launch_bounds__(kMoveThreads) void paged_evict_in_place_kernel(PagedEvictArgs a) {
  const PagedView &c = a.c;
  const int head = blockIdx.x % c.n_kv, b = (blockIdx.x / c.n_kv) % c.batch, layer = blockIdx.x / c.n_kv / c.batch;
  const int n = a.lens[b];
  if (n <= a.budget || n > a.max_len) return;
  const int32_t *kept = a.kept + (size_t)blockIdx.x * a.budget;
  const int esz = c.bf16 ? 2 : 4, slices = c.dh * esz / 16 / SLICE;
  const int part = blockIdx.y;  // slices of k, slices of v, weights
  const int64_t base = (layer * c.layer_stride + head * c.head_stride) * esz;
  if (part < 2 * slices)
    evict_in_place<false, SLICE>(a, b, layer, head, kept, a.budget, part < slices ? c.k : c.v, base, esz, part % slices);
  else
    evict_in_place<true, SLICE>(a, b, layer, head, kept, a.budget, nullptr, 0, 0, 0);
}

__global__ __launch_bounds__(kMoveThreads) void paged_evict_gather_kernel(PagedEvictArgs a) {
  const PagedView &c = a.c;
  const int head = blockIdx.x % c.n_kv, b = (blockIdx.x / c.n_kv) % c.batch, layer = blockIdx.x / c.n_kv / c.batch;
  const int n = a.lens[b], tid = threadIdx.x;
  if (n < 0 || n > a.max_len) return;
  const int count = min(n, a.budget), r0 = blockIdx.y * kEvictMoveRows;
  if (r0 >= count) return;
  const int rows = min(kEvictMoveRows, count - r0);
  const int32_t *kept = a.kept + (size_t)blockIdx.x * a.budget;
  __shared__ int64_t from[kEvictMoveRows], to[kEvictMoveRows];
  if (tid < rows) {
    const int s = kept[r0 + tid], i = r0 + tid;
    const int pf = page_of(c, b, s), pt = a.new_table[(int64_t)b * a.new_pages + (i >> c.page_shift)];
    from[tid] = -1;
    if (pf >= 0 && (unsigned)pt < (unsigned)c.n_pages) {
      from[tid] = slot_offset(c, pf, s);
      to[tid] = slot_offset(c, pt, i);
      c.weights[weight_offset(c, layer, pt, head, i)] = c.weights[weight_offset(c, layer, pf, head, s)];
    } else {
      raise_error(a.err, DEV_BAD_PAGE);
    }
  }
  __syncthreads();
  const int esz = c.bf16 ? 2 : 4, shift = __builtin_ctz(c.dh * esz / 16), half = rows << shift;
  const int64_t base = (layer * c.layer_stride + head * c.head_stride) * esz;
  for (int it = tid; it < 2 * half; it += kMoveThreads) {
    const int rem = it < half ? it : it - half, d = rem >> shift;
    if (from[d] < 0) continue;
    char *p = (it < half ? c.k : c.v) + base + (rem & ((1 << shift) - 1)) * 16;
    *(u32x4 *)(p + to[d] * esz) = *(const u32x4 *)(p + from[d] * esz);
  }
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
template <typename T, int DH>
static void append_of(const PagedAppendArgs &a, hipStream_t st) {
  constexpr int GROUPS = kAppendThreads / (DH / 8);
  const int heads = a.nq + 2 * a.c.n_kv;
  const int ys = a.tokens < 1024 ? min((heads + GROUPS - 1) / GROUPS, 16383) : 1;  // (a grid holds 1024 x 16383 workgroups of 256)
  hipLaunchKernelGGL((paged_append_kernel<T, DH>), dim3(a.tokens + 1, ys), dim3(kAppendThreads), 0, st, a);
}
void launch_paged_append(const PagedAppendArgs &a, hipStream_t st) {
  if (a.c.bf16) a.c.dh == 128 ? append_of<bf16_t, 128>(a, st) : append_of<bf16_t, 64>(a, st);
  else a.c.dh == 128 ? append_of<float, 128>(a, st) : append_of<float, 64>(a, st);
}

void launch_paged_commit(const PagedView &c, int n_nodes, int max_depth, const int32_t *ctx_lens, const int32_t *accept_len,
                         const int32_t *accepted, int32_t *new_lens, int32_t *err, hipStream_t st) {
  const dim3 grid(c.n_layers * c.batch * c.n_kv), block(kMoveThreads);
  const int items = 2 * max_depth * (c.dh * (c.bf16 ? 2 : 4) / 16);
  if (items <= 4 * kMoveThreads)
    hipLaunchKernelGGL(paged_commit_kernel<4>, grid, block, 0, st, c, n_nodes, max_depth, ctx_lens, accept_len, accepted, new_lens, err);
  else
    hipLaunchKernelGGL(paged_commit_kernel<16>, grid, block, 0, st, c, n_nodes, max_depth, ctx_lens, accept_len, accepted, new_lens, err);
}

void launch_paged_evict(const PagedEvictArgs &a, hipStream_t st) {
  const int heads = a.c.n_layers * a.c.batch * a.c.n_kv;
  const bool tiny = a.c.page_shift < 2;
  const int slices = (a.max_len + kEvictSlice - 1) / kEvictSlice;
  if (slices == 1) {
    if (tiny) hipLaunchKernelGGL(paged_evict_select_kernel<true>, dim3(heads), dim3(kSelThreads), 0, st, a);
    else hipLaunchKernelGGL(paged_evict_select_kernel<false>, dim3(heads), dim3(kSelThreads), 0, st, a);
  } else {
    for (int phase = 0; phase < 4; ++phase) {
      if (tiny) hipLaunchKernelGGL(paged_evict_phase_kernel<true>, dim3(heads * slices), dim3(kSelThreads), 0, st, a, phase, slices);
      else hipLaunchKernelGGL(paged_evict_phase_kernel<false>, dim3(heads * slices), dim3(kSelThreads), 0, st, a, phase, slices);
    }
  }
  if (a.new_table) {
    hipLaunchKernelGGL(paged_evict_gather_kernel, dim3(heads, (min(a.budget, a.max_len) + kEvictMoveRows - 1) / kEvictMoveRows),
                       dim3(kMoveThreads), 0, st, a);
  } else {
    const int wide = a.c.dh * (a.c.bf16 ? 2 : 4) / 64, parts = evict_in_place_parts(a.c.dh, a.c.bf16, heads);
    if (parts == 4 * wide + 1) hipLaunchKernelGGL(paged_evict_in_place_kernel<2>, dim3(heads, parts), dim3(kMoveThreads), 0, st, a);
    else hipLaunchKernelGGL(paged_evict_in_place_kernel<4>, dim3(heads, parts), dim3(kMoveThreads), 0, st, a);
  }
}

}  // namespace dk
