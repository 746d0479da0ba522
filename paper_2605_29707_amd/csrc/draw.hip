// Drawing a token of rows of logits under temperature, top-k, top-p and min-p.
//
// In the order (value desc, id asc), with e = exp((l - max) / T): every filter keeps a prefix,
// and the token is where the running sum of e passes u times the kept prefix's sum.  Sums are of
// whole numbers, e in units of 2^-44, so that their order does not matter and a prefix is told
// by its sum.  e comes from 64-bit arithmetic: in 32 bits the errors of a flat row's sums are as
// wide as its tokens' weights in one row of a few hundred, and the token another one.
//
// Launches:
//   groups  as for the top entries (logits.hip)
//   first   a workgroup a row: the first C entries (select.h), C = top_k where that is at most 1024,
//           or 64; the filters and the draw in their running sums.  Nearly all rows of a model
//           end here.
//   whole   the other rows (flat ones, whose kept entries or draw lie behind the first 64), several
//           workgroups a row: sums of e by bins of log2 e, in LDS, then added in memory; the last
//           workgroup to finish a row finds the bin where a running sum passes its target, and the entry
//           among the bin's, sorted, or first by parts of the bin while they are too many.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "select.h"

namespace dk {

constexpr int kWeightBits = 44;                       // a weight of 1 is 2^44; a row's sum stays below 2^63
static_assert(kRowsMaxVocab <= 1 << 19, "sums of weights must fit 63 bits");
constexpr int kBinsLog = 6;                           // bins of 1/64 in log2 of the weight
constexpr int kBins = (kWeightBits + 2) << kBinsLog;  // a weight past them rounds to 0
static_assert(sizeof(DrawSums::mass) == kBins * 8, "the bins in memory");
constexpr int kSplitLog = 11;                         // parts a bin is split into, level by level
constexpr int kSplit = 1 << kSplitLog;
constexpr int kFirst = 64;                            // entries looked at first where top_k is off
constexpr int kWholeThreads = 1024;
constexpr int kWholeWaves = kWholeThreads / 64;
constexpr double kOne = (double)(1ull << kWeightBits);

// round(2^44 2^-x), x >= 0.  2^f on [-1/2, 1/2] by its Taylor sum to the 11th power, whose next
// term is 2^-50; the rest is exact or rounded to 53 bits.
DEVI unsigned long long weight_of(double x) {
  if (!(x < kWeightBits + 1.5)) return 0ull;
  const double n = rint(x), t = (n - x) * 0.69314718055994530942;
  double p = 1.0 / 39916800.0;
  p = fma(p, t, 1.0 / 3628800.0);
  p = fma(p, t, 1.0 / 362880.0);
  p = fma(p, t, 1.0 / 40320.0);
  p = fma(p, t, 1.0 / 5040.0);
  p = fma(p, t, 1.0 / 720.0);
  p = fma(p, t, 1.0 / 120.0);
  p = fma(p, t, 1.0 / 24.0);
  p = fma(p, t, 1.0 / 6.0);
  p = fma(p, t, 0.5);
  p = fma(p, t, 1.0);
  p = fma(p, t, 1.0);
  const double scale = __longlong_as_double((unsigned long long)(1023 + kWeightBits - (int)n) << 52);
  // adding 2^52 rounds to a whole number in the low bits
  return (unsigned long long)__double_as_longlong(fma(p, scale, 4503599627370496.0)) & ((1ull << 52) - 1);
}

// A row's parameters; T = 0 is top_k = 1 at T = 1.
struct DrawRow {
  float T, u, top_p, min_p;
  int top_k;
  bool ok, has_k, use_p, use_m;
  float m;     // the row's maximum
  double cd;   // log2(e) / T
  float cf;    // the same in units of the bins' parts
  double min_d;  // max - l up to this stays under min-p

  DEVI void read(const RowsArgs &a, const SampleArgs &p, int row) {
    T = a.temps ? a.temps[row] : 1.f;
    u = p.uniforms[row];
    top_p = p.top_p ? p.top_p[row] : 1.f;
    min_p = p.min_p ? p.min_p[row] : 0.f;
    top_k = p.top_k ? p.top_k[row] : 0;
    ok = T >= 0.f && T < INFINITY && u >= 0.f && u < 1.f && top_p >= 0.f && top_p <= 1.f && min_p >= 0.f && min_p <= 1.f;
    if (T == 0.f) {
      top_k = 1;
      T = 1.f;
    }
    has_k = top_k > 0 && top_k < a.V;
    use_p = top_p < 1.f;
    use_m = min_p > 0.f;
  }
  DEVI void set_max(float max) {
    m = max;
    cd = 1.44269504088896340736 / (double)T;
    cf = fminf((float)(cd * (double)(1 << (kBinsLog + kSplitLog))), 1e30f);
    min_d = use_m ? -log((double)min_p) * (double)T : INFINITY;
  }
  // of a value that is no NaN; logits of +inf have all the weight
  DEVI unsigned long long weight(float v) const {
    if (m == INFINITY) return v == m ? 1ull << kWeightBits : 0ull;
    return weight_of(((double)m - (double)v) * cd);
  }
  DEVI bool stays(float v) const { return v == m || (double)m - (double)v <= min_d; }
  DEVI float logprob(float v, unsigned long long total) const {
    return (float)((v == m ? 0.0 : ((double)v - (double)m) / (double)T) - log((double)total / kOne));
  }
  DEVI void finish(const SampleArgs &p, int row, int token, float lp) const {
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = lp;
  }
};

// ---------------------------------------------------------------------------
// the first entries
// ---------------------------------------------------------------------------
template <typename LT, int NR>
__global__ __launch_bounds__(kSelThreads) void draw_first_kernel(RowsArgs a, SampleArgs p) {
  __shared__ SelShared sh;
  __shared__ unsigned long long run[kTopMax];  // running sums of the first C
  __shared__ unsigned long long redu[kSelWaves];
  __shared__ int first[4];
  constexpr int kPer = kTopMax / kSelThreads;
  const int row = blockIdx.x, tid = threadIdx.x;
  DrawRow d;
  d.read(a, p, row);
  if (tid == 0) p.state[row] = 0;
  if (!d.ok) {
    if (tid == 0) {
      raise_error(a.err, DEV_BAD_PARAM);
      d.finish(p, row, -1, NAN);
    }
    return;
  }
  const int C = min(a.V, d.has_k && d.top_k <= kTopMax ? d.top_k : kFirst);
  float rm = 0.f;
  double rs = 0.0;
  select_top<LT, NR>((const LT *)a.logits + (size_t)row * a.ld, a.groups + (size_t)row * a.G, a.V, a.G, C,
                     row_scale(d.T), sh, rm, rs);
  d.set_max(entry_value(sh.list[0]));
  if (d.m == -INFINITY) {  // nothing to draw from
    if (tid == 0) d.finish(p, row, -1, -INFINITY);
    return;
  }
  // entry i is of thread i / per; with the running sums, the first of them that ...
  const int per = C <= kSelThreads ? 1 : kPer;
  float v[kPer];
  unsigned long long w[kPer], sum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int i = tid * per + j;
    const bool on = j < per && i < C;
    v[j] = on ? entry_value(sh.list[i]) : -INFINITY;
    w[j] = on ? d.weight(v[j]) : 0ull;
    sum += w[j];
  }
  if (tid < 4) first[tid] = C;
  unsigned long long r = block_scan<kSelWaves>(sum, redu) - sum;
  auto each = [&](auto f) {  // f(entry, its value, weight)
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (j < per && tid * per + j < C) f(tid * per + j, v[j], w[j]);
  };
  each([&](int i, float x, unsigned long long wi) {
    run[i] = r += wi;
    if (wi == 0ull) atomicMin(&first[0], i);       // ... has no weight
    if (!d.stays(x)) atomicMin(&first[1], i);      // ... does not stay under min-p
  });
  __syncthreads();
  const unsigned long long sum_c = run[C - 1], kUnknown = ~0ull;
  const int weighty = first[0], n_m = first[1];    // C: all of them
  const bool all = C == a.V || weighty < C;        // no weight lies behind the first C
  // the whole row's sum: of the first C exactly, of the rest from the groups' sums
  unsigned long long whole = sum_c;
  if (!all && rs != 0.0) whole += (unsigned long long)(rs * exp2(((double)rm - (double)d.m) * d.cd) * kOne);
  unsigned long long total = all ? sum_c : kUnknown;  // the kept prefix's sum
  bool decided = true;
  if (d.has_k && d.top_k <= C) whole = total = min(total, run[d.top_k - 1]);
  if (d.use_p) {
    if (!d.has_k || d.top_k <= C || all) {
      const unsigned long long want = (unsigned long long)ceil((double)d.top_p * (double)whole);
      each([&](int i, float, unsigned long long) {
        if (run[i] >= want) atomicMin(&first[2], i);
      });
    } else {
      decided = false;  // the sum of the first top_k is not known
    }
    __syncthreads();
    if (first[2] < C) total = min(total, run[first[2]]);
  }
  if (d.use_m && n_m < C) total = min(total, run[n_m - 1]);
  // no filter ends within the first C: without any, the draw may still fall there
  if (total == kUnknown) {
    total = whole;
    if (d.use_p || d.use_m || d.has_k) decided = false;
  }
  if (decided) {
    const unsigned long long target = (unsigned long long)floor((double)d.u * (double)total);
    each([&](int i, float, unsigned long long) {
      if (run[i] > target) atomicMin(&first[3], i);
    });
    __syncthreads();
    const int i = first[3];
    if (i < C) {
      if (tid == 0) {
        const unsigned long long key = sh.list[i];
        d.finish(p, row, (int)entry_id(key), d.logprob(entry_value(key), total));
      }
      return;
    }
  }
  // for the next launch: the row's maximum, and its sums cleared
  if (tid == 0) p.state[row] = order_key(d.m);
  if (p.slices > 1) {
    uint32_t *g = (uint32_t *)(p.sums + row);
    for (int i = tid; i < (int)(sizeof(DrawSums) / 4); i += kSelThreads) g[i] = 0;
  }
}

// ---------------------------------------------------------------------------
// the whole row
// ---------------------------------------------------------------------------
struct WholeShared {
  union {
    alignas(16) unsigned long long list[kListMax + 2];
    struct {                     // a bin by parts
      unsigned long long mass[kSplit];
      uint32_t count[kSplit];
    } part;
  };
  unsigned long long mass[kBins];  // the row by bins
  uint32_t count[kBins];           // (where top-k is on)
  unsigned long long redu[2][kWholeWaves];
  unsigned long long hit[3];
  int hit_i, n, last;
};
static_assert(sizeof(WholeShared) <= 65536, "two workgroups a CU, static LDS");

// f(value, id) for the values of ids [v0, v1); the next 16-byte loads are on their way meanwhile.
// NaN comes as -inf.
template <typename LT, typename F>
DEVI void each_of_row(const LT *lr, uint32_t V, uint32_t v0, uint32_t v1, F f) {
  constexpr int N = RowVec<LT>::N, U = 2;
  constexpr uint32_t step = kWholeThreads * N;
  u32x4 x[U], y[U];
  auto load = [&](u32x4 (&z)[U], uint32_t c0) {
    if (c0 + U * step <= V) {  // uniform
#pragma unroll
      for (int q = 0; q < U; ++q) z[q] = row_load(lr + c0 + q * step + threadIdx.x * N);
    } else {
#pragma unroll
      for (int q = 0; q < U; ++q) z[q] = row_load_end(lr, c0 + q * step + threadIdx.x * N, V);
    }
  };
  load(x, v0);
#pragma unroll 1
  for (uint32_t c0 = v0; c0 < v1; c0 += U * step) {
    if (c0 + U * step < v1) load(y, c0 + U * step);
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const uint32_t id = c0 + q * step + threadIdx.x * N;
      if (id < v1) {
#pragma unroll
        for (int e = 0; e < N; ++e) f(fmaxf(RowVec<LT>::get(x[q], e), -INFINITY), id + e);
      }
    }
#pragma unroll
    for (int q = 0; q < U; ++q) x[q] = y[q];
  }
}

// The order in digits, each ascending: the bin and its part (of the distance to the
// maximum), the value's key, the id; `level` says which digit, `near` whether those before it agree.
struct Digits {
  uint32_t y, k, id;
};
// the distance in parts of a bin, not above what 24 bits hold (max = +inf: NaN for its equals, which are at 0)
DEVI float distance(const DrawRow &s, float v) { return fminf(fmaxf((s.m - v) * s.cf, 0.f), 1.6e7f); }
constexpr float kFar = (float)(kBins << kSplitLog);
DEVI bool near(const Digits &a, const Digits &b, int level) {
  const uint32_t my = level == 0 ? 0u : level == 1 ? ~2047u : ~0u;
  const uint32_t mk = level < 3 ? 0u : level == 3 ? ~0u << 21 : level == 4 ? ~0u << 10 : ~0u;
  const uint32_t mi = level < 6 ? 0u : level == 6 ? ~2047u : ~0u;
  return (((a.y ^ b.y) & my) | ((a.k ^ b.k) & mk) | ((a.id ^ b.id) & mi)) == 0;
}
DEVI uint32_t digit_of(const Digits &a, int level) {
  switch (level) {
    case 1: return a.y & 2047;
    case 2: return a.k >> 21;
    case 3: return a.k >> 10 & 2047;
    case 4: return a.k & 1023;
    case 5: return a.id >> 11;
    default: return a.id & 2047;
  }
}
DEVI void set_digit(Digits &a, int level, uint32_t d) {
  switch (level) {
    case 0: a.y = d << 11; break;
    case 1: a.y |= d; break;
    case 2: a.k = d << 21; break;
    case 3: a.k |= d << 10; break;
    case 4: a.k |= d; break;
    case 5: a.id = d << 11; break;
    default: a.id |= d; break;
  }
}

// Where a running sum in the order ends: the sum and the last entry.
struct Prefix {
  unsigned long long mass, key;
};

// The shortest prefix of the whole row's order whose count (by_count) or sum is above `target`; one exists.
template <typename LT>
DEVI Prefix find_in_row(const LT *lr, uint32_t V, const DrawRow &s, bool by_count, unsigned long long target,
                        WholeShared &sh) {
  const int tid = threadIdx.x;
  Digits at = {0, 0, 0};
  unsigned long long n0 = 0, m0 = 0;  // before the part in work
  // f(value, its digits) of the entries with a weight that agree with `at` before `level`
  auto each_near = [&](int level, auto f) {
    const float from = (float)at.y, to = (float)(at.y + (level == 1 ? kSplit : 1));
    each_of_row(lr, V, 0, V, [&](float v, uint32_t id) {
      const float y = distance(s, v);
      if (y >= from && y < to) {
        const Digits d = {(uint32_t)y, ~order_key(v), id};
        if (near(d, at, level)) f(v, d);
      }
    });
  };
  for (int level = 0;; ++level) {
    unsigned long long *mass = level == 0 ? sh.mass : sh.part.mass;
    uint32_t *count = level == 0 ? sh.count : sh.part.count;
    const int bins = level == 0 ? kBins : kSplit;
    if (level > 0) {
      for (int i = tid; i < kSplit; i += kWholeThreads) {
        mass[i] = 0;
        count[i] = 0;
      }
      __syncthreads();
      each_near(level, [&](float v, const Digits &d) {
        const unsigned long long w = s.weight(v);
        if (w) {
          atomicAdd(&mass[digit_of(d, level)], w);
          atomicAdd(&count[digit_of(d, level)], 1u);
        }
      });
      __syncthreads();
    }
    // the digit in which the target is passed: kPer of them a thread
    constexpr int kPer = (kBins + kWholeThreads - 1) / kWholeThreads;
    unsigned long long pm = 0, pn = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = tid * kPer + j;
      if (b < bins) {
        pm += mass[b];
        if (by_count) pn += count[b];
      }
    }
    unsigned long long em = block_scan<kWholeWaves>(pm, sh.redu[0]) - pm + m0, en = n0;
    if (by_count) en += block_scan<kWholeWaves>(pn, sh.redu[1]) - pn;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = tid * kPer + j;
      if (b < bins) {
        const unsigned long long a0 = by_count ? en : em, a1 = a0 + (by_count ? count[b] : mass[b]);
        if (a0 <= target && target < a1) {  // one bin of all
          sh.hit[0] = en;
          sh.hit[1] = em;
          sh.hit_i = b;
        }
        em += mass[b];
        if (by_count) en += count[b];
      }
    }
    if (tid == 0) sh.n = 0;
    __syncthreads();
    n0 = sh.hit[0];
    m0 = sh.hit[1];
    set_digit(at, level, sh.hit_i);
    __syncthreads();
    // its entries, sorted, with their running sums
    each_near(level + 1, [&](float v, const Digits &d) {
      if (s.weight(v)) {
        const int to = atomicAdd(&sh.n, 1);
        if (to < kListMax) sh.list[to] = entry_key(v, d.id);
      }
    });
    __syncthreads();
    const int n = sh.n;
    if (n > kListMax) continue;  // (at the last level a part is one entry)
    sort_list<kWholeWaves>(n, sh.list);
    constexpr int kTwo = kListMax / kWholeThreads;
    unsigned long long w[kTwo], ws = 0;
#pragma unroll
    for (int j = 0; j < kTwo; ++j) {
      const int i = tid * kTwo + j;
      w[j] = i < n ? s.weight(entry_value(sh.list[i])) : 0ull;
      ws += w[j];
    }
    unsigned long long e = block_scan<kWholeWaves>(ws, sh.redu[0]) - ws + m0;
#pragma unroll
    for (int j = 0; j < kTwo; ++j) {
      const int i = tid * kTwo + j;
      if (i < n) {
        const unsigned long long a0 = by_count ? n0 + i : e, a1 = by_count ? a0 + 1 : e + w[j];
        if (a0 <= target && target < a1) {
          sh.hit[0] = e + w[j];
          sh.hit[1] = sh.list[i];
        }
        e += w[j];
      }
    }
    __syncthreads();
    const Prefix p = {sh.hit[0], sh.hit[1]};
    __syncthreads();
    return p;
  }
}

template <typename LT>
__global__ __launch_bounds__(kWholeThreads) void draw_whole_kernel(RowsArgs a, SampleArgs p) {
  __shared__ WholeShared sh;
  constexpr int N = RowVec<LT>::N;
  const int row = blockIdx.x / p.slices, slice = blockIdx.x % p.slices, tid = threadIdx.x;
  const uint32_t state = p.state[row];
  if (state == 0) return;  // the first entries have decided
  const LT *lr = (const LT *)a.logits + (size_t)row * a.ld;
  DrawRow d;
  d.read(a, p, row);
  d.set_max(order_key_value(state));
  for (int i = tid; i < kBins; i += kWholeThreads) {
    sh.mass[i] = 0;
    sh.count[i] = 0;
  }
  __syncthreads();
  unsigned long long mm = 0;  // the sum that stays under min-p
  const uint32_t len = ((uint32_t)a.V / p.slices / N + 1) * N, v0 = slice * len, v1 = min((uint32_t)a.V, v0 + len);
  if (v0 < v1)
    each_of_row(lr, a.V, v0, v1, [&](float x, uint32_t) {
      const float y = distance(d, x);
      if (y < kFar) {
        const unsigned long long w = d.weight(x);
        if (w) {
          const int b = (int)y >> kSplitLog;
          atomicAdd(&sh.mass[b], w);
          if (d.has_k) atomicAdd(&sh.count[b], 1u);
          if (d.use_m && d.stays(x)) mm += w;
        }
      }
    });
  __syncthreads();
  mm = block_reduce_sum<kWholeWaves>(mm, sh.redu[0]);
  if (p.slices > 1) {
    // to memory; the last workgroup to add its own takes all of them up again
    DrawSums *g = p.sums + row;
    for (int i = tid; i < kBins; i += kWholeThreads) {
      if (sh.mass[i]) atomicAdd(&g->mass[i], sh.mass[i]);
      if (d.has_k && sh.count[i]) atomicAdd(&g->count[i], sh.count[i]);
    }
    if (tid == 0 && mm) atomicAdd(&g->stays, mm);
    __threadfence();
    __syncthreads();
    if (tid == 0) sh.last = atomicAdd(&g->done, 1u) == (unsigned)p.slices - 1;
    __syncthreads();
    if (!sh.last) return;
    __threadfence();
    for (int i = tid; i < kBins; i += kWholeThreads) {
      sh.mass[i] = __hip_atomic_load(&g->mass[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (d.has_k) sh.count[i] = __hip_atomic_load(&g->count[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    mm = __hip_atomic_load(&g->stays, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
  }
  unsigned long long tn = 0, tm = 0;
  for (int i = tid; i < kBins; i += kWholeThreads) {
    tn += sh.count[i];
    tm += sh.mass[i];
  }
  const unsigned long long entries = block_reduce_sum<kWholeWaves>(tn, sh.redu[1]);
  unsigned long long total = block_reduce_sum<kWholeWaves>(tm, sh.redu[0]);
  __syncthreads();
  // top-k, top-p, then (the shorter of it and min-p kept) the draw
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {
    unsigned long long target;
    if (step == 0) {
      if (!d.has_k || (unsigned long long)d.top_k >= entries) continue;
      target = d.top_k - 1;
    } else if (step == 1) {
      if (!d.use_p) continue;
      target = (unsigned long long)ceil((double)d.top_p * (double)total);
      target = target == 0 ? 0 : min(target, total) - 1;
    } else {
      if (d.use_m) total = min(total, mm);
      target = min((unsigned long long)floor((double)d.u * (double)total), total - 1);
    }
    const Prefix f = find_in_row(lr, a.V, d, step == 0, target, sh);
    if (step < 2) total = f.mass;
    else if (tid == 0) d.finish(p, row, (int)entry_id(f.key), d.logprob(entry_value(f.key), total));
  }
}

// Workgroups a row of the last launch: for few rows as many as cut a row of 128K ids to 8K each (64
// rows of 128256 fp32 logits, the flat ones 120 us with one workgroup), for many enough to fill the chip.
static int draw_slices(int rows, int V) { return std::max(1, std::min({16, 1024 / rows, V / 8192})); }

// [error word and groups][state][sums, where a row has several workgroups]
struct DrawLayout {
  size_t state, sums, bytes;
};
static DrawLayout draw_layout(int rows, int V) {
  DrawLayout l;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  l.state = up(rows_ws_bytes(rows, V));
  l.sums = up(l.state + (size_t)rows * 4);
  l.bytes = l.sums + (draw_slices(rows, V) > 1 ? (size_t)rows * sizeof(DrawSums) : 0);
  return l;
}
size_t draw_ws_bytes(int rows, int V) { return draw_layout(rows, V).bytes; }

void launch_sample_logits(RowsArgs a, bool bf16, SampleArgs p, void *ws, hipStream_t st) {
  const DrawLayout l = draw_layout(a.rows, a.V);
  p.state = (uint32_t *)((char *)ws + l.state);
  p.sums = (DrawSums *)((char *)ws + l.sums);
  p.slices = draw_slices(a.rows, a.V);
  a = launch_row_groups(a, bf16, ws, st);
  auto go = [&](auto t) {
    using LT = decltype(t);
    by_vocab(a.V, [&](auto nr) {
      constexpr int NR = decltype(nr)::value;
      hipLaunchKernelGGL((draw_first_kernel<LT, NR>), dim3(a.rows), dim3(kSelThreads), 0, st, a, p);
    });
    hipLaunchKernelGGL(draw_whole_kernel<LT>, dim3(a.rows * p.slices), dim3(kWholeThreads), 0, st, a, p);
  };
  if (bf16) go(bf16_t{});
  else go(0.f);
}

}  // namespace dk
