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
//           or 64; the filters and the draw in their running sums.  A row ends here if they all fall among
//           those, clear of what the sum of the others may be off by, since that is of single-precision
//           exponentials.  Bound by the chain of its steps (one row of 151936 11 us, 512 19).
//   whole   the other rows (flat ones, whose kept entries or draw lie behind the first 64), several
//           workgroups a row: sums of e by bins of log2 e, in LDS, then added in memory; the last
//           workgroup to finish a row finds the bin where a running sum passes its target, and the entry
//           among the bin's, sorted, or first by parts of their range while they are too many.  Bound by the
//           polynomials and LDS atomics of the sums, then by one CU's pass over a row for each border (64 of
//           512 rows of 151936 bf16 logits flat: 67 us, 21 of them for the sums, 6 to join them, 14 a pass
//           and 6 for the list it leaves).
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
constexpr int kSplitLog = 11;                         // parts of a bin
constexpr int kSplit = 1 << kSplitLog;
constexpr int kFirst = 64;                            // entries looked at first where top_k is off
constexpr int kWholeThreads = 1024;
constexpr int kWholeWaves = kWholeThreads / 64;
constexpr double kOne = (double)(1ull << kWeightBits);
// What a row's sum behind its first entries may be off by where it comes from single-precision exponentials, of itself.
// In units of 2^-24: an exponent is off by 2.3 of itself (the factor, the difference, the product), and the
// weighted mean of the exponents is log2 V < 18.4 at most, so 29 of the sum; two exponentials 4; sums of 10 in a group, of
// 20 groups and of 132 values in a thread 162.  Together 195, below 256.
constexpr double kRestOff = 0x1p-16;

// round(2^44 2^-x) for 0 <= x < 2^10.  2^f on [-1/2, 1/2] as 1 + f q(f), q interpolating (2^f - 1) / f at the
// zeros of the Chebyshev polynomial of degree 8: 2^-38.8 of the value off at most, and exactly 1 at 0.
// The whole part of x is rounded off by adding 1.5 2^52, which leaves it in the low word.
DEVI unsigned long long weight_of(double x) {
  const double big = 6755399441055744.0, r = x + big, f = (r - big) - x;
  const int n = (int)(uint32_t)__double_as_longlong(r);
  double p = 1.325080551750225e-06;
  p = fma(p, f, 1.5303700711365693e-05);
  p = fma(p, f, 0.00015403475186530786);
  p = fma(p, f, 0.0013333478473685416);
  p = fma(p, f, 0.00961812913523614);
  p = fma(p, f, 0.055504109063258665);
  p = fma(p, f, 0.24022650695888503);
  p = fma(p, f, 0.6931471805568324);
  p = fma(p, f, 1.0);
  const double scale = __hiloint2double((1023 + kWeightBits - n) << 20, 0);
  // adding 2^52 rounds to a whole number in the low bits
  return (unsigned long long)__double_as_longlong(fma(p, scale, 4503599627370496.0)) & ((1ull << 52) - 1);
}

// a value that is the same in every lane, in scalar registers
DEVI uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
DEVI float scalar(float x) { return __uint_as_float(scalar(__float_as_uint(x))); }
DEVI double scalar(double x) {
  return __hiloint2double((int)scalar((uint32_t)__double2hiint(x)), (int)scalar((uint32_t)__double2loint(x)));
}
DEVI unsigned long long scalar(unsigned long long x) {
  return (unsigned long long)scalar((uint32_t)(x >> 32)) << 32 | scalar((uint32_t)x);
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
    ok = (T == 0.f || row_temperature_ok(T)) && u >= 0.f && u < 1.f && top_p >= 0.f && top_p <= 1.f && min_p >= 0.f && min_p <= 1.f;
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
    cd = scalar(1.44269504088896340736 / (double)T);
    cf = scalar((float)(cd * (double)(1 << (kBinsLog + kSplitLog))));
    min_d = scalar(use_m ? -log((double)min_p) * (double)T : (double)INFINITY);
  }
  // of a value that is no NaN; logits of +inf have all the weight
  DEVI unsigned long long weight(float v) const {
    if (m == INFINITY) return v == m ? 1ull << kWeightBits : 0ull;
    const double x = ((double)m - (double)v) * cd;
    return x < kWeightBits + 2 ? weight_of(x) : 0ull;
  }
  // above every weight of a bin
  DEVI unsigned long long weight_at(int bin) const { return weight_of((double)bin / (1 << kBinsLog)) + (1ull << (kWeightBits - 20)); }
  // whether a bin of this sum may hold few enough entries for a list
  DEVI bool few(unsigned long long mass, int bin) const { return mass <= weight_at(bin) * (kListMax * 15 / 16); }
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
  __shared__ int first[6];
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
                     row_scale(d.T), !d.has_k || d.top_k > C, sh, rm, rs);
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
  if (tid < 6) first[tid] = C;
  unsigned long long r = block_scan<kSelWaves>(sum, redu) - sum;
  // the first entry that on(entry, its value, weight) takes, by one lane of each wave (entries are in the lanes' order)
  auto first_of = [&](int slot, auto on) {
    int i = C;
#pragma unroll
    for (int j = kPer - 1; j >= 0; --j)
      if (j < per && tid * per + j < C && on(tid * per + j, v[j], w[j])) i = tid * per + j;
    const unsigned long long mk = __ballot(i < C);
    if (mk && (tid & 63) == __ffsll(mk) - 1) atomicMin(&first[slot], i);
  };
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (j < per && tid * per + j < C) run[tid * per + j] = r += w[j];
  first_of(0, [&](int, float, unsigned long long wi) { return wi == 0ull; });   // ... has no weight
  first_of(1, [&](int, float x, unsigned long long) { return !d.stays(x); });   // ... does not stay under min-p
  __syncthreads();
  const unsigned long long sum_c = run[C - 1], kUnknown = ~0ull;
  const int weighty = first[0], n_m = first[1];    // C: all of them
  const bool all = C == a.V || weighty < C;        // no weight lies behind the first C
  // The whole row's sum, of the first C as the next launch has it, of the rest from the groups' sums: that launch's
  // is within `off` of it, half a unit an entry for the rounding of its weights.  A border or a draw that falls among
  // the first C decides here where it is the same entry for the least and the most that the sum can be.
  unsigned long long whole = sum_c, off = 0;
  if (!all && rs != 0.0) {
    const double rest = rs * (rm == d.m ? 1.0 : exp2(((double)rm - (double)d.m) * d.cd)) * kOne;
    whole += (unsigned long long)rest;
    off = (unsigned long long)(rest * kRestOff) + (unsigned)a.V;
  }
  unsigned long long least = all ? sum_c : kUnknown, most = least;  // the kept prefix's sum
  bool decided = true;
  if (d.has_k && d.top_k <= C) {
    whole = least = most = min(least, run[d.top_k - 1]);
    off = 0;
  }
  if (d.use_p) {
    if (!d.has_k || d.top_k <= C || all) {
      auto border = [&](int slot, unsigned long long sum) {
        const unsigned long long want = (unsigned long long)ceil((double)d.top_p * (double)sum);
        first_of(slot, [&](int i, float, unsigned long long) { return run[i] >= want; });
      };
      border(2, whole - off);
      if (off) border(4, whole + off);
    } else {
      decided = false;  // the sum of the first top_k is not known
    }
    __syncthreads();
    const int p0 = first[2], p1 = off ? first[4] : p0;
    if (p0 < C) least = min(least, run[p0]);
    if (p1 < C) most = min(most, run[p1]);
  }
  if (d.use_m && n_m < C) {
    least = min(least, run[n_m - 1]);
    most = min(most, run[n_m - 1]);
  }
  if (least != most) decided = false;
  // no filter ends within the first C: without any, the draw may still fall there
  unsigned long long total = least;
  if (total == kUnknown) {
    total = whole;
    least = whole - off;
    most = whole + off;
    if (d.use_p || d.use_m || d.has_k) decided = false;
  }
  if (decided) {
    auto drawn = [&](int slot, unsigned long long sum) {
      const unsigned long long target = (unsigned long long)floor((double)d.u * (double)sum);
      first_of(slot, [&](int i, float, unsigned long long) { return run[i] > target; });
    };
    drawn(3, least);
    if (least != most) drawn(5, most);
    __syncthreads();
    const int i = first[3];
    if (i < C && (least == most || i == first[5])) {
      if (tid == 0) {
        const unsigned long long key = sh.list[i];
        d.finish(p, row, (int)entry_id(key), d.logprob(entry_value(key), total));
      }
      return;
    }
  }
  // for the next launch
  if (tid == 0) {
    p.state[row] = order_key(d.m);
    p.done[row] = 0;
  }
}

// ---------------------------------------------------------------------------
// the whole row
// ---------------------------------------------------------------------------
struct WholeShared {
  unsigned long long mass[kBins];  // the row by bins
  union {
    struct {
      alignas(16) unsigned long long list[kListMax + 2];
      union {
        alignas(16) unsigned long long draw[kListMax + 2];  // a second list, of the draw's bin
        uint32_t count[kBins];                              // (for top-k, which comes before the draw)
      };
    };
    struct {                       // a bin by parts
      unsigned long long mass[kSplit];
      uint32_t count[kSplit];
    } part;
  };
  unsigned long long redu[2][kWholeWaves];
  unsigned long long hit[2];
  uint32_t sort[kWholeThreads], red[kWholeWaves];  // of sort_list
  int hit_i, last, n[2], wave_n[2][kWholeWaves];
};
static_assert(sizeof(WholeShared) <= 65536, "static LDS");
constexpr int kBinsPer = (kBins + kWholeThreads - 1) / kWholeThreads;  // bins a thread
constexpr int kSeg = 2 * kListMax / kWholeWaves;                      // a wave's part of a list while it is ids

// f(16 bytes of values, first id) for the ids [v0, v1) of a row of at least a vector; -inf follows its last
// value.  The next U loads are on their way meanwhile: they go to clamped places without a branch, since
// the compiler waits for all loads where one is on some path only (19 us instead of 9 for 38K values).  The row's end is
// in the loop, and its rarer users have U = 1: this code is long, and comes from memory at its first run.
template <int U, typename LT, typename F>
DEVI void each_of_row(const LT *lr, uint32_t V, uint32_t v0, uint32_t v1, F f) {
  constexpr uint32_t N = RowVec<LT>::N, step = kWholeThreads * N;
  u32x4 x[U], y[U];
  auto load = [&](u32x4 (&z)[U], uint32_t c0) {
#pragma unroll
    for (int q = 0; q < U; ++q) z[q] = row_load(lr + min(c0 + q * step + threadIdx.x * N, V - N));
  };
  load(x, v0);
#pragma unroll 1
  for (uint32_t c0 = v0; c0 < v1; c0 += U * step) {
    load(y, c0 + U * step);
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const uint32_t id = c0 + q * step + threadIdx.x * N;
      if (id < v1) f(id + N <= V ? x[q] : row_move_end<LT>(x[q], id + N - V), id);
    }
#pragma unroll
    for (int q = 0; q < U; ++q) x[q] = y[q];
  }
}

// the distance to the maximum in parts of a bin; NaN and -inf are far
constexpr float kFar = (float)(kBins << kSplitLog);
DEVI float distance(const DrawRow &s, float v) { return (s.m - v) * s.cf; }
DEVI bool in_bin(const DrawRow &s, float v, int bin) {
  const float y = distance(s, v);
  return y < kFar && (int)y >> kSplitLog == bin;
}

// Bounds of the values of the bins [from, to), a little wider: the distance is off by 2^-23 of itself, and its factor
// by 2^-24, together less than two parts.
struct Between {
  float lo, hi;
  DEVI static Between bins(const DrawRow &s, int from, int to) {
    const double part = (double)s.T * (0.6931471805599453 / (1 << (kBinsLog + kSplitLog)));
    const double top = (double)s.m - ((double)(from << kSplitLog) - 2.0) * part, end = (double)s.m - ((double)(to << kSplitLog) + 2.0) * part;
    return {scalar((float)(end - fabs(end) * 0x1p-22)), scalar((float)(top + fabs(top) * 0x1p-22))};
  }
  DEVI static Between none() { return {INFINITY, INFINITY}; }  // (rows with a logit of +inf are done without)
  DEVI bool some() const { return lo < INFINITY; }
  // (no value is its own median of these if it is NaN)
  DEVI bool has(float v) const { return __builtin_amdgcn_fmed3f(v, lo, hi) == v; }
};
// which of a vector's values are between the bounds, the last one in the lowest bit; without a branch: one for every
// value took 24 us a row of 151936, three times as long
template <typename LT>
DEVI uint32_t hits(const u32x4 &x, const Between &of) {
  uint32_t b = 0;
#pragma unroll
  for (int e = 0; e < RowVec<LT>::N; ++e) b = b + b + (of.has(RowVec<LT>::get(x, e)) ? 1u : 0u);
  return b;
}
// f(value, id) of the values between the bounds
template <typename LT, typename F>
DEVI void each_between(const LT *lr, uint32_t V, const Between &of, F f) {
  constexpr int N = RowVec<LT>::N;
  each_of_row<1>(lr, V, 0, V, [&](const u32x4 &x, uint32_t id0) {
    for (uint32_t b = hits<LT>(x, of); b; b &= b - 1) {
      const int e = N - 1 - (__ffs(b) - 1), i = e * 4 / N;
      const uint32_t w = i < 2 ? (i == 0 ? x[0] : x[1]) : (i == 2 ? x[2] : x[3]);
      f(RowVec<LT>::get(u32x4{w, w, w, w}, 0 + (N == 8 && (e & 1))), id0 + e);
    }
  });
}
// Collects the ids of the values between the bounds of A in sh.list, and of B in sh.draw, by waves: each has a
// part of its own, so that no lane waits for a place.  Bit 0, bit 1: A's, B's are all there.
template <typename LT>
DEVI int collect(const LT *lr, uint32_t V, const Between &A, const Between &B, WholeShared &sh) {
  constexpr int N = RowVec<LT>::N;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int na = 0, nb = 0;
  each_of_row<2>(lr, V, 0, V, [&](const u32x4 &x, uint32_t id0) {
    auto put = [&](uint32_t bits, unsigned long long *list, int &n) {
      while (true) {
        const unsigned long long mk = __ballot(bits != 0);
        if (!mk) break;
        if (bits) {
          const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(mk >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mk, 0));
          if (at < kSeg) ((uint32_t *)list)[wave * kSeg + at] = id0 + (N - 1) - (__ffs(bits) - 1);
          bits &= bits - 1;
        }
        n += __popcll(mk);
      }
    };
    put(hits<LT>(x, A), sh.list, na);
    if (B.some()) put(hits<LT>(x, B), sh.draw, nb);  // (uniform; the loop is bound by its instructions)
  });
  if (lane == 0) {
    sh.wave_n[0][wave] = na;
    sh.wave_n[1][wave] = nb;
  }
  __syncthreads();
  int most[2] = {0, 0}, all[2] = {0, 0};
  for (int w = 0; w < kWholeWaves; ++w)
    for (int i = 0; i < 2; ++i) {
      most[i] = max(most[i], sh.wave_n[i][w]);
      all[i] += sh.wave_n[i][w];
    }
  return (most[0] <= kSeg && all[0] <= kListMax ? 1 : 0) | (most[1] <= kSeg && all[1] <= kListMax ? 2 : 0);
}
// The entries of a collected list that are of `bin` and have a weight, as keys in descending order; their number.
template <typename LT>
DEVI int pack_list(const LT *lr, uint32_t V, const DrawRow &s, unsigned long long *list, int bin, const Between &of,
                   const int *wave_n, WholeShared &sh, int slot) {
  constexpr int kPer = 2 * kListMax / kWholeThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, have = wave_n[wave];  // (its own part)
  unsigned long long k[kPer];
  uint32_t id[kPer];
  float v[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    id[j] = ((const uint32_t *)list)[wave * kSeg + j * 64 + lane];
    v[j] = to_f32(lr[min(id[j], V - 1)]);  // (at any place of the row where there is none)
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    k[j] = 0;
    if (j * 64 + lane < have && id[j] < V && in_bin(s, v[j], bin) && s.weight(v[j])) k[j] = entry_key(v[j], id[j]);
  }
  if (tid == 0) sh.n[slot] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (k[j]) list[atomicAdd(&sh.n[slot], 1)] = k[j];
  __syncthreads();
  const int n = sh.n[slot];
  sort_list<kWholeWaves, LT>(n, list, order_key(of.lo), order_key(of.hi), sh.sort, sh.red);
  return n;
}

// Where a running sum in the order ends: the sum and the last entry.
struct Prefix {
  unsigned long long mass, key;
};

// Where the running sum of a sorted list (or its count, from n0) that starts at m0 passes `target`; it does.
DEVI Prefix pass_in_list(const DrawRow &s, const unsigned long long *list, int n, bool by_count, unsigned long long target,
                         unsigned long long m0, unsigned long long n0, WholeShared &sh) {
  constexpr int kTwo = kListMax / kWholeThreads;
  const int tid = threadIdx.x;
  unsigned long long w[kTwo], ws = 0;
#pragma unroll
  for (int j = 0; j < kTwo; ++j) {
    const int i = tid * kTwo + j;
    w[j] = i < n ? s.weight(entry_value(list[i])) : 0ull;
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
        sh.hit[1] = list[i];
      }
      e += w[j];
    }
  }
  __syncthreads();
  const Prefix p = {scalar(sh.hit[0]), scalar(sh.hit[1])};
  __syncthreads();
  return p;
}

// The bin (or part of one) in which a running sum passes a target, and the sum and count before it.
struct Bin {
  int i;
  unsigned long long m0, n0;
};
template <int PER>
DEVI Bin pass_in_bins(const unsigned long long *mass, const uint32_t *count, int bins, bool by_count, unsigned long long target,
                      unsigned long long em, unsigned long long en, WholeShared &sh) {
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int b = threadIdx.x * PER + j;
    if (b < bins) {
      const unsigned long long mb = mass[b], a0 = by_count ? en : em, a1 = a0 + (by_count ? count[b] : mb);
      if (a0 <= target && target < a1) {  // one bin of all
        sh.hit[0] = en;
        sh.hit[1] = em;
        sh.hit_i = b;
      }
      em += mb;
      if (by_count) en += count[b];
    }
  }
  __syncthreads();
  const Bin r = {(int)scalar((uint32_t)sh.hit_i), scalar(sh.hit[1]), scalar(sh.hit[0])};
  __syncthreads();
  return r;
}

// The ids of the values with a key, counted by 256s in sh.part.count; their number.
constexpr int kIdsLog = 8;
static_assert(kRowsMaxVocab <= kSplit << kIdsLog, "a row's ids in the parts");
template <typename LT>
DEVI uint32_t count_equal(const LT *lr, uint32_t V, uint32_t key, WholeShared &sh) {
  const int tid = threadIdx.x;
  __syncthreads();
  for (int i = tid; i < kSplit; i += kWholeThreads) sh.part.count[i] = 0;
  __syncthreads();
  const float v = order_key_value(key);
  each_between<LT>(lr, V, Between{v, v}, [&](float, uint32_t id) { atomicAdd(&sh.part.count[id >> kIdsLog], 1u); });
  __syncthreads();
  const uint32_t n = sh.part.count[2 * tid] + sh.part.count[2 * tid + 1];
  return block_reduce_sum<kWholeWaves>(n, sh.red);
}
static_assert(kSplit == 2 * kWholeThreads, "two parts a thread");
// The at-th id of those, of as many and more.
template <typename LT>
DEVI uint32_t equal_at(const LT *lr, uint32_t V, uint32_t key, uint32_t at, WholeShared &sh) {
  const int tid = threadIdx.x;
  __syncthreads();
  const uint32_t c0 = sh.part.count[2 * tid], c1 = sh.part.count[2 * tid + 1];
  const uint32_t before = block_scan<kWholeWaves>(c0 + c1, sh.red) - c0 - c1;
  if (before <= at && at < before + c0 + c1) {
    sh.hit_i = 2 * tid + (at >= before + c0);
    sh.hit[0] = at - before - (at >= before + c0 ? c0 : 0);
  }
  __syncthreads();
  const uint32_t id = ((uint32_t)sh.hit_i << kIdsLog) + tid;
  const bool on = tid < 1 << kIdsLog && id < V && order_key(to_f32(lr[min(id, V - 1)])) == key;
  const uint32_t place = (uint32_t)sh.hit[0], upto = block_scan<kWholeWaves>(on ? 1u : 0u, sh.sort);
  if (on && upto == place + 1) sh.hit[1] = id;
  __syncthreads();
  const uint32_t r = scalar((uint32_t)sh.hit[1]);
  __syncthreads();
  return r;
}

// The shortest prefix of the whole row's order whose count (by_count) or sum is above `target`, which is passed in
// `bin`: among its entries, sorted, where they are not too many; or of a part of their keys' range, cut in 2048 parts
// again and again, or of equal values by their place among the ids (bf16 logits above 16 are 1/8 apart: a flat row of
// 151936 has thousands of each; 64 such rows without filters 210 us in all, 700 with a level for every 11 bits of
// the order).  The values of `also` come into sh.draw on the way; it is set to none if they did not.
template <typename LT>
DEVI Prefix find_in_row(const LT *lr, uint32_t V, const DrawRow &s, bool by_count, unsigned long long target, Bin bin,
                        Between &also, WholeShared &sh) {
  const int tid = threadIdx.x, b = bin.i;
  const Between of = Between::bins(s, b, b + 1);
  int got = 0;
  if (s.few(sh.mass[b], b)) {
    got = collect<LT>(lr, V, of, also, sh);
    if (!(got & 2)) also = Between::none();
    if (got & 1) {
      const int n = pack_list(lr, V, s, sh.list, b, of, sh.wave_n[0], sh, 0);
      return pass_in_list(s, sh.list, n, by_count, target, bin.m0, bin.n0, sh);
    }
  }
  also = Between::none();
  uint32_t lo = order_key(of.lo), hi = order_key(of.hi);
  // f(value, id) of the bin's entries with a key in [lo, hi]
  auto each = [&](auto f) {
    each_between<LT>(lr, V, of, [&](float v, uint32_t id) {
      const uint32_t key = order_key(v);
      if (in_bin(s, v, b) && key >= lo && key <= hi) f(v, id);
    });
  };
  while (true) {
    const uint32_t range = hi - lo;
    const int shift = range < kSplit ? 0 : 32 - kSplitLog - __builtin_clz(range);
    __syncthreads();
    for (int i = tid; i < kSplit; i += kWholeThreads) {
      sh.part.mass[i] = 0;
      sh.part.count[i] = 0;
    }
    if (tid == 0) sh.n[0] = 0;
    __syncthreads();
    each([&](float v, uint32_t) {
      const unsigned long long w = s.weight(v);
      if (w) {
        const uint32_t i = kSplit - 1 - ((order_key(v) - lo) >> shift);
        atomicAdd(&sh.part.mass[i], w);
        atomicAdd(&sh.part.count[i], 1u);
      }
    });
    __syncthreads();
    const unsigned long long pm = sh.part.mass[2 * tid] + sh.part.mass[2 * tid + 1];
    const uint32_t pn = sh.part.count[2 * tid] + sh.part.count[2 * tid + 1];
    const unsigned long long em = bin.m0 + block_scan<kWholeWaves>(pm, sh.redu[0]) - pm;
    const unsigned long long en = bin.n0 + block_scan<kWholeWaves, unsigned long long>(pn, sh.redu[1]) - pn;
    bin = pass_in_bins<2>(sh.part.mass, sh.part.count, kSplit, by_count, target, em, en, sh);
    const int n = (int)scalar(sh.part.count[bin.i]);
    lo += (uint32_t)(kSplit - 1 - bin.i) << shift;
    hi = min(hi, lo + ((1u << shift) - 1u));
    __syncthreads();
    if (n <= kListMax) {
      each([&](float v, uint32_t id) {
        if (s.weight(v)) sh.list[min(atomicAdd(&sh.n[0], 1), kListMax - 1)] = entry_key(v, id);  // (n of them)
      });
      __syncthreads();
      sort_list<kWholeWaves, LT>(n, sh.list, lo, hi, sh.sort, sh.red);
      return pass_in_list(s, sh.list, n, by_count, target, bin.m0, bin.n0, sh);
    }
    if (shift == 0) break;
  }
  // one value: the place among its ids
  const float v = order_key_value(lo);
  const unsigned long long w = s.weight(v), at = by_count ? target - bin.n0 : (target - bin.m0) / w;
  count_equal<LT>(lr, V, lo, sh);
  return {bin.m0 + (at + 1) * w, entry_key(v, equal_at<LT>(lr, V, lo, (uint32_t)at, sh))};
}

// A row whose maximum is +inf: its n logits of +inf have a weight of 1 each, in the order of their ids.
template <typename LT>
DEVI void draw_of_infinities(const LT *lr, const SampleArgs &p, const DrawRow &d, int V, int row, WholeShared &sh) {
  const uint32_t key = order_key(INFINITY);
  uint32_t n = count_equal<LT>(lr, V, key, sh);
  if (d.has_k) n = min(n, (uint32_t)d.top_k);
  if (d.use_p) n = max(1u, min(n, (uint32_t)ceil((double)d.top_p * n)));
  const uint32_t at = min((uint32_t)floor((double)d.u * n), n - 1);  // the draw's place among them
  const uint32_t id = equal_at<LT>(lr, V, key, at, sh);
  if (threadIdx.x == 0) d.finish(p, row, (int)id, d.logprob(INFINITY, (unsigned long long)n << kWeightBits));
}

template <typename LT>
DEVI void draw_whole(const RowsArgs &a, const SampleArgs &p, const DrawRow &d, int row, int slice, int slices, DrawSums *g,
                     WholeShared &sh) {
  constexpr int N = RowVec<LT>::N;
  const int tid = threadIdx.x;
  const LT *lr = (const LT *)a.logits + (size_t)row * a.ld;
  if (d.m == INFINITY) {
    if (slice == 0) draw_of_infinities(lr, p, d, a.V, row, sh);
    return;
  }
  for (int i = tid; i < kBins; i += kWholeThreads) {
    sh.mass[i] = 0;
    sh.count[i] = 0;
  }
  __syncthreads();
  const uint32_t len = ((uint32_t)a.V / slices / N + 1) * N, v0 = slice * len, v1 = min((uint32_t)a.V, v0 + len);
  // f(bin, weight), four values at a time: their weights are formed side by side
  auto each_weight = [&](auto f) {
    each_of_row<2>(lr, a.V, v0, v1, [&](const u32x4 &x, uint32_t) {
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        float y[4];
        unsigned long long w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = RowVec<LT>::get(x, e + j);
          y[j] = distance(d, v);
          w[j] = weight_of(((double)d.m - (double)v) * d.cd);  // (any number where y is far)
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (y[j] < kFar) f((int)y[j] >> kSplitLog, w[j]);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
  };
  if (v0 < v1) {
    each_weight([&](int b, unsigned long long w) { atomicAdd(&sh.mass[b], w); });
    if (d.has_k)
      each_weight([&](int b, unsigned long long w) {
        if (w) atomicAdd(&sh.count[b], 1u);
      });
  }
  __syncthreads();
  if (slices > 1) {
    // To memory; the last workgroup of the row adds them all up.  Stores and loads are device-scope ones,
    // complete when the count of the storing thread's drains: 64 rows at once took 17 to 37 us by
    // 64-bit atomics into one place, and as long by plain stores between fences, which write back and
    // drop the whole cache of an XCD.  Relaxed accesses say nothing of the order of sums and count: it comes from this
    // chip's counter of stores, the barrier, and fences for the compiler alone, which emit no instruction.
    for (int i = tid; i < kBins; i += kWholeThreads) {
      __hip_atomic_store(&g[slice].mass[i], sh.mass[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (d.has_k) __hip_atomic_store(&g[slice].count[i], sh.count[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);  // this thread's sums are there
    asm volatile("" ::: "memory");
    __syncthreads();
    if (tid == 0)
      sh.last = __hip_atomic_fetch_add(&p.done[row], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)slices - 1;
    __syncthreads();
    asm volatile("" ::: "memory");
    if (!sh.last) return;
    unsigned long long m[kBinsPer] = {};
    uint32_t n[kBinsPer] = {};
    for (int q0 = 0; q0 < slices; q0 += 8) {  // (eight of every bin in flight: each waits a microsecond or two)
      unsigned long long x[8][kBinsPer];
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int j = 0; j < kBinsPer; ++j)
          x[q][j] = __hip_atomic_load(&g[min(q0 + q, slices - 1)].mass[min(j * kWholeThreads + tid, kBins - 1)],
                                      __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int j = 0; j < kBinsPer; ++j) m[j] += q0 + q < slices ? x[q][j] : 0ull;
    }
    if (d.has_k)
      for (int q = 0; q < slices; ++q)
#pragma unroll
        for (int j = 0; j < kBinsPer; ++j)
          n[j] += __hip_atomic_load(&g[q].count[min(j * kWholeThreads + tid, kBins - 1)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int j = 0; j < kBinsPer; ++j)
      if (j * kWholeThreads + tid < kBins) {
        sh.mass[j * kWholeThreads + tid] = m[j];
        sh.count[j * kWholeThreads + tid] = n[j];
      }
    __syncthreads();
  }
  // what lies before each thread's bins, and in all of them
  unsigned long long pm = 0, pn = 0;
  for (int b = tid * kBinsPer; b < min((tid + 1) * kBinsPer, kBins); ++b) {
    pm += sh.mass[b];
    pn += sh.count[b];
  }
  const unsigned long long em = block_scan<kWholeWaves>(pm, sh.redu[0]), en = block_scan<kWholeWaves>(pn, sh.redu[1]);
  if (tid == kWholeThreads - 1) {
    sh.hit[0] = en;
    sh.hit[1] = em;
  }
  __syncthreads();
  const unsigned long long entries = scalar(sh.hit[0]);
  unsigned long long total = scalar(sh.hit[1]);
  __syncthreads();
  auto bin_of = [&](bool by_count, unsigned long long target) {
    return pass_in_bins<kBinsPer>(sh.mass, sh.count, kBins, by_count, target, em - pm, en - pn, sh);
  };
  auto drawn = [&](unsigned long long sum) { return min((unsigned long long)floor((double)d.u * (double)sum), sum - 1); };
  // top-k, top-p, then (the shorter of it and min-p kept) the draw
#pragma unroll 1
  for (int step = d.has_k && (unsigned long long)d.top_k < entries ? 0 : d.use_p ? 1 : 2;; step = step == 0 && d.use_p ? 1 : 2) {
    unsigned long long target = d.top_k - 1;
    if (step == 1) {
      const unsigned long long want = (unsigned long long)ceil((double)d.top_p * (double)total);
      target = want == 0 ? 0 : min(want, total) - 1;
    } else if (step == 2) {
      if (d.use_m) {
        // the sum that stays under min-p: whole bins, and of the bins around the border the entries that stay
        const double border = d.min_d * (double)d.cf / kSplit;
        const int b0 = (int)fmin(fmax(border - 1.0, 0.0), (double)kBins), b1 = min(b0 + 3, kBins);
        unsigned long long mm = 0;
        for (int b = tid; b < b0; b += kWholeThreads) mm += sh.mass[b];
        if (b0 < kBins)
          each_between<LT>(lr, a.V, Between::bins(d, b0, b1), [&](float v, uint32_t) {
            const float y = distance(d, v);
            if (y < kFar && (int)y >> kSplitLog >= b0 && (int)y >> kSplitLog < b1 && d.stays(v)) mm += d.weight(v);
          });
        total = min(total, block_reduce_sum<kWholeWaves>(mm, sh.redu[0]));
        __syncthreads();
      }
      target = drawn(total);
    }
    Bin bin = {}, next = {};
    // The sum that top-p keeps is target + 1 at least, and less than the weight of the bin's first part above it:
    // where the draw falls into one bin in both cases, one pass collects both bins.
    Between also = Between::none();
    const int both = step == 1 && !d.use_m ? 3 : 1;
#pragma unroll 1
    for (int t = 0; t < both; ++t) {  // (a loop: three copies of the search come from memory three times)
      const Bin r = bin_of(step == 0, t == 0 ? target : drawn(t == 1 ? target + 1 : min(total, target + 1 + d.weight_at(bin.i))));
      if (t == 0) bin = r;
      else if (t == 1) next = r;
      else if (next.i == r.i && d.few(sh.mass[r.i], r.i)) also = Between::bins(d, r.i, r.i + 1);
    }
    Prefix f = find_in_row<LT>(lr, a.V, d, step == 0, target, bin, also, sh);
    bool end = step == 2;
    if (!end) total = f.mass;
    if (also.some()) {
      const int n = pack_list(lr, a.V, d, sh.draw, next.i, also, sh.wave_n[1], sh, 1);
      f = pass_in_list(d, sh.draw, n, false, drawn(total), next.m0, next.n0, sh);
      end = true;
    }
    if (end) {
      if (tid == 0) d.finish(p, row, (int)entry_id(f.key), d.logprob(entry_value(f.key), total));
      return;
    }
  }
}

// The rows that are left, a workgroup a slice of each.  (Slices that go by how many rows are left, from a
// list of them, are no faster: their parameters come three dependent loads later.)  Its 128 registers, all that
// 16 waves can have, keep it to one workgroup a CU, and it spills 37 of them (35 with fp32 logits).
template <typename LT>
__global__ __launch_bounds__(kWholeThreads) void draw_whole_kernel(RowsArgs a, SampleArgs p) {
  __shared__ WholeShared sh;
  const int row = blockIdx.x / p.slices, slice = blockIdx.x % p.slices;
  const uint32_t state = p.state[row];
  if (state == 0) return;  // the first entries have decided
  DrawRow d;
  d.read(a, p, row);
  d.set_max(order_key_value(state));
  draw_whole<LT>(a, p, d, row, slice, p.slices, p.sums + (size_t)row * p.slices, sh);
}

// Workgroups a row of the last launch: for few rows as many as cut a row of 128K ids to 8K each (64
// rows of 128256 fp32 logits, the flat ones: 46 us, 66 with one), for many enough to fill the chip
// (512 rows of 151936 bf16 logits, 64 of them flat: 78 us with one, 67 with two, 99 with four.  What four
// cost is not the work of a slice; most likely it is the many workgroups without a row left, each of which takes
// a CU to itself.  Not traced.)
static int draw_slices(int rows, int V) { return std::max(1, std::min({16, 1024 / rows, V / 8192})); }

// [error word and groups][a row each: state, workgroups done][sums, where a row has several workgroups]
struct DrawLayout {
  size_t state, done, sums, bytes;
};
static DrawLayout draw_layout(int rows, int V) {
  DrawLayout l;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  const int slices = draw_slices(rows, V);
  l.state = up(rows_ws_bytes(rows, V));
  l.done = l.state + (size_t)rows * 4;
  l.sums = up(l.done + (size_t)rows * 4);
  l.bytes = l.sums + (slices > 1 ? (size_t)rows * slices * sizeof(DrawSums) : 0);
  return l;
}
size_t draw_ws_bytes(int rows, int V) { return draw_layout(rows, V).bytes; }

void launch_sample_logits(RowsArgs a, bool bf16, SampleArgs p, void *ws, hipStream_t st) {
  const DrawLayout l = draw_layout(a.rows, a.V);
  char *w = (char *)ws;
  p.state = (uint32_t *)(w + l.state);
  p.done = (uint32_t *)(w + l.done);
  p.sums = (DrawSums *)(w + l.sums);
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
