// The top entries of rows of logits, and drawing a token under temperature, top-k,
// top-p and min-p.  Both read a row once for the maximum and the sum of exp of its
// groups of 32 ids, and select from those:
//
//   The first C entries of a row in the order (value desc, id asc) lie in the first C
//   groups in the order (maximum desc, group asc).  (An entry outside them is behind
//   the maximum of each of them.)  So a row of V values is cut to 32 C of them after
//   one pass, whatever its values.
//
// Launches:
//   groups  bound by the logits' bytes: 16-byte loads, a group in the registers of 4 (bf16)
//           or 8 (fp32) lanes
//   top     a workgroup a row: the C-th best group by binary search over the groups' maxima,
//           the values of the first C groups in registers, those that can be among the
//           first C sorted in LDS; the sum of the rest from the other groups' sums and
//           the registers, never as a total less the entries
//   sample  the same with C = top_k, or 256 where it is off; the filters and the draw are
//           running sums over the sorted entries, in integers (weights of 2^-44 of the
//           row's best), so that their order does not matter.  Rows that this does not
//           decide (flat ones whose nucleus or draw lies behind 256 entries) go on over the
//           whole row: sums by bins of exp(-(max - l) / T), the bin where the running sum
//           passes the target, and its entries sorted, or split again while they are too many.
#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace dk {

constexpr int kGroup = 32;        // ids a group
constexpr int kGrThreads = 256;
constexpr int kGrChunk = 8192;    // ids a workgroup of the first launch
constexpr int kSelThreads = 1024; // a workgroup a row
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kSelRegs = kRowsMaxVocab / (kGroup * kSelThreads);  // group maxima a thread
static_assert(kRowsMaxVocab % (kGroup * kSelThreads) == 0, "whole registers of groups");
constexpr int kTopMax = 1024;     // entries at most: one a thread
constexpr int kListMax = 2048;    // candidates sorted in LDS
constexpr int kSelMax = 2048;     // groups read
constexpr uint32_t kIdMask = 0xfffffu;
static_assert(kRowsMaxVocab <= kIdMask, "ids in 20 bits");

// log2(e) / T, kept finite: a difference of 0 has to stay 0
DEVI float row_scale(float T) { return fminf(kRowLog2e / T, 1e30f); }

// ---------------------------------------------------------------------------
// (1) (max, sum of exp((l - max) / T)) of every group of every row
// ---------------------------------------------------------------------------
template <typename LT>
__global__ __launch_bounds__(kGrThreads) void row_groups_kernel(RowsArgs a) {
  constexpr int N = RowVec<LT>::N, NV = kGrChunk / kGrThreads / N, LPG = kGroup / N;
  const int row = blockIdx.x / a.nch, ch = blockIdx.x % a.nch, tid = threadIdx.x;
  if (blockIdx.x == 0 && tid == 0) *a.err = 0;
  const uint32_t c0 = (uint32_t)ch * kGrChunk, V = a.V;
  const LT *lr = (const LT *)a.logits + (size_t)row * a.ld;
  u32x4 x[NV];
  if (c0 + kGrChunk <= V) {  // workgroup-uniform: every load goes out at once
#pragma unroll
    for (int q = 0; q < NV; ++q) x[q] = row_load(lr + c0 + (q * kGrThreads + tid) * N);
  } else {
#pragma unroll
    for (int q = 0; q < NV; ++q) x[q] = row_load_end(lr, c0 + (q * kGrThreads + tid) * N, V);
  }
  const float c = row_scale(a.temps ? a.temps[row] : a.T);
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, RowVec<LT>::get(x[q], e));
    // over the group's lanes: 4 by quads, 8 by half rows
    m = fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0xB1, 0xf, 0xf, false)));
    m = fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0x4E, 0xf, 0xf, false)));
    if (LPG == 8) m = fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0x141, 0xf, 0xf, false)));
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      // (v = m = +inf: the difference is NaN and counts as 0)
      const float v = fmaxf(RowVec<LT>::get(x[q], e), -INFINITY);
      s += __builtin_amdgcn_exp2f(fminf((v - m) * c, 0.f));
    }
    s += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(s), 0xB1, 0xf, 0xf, false));
    s += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(s), 0x4E, 0xf, 0xf, false));
    if (LPG == 8) s += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(s), 0x141, 0xf, 0xf, false));
    const uint32_t g = (c0 + (q * kGrThreads + tid) * N) / kGroup;
    if (tid % LPG == 0 && g < (uint32_t)a.G) a.groups[(size_t)row * a.G + g] = make_float2(m, m == -INFINITY ? 0.f : s);
  }
}

// ---------------------------------------------------------------------------
// (2) selection within a row
// ---------------------------------------------------------------------------
// What bounds it is the chain of steps of one workgroup, and the first run of each
// instruction, which comes from memory: loops stay loops where that costs nothing (a first
// version with every loop unrolled, 74 to 280 KB of code, took 23 us for one row).
struct SelShared {
  unsigned long long list[kListMax];  // keys: order_key of the value, complement of the id
  int sel[kSelMax];                   // the selected groups
  uint32_t hist[kSelThreads];
  uint32_t wave[2][kSelWaves];
  float redf[kSelWaves];
  double redd[kSelWaves];
  uint32_t hit[3];
  int n;
};

DEVI unsigned long long entry_key(float v, uint32_t id) { return ((unsigned long long)order_key(v) << 32) | (0xffffffffu - id); }
DEVI float entry_value(unsigned long long k) { return order_key_value((uint32_t)(k >> 32)); }
DEVI uint32_t entry_id(unsigned long long k) { return 0xffffffffu - (uint32_t)k; }

// inclusive running sum over the workgroup's threads; `red` is free again after the next barrier
template <typename T>
DEVI T block_scan(T v, T *red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  if (lane == 63) red[wave] = v;
  __syncthreads();
  T base = 0;
  for (int w = 0; w < wave; ++w) base += red[w];
  return base + v;
}

// Those with a key above `key`, or with this key and an id up to `id`.
struct Cut {
  uint32_t key, id;
  DEVI bool has(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= id); }
};

// A cut that takes at least `want` items, and at most `cap` (want <= cap): by counts in 1024
// equal parts of [lo, hi], which holds the key of the want-th, and again of the part that holds
// it while there are more than `cap` up to its end; among equal keys the same by ids.
// each(f) calls f(key, id) for every item.
template <typename Each>
DEVI Cut cut_at(uint32_t lo, uint32_t hi, int want, int cap, SelShared &sh, Each each) {
  const int tid = threadIdx.x;
  bool by_id = false;
  uint32_t key = 0;
  int above = 0;  // items beyond hi
  while (true) {
    const uint32_t range = hi - lo;
    const int shift = range < kSelThreads ? 0 : 22 - __builtin_clz(range);
    sh.hist[tid] = 0;
    __syncthreads();
    each([&](uint32_t k, uint32_t id) {
      const uint32_t x = by_id ? kIdMask - id : k;
      if (x >= lo && x <= hi && (!by_id || k == key)) atomicAdd(&sh.hist[kSelThreads - 1 - ((x - lo) >> shift)], 1u);
    });
    __syncthreads();
    const int c = sh.hist[tid];
    const int n = above + block_scan<uint32_t>(c, sh.wave[0]);
    if (n >= want && n - c < want) {  // one thread of all
      sh.hit[0] = kSelThreads - 1 - tid;
      sh.hit[1] = n;
      sh.hit[2] = n - c;
    }
    __syncthreads();
    const uint32_t part = lo + (sh.hit[0] << shift);
    const int upto = sh.hit[1], before = sh.hit[2];
    if (upto <= cap) return by_id ? Cut{key, kIdMask - part} : Cut{part, 0xffffffffu};
    above = before;
    if (shift > 0) {
      hi = min(hi, part + ((1u << shift) - 1u));
      lo = part;
    } else {  // (a part of ids holds one item: it would have been taken)
      by_id = true;
      key = part;
      lo = 0;
      hi = kIdMask;
    }
  }
}

// sh.list[0 .. n) in descending order (keys are distinct).  Up to 256 a key counts those before
// it (n^2 / 64 reads of 4 cycles), by several threads where there are enough; more by a bitonic
// network, whose short steps stay within a wave and need no barrier.
DEVI void sort_list(int n, SelShared &sh) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (n <= 256) {
    const int lg = n <= 64 ? 4 : n <= 128 ? 3 : 2, i = tid >> lg, parts = 1 << lg;
    unsigned long long k = 0;
    int r = 0;
    if (i < n) {
      k = sh.list[i];
      for (int j = tid & (parts - 1); j < n; j += parts) r += sh.list[j] > k;
    }
    for (int o = 1; o < parts; o <<= 1) r += __shfl_xor(r, o, 64);
    __syncthreads();
    if (i < n && (tid & (parts - 1)) == 0) sh.list[r] = k;
    __syncthreads();
    return;
  }
  int size = 512;
  while (size < n) size <<= 1;
  for (int i = n + tid; i < size; i += kSelThreads) sh.list[i] = 0;
  __syncthreads();
  for (int len = 2; len <= size; len <<= 1)
    for (int step = len >> 1; step >= 1; step >>= 1) {
      if (tid < size / 2) {
        const int i = (tid & ~(step - 1)) * 2 + (tid & (step - 1)), j = i + step;
        const unsigned long long x = sh.list[i], y = sh.list[j];
        const bool desc = (i & len) == 0;
        if ((x < y) == desc) {
          sh.list[i] = y;
          sh.list[j] = x;
        }
      }
      // a wave's 128 keys are its own up to steps of 64
      if (step > 64 || (step == 1 && len >= 128)) __syncthreads();
      else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    }
  __syncthreads();
}

// The first C entries of a row, sorted, in sh.list; of the others the largest value (rest_m)
// and the sum of exp((l - rest_m) / T) (rest_s).  C <= min(V, kTopMax).
template <typename LT>
DEVI void select_top(const LT *lr, const float2 *groups, int V, int G, int C, float c, SelShared &sh, float &rest_m,
                     double &rest_s) {
  constexpr int N = RowVec<LT>::N, LPG = kGroup / N;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the groups, group i * 1024 + tid in register i
  uint32_t gk[kSelRegs];
  float gs[kSelRegs];
  const int nr = (G + kSelThreads - 1) / kSelThreads;
  uint32_t hi = 0;
#pragma unroll
  for (int i = 0; i < kSelRegs; ++i) {
    gk[i] = 0;  // (no value has the key 0)
    gs[i] = 0.f;
    if (i < nr) {
      const int g = i * kSelThreads + tid;
      if (g < G) {
        const float2 x = groups[g];
        gk[i] = order_key(x.x);
        gs[i] = x.y;
      }
      hi = max(hi, gk[i]);
    }
  }
  // Bounds of the C-th group's key.  From below: the least of 1024 / s maxima, each of the groups
  // of s threads, with 1024 / s >= C of them (where every thread has one).
  uint32_t lo = hi;
  if (G >= kSelThreads) {
    for (int s = 1; s < 64 && kSelThreads / (2 * s) >= C; s <<= 1) lo = max(lo, (uint32_t)__shfl_xor((int)lo, s, 64));
  } else if (lo == 0) {
    lo = 0xffffffffu;  // (a thread without a group)
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
  }
  if (lane == 0) {
    sh.wave[0][wave] = lo;
    sh.wave[1][wave] = hi;
  }
  __syncthreads();
#pragma unroll 4
  for (int w = 0; w < kSelWaves; ++w) {
    lo = min(lo, sh.wave[0][w]);
    hi = max(hi, sh.wave[1][w]);
  }
  auto every_group = [&](auto f) {
#pragma unroll
    for (int i = 0; i < kSelRegs; ++i)
      if (i < nr && gk[i]) f(gk[i], (uint32_t)(i * kSelThreads + tid));
  };
  Cut gc = {0, 0xffffffffu};
  if (G > kSelMax || C < G) gc = cut_at(lo, hi, min(C, G), kSelMax, sh, every_group);
  // their list, by waves
  uint32_t chosen = 0;
  int nw = 0;
#pragma unroll
  for (int i = 0; i < kSelRegs; ++i)
    if (i < nr) {
      const bool on = gk[i] && gc.has(gk[i], i * kSelThreads + tid);
      chosen |= on ? 1u << i : 0u;
      nw += __popcll(__ballot(on));
    }
  __syncthreads();
  if (lane == 0) sh.wave[0][wave] = nw;
  if (tid == 0) sh.n = 0;
  __syncthreads();
  int at = 0, nsel = 0;
#pragma unroll 4
  for (int w = 0; w < kSelWaves; ++w) {
    const int x = sh.wave[0][w];
    if (w < wave) at += x;
    nsel += x;
  }
#pragma unroll
  for (int i = 0; i < kSelRegs; ++i)
    if (i < nr) {
      const unsigned long long mk = __ballot(chosen >> i & 1);
      if (chosen >> i & 1) sh.sel[at + __popcll(mk & ((1ull << lane) - 1))] = i * kSelThreads + tid;
      at += __popcll(mk);
    }
  __syncthreads();
  // Their values: vector u is part u % LPG of group u / LPG.  The first kHeld a thread (256 groups)
  // stay in registers from pass to pass; where there are more, every pass loads them again.
  constexpr int kHeld = LPG / 4;
  const int nu = nsel * LPG;
  u32x4 x[kHeld];
  uint32_t id0[kHeld];
  auto load = [&](int u0) {
#pragma unroll
    for (int q = 0; q < kHeld; ++q) {
      const int u = u0 + q * kSelThreads + tid;
      id0[q] = 0x7fffffffu;  // past every row: no value of it counts
      if (u < nu) {
        id0[q] = (uint32_t)sh.sel[u / LPG] * kGroup + (u % LPG) * N;
        x[q] = row_load_end(lr, id0[q], V);
      }
    }
  };
  load(0);
  auto every_vec = [&](auto f) {  // f(vector, its first id)
    if (nu > kHeld * kSelThreads) load(0);
#pragma unroll 1
    for (int u0 = 0;;) {
#pragma unroll
      for (int q = 0; q < kHeld; ++q)
        if (id0[q] < (uint32_t)V) f(x[q], id0[q]);
      u0 += kHeld * kSelThreads;
      if (u0 >= nu) break;
      load(u0);
    }
  };
  auto every_value = [&](auto f) {  // f(key, id)
    every_vec([&](const u32x4 &y, uint32_t id) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (id + e < (uint32_t)V) f(order_key(RowVec<LT>::get(y, e)), id + e);
    });
  };
  // The values that can be among the first C: those the cut of the groups' maxima takes by their
  // key; where they are more than the list holds, those of a cut of their own.
  Cut ec = {gc.key, 0xffffffffu};
  float m;
  for (bool cut = gc.key == 0 && V > kListMax;; cut = true) {  // (no cut of the groups: every value)
    if (cut) {
      lo = max(ec.key, 1u);
      ec = cut_at(lo, hi, C, kListMax, sh, every_value);
      if (tid == 0) sh.n = 0;
      __syncthreads();
    }
    m = -INFINITY;
    every_vec([&](const u32x4 &y, uint32_t id) {
      uint32_t on = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = RowVec<LT>::get(y, e);
        const bool in = id + e < (uint32_t)V, has = in && ec.has(order_key(v), id + e);
        on |= has ? 1u << e : 0u;
        if (in && !has) m = fmaxf(m, v);
      }
      if (on) {
        int to = atomicAdd(&sh.n, __popc(on));
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (on >> e & 1) {
            if (to < kListMax) sh.list[to] = entry_key(RowVec<LT>::get(y, e), id + e);
            ++to;
          }
      }
    });
    __syncthreads();
    if (sh.n <= kListMax) break;
  }
  const int n = sh.n;
  sort_list(n, sh);
  // The rest: the groups not read, the values not listed, the list behind C.
#pragma unroll
  for (int i = 0; i < kSelRegs; ++i)
    if (i < nr && gk[i] && !(chosen >> i & 1)) m = fmaxf(m, order_key_value(gk[i]));
  if (n > C) m = fmaxf(m, entry_value(sh.list[C]));
  m = block_reduce_max<kSelWaves>(m, sh.redf);
  double s = 0.0;
  if (m > -INFINITY) {  // uniform
    float t = 0.f;
    auto add = [&](float v, float by) { t += by * __builtin_amdgcn_exp2f(fminf((fmaxf(v, -INFINITY) - m) * c, 0.f)); };
#pragma unroll
    for (int i = 0; i < kSelRegs; ++i)
      if (i < nr && gk[i] && !(chosen >> i & 1)) add(order_key_value(gk[i]), gs[i]);
    s = t;
    t = 0.f;
    every_vec([&](const u32x4 &y, uint32_t id) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = RowVec<LT>::get(y, e);
        if (id + e < (uint32_t)V && !ec.has(order_key(v), id + e)) add(v, 1.f);
      }
    });
    for (int i = C + tid; i < n; i += kSelThreads) add(entry_value(sh.list[i]), 1.f);
    s += t;
  }
  rest_m = m;
  rest_s = block_reduce_sum<kSelWaves>(s, sh.redd);
}

template <typename LT>
__global__ __launch_bounds__(kSelThreads) void top_select_kernel(RowsArgs a, int k, int32_t *__restrict__ ids,
                                                                 float *__restrict__ vals, float *__restrict__ rest) {
  __shared__ SelShared sh;
  const int row = blockIdx.x, tid = threadIdx.x;
  const LT *lr = (const LT *)a.logits + (size_t)row * a.ld;
  const float2 *groups = a.groups + (size_t)row * a.G;
  const float c = row_scale(a.T);
  float rm = 0.f;
  double rs = 0.0;
  select_top<LT>(lr, groups, a.V, a.G, k, c, sh, rm, rs);
  if (tid < k) {
    const unsigned long long key = sh.list[tid];
    ids[(size_t)row * k + tid] = (int32_t)entry_id(key);
    vals[(size_t)row * k + tid] = entry_value(key);
  }
  if (rest && tid == 0)
    rest[row] = rs == 0.0 ? -INFINITY : rm == INFINITY ? INFINITY : (float)((double)rm / (double)a.T + log(rs));
}

// ---------------------------------------------------------------------------
// (3) sampling
// ---------------------------------------------------------------------------
constexpr int kWeightBits = 44;                        // a weight of 1 is 2^44; a row's sum stays below 2^63
static_assert(kRowsMaxVocab <= 1 << 19, "sums of weights must fit 63 bits");
constexpr int kBinsLog = 6;                            // bins of 1/64 in log2 of the weight
constexpr int kBins = (kWeightBits + 2) << kBinsLog;   // a weight past them rounds to 0
constexpr int kSplit = 2048;                           // parts a bin is split into, level by level
constexpr int kSampleTop = 256;                        // entries looked at first where top_k is off

// round(2^44 exp(-(max - l) / T)): x = (max - l) log2(e) / T >= 0.  2^f on [-1/2, 1/2] by its Taylor sum
// to the 11th power, whose next term is 2^-50; the rest is exact or rounded to 53 bits.
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

struct SampleRow {
  float m;      // the row's maximum
  double cd;    // log2(e) / T
  float cf;     // the same by 2^17, for the bins
  DEVI unsigned long long weight(float v) const {
    return v == m ? 1ull << kWeightBits : weight_of(((double)m - (double)v) * cd);
  }
};

struct SampleShared {
  union {
    SelShared sel;
    struct {                          // a bin of the whole row, by parts
      unsigned long long mass[kSplit];
      uint32_t count[kSplit];
    } part;
  };
  union {
    unsigned long long run[kTopMax];  // running sums of the first entries
    struct {                          // the whole row by bins
      unsigned long long mass[kBins];
      uint32_t count[kBins];
    } row;
  };
  unsigned long long redu[2][kSelWaves];
  unsigned long long hit[3];
  int hit_i, first[4];
};
static_assert(sizeof(SampleShared) <= 65536, "two workgroups a CU, static LDS");

// Where a running sum in the order ends: after n entries of together `mass`, the last one `key`.
struct Prefix {
  unsigned long long n, mass, key;
};

// f(value, id, is one) for every value of the row; the next 16-byte loads are on their way meanwhile
template <typename LT, typename F>
DEVI void each_of_row(const LT *lr, uint32_t V, F f) {
  constexpr int N = RowVec<LT>::N, U = 2;
  constexpr uint32_t step = kSelThreads * N;
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
  load(x, 0);
#pragma unroll 1
  for (uint32_t c0 = 0; c0 < V; c0 += U * step) {
    load(y, c0 + U * step);
#pragma unroll
    for (int q = 0; q < U; ++q)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint32_t id = c0 + q * step + threadIdx.x * N + e;
        f(RowVec<LT>::get(x[q], e), id, id < V);
      }
#pragma unroll
    for (int q = 0; q < U; ++q) x[q] = y[q];
  }
}

// The order in digits, each ascending: the bin and its fraction (of the distance to the
// maximum), the value's key, the id; `level` says which digit, `near` whether those before it agree.
struct Digits {
  uint32_t y, k, id;
};
DEVI Digits digits_of(const SampleRow &s, float v, uint32_t id) {
  const float d = (s.m - v) * s.cf;  // (max = +inf: NaN for its equals, which are at distance 0)
  return {v == s.m ? 0u : (uint32_t)fminf(d, 1.6e7f), ~order_key(v), id};
}
DEVI bool near(const Digits &a, const Digits &b, int level) {
  const uint32_t my = level == 0 ? 0u : level == 1 ? ~2047u : ~0u;
  const uint32_t mk = level < 3 ? 0u : level == 3 ? ~0u << 21 : level == 4 ? ~0u << 10 : ~0u;
  const uint32_t mi = level < 6 ? 0u : level == 6 ? ~2047u : ~0u;
  return (((a.y ^ b.y) & my) | ((a.k ^ b.k) & mk) | ((a.id ^ b.id) & mi)) == 0;
}
DEVI uint32_t digit_of(const Digits &a, int level) {
  switch (level) {
    case 0: return a.y >> 11;
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

// The shortest prefix of the whole order whose count (by_count) or mass is above `target`; one exists.
template <typename LT>
DEVI Prefix find_in_row(const LT *lr, uint32_t V, const SampleRow &s, bool by_count, unsigned long long target,
                        SampleShared &sh) {
  const int tid = threadIdx.x;
  Digits at = {0, 0, 0};
  unsigned long long n0 = 0, m0 = 0;  // before the part in work
  for (int level = 0;; ++level) {
    unsigned long long *mass = level == 0 ? sh.row.mass : sh.part.mass;
    uint32_t *count = level == 0 ? sh.row.count : sh.part.count;
    const int bins = level == 0 ? kBins : kSplit;
    if (level > 0) {
      for (int i = tid; i < kSplit; i += kSelThreads) {
        mass[i] = 0;
        count[i] = 0;
      }
      __syncthreads();
      each_of_row(lr, V, [&](float v, uint32_t id, bool in) {
        const Digits d = digits_of(s, v, id);
        if (in && d.y < (uint32_t)kBins << 11 && near(d, at, level)) {
          const unsigned long long w = s.weight(order_val(v));
          if (w) {
            atomicAdd(&mass[digit_of(d, level)], w);
            atomicAdd(&count[digit_of(d, level)], 1u);
          }
        }
      });
      __syncthreads();
    }
    // the digit in which the target is passed: kBinsPer of them a thread
    constexpr int kPer = (kBins + kSelThreads - 1) / kSelThreads;
    unsigned long long pm = 0, pn = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = tid * kPer + j;
      if (b < bins) {
        pm += mass[b];
        pn += count[b];
      }
    }
    unsigned long long em = block_scan(pm, sh.redu[0]) - pm + m0, en = block_scan(pn, sh.redu[1]) - pn + n0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = tid * kPer + j;
      if (b < bins) {
        const unsigned long long a0 = by_count ? en : em, a1 = a0 + (by_count ? count[b] : mass[b]);
        if (a0 <= target && target < a1) {  // one bin of all
          sh.hit[0] = en;
          sh.hit[1] = em;
          sh.hit[2] = count[b];
          sh.hit_i = b;
        }
        em += mass[b];
        en += count[b];
      }
    }
    __syncthreads();
    n0 = sh.hit[0];
    m0 = sh.hit[1];
    const unsigned long long inside = sh.hit[2];
    set_digit(at, level, sh.hit_i);
    __syncthreads();
    if (inside > kListMax) continue;  // (at level 6 a part is one entry)
    // its entries, sorted, with their running sums
    if (tid == 0) sh.sel.n = 0;
    __syncthreads();
    each_of_row(lr, V, [&](float v, uint32_t id, bool in) {
      const Digits d = digits_of(s, v, id);
      const bool on = in && d.y < (uint32_t)kBins << 11 && near(d, at, level + 1) && s.weight(order_val(v));
      if (on) {
        const int to = atomicAdd(&sh.sel.n, 1);
        if (to < kListMax) sh.sel.list[to] = entry_key(v, id);
      }
    });
    __syncthreads();
    const int n = sh.sel.n;
    sort_list(n, sh.sel);
    constexpr int kTwo = kListMax / kSelThreads;
    unsigned long long w[kTwo], ws = 0;
#pragma unroll
    for (int j = 0; j < kTwo; ++j) {
      const int i = tid * kTwo + j;
      w[j] = i < n ? s.weight(entry_value(sh.sel.list[i])) : 0ull;
      ws += w[j];
    }
    unsigned long long e = block_scan(ws, sh.redu[0]) - ws + m0;
#pragma unroll
    for (int j = 0; j < kTwo; ++j) {
      const int i = tid * kTwo + j;
      if (i < n) {
        const unsigned long long a0 = by_count ? n0 + i : e, a1 = by_count ? a0 + 1 : e + w[j];
        if (a0 <= target && target < a1) {
          sh.hit[0] = n0 + i + 1;
          sh.hit[1] = e + w[j];
          sh.hit[2] = sh.sel.list[i];
        }
        e += w[j];
      }
    }
    __syncthreads();
    const Prefix p = {sh.hit[0], sh.hit[1], sh.hit[2]};
    __syncthreads();
    return p;
  }
}

template <typename LT>
__global__ __launch_bounds__(kSelThreads) void sample_kernel(RowsArgs a, SampleArgs p) {
  __shared__ SampleShared sh;
  const int row = blockIdx.x, tid = threadIdx.x;
  const LT *lr = (const LT *)a.logits + (size_t)row * a.ld;
  const float2 *groups = a.groups + (size_t)row * a.G;
  // the row's parameters; one out of range leaves the row without a token
  float T = a.temps ? a.temps[row] : 1.f;
  const float u = p.uniforms[row], top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  int top_k = p.top_k ? p.top_k[row] : 0;
  auto finish = [&](int token, float logprob) {  // one thread
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = logprob;
  };
  if (!(T >= 0.f && T < INFINITY && u >= 0.f && u < 1.f && top_p >= 0.f && top_p <= 1.f && min_p >= 0.f && min_p <= 1.f)) {
    if (tid == 0) {
      raise_error(a.err, DEV_BAD_PARAM);
      finish(-1, NAN);
    }
    return;
  }
  if (T == 0.f) {
    top_k = 1;
    T = 1.f;
  }
  const bool has_k = top_k > 0 && top_k < a.V, use_p = top_p < 1.f, use_m = min_p > 0.f;
  const int C = min(a.V, has_k && top_k <= kTopMax ? top_k : kSampleTop);
  float rm = 0.f;
  double rs = 0.0;
  select_top<LT>(lr, groups, a.V, a.G, C, row_scale(T), sh.sel, rm, rs);
  SampleRow s;
  s.m = entry_value(sh.sel.list[0]);
  s.cd = 1.44269504088896340736 / (double)T;
  s.cf = fminf((float)(s.cd * (double)(1 << (kBinsLog + 11))), 1e30f);
  if (s.m == -INFINITY) {  // nothing to draw from
    if (tid == 0) finish(-1, -INFINITY);
    return;
  }
  constexpr double kOne = (double)(1ull << kWeightBits);
  auto logprob = [&](float v, unsigned long long total) {
    return (float)((v == s.m ? 0.0 : ((double)v - (double)s.m) / (double)T) - log((double)total / kOne));
  };
  // running sums over the first C, and the first of them that ...
  const unsigned long long key = tid < C ? sh.sel.list[tid] : 0ull;
  const float v = tid < C ? entry_value(key) : -INFINITY;
  const unsigned long long w = tid < C ? s.weight(v) : 0ull;
  if (tid < 4) sh.first[tid] = C;
  const unsigned long long run = block_scan(w, sh.redu[0]);
  if (tid < C) sh.run[tid] = run;
  auto first = [&](int slot, bool on) {
    const unsigned long long mk = __ballot(on && tid < C);
    if (mk && (tid & 63) == 0) atomicMin(&sh.first[slot], (tid & ~63) + __ffsll(mk) - 1);
  };
  const double min_d = use_m ? -log((double)min_p) * (double)T : INFINITY;  // max - l up to this stays
  auto stays = [&](float x) { return x == s.m || (double)s.m - (double)x <= min_d; };
  first(0, w == 0ull);
  first(1, !stays(v));
  __syncthreads();
  const unsigned long long sum_c = sh.run[C - 1], kUnknown = ~0ull;
  const int weighty = sh.first[0], n_m = sh.first[1];  // C: all of them
  const bool all = C == a.V || weighty < C;            // no weight lies behind the first C
  // the whole row's sum: of the first C exactly, of the rest from the groups' sums
  unsigned long long whole = sum_c;
  if (!all && rs != 0.0) whole += (unsigned long long)(rs * exp2(((double)rm - (double)s.m) * s.cd) * kOne);
  unsigned long long keep = all ? weighty : kUnknown, total = all ? sum_c : kUnknown;
  auto shorten = [&](int n) {  // n in [1, C]
    if ((unsigned long long)n < keep) {
      keep = n;
      total = sh.run[n - 1];
    }
  };
  bool decided = true;
  if (has_k && top_k <= C) {
    shorten(top_k);
    whole = total;
  }
  if (use_p) {
    if (!has_k || top_k <= C || all) first(2, run >= (unsigned long long)ceil((double)top_p * (double)whole));
    else decided = false;  // the sum of the first top_k is not known
    __syncthreads();
    if (sh.first[2] < C) shorten(sh.first[2] + 1);
  }
  if (use_m && n_m < C) shorten(n_m);
  // no filter ends within the first C: without any, the draw may still fall there
  if (keep == kUnknown) {
    total = whole;
    if (use_p || use_m || has_k) decided = false;
  }
  if (decided) {
    first(3, run > (unsigned long long)floor((double)u * (double)total));
    __syncthreads();
    const int i = keep == kUnknown ? sh.first[3] : min(sh.first[3], (int)keep - 1);
    if (i < C) {
      if (tid == i) finish((int)entry_id(key), logprob(v, total));
      return;
    }
  }
  __syncthreads();
  // The whole row.
  for (int i = tid; i < kBins; i += kSelThreads) {
    sh.row.mass[i] = 0;
    sh.row.count[i] = 0;
  }
  __syncthreads();
  unsigned long long mn = 0, mm = 0;
  each_of_row(lr, a.V, [&](float x, uint32_t id, bool in) {
    x = order_val(x);
    const Digits d = digits_of(s, x, id);
    if (in && d.y < (uint32_t)kBins << 11) {
      const unsigned long long wx = s.weight(x);
      if (wx) {
        atomicAdd(&sh.row.mass[d.y >> 11], wx);
        atomicAdd(&sh.row.count[d.y >> 11], 1u);
        if (use_m && stays(x)) {
          ++mn;
          mm += wx;
        }
      }
    }
  });
  __syncthreads();
  unsigned long long tn = 0, tm = 0;
  for (int i = tid; i < kBins; i += kSelThreads) {
    tn += sh.row.count[i];
    tm += sh.row.mass[i];
  }
  keep = block_reduce_sum<kSelWaves>(tn, sh.redu[0]);
  total = block_reduce_sum<kSelWaves>(tm, sh.redu[1]);
  __syncthreads();
  mn = block_reduce_sum<kSelWaves>(mn, sh.redu[0]);
  mm = block_reduce_sum<kSelWaves>(mm, sh.redu[1]);
  __syncthreads();
  // top-k, top-p, then (the shorter of it and min-p kept) the draw
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {
    unsigned long long target;
    if (step == 0) {
      if (!has_k || (unsigned long long)top_k >= keep) continue;
      target = top_k - 1;
    } else if (step == 1) {
      target = (unsigned long long)ceil((double)top_p * (double)total);
      if (!use_p) continue;
      target = target == 0 ? 0 : min(target, total) - 1;
    } else {
      if (use_m && mn < keep) total = mm;
      target = min((unsigned long long)floor((double)u * (double)total), total - 1);
    }
    const Prefix f = find_in_row(lr, a.V, s, step == 0, target, sh);
    if (step == 2) {
      if (tid == 0) finish((int)entry_id(f.key), logprob(entry_value(f.key), total));
    } else if (f.n < keep) {
      keep = f.n;
      total = f.mass;
    }
  }
}

// [error word, padded to 256][groups]
int rows_groups(int V) { return (V + kGroup - 1) / kGroup; }
size_t rows_ws_bytes(int rows, int V) { return 256 + (size_t)rows * rows_groups(V) * sizeof(float2); }

static RowsArgs rows_args(RowsArgs a, void *ws) {
  a.err = (int32_t *)ws;
  a.groups = (float2 *)((char *)ws + 256);
  a.G = rows_groups(a.V);
  a.nch = (a.V + kGrChunk - 1) / kGrChunk;
  return a;
}

template <typename Go>
static void by_type(bool bf16, Go go) {
  if (bf16) go(bf16_t{});
  else go(0.f);
}

void launch_top_logits(RowsArgs a, bool bf16, int k, int32_t *ids, float *vals, float *rest, void *ws, hipStream_t st) {
  a = rows_args(a, ws);
  by_type(bf16, [&](auto t) {
    using LT = decltype(t);
    hipLaunchKernelGGL(row_groups_kernel<LT>, dim3(a.rows * a.nch), dim3(kGrThreads), 0, st, a);
    hipLaunchKernelGGL(top_select_kernel<LT>, dim3(a.rows), dim3(kSelThreads), 0, st, a, k, ids, vals, rest);
  });
}

void launch_sample_logits(RowsArgs a, bool bf16, const SampleArgs &p, void *ws, hipStream_t st) {
  a = rows_args(a, ws);
  by_type(bf16, [&](auto t) {
    using LT = decltype(t);
    hipLaunchKernelGGL(row_groups_kernel<LT>, dim3(a.rows * a.nch), dim3(kGrThreads), 0, st, a);
    hipLaunchKernelGGL(sample_kernel<LT>, dim3(a.rows), dim3(kSelThreads), 0, st, a, p);
  });
}

}  // namespace dk
