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
struct SelShared {
  unsigned long long list[kListMax];  // keys: order_key of the value, complement of the id
  unsigned long long cnt[2][kSelWaves];
  int sel[kTopMax];                   // the selected groups
  int gcnt[kSelRegs * kSelWaves];
  float redf[2][kSelWaves];
  double redd[kSelWaves];
  unsigned long long redu[kSelWaves];
  uint32_t mm[2][kSelWaves];
  int n;
};

DEVI unsigned long long entry_key(float v, uint32_t id) { return ((unsigned long long)order_key(v) << 32) | (0xffffffffu - id); }
DEVI float entry_value(unsigned long long k) { return order_key_value((uint32_t)(k >> 32)); }
DEVI uint32_t entry_id(unsigned long long k) { return 0xffffffffu - (uint32_t)k; }

// the largest t with at least `want` of the workgroup's numbers >= t, two bits a
// step from the highest bit in which the numbers can differ.  count(t1, t2, t3)
// gives a wave's numbers >= each, packed by 20 bits; [lo, hi] holds them all.
template <typename Count>
DEVI uint32_t kth_largest(uint32_t lo, uint32_t hi, int want, SelShared &sh, Count count) {
  if (lo >= hi) return hi;
  int shift = (31 - __builtin_clz(lo ^ hi)) & ~1;
  uint32_t t = shift == 30 ? 0u : hi & ~((4u << shift) - 1u);
  for (int it = 0; shift >= 0; shift -= 2, it ^= 1) {
    const uint32_t t1 = t | (1u << shift), t2 = t | (2u << shift), t3 = t | (3u << shift);
    const unsigned long long c = count(t1, t2, t3);
    if ((threadIdx.x & 63) == 0) sh.cnt[it][threadIdx.x >> 6] = c;
    __syncthreads();
    unsigned long long s = 0;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) s += sh.cnt[it][w];
    const int n1 = (int)(s & 0xfffff), n2 = (int)(s >> 20 & 0xfffff), n3 = (int)(s >> 40);
    t = n3 >= want ? t3 : n2 >= want ? t2 : n1 >= want ? t1 : t;
  }
  __syncthreads();  // sh.cnt is free again
  return t;
}
DEVI unsigned long long pack3(int a, int b, int c) {
  return (unsigned long long)a | (unsigned long long)b << 20 | (unsigned long long)c << 40;
}
// a count over the workgroup, from each wave's
DEVI int block_count(int wave_n, int slot, SelShared &sh) {
  if ((threadIdx.x & 63) == 0) sh.cnt[slot][threadIdx.x >> 6] = wave_n;
  __syncthreads();
  unsigned long long s = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) s += sh.cnt[slot][w];
  __syncthreads();
  return (int)s;
}
// (min, max) over the workgroup
DEVI void block_range(uint32_t &lo, uint32_t &hi, SelShared &sh) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
  }
  if ((threadIdx.x & 63) == 0) {
    sh.mm[0][threadIdx.x >> 6] = lo;
    sh.mm[1][threadIdx.x >> 6] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    lo = min(lo, sh.mm[0][w]);
    hi = max(hi, sh.mm[1][w]);
  }
  __syncthreads();
}

// sh.list[0 .. n) in descending order (keys are distinct), n <= kListMax.  Up to 512 each
// key counts those before it; more by a bitonic network.
DEVI void sort_list(int n, SelShared &sh) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (n <= 512) {
    unsigned long long k = 0;
    int r = 0;
    if (tid < n) {
      k = sh.list[tid];
      for (int i = 0; i < n; ++i) r += sh.list[i] > k;
    }
    __syncthreads();
    if (tid < n) sh.list[r] = k;
    __syncthreads();
    return;
  }
  const int size = n <= 1024 ? 1024 : 2048;
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
      __syncthreads();
    }
}

// push of the lanes whose `on` is set; sh.n counts (past kListMax nothing is stored)
DEVI void push_list(bool on, unsigned long long key, SelShared &sh) {
  const unsigned long long mk = __ballot(on);
  if (!mk) return;
  const int lane = threadIdx.x & 63;
  int at = 0;
  if (lane == 0) at = atomicAdd(&sh.n, __popcll(mk));
  at = __builtin_amdgcn_readfirstlane(at) + __popcll(mk & ((1ull << lane) - 1));
  if (on && at < kListMax) sh.list[at] = key;
}

// The first C entries of a row, sorted, in sh.list; with REST also their complement's
// sum: max in rest_m, sum of exp((l - rest_m) / T) in rest_s.  C <= min(V, kTopMax).
template <typename LT, bool REST>
DEVI void select_top(const LT *lr, const float2 *groups, int V, int G, int C, float c, SelShared &sh, float &rest_m,
                     double &rest_s) {
  constexpr int N = RowVec<LT>::N, LPG = kGroup / N;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the groups' maxima, group i * 1024 + tid in register i
  uint32_t gk[kSelRegs];
  const int nr = (G + kSelThreads - 1) / kSelThreads;
#pragma unroll
  for (int i = 0; i < kSelRegs; ++i) {
    gk[i] = 0;  // (no value has the key 0)
    if (i < nr) {
      const int g = i * kSelThreads + tid;
      if (g < G) gk[i] = order_key(groups[g].x);
    }
  }
  const int take = min(C, G);  // groups to read
  uint32_t gt = 0;             // the key of the last of them
  int over = 0;                // of those with just this key, how many are read
  if (take < G) {
    uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int i = 0; i < kSelRegs; ++i)
      if (gk[i]) {
        lo = min(lo, gk[i]);
        hi = max(hi, gk[i]);
      }
    block_range(lo, hi, sh);
    gt = kth_largest(lo, hi, take, sh, [&](uint32_t t1, uint32_t t2, uint32_t t3) {
      int n1 = 0, n2 = 0, n3 = 0;
#pragma unroll
      for (int i = 0; i < kSelRegs; ++i)
        if (i < nr) {
          n1 += __popcll(__ballot(gk[i] >= t1));
          n2 += __popcll(__ballot(gk[i] >= t2));
          n3 += __popcll(__ballot(gk[i] >= t3));
        }
      return pack3(n1, n2, n3);
    });
    int n = 0;
#pragma unroll
    for (int i = 0; i < kSelRegs; ++i)
      if (i < nr) n += __popcll(__ballot(gk[i] > gt));
    over = take - block_count(n, 0, sh);
  }
  // Places in group order (so that sums over the groups have one order): first those
  // with the last key are counted, then the chosen ones.
  uint32_t chosen = 0;  // a bit a register
  for (int pass = take < G ? 0 : 1; pass < 2; ++pass) {
#pragma unroll
    for (int i = 0; i < kSelRegs; ++i)
      if (i < nr) {
        const bool on = pass == 0 ? gk[i] == gt : take == G ? gk[i] != 0 : gk[i] > gt || (chosen >> i & 1);
        const int n = __popcll(__ballot(on));
        if (lane == 0) sh.gcnt[i * kSelWaves + wave] = n;
      }
    __syncthreads();
    if (wave == 0) {  // exclusive running sums over (register, wave)
      int base = 0;
      for (int j0 = 0; j0 < nr * kSelWaves; j0 += 64) {
        const int n = j0 + lane < nr * kSelWaves ? sh.gcnt[j0 + lane] : 0;
        int x = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(x, o, 64);
          if (lane >= o) x += y;
        }
        if (j0 + lane < nr * kSelWaves) sh.gcnt[j0 + lane] = base + x - n;
        base += __shfl(x, 63, 64);
      }
    }
    __syncthreads();
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < kSelRegs; ++i)
      if (i < nr) {
        const bool on = pass == 0 ? gk[i] == gt : take == G ? gk[i] != 0 : gk[i] > gt || (chosen >> i & 1);
        const int at = sh.gcnt[i * kSelWaves + wave] + __popcll(__ballot(on) & below);
        if (pass == 0) {
          if (on && at < over) chosen |= 1u << i;
        } else {
          if (on) sh.sel[at] = i * kSelThreads + tid;
          if (on) chosen |= 1u << i;
        }
      }
    __syncthreads();
  }
  // their values, from memory in each pass (the caches hold them; 32 values a thread
  // in registers beside the groups' maxima spill): vector u is part u % LPG of group u / LPG
  const int nu = take * LPG;
  auto each = [&](auto f) {  // f(value, its key, id, is one)
    constexpr int U = 4;
#pragma unroll 1
    for (int u0 = 0; u0 < nu; u0 += U * kSelThreads) {
      u32x4 x[U];
      uint32_t id0[U];
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int u = u0 + q * kSelThreads + tid;
        id0[q] = 0x7fffffffu;  // past every row: no value of it counts
        if (u < nu) {
          id0[q] = (uint32_t)sh.sel[u / LPG] * kGroup + (u % LPG) * N;
          x[q] = row_load_end(lr, id0[q], V);
        }
      }
#pragma unroll
      for (int q = 0; q < U; ++q)
        if (u0 + q * kSelThreads < nu) {  // uniform
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const uint32_t id = id0[q] + e;
            const float v = RowVec<LT>::get(x[q], e);
            f(v, order_key(v), id, id < (uint32_t)V);
          }
        }
    }
  };
  // Those that can be among the first C: not behind the last group's maximum.  Where they are
  // more than the list holds, the C-th value itself, then the C-th id of that value.
  uint32_t et = gt, eid = 0xffffffffu;  // entries with a key above et, or et and an id up to eid
  for (int tries = 0;; ++tries) {
    if (tid == 0) sh.n = 0;
    __syncthreads();
    each([&](float, uint32_t k, uint32_t id, bool in) {
      push_list(in && (k > et || (k == et && id <= eid)), ((unsigned long long)k << 32) | (0xffffffffu - id), sh);
    });
    __syncthreads();
    if (sh.n <= kListMax || tries == 2) break;
    uint32_t lo = 0xffffffffu, hi = 0;
    if (tries == 0) {
      each([&](float, uint32_t k, uint32_t, bool in) {
        if (in) {
          lo = min(lo, k);
          hi = max(hi, k);
        }
      });
      block_range(lo, hi, sh);
      lo = max(lo, et);
      et = kth_largest(lo, hi, C, sh, [&](uint32_t t1, uint32_t t2, uint32_t t3) {
        int n1 = 0, n2 = 0, n3 = 0;
        each([&](float, uint32_t k, uint32_t, bool in) {
          n1 += __popcll(__ballot(in && k >= t1));
          n2 += __popcll(__ballot(in && k >= t2));
          n3 += __popcll(__ballot(in && k >= t3));
        });
        return pack3(n1, n2, n3);
      });
    } else {
      int n = 0;
      each([&](float, uint32_t k, uint32_t, bool in) { n += __popcll(__ballot(in && k > et)); });
      const int left = C - block_count(n, 0, sh);
      // the left-th smallest id, as the left-th largest of the complements
      eid = 0xfffffu - kth_largest(0, 0xfffffu, left, sh, [&](uint32_t t1, uint32_t t2, uint32_t t3) {
              int n1 = 0, n2 = 0, n3 = 0;
              each([&](float, uint32_t k, uint32_t id, bool in) {
                const uint32_t r = 0xfffffu - id;
                n1 += __popcll(__ballot(in && k == et && r >= t1));
                n2 += __popcll(__ballot(in && k == et && r >= t2));
                n3 += __popcll(__ballot(in && k == et && r >= t3));
              });
              return pack3(n1, n2, n3);
            });
    }
  }
  const int n = min(sh.n, kListMax);
  sort_list(n, sh);
  if (!REST) return;
  // The rest: the groups not read, the values not listed, the list behind C.
  float m = -INFINITY;
  float2 gs[kSelRegs];
#pragma unroll
  for (int i = 0; i < kSelRegs; ++i)
    if (i < nr) {
      const int g = i * kSelThreads + tid;
      gs[i] = g < G && !(chosen >> i & 1) ? groups[g] : make_float2(-INFINITY, 0.f);
      m = fmaxf(m, gs[i].x);
    }
  each([&](float v, uint32_t k, uint32_t id, bool in) {
    if (in && !(k > et || (k == et && id <= eid))) m = fmaxf(m, v);
  });
  if (n > C) m = fmaxf(m, entry_value(sh.list[C]));
  m = block_reduce_max<kSelWaves>(m, sh.redf[0]);
  double s = 0.0;
  if (m > -INFINITY) {  // uniform
#pragma unroll
    for (int i = 0; i < kSelRegs; ++i)
      if (i < nr && gs[i].x > -INFINITY)
        s += (double)gs[i].y * (double)__builtin_amdgcn_exp2f(fminf((gs[i].x - m) * c, 0.f));
    float t = 0.f;
    each([&](float v, uint32_t k, uint32_t id, bool in) {
      if (in && !(k > et || (k == et && id <= eid)))
        t += __builtin_amdgcn_exp2f(fminf((fmaxf(v, -INFINITY) - m) * c, 0.f));
    });
    s += t;
    for (int i = C + tid; i < n; i += kSelThreads)
      s += __builtin_amdgcn_exp2f(fminf((entry_value(sh.list[i]) - m) * c, 0.f));
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
  if (rest) select_top<LT, true>(lr, groups, a.V, a.G, k, c, sh, rm, rs);
  else select_top<LT, false>(lr, groups, a.V, a.G, k, c, sh, rm, rs);
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
  unsigned long long mass[kBins];   // of the whole row by bins
  uint32_t count[kBins];
  union {
    struct {
      unsigned long long mass[kSplit];
      uint32_t count[kSplit];
    } part;
    SelShared sel;
  };
  unsigned long long redu[2][kSelWaves];
  unsigned long long hit[4];
  int hit_i;
};

// inclusive running sum over the threads of the workgroup
DEVI unsigned long long block_scan(unsigned long long v, unsigned long long *red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  if (lane == 63) red[wave] = v;
  __syncthreads();
  unsigned long long base = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) base += w < wave ? red[w] : 0ull;
  __syncthreads();
  return base + v;
}

// Where a running sum in the order ends: after n entries of together `mass`, the last one `key`.
struct Prefix {
  unsigned long long n, mass, key;
};

// f(value, id) for every value of the row, four 16-byte loads in flight a thread
template <typename LT, typename F>
DEVI void each_of_row(const LT *lr, uint32_t V, F f) {
  constexpr int N = RowVec<LT>::N, U = 4;
  const uint32_t step = kSelThreads * N;
  uint32_t v0 = threadIdx.x * N;
  for (; v0 - threadIdx.x * N + U * step <= V; v0 += U * step) {
    u32x4 x[U];
#pragma unroll
    for (int q = 0; q < U; ++q) x[q] = row_load(lr + v0 + q * step);
#pragma unroll
    for (int q = 0; q < U; ++q)
#pragma unroll
      for (int e = 0; e < N; ++e) f(RowVec<LT>::get(x[q], e), v0 + q * step + e, true);
  }
  for (; v0 - threadIdx.x * N < V; v0 += step) {
    const u32x4 x = row_load_end(lr, v0, V);
#pragma unroll
    for (int e = 0; e < N; ++e) f(RowVec<LT>::get(x, e), v0 + e, v0 + e < V);
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
    unsigned long long *mass = level == 0 ? sh.mass : sh.part.mass;
    uint32_t *count = level == 0 ? sh.count : sh.part.count;
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
      push_list(on, entry_key(v, id), sh.sel);
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
  float T = a.temps ? a.temps[row] : 1.f, u = p.uniforms[row];
  const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  int top_k = p.top_k ? p.top_k[row] : 0;
  const bool ok = T >= 0.f && T < INFINITY && u >= 0.f && u < 1.f && top_p >= 0.f && top_p <= 1.f && min_p >= 0.f &&
                  min_p <= 1.f;
  if (!ok) {
    if (tid == 0) {
      raise_error(a.err, DEV_BAD_PARAM);
      p.tokens[row] = -1;
      if (p.logprobs) p.logprobs[row] = NAN;
    }
    return;
  }
  if (T == 0.f) {
    top_k = 1;
    T = 1.f;
  }
  const bool has_k = top_k > 0 && top_k < a.V;
  const int C = min(a.V, has_k && top_k <= kTopMax ? top_k : kSampleTop);
  float rm = 0.f;
  double rs = 0.0;
  select_top<LT, true>(lr, groups, a.V, a.G, C, row_scale(T), sh.sel, rm, rs);
  SampleRow s;
  s.m = entry_value(sh.sel.list[0]);
  s.cd = 1.44269504088896340736 / (double)T;
  s.cf = fminf((float)(s.cd * (double)(1 << (kBinsLog + 11))), 1e30f);
  if (s.m == -INFINITY) {  // nothing to draw from
    if (tid == 0) {
      p.tokens[row] = -1;
      if (p.logprobs) p.logprobs[row] = -INFINITY;
    }
    return;
  }
  // running sums over the first C; entries of no weight end them
  const unsigned long long key = tid < C ? sh.sel.list[tid] : 0ull;
  const float v = tid < C ? entry_value(key) : -INFINITY;
  const unsigned long long w = tid < C ? s.weight(v) : 0ull;
  __syncthreads();  // (the list's memory is used again below)
  const unsigned long long run = block_scan(w, sh.redu[0]);
  auto at_thread = [&](int t) {  // `run` of thread t
    if (tid == t) sh.hit[3] = run;
    __syncthreads();
    const unsigned long long x = sh.hit[3];
    __syncthreads();
    return x;
  };
  // first thread (< C) whose `on` is set, C if none
  auto first = [&](bool on) {
    if (tid == 0) sh.hit_i = C;
    __syncthreads();
    const unsigned long long mk = __ballot(on && tid < C);
    if (mk && (tid & 63) == 0) atomicMin(&sh.hit_i, (tid & ~63) + __ffsll((unsigned long long)mk) - 1);
    __syncthreads();
    const int x = sh.hit_i;
    __syncthreads();
    return x;
  };
  const unsigned long long sum_c = at_thread(C - 1);
  const int weighty = first(w == 0ull);          // entries with a weight among the first C
  const bool all = C == a.V || weighty < C;      // no weight lies behind them
  // the whole row's sum: of the first C exactly, of the rest from the groups' sums
  double rest = 0.0;
  if (!all && rs != 0.0) rest = rs * exp2((rm - (double)s.m) * s.cd) * (double)(1ull << kWeightBits);
  const bool use_p = top_p < 1.f, use_m = min_p > 0.f;
  const double min_d = use_m ? -log((double)min_p) * (double)T : INFINITY;  // max - l up to this stays
  auto stays = [&](float x) { return x == s.m || (double)s.m - (double)x <= min_d; };
  const unsigned long long kUnknown = ~0ull;
  unsigned long long keep = all ? weighty : kUnknown, keep_mass = all ? sum_c : kUnknown;
  unsigned long long whole = all ? sum_c : (unsigned long long)((double)sum_c + rest);
  bool decided = true;
  // prefix of n <= C entries
  auto shorten = [&](int n) {
    if ((unsigned long long)n < keep) {
      keep = n;
      keep_mass = at_thread(n - 1);
    }
  };
  if (has_k && top_k <= C) {
    shorten(top_k);
    whole = keep_mass;
  }
  const bool whole_known = !has_k || top_k <= C || all;
  if (use_p) {
    if (whole_known) {
      const unsigned long long want = (unsigned long long)ceil((double)top_p * (double)whole);
      const int n = first(run >= want) + 1;
      if (n <= C) shorten(n);
    } else {
      decided = false;
    }
  }
  if (use_m) {
    const int n = first(!stays(v));
    if (n < C) shorten(n);
  }
  // keep unknown: no filter ends within the first C.  Without any, the draw may still fall there.
  unsigned long long total = keep_mass;
  if (keep == kUnknown) {
    total = whole;
    if (use_p || use_m || has_k) decided = false;
  }
  if (decided) {
    const unsigned long long target = (unsigned long long)floor((double)u * (double)total);
    int i = first(run > target);
    if (keep != kUnknown) i = min(i, (int)keep - 1);
    if (i < C) {
      if (tid == i) {
        p.tokens[row] = (int32_t)entry_id(key);
        if (p.logprobs)
          p.logprobs[row] =
              v == s.m ? (float)-log((double)total / (double)(1ull << kWeightBits))
                       : (float)(((double)v - (double)s.m) / (double)T - log((double)total / (double)(1ull << kWeightBits)));
      }
      return;
    }
  }
  // The whole row.
  for (int i = tid; i < kBins; i += kSelThreads) {
    sh.mass[i] = 0;
    sh.count[i] = 0;
  }
  __syncthreads();
  unsigned long long mn = 0, mm = 0;
  each_of_row(lr, a.V, [&](float x, uint32_t id, bool in) {
    x = order_val(x);
    const Digits d = digits_of(s, x, id);
    if (in && d.y < (uint32_t)kBins << 11) {
      const unsigned long long wx = s.weight(x);
      if (wx) {
        atomicAdd(&sh.mass[d.y >> 11], wx);
        atomicAdd(&sh.count[d.y >> 11], 1u);
        if (stays(x)) {
          ++mn;
          mm += wx;
        }
      }
    }
  });
  __syncthreads();
  unsigned long long tn = 0, tm = 0;
  for (int i = tid; i < kBins; i += kSelThreads) {
    tn += sh.count[i];
    tm += sh.mass[i];
  }
  keep = block_reduce_sum<kSelWaves>(tn, sh.redu[0]);
  keep_mass = block_reduce_sum<kSelWaves>(tm, sh.redu[1]);
  __syncthreads();
  mn = block_reduce_sum<kSelWaves>(mn, sh.redu[0]);
  mm = block_reduce_sum<kSelWaves>(mm, sh.redu[1]);
  __syncthreads();
  if (has_k && (unsigned long long)top_k < keep) {
    const Prefix f = find_in_row(lr, a.V, s, true, top_k - 1, sh);
    keep = f.n;
    keep_mass = f.mass;
  }
  if (use_p) {
    const unsigned long long want = (unsigned long long)ceil((double)top_p * (double)keep_mass);
    if (want > 0) {
      const Prefix f = find_in_row(lr, a.V, s, false, min(want, keep_mass) - 1, sh);
      if (f.n < keep) {
        keep = f.n;
        keep_mass = f.mass;
      }
    }
  }
  if (use_m && mn < keep) {
    keep = mn;
    keep_mass = mm;
  }
  const unsigned long long target = min((unsigned long long)floor((double)u * (double)keep_mass), keep_mass - 1);
  const Prefix f = find_in_row(lr, a.V, s, false, target, sh);
  if (tid == 0) {
    const float x = entry_value(f.key);
    p.tokens[row] = (int32_t)entry_id(f.key);
    if (p.logprobs)
      p.logprobs[row] = (float)((x == s.m ? 0.0 : ((double)x - (double)s.m) / (double)T) -
                                log((double)keep_mass / (double)(1ull << kWeightBits)));
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
