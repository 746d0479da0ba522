// Selection within a row of logits, from the maxima and sums of its groups of 32 ids.
//
//   The first C entries of a row in the order (value desc, id asc) lie in the first C
//   groups in the order (maximum desc, group asc).  (An entry outside them is behind
//   the maximum of each of them.)  So a row of V values is cut to 32 C of them after
//   one pass over it, whatever its values.
//
// One workgroup of eight waves a row.  What bounds it is the chain of its steps: every
// instruction that all waves repeat takes 4 cycles a wave on its SIMD.  16 waves a row took 9 us for
// a row of 128 groups where four take 5; of four and eight, four are slower for wide rows (16 rows
// of 151936 logits 14.8 us against 11.9, 960 rows 86 against 48).
#pragma once
#include "kernels.h"
#include "rows.h"

namespace dk {

constexpr int kGroup = 32;         // ids a group
constexpr int kSelLog = 9, kSelThreads = 1 << kSelLog;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kTopMax = 1024;      // entries at most
constexpr int kListMax = 2048;     // candidates sorted in LDS
constexpr int kSelMax = 2048;      // groups read
constexpr uint32_t kIdMask = 0xfffffu;
static_assert(kRowsMaxVocab <= kIdMask, "ids in 20 bits");
constexpr int rows_groups(int V) { return (V + kGroup - 1) / kGroup; }

// log2(e) / T: finite, since T >= 1e-30
DEVI float row_scale(float T) { return kRowLog2e / T; }

// An entry as a number whose order is the entries': order_key of the value, complement of the id.
DEVI unsigned long long entry_key(float v, uint32_t id) {
  return ((unsigned long long)order_key(v) << 32) | (0xffffffffu - id);
}
DEVI float entry_value(unsigned long long k) { return order_key_value((uint32_t)(k >> 32)); }
DEVI uint32_t entry_id(unsigned long long k) { return 0xffffffffu - (uint32_t)k; }

// inclusive running sum over the W waves' threads; `red` is free again after the next barrier
template <int W, typename T>
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
#pragma unroll
  for (int w = 0; w < W - 1; ++w) base += w < wave ? red[w] : T(0);
  return base + v;
}

// list[0 .. n), n <= kListMax, in descending order (keys are distinct, their upper halves in [lo, hi]), by
// W waves.  Up to 128 a key counts those before it, by several threads where there are enough.  More
// are dealt into as many equal parts of [lo, hi] as there are threads, and a key counts those before it in
// its part (270 keys in 2.5K cycles; all against all, 11K beside another workgroup).  The ids follow in the
// parts, and bf16 values leave out the bits they do not have, so that equal values fall into many.  Where a part
// holds many all the same, a bitonic network, whose short steps stay within a wave and need no barrier (2048 keys: 20 us).
// Rows that are listed whole, without a cut of the groups (up to 2048 ids, unless C is less than their groups), always
// come to that: their keys lie over the whole range, a part of it is about a binade, and several hundred values have one
// (16 rows of 2048 logits, top-p 38 us and 64 entries 32; of 2049 17.7 and 12.4; of 1000 28 and 22).
constexpr int kPartMax = 64;
template <int W, typename LT>
DEVI void sort_list(int n, unsigned long long *list, uint32_t lo, uint32_t hi, uint32_t *hist, uint32_t *red) {
  constexpr int kThreads = 64 * W, kEach = kListMax / kThreads, kLog = W == 16 ? 10 : 9;
  static_assert(W == 8 || W == 16, "log2 of the threads");
  const int tid = threadIdx.x;
  if (tid == 0) list[n] = 0;  // (before every key; the place behind the longest list is there)
  hist[tid] = 0;
  __syncthreads();
  if (n <= 128) {
    int lg = 0;
    while (lg < 4 && (n << (lg + 1)) <= kThreads) ++lg;
    const int i = tid >> lg, parts = 1 << lg;
    const unsigned long long k = i < n ? list[i] : ~0ull;
    int r = 0;
#pragma unroll 4
    for (int q = (tid & ~63) >> lg < n ? 2 * (tid & (parts - 1)) : n; q < n; q += 2 * parts)  // (a wave without keys: none)
      r += (list[q] > k) + (list[q + 1] > k);
    for (int o = 1; o < parts; o <<= 1) r += __shfl_xor(r, o, 64);
    __syncthreads();
    if (i < n && (tid & (parts - 1)) == 0) list[r] = k;
    __syncthreads();
    return;
  }
  constexpr int kDrop = RowVec<LT>::N == 8 ? 16 : 0;
  constexpr uint32_t kIds = (1u << 19) - 1;
  static_assert(kRowsMaxVocab <= (int)kIds, "ids in 19 bits");
  const unsigned long long range = (unsigned long long)((hi >> kDrop) - (lo >> kDrop)) << 19 | kIds;
  const int shift = 64 - kLog - __builtin_clzll(range);
  unsigned long long k[kEach];
  int part[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int i = j * kThreads + tid;
    if (i < n) {
      k[j] = list[i];
      const unsigned long long at = (unsigned long long)(((uint32_t)(k[j] >> 32) >> kDrop) - (lo >> kDrop)) << 19 | ((uint32_t)k[j] & kIds);
      part[j] = kThreads - 1 - (int)(at >> shift);
      atomicAdd(&hist[part[j]], 1u);
    }
  }
  __syncthreads();
  const uint32_t c = hist[tid], before = block_scan<W>(c, red) - c;
  const bool many = __syncthreads_or(c > kPartMax);
  if (!many) {
    hist[tid] = before;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (j * kThreads + tid < n) list[atomicAdd(&hist[part[j]], 1u)] = k[j];  // (then hist has the parts' ends)
    __syncthreads();
    int r[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (j * kThreads + tid < n) {
        r[j] = part[j] ? hist[part[j] - 1] : 0;
        for (int q = r[j]; q < (int)hist[part[j]]; ++q) r[j] += list[q] > k[j];
      }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (j * kThreads + tid < n) list[r[j]] = k[j];
    __syncthreads();
    return;
  }
  int size = 256;
  while (size < n) size <<= 1;
  for (int i = n + tid; i < size; i += kThreads) list[i] = 0;
  __syncthreads();
  for (int len = 2; len <= size; len <<= 1)
    for (int step = len >> 1; step >= 1; step >>= 1) {
      for (int t = tid; t < size / 2; t += kThreads) {
        const int i = (t & ~(step - 1)) * 2 + (t & (step - 1)), j = i + step;
        const unsigned long long x = list[i], y = list[j];
        if ((x < y) == ((i & len) == 0)) {
          list[i] = y;
          list[j] = x;
        }
      }
      // up to steps of 64 each run of 64 pairs is a wave's own
      if (step > 64 || (step == 1 && len >= 128)) __syncthreads();
      else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    }
  __syncthreads();
}

struct SelShared {
  alignas(16) unsigned long long list[kListMax + 2];  // keys
  int sel[kSelMax];                   // the selected groups
  uint32_t hist[kSelThreads];
  uint32_t wave[2][kSelWaves];
  float redf[kSelWaves];
  double redd[kSelWaves];
  uint32_t hit[3];
  int n;
};

// Those with a key above `key`, or with this key and an id up to `id`.
struct Cut {
  uint32_t key, id;
  DEVI bool has(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= id); }
};

// A cut that takes at least `want` items, and at most `cap` (want <= cap): by counts in 512
// equal parts of [lo, hi], which holds the key of the want-th, and again of the part that holds
// it while there are more than `cap` up to its end; among equal keys the same by ids.
// each(f) calls f(key, id) for every item.  sh.hist is clear, before and after.
template <typename Each>
DEVI Cut cut_at(uint32_t lo, uint32_t hi, int want, int cap, SelShared &sh, Each each) {
  const int tid = threadIdx.x;
  bool by_id = false;
  uint32_t key = 0;
  int above = 0;  // items beyond hi
  while (true) {
    const uint32_t range = hi - lo;
    const int shift = range < kSelThreads ? 0 : 32 - kSelLog - __builtin_clz(range);
    each([&](uint32_t k, uint32_t id) {
      const uint32_t x = by_id ? kIdMask - id : k;
      if (x >= lo && x <= hi && (!by_id || k == key)) atomicAdd(&sh.hist[kSelThreads - 1 - ((x - lo) >> shift)], 1u);
    });
    __syncthreads();
    const int c = sh.hist[tid];
    sh.hist[tid] = 0;  // (for the next counts, after a barrier)
    const int n = above + block_scan<kSelWaves, uint32_t>(c, sh.wave[0]);
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

// The first C entries of a row, sorted, in sh.list; where it is wanted, of the others the largest value
// (rest_m) and the sum of exp((l - rest_m) / T) (rest_s).  C <= min(V, kTopMax); a thread holds NR groups.
template <typename LT, int NR>
DEVI void select_top(const LT *lr, const float2 *groups, int V, int G, int C, float c, bool want_rest, SelShared &sh,
                     float &rest_m, double &rest_s) {
  constexpr int N = RowVec<LT>::N, LPG = kGroup / N;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // the groups, group i * 512 + tid in register i (loads at clamped places, so that none waits for another)
  uint32_t gk[NR];
  float gs[NR];
  const int nr = (G + kSelThreads - 1) / kSelThreads;
  float2 g2[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) g2[i] = groups[min(i * kSelThreads + tid, G - 1)];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const bool in = i * kSelThreads + tid < G;
    gk[i] = in ? order_key(g2[i].x) : 0;  // (no value has the key 0, which is the key of a NaN)
    gs[i] = in ? g2[i].y : 0.f;
  }
  uint32_t hi = 0;
#pragma unroll
  for (int i = 0; i < NR; ++i) hi = max(hi, gk[i]);
  // Bounds of the C-th group's key.  From below, where every thread has a group: the least of 512 / s
  // maxima, each of the groups of s threads, with 512 / s >= C of them; or the least key of all.
  uint32_t lo = hi;
  if (C <= kSelThreads && G >= kSelThreads) {
    for (int s = 1; s < 64 && kSelThreads / (2 * s) >= C; s <<= 1) lo = max(lo, (uint32_t)__shfl_xor((int)lo, s, 64));
  } else {
    lo = 0xfffffffeu;
#pragma unroll
    for (int i = 0; i < NR; ++i) lo = min(lo, gk[i] - 1u);
    lo += 1u;
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
  sh.hist[tid] = 0;
  if (tid == 0) sh.n = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    lo = min(lo, sh.wave[0][w]);
    hi = max(hi, sh.wave[1][w]);
  }
  auto every_group = [&](auto f) {
#pragma unroll
    for (int i = 0; i < NR; ++i)
      if (i < nr) f(gk[i], (uint32_t)(i * kSelThreads + tid));
  };
  Cut gc = {1, 0xffffffffu};
  if (C < G) gc = cut_at(lo, hi, C, kSelMax, sh, every_group);
  // their list, by threads
  uint32_t chosen = 0;
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (gc.has(gk[i], i * kSelThreads + tid)) chosen |= 1u << i;
  const int mine = __popc(chosen);
  __syncthreads();
  const int upto = block_scan<kSelWaves, uint32_t>(mine, sh.wave[0]);
  int at = upto - mine;
  for (uint32_t b = chosen; b; b &= b - 1) sh.sel[at++] = (__ffs(b) - 1) * kSelThreads + tid;
  if (tid == kSelThreads - 1) sh.hit[0] = upto;
  __syncthreads();
  const int nsel = sh.hit[0];
  // Their values: vector u is part u % LPG of group u / LPG.  A thread's first two stay in registers from
  // pass to pass; where there are more, each pass loads them again (the caches hold them; all of them
  // in registers make the code several times as long).  That is 256 groups of bf16 or 128 of fp32: a cut takes a
  // few more groups than C, so that C = 256 and 128 are just past it.
  const int nu = nsel * LPG;
  constexpr int U = 2;
  u32x4 x[U], y[U];
  uint32_t ix[U], iy[U];
  auto load = [&](int u0, u32x4 (&z)[U], uint32_t (&iz)[U]) {
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int u = u0 + q * kSelThreads + tid;
      iz[q] = (uint32_t)sh.sel[min(u, nu - 1) / LPG] * kGroup + (u % LPG) * N;
      z[q] = row_load_end(lr, iz[q], V);
      if (u >= nu) iz[q] = 0x7fffffffu;  // past every row: no value of it counts
    }
  };
  load(0, x, ix);
  bool held = true;
  auto every_vec = [&](auto f) {  // f(vector, its first id)
    if (!held) load(0, x, ix);
    held = nu <= U * kSelThreads;
#pragma unroll 1
    for (int u0 = 0;;) {
      u0 += U * kSelThreads;
      if (u0 < nu) load(u0, y, iy);
#pragma unroll
      for (int q = 0; q < U; ++q)
        if (ix[q] < (uint32_t)V) f(x[q], ix[q]);
      if (u0 >= nu) break;
#pragma unroll
      for (int q = 0; q < U; ++q) {
        x[q] = y[q];
        ix[q] = iy[q];
      }
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
  for (bool cut = C >= G && V > kListMax;; cut = true) {  // (no cut of the groups: every value)
    if (cut) {
      ec = cut_at(ec.key, hi, C, kListMax, sh, every_value);
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
  sort_list<kSelWaves, LT>(n, sh.list, ec.key, hi, sh.hist, sh.wave[0]);
  if (!want_rest) return;
  // The rest: the groups not read, the values not listed, the list behind C.
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (!(chosen >> i & 1)) m = fmaxf(m, order_key_value(gk[i]));
  if (n > C) m = fmaxf(m, entry_value(sh.list[C]));
  m = block_reduce_max<kSelWaves>(m, sh.redf);
  double s = 0.0;
  if (m > -INFINITY) {  // uniform
    float t = 0.f;
    // (m = +inf: the difference of its equals is NaN and counts as 0)
    auto add = [&](float v, float by) { t += by * __builtin_amdgcn_exp2f(fminf((v - m) * c, 0.f)); };
#pragma unroll
    for (int i = 0; i < NR; ++i)
      add(order_key_value(gk[i]), chosen >> i & 1 ? 0.f : gs[i]);
    s = t;
    t = 0.f;
    every_vec([&](const u32x4 &y, uint32_t id) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = order_val(RowVec<LT>::get(y, e));
        if (id + e < (uint32_t)V && !ec.has(order_key(v), id + e)) add(v, 1.f);
      }
    });
    for (int i = C + tid; i < n; i += kSelThreads) add(entry_value(sh.list[i]), 1.f);
    s += t;
  }
  rest_m = m;
  rest_s = block_reduce_sum<kSelWaves>(s, sh.redd);
}

// f(integral constant): the groups a thread holds, by the vocabulary
template <typename F>
void by_vocab(int V, F f) {
  const int per = (rows_groups(V) + kSelThreads - 1) / kSelThreads;
  if (per <= 2) f(std::integral_constant<int, 2>{});
  else if (per <= 10) f(std::integral_constant<int, 10>{});
  else f(std::integral_constant<int, 20>{});
}
static_assert(kRowsMaxVocab <= 20 * kSelThreads * kGroup, "the groups of the largest vocabulary in 20 registers a thread");

}  // namespace dk
