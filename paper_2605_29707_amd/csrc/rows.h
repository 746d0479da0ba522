// Rows of logits as the row operators read them (top entries, filtered sampling,
// distillation): fp32 or bf16 values, rows `ld` elements apart, at any address a
// value may have.  NaN counts as -inf everywhere.
#pragma once
#include "common.h"

namespace dk {

constexpr float kRowLog2e = 1.4426950408889634f;

// 16 bytes of a row: 8 bf16 or 4 fp32 values
template <typename LT>
struct RowVec;
template <>
struct RowVec<bf16_t> {
  static constexpr int N = 8;
  DEVI static float get(const u32x4 &x, int e) {
    const uint32_t w = x[e >> 1];
    return __uint_as_float((e & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  DEVI static void set(u32x4 &x, int e, bf16_t v) {
    x[e >> 1] = (e & 1) ? (x[e >> 1] & 0xffffu) | ((uint32_t)v.v << 16) : (x[e >> 1] & 0xffff0000u) | v.v;
  }
  DEVI static bf16_t at(const u32x4 &x, int e) { return bf16_t{(uint16_t)(x[e >> 1] >> (16 * (e & 1)))}; }
  DEVI static bf16_t low() { return bf16_t{0xff80}; }
  static constexpr uint32_t kLow = 0xff80ff80u;  // -inf twice
};
template <>
struct RowVec<float> {
  static constexpr int N = 4;
  DEVI static float get(const u32x4 &x, int e) { return __uint_as_float(x[e]); }
  DEVI static void set(u32x4 &x, int e, float v) { x[e] = __float_as_uint(v); }
  DEVI static float at(const u32x4 &x, int e) { return __uint_as_float(x[e]); }
  DEVI static float low() { return -INFINITY; }
  static constexpr uint32_t kLow = 0xff800000u;
};

// 16 bytes at any address of a value: the wide loads and stores of this chip
// need no alignment of their own, and an odd vocabulary has rows at odd addresses.
template <typename LT>
DEVI u32x4 row_load(const LT *p) {
  u32x4 x;
  __builtin_memcpy(&x, p, 16);
  return x;
}
template <typename LT>
DEVI void row_store(LT *p, const u32x4 &x) {
  __builtin_memcpy(p, &x, 16);
}
// The row's last 16 bytes as the vector that begins `by` values later, -inf past the row's end.
template <typename LT>
DEVI u32x4 row_move_end(u32x4 x, uint32_t by) {
  constexpr int N = RowVec<LT>::N;
  constexpr uint32_t kLow = RowVec<LT>::kLow;
  if (by & (N / 2)) x = u32x4{x[2], x[3], kLow, kLow};
  if (by & (N / 4)) x = u32x4{x[1], x[2], x[3], kLow};
  if (N == 8 && (by & 1)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_alignbit(e < 3 ? x[e + 1] : kLow, x[e], 16);
  }
  return x;
}
// The vector at v0 < V of a row of V values, -inf past its end.  Where it crosses the end the row's
// last 16 bytes are loaded and moved down, in a few instructions: this code is in many loops.
template <typename LT>
DEVI u32x4 row_load_end(const LT *row, uint32_t v0, uint32_t V) {
  constexpr int N = RowVec<LT>::N;
  constexpr uint32_t kLow = RowVec<LT>::kLow;
  if (v0 + N <= V) return row_load(row + v0);
  u32x4 x = {kLow, kLow, kLow, kLow};
  if (v0 >= V) return x;
  const uint32_t by = v0 + N - V;  // values past the end
  if (V >= N) {
    x = row_move_end<LT>(row_load(row + (V - N)), by);
  } else {  // (v0 = 0, fewer values than a vector has)
#pragma unroll 1
    for (uint32_t i = V; i-- > 0;) {
      const u32x4 y = x;
      if (N == 8) {
#pragma unroll
        for (int e = 3; e >= 0; --e) x[e] = __builtin_amdgcn_alignbit(y[e], e > 0 ? y[e - 1] : 0u, 16);
      } else {
        x = u32x4{0, y[0], y[1], y[2]};
      }
      RowVec<LT>::set(x, 0, row[i]);
    }
  }
  return x;
}

// The first part of the selection order as an unsigned number: larger value,
// larger key; the zeros of both signs are equal, NaN is -inf.
DEVI uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(order_val(v) + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
DEVI float order_key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k ^ 0x80000000u) : ~k); }

// Sums and maxima of a workgroup of W waves, in a fixed order; every thread gets
// the result.  `red` holds W values and is free again after the next barrier.
template <int W, typename T>
DEVI T block_reduce_sum(T v, T *red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T s = red[0];
#pragma unroll
  for (int w = 1; w < W; ++w) s += red[w];
  return s;
}
template <int W>
DEVI float block_reduce_max(float v, float *red) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = red[0];
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, red[w]);
  return m;
}

}  // namespace dk
