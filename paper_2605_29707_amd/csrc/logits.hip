// The top entries of rows of logits: one pass over a row for the maximum and the sum of exp of
// its groups of 32 ids, then a workgroup a row that selects from those (select.h).
//   groups  bound by the logits' bytes: 16-byte loads, a group in the registers of 4 (bf16)
//           or 8 (fp32) lanes (960 rows of 151936 bf16 logits 63.6 us, 4.6 TB/s)
//   top     the first C groups' values in registers, those that can be among the first C entries
//           sorted in LDS; the sum of the rest from the other groups' sums and the registers, never as
//           a total less the entries.  At few rows bound by the chain of its steps (one row of 128 groups
//           6.8 us, 16 of 4748 12), at many by their instructions (960 rows, 256 entries 42 us)
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "select.h"

namespace dk {

constexpr int kGrThreads = 256;
constexpr int kGrChunk = 8192;  // ids a workgroup of the first launch

// (max, sum of exp((l - max) / T)) of every group of every row
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

template <typename LT, int NR>
__global__ __launch_bounds__(kSelThreads) void top_select_kernel(RowsArgs a, int k, int32_t *__restrict__ ids,
                                                                 float *__restrict__ vals, float *__restrict__ rest) {
  __shared__ SelShared sh;
  const int row = blockIdx.x, tid = threadIdx.x;
  float rm = 0.f;
  double rs = 0.0;
  select_top<LT, NR>((const LT *)a.logits + (size_t)row * a.ld, a.groups + (size_t)row * a.G, a.V, a.G, k, row_scale(a.T),
                     rest != nullptr, sh, rm, rs);
  for (int i = tid; i < k; i += kSelThreads) {
    const unsigned long long key = sh.list[i];
    ids[(size_t)row * k + i] = (int32_t)entry_id(key);
    vals[(size_t)row * k + i] = entry_value(key);
  }
  if (rest && tid == 0)
    rest[row] = rs == 0.0 ? -INFINITY : rm == INFINITY ? INFINITY : (float)((double)rm / (double)a.T + log(rs));
}

size_t rows_ws_bytes(int rows, int V) { return 256 + (size_t)rows * rows_groups(V) * sizeof(float2); }

// [error word, padded to 256][groups]
RowsArgs launch_row_groups(RowsArgs a, bool bf16, void *ws, hipStream_t st) {
  a.err = (int32_t *)ws;
  a.groups = (float2 *)((char *)ws + 256);
  a.G = rows_groups(a.V);
  a.nch = (a.V + kGrChunk - 1) / kGrChunk;
  const dim3 grid(a.rows * a.nch), block(kGrThreads);
  if (bf16) hipLaunchKernelGGL(row_groups_kernel<bf16_t>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(row_groups_kernel<float>, grid, block, 0, st, a);
  return a;
}

void launch_top_logits(RowsArgs a, bool bf16, int k, int32_t *ids, float *vals, float *rest, void *ws, hipStream_t st) {
  a = launch_row_groups(a, bf16, ws, st);
  by_vocab(a.V, [&](auto nr) {
    constexpr int NR = decltype(nr)::value;
    if (bf16)
      hipLaunchKernelGGL((top_select_kernel<bf16_t, NR>), dim3(a.rows), dim3(kSelThreads), 0, st, a, k, ids, vals, rest);
    else
      hipLaunchKernelGGL((top_select_kernel<float, NR>), dim3(a.rows), dim3(kSelThreads), 0, st, a, k, ids, vals, rest);
  });
}

}  // namespace dk
