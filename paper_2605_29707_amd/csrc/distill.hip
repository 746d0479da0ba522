// Distillation from a teacher's top entries: loss and gradient.
//
// A row has V student logits l and k teacher entries (id i, logit t_i), with the
// log-sum-exp rest_t of the teacher's other ids (-inf when it is not given).  Both
// distributions are taken over k + 1 buckets, the entries and one bucket of every
// other id:
//   p = softmax(t_1 / T, .., t_k / T, rest_t)
//   q_i = exp(l_i / T) / Z,  q_rest = R / Z,  R = sum_{v not an entry} exp(l_v / T),
//   Z = R + sum_i exp(l_i / T)
//   row_loss = T^2 (sum_i p_i log(p_i / q_i) + p_rest log(p_rest / q_rest))
//   loss = sum_r w_r row_loss_r / W,  W = sum_r w_r
//   dloss/dl_i = T w_r / W (q_i - p_i)
//   dloss/dl_v = T w_r / W (exp(l_v / T) / R) (q_rest - p_rest),  v not an entry
// R is summed over the other ids alone, never as a total less the entries, so that
// it keeps its precision where the entries hold nearly everything.
//
// Three launches:
//   part  (row, chunk of the vocabulary): max and sum of exp of the chunk's values that
//         are no entries (a bit each in LDS marks the entries), and the entries' values
//   row   a workgroup a row: R, Z, the loss and the gradients of the entries
//   grad  (row, chunk): the gradient, the entries' own through LDS; its last workgroup
//         adds the rows' losses.  Without a gradient that workgroup is all there is.
#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace dk {

constexpr int kDsThreads = 256;
constexpr int kDsChunk = 4096;  // vocabulary ids a workgroup
constexpr int kDsWaves = kDsThreads / 64;
constexpr int kDsMaxK = 1024;   // entries at most

template <typename LT>
constexpr int kDsVecs = kDsChunk / kDsThreads / RowVec<LT>::N;

// this thread's vectors of chunk ch: vector q at ids id0 + q * step
template <typename LT>
DEVI void ds_load(const LT *row, uint32_t c0, uint32_t V, u32x4 (&x)[kDsVecs<LT>]) {
  constexpr int N = RowVec<LT>::N;
  if (c0 + kDsChunk <= V) {  // workgroup-uniform: every load goes out at once
#pragma unroll
    for (int q = 0; q < kDsVecs<LT>; ++q) x[q] = row_load(row + c0 + (q * kDsThreads + threadIdx.x) * N);
  } else {
#pragma unroll
    for (int q = 0; q < kDsVecs<LT>; ++q) x[q] = row_load_end(row, c0 + (q * kDsThreads + threadIdx.x) * N, V);
  }
}

// a weight that counts: not negative, finite; anything else counts as 0
DEVI float ds_weight(float w) { return w >= 0.f && w < INFINITY ? w : 0.f; }

// the N bits of the vector at in-chunk place `at` (a multiple of N)
template <int N>
DEVI uint32_t ds_bits(const uint32_t *bits, uint32_t at) {
  return (bits[at >> 5] >> (at & 31)) & ((1u << N) - 1u);
}

// (1) One chunk of one row.  An id given twice, or outside [-1, V), is marked by a NaN
// (as its max: errors are raised by the next launch, since this one clears the error
// word).  The workgroup after the last chunk adds the rows' weights.
// Bound by the logits' bytes: 240 rows of 151936 fp32 logits 39 us, 480 of as many bf16 34 us (39 with the ids
// loaded after the values, on which they then wait, and the entries' values by a load of their own).
template <typename LT>
__global__ __launch_bounds__(kDsThreads) void distill_part_kernel(DistillArgs a, int chunks) {
  constexpr int N = RowVec<LT>::N, NV = kDsVecs<LT>;
  const int row = blockIdx.x / a.nch, ch = blockIdx.x % a.nch, tid = threadIdx.x;
  __shared__ uint32_t bits[kDsChunk / 32];
  __shared__ uint16_t entry[kDsChunk];  // which one, where there is a bit
  __shared__ float red[2][kDsWaves];
  __shared__ double redw[2][kDsWaves];
  __shared__ int bad;
  if ((int)blockIdx.x == chunks) {
    double W = 0.0, odd = 0.0;
    for (int r = tid; r < a.rows; r += kDsThreads) {
      const float w = a.weights ? a.weights[r] : 1.f;
      if (ds_weight(w) == w) W += w;
      else odd = 1.0;
    }
    W = block_reduce_sum<kDsWaves>(W, redw[0]);
    odd = block_reduce_sum<kDsWaves>(odd, redw[1]);
    if (tid == 0) {
      *a.err = 0;
      a.wsum[0] = W;
      a.wsum[1] = odd;
    }
    return;
  }
  const uint32_t c0 = (uint32_t)ch * kDsChunk, V = a.V;
  const LT *lr = (const LT *)a.logits + (size_t)row * a.ld;
  const size_t r0 = (size_t)row * a.k;
  int id = a.ids[r0 + min(tid, a.k - 1)];  // before the values: loads end in order
  u32x4 x[NV];
  ds_load<LT>(lr, c0, V, x);
  if (tid < kDsChunk / 32) bits[tid] = 0;
  if (tid == 0) bad = 0;
  __syncthreads();
  for (int i = tid; i < a.k;) {
    const uint32_t at = (uint32_t)id - c0;
    if (id >= 0 && id < a.V) {
      if (at < kDsChunk) {
        const uint32_t bit = 1u << (at & 31);
        if (atomicOr(&bits[at >> 5], bit) & bit) bad = 1;
        entry[at] = (uint16_t)i;
      }
    } else if (ch == 0 && id != -1) {
      bad = 1;
    }
    i += kDsThreads;
    if (i < a.k) id = a.ids[r0 + i];
  }
  __syncthreads();
  float m = -INFINITY;
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    const uint32_t mine = ds_bits<N>(bits, (q * kDsThreads + tid) * N);
    if (mine) {  // few lanes: the entries out of the sum
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (mine >> e & 1) {
          a.z[r0 + entry[(q * kDsThreads + tid) * N + e]] = order_val(RowVec<LT>::get(x[q], e));
          RowVec<LT>::set(x[q], e, RowVec<LT>::low());
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, RowVec<LT>::get(x[q], e));
  }
  m = block_reduce_max<kDsWaves>(m, red[0]);
  const float ref = m == -INFINITY ? 0.f : m;
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < NV; ++q)
#pragma unroll
    for (int e = 0; e < N; ++e)
      s += __builtin_amdgcn_exp2f((order_val(RowVec<LT>::get(x[q], e)) - ref) * a.c);
  s = block_reduce_sum<kDsWaves>(s, red[1]);
  if (tid == 0) a.part[(size_t)row * a.nch + ch] = make_float2(bad ? NAN : m, s);
}

// maxima (of NF values) and sums (of ND) over the workgroup, one barrier each; every thread gets them
template <int NF>
DEVI void block_maxima(float (&v)[NF], float (*red)[kDsWaves]) {
#pragma unroll
  for (int i = 0; i < NF; ++i) v[i] = wave_max(v[i]);
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < NF; ++i) red[i][threadIdx.x >> 6] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NF; ++i)
#pragma unroll
    for (int w = 0; w < kDsWaves; ++w) v[i] = fmaxf(v[i], red[i][w]);
}
template <int ND>
DEVI void block_sums(double (&v)[ND], double (*red)[kDsWaves]) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
#pragma unroll
    for (int i = 0; i < ND; ++i) v[i] += __shfl_xor(v[i], o, 64);
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < ND; ++i) red[i][threadIdx.x >> 6] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ND; ++i) {
    v[i] = 0.0;
#pragma unroll
    for (int w = 0; w < kDsWaves; ++w) v[i] += red[i][w];
  }
}

// (2) One row, in 64 bits: a few hundred values, and differences of logarithms.  Bound by its chain of
// steps: its loads go out together, an entry's exponentials are formed once, and three barriers
// part the maxima, the sums and the loss (15 rows 5.7 us, 480 6.7; 240 rows 6.2, 7.2 with a barrier for each of them).
__global__ __launch_bounds__(kDsThreads) void distill_row_kernel(DistillArgs a) {
  constexpr int kPer = kDsMaxK / kDsThreads;
  const int row = blockIdx.x, tid = threadIdx.x;
  __shared__ float redf[4][kDsWaves];
  __shared__ double red[4][kDsWaves];
  const float2 *part = a.part + (size_t)row * a.nch;
  const size_t r0 = (size_t)row * a.k;
  float *z = a.z + r0;
  // entry i of thread i % 256: student's and teacher's logit, -inf where there is none
  float zi[kPer], ti[kPer];
  uint32_t used = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    zi[j] = ti[j] = -INFINITY;
    const int i = j * kDsThreads + tid;
    if (i < a.k) {
      const int id = a.ids[r0 + i];
      const float zv = z[i], tv = a.t_vals[r0 + i];
      if (id >= 0 && id < a.V) {  // (another one's z is not set)
        used |= 1u << j;
        zi[j] = zv;
        ti[j] = order_val(tv);
      }
    }
  }
  const double W = a.wsum[0], odd_weights = a.wsum[1];
  const float w = ds_weight(a.weights ? a.weights[row] : 1.f), rt = a.t_rest ? order_val(a.t_rest[row]) : -INFINITY;
  // the first chunks' pairs, one a thread; the others below
  const float2 p0 = tid < a.nch ? part[tid] : make_float2(-INFINITY, 0.f);
  const double inv_t = 1.0 / (double)a.T;
  // maxima: the other ids', the entries', the teacher's; whether an id was bad
  float mx[4] = {p0.x, -INFINITY, -INFINITY, p0.x != p0.x ? 1.f : 0.f};
  for (int c = kDsThreads + tid; c < a.nch; c += kDsThreads) {
    const float x = part[c].x;
    mx[3] = x != x ? 1.f : mx[3];
    mx[0] = fmaxf(mx[0], x);
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    mx[1] = fmaxf(mx[1], zi[j]);
    mx[2] = fmaxf(mx[2], ti[j]);
  }
  mx[0] = fmaxf(mx[0], -INFINITY);  // (a NaN is not a maximum)
  block_maxima(mx, redf);
  const float mr = mx[0], m = fmaxf(mx[0], mx[1]);
  const bool bad = mx[3] != 0.f;
  // The teacher's logits over T relative to the largest of them and the rest: differences first, since t / T alone may
  // be 1e38, where one step is more than the differences.  (Products and sums contract: without the minimum
  // what rounds to 0 could be a step above it.)
  const double te = (double)mx[2] * inv_t, tm = fmax(te, (double)rt);
  const bool by_rest = rt > te;
  auto teacher = [&](float t) { return by_rest ? fmin((double)t * inv_t - rt, 0.0) : ((double)t - mx[2]) * inv_t; };
  const double tr = by_rest ? 0.0 : fmin(rt - te, 0.0);
  const bool none = tm == -INFINITY;  // the teacher says nothing of this row
  const bool lost = bad || m == INFINITY || tm == INFINITY;  // its loss and gradient are NaN
  // sums relative to the maxima: R / exp(mr / T), the entries' part of Z / exp(m / T), the teacher's P
  double e[kPer], pe[kPer], sum[3] = {0.0, 0.0, 0.0};
  if (p0.x != -INFINITY) sum[0] = (double)p0.y * exp(((double)p0.x - mr) * inv_t);  // (NaN in a row of +inf)
  for (int c = kDsThreads + tid; c < a.nch; c += kDsThreads) {
    const float2 p = part[c];
    if (p.x != -INFINITY) sum[0] += (double)p.y * exp(((double)p.x - mr) * inv_t);
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    e[j] = pe[j] = 0.0;
    if (j * kDsThreads < a.k) {  // uniform
      if (zi[j] != -INFINITY) e[j] = exp(((double)zi[j] - m) * inv_t);
      if (ti[j] != -INFINITY) pe[j] = exp(teacher(ti[j]));
      sum[1] += e[j];
      sum[2] += pe[j];
    }
  }
  block_sums(sum, red);
  const double R = sum[0], P = sum[2] + (rt != -INFINITY ? exp(tr) : 0.0);
  // logarithms relative to the maxima: beside values near the type's lowest log(V) would be lost
  const double r_m = ((double)mr - m) * inv_t, Zr = R != 0.0 ? R * exp(r_m) : 0.0, Z = sum[1] + Zr;
  const double log_Z = log(Z), log_P = log(P);  // Z = 0: no student logit above -inf
  const double scale = W > 0.0 && !none ? (double)a.T * (double)w / W * (double)a.grad_scale : 0.0;
  double kl[1] = {0.0};
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    if (j * kDsThreads >= a.k) break;  // uniform
    const double p = pe[j] / P, q = zi[j] == -INFINITY ? 0.0 : e[j] / Z;
    const double lp = teacher(ti[j]) - log_P;
    const double lq = zi[j] == -INFINITY ? -INFINITY : ((double)zi[j] - m) * inv_t - log_Z;
    if ((used >> j & 1) && !none && p != 0.0) kl[0] += p * (lp - lq);
    const int i = j * kDsThreads + tid;
    if (i < a.k)  // the entry's value is read, its gradient takes its place
      z[i] = scale == 0.0 ? 0.f : lost ? NAN : used >> j & 1 ? (float)(scale * (q - p)) : 0.f;
  }
  if (tid == 64) {  // the bucket of the other ids, beside the entries' of the first wave
    const double lpr = tr - log_P, lqr = R == 0.0 ? -INFINITY : r_m + (log(R) - log_Z);
    const double pr = none || rt == -INFINITY ? 0.0 : exp(lpr);
    if (!none && pr != 0.0) kl[0] += pr * (lpr - lqr);
    // the gradient of any other id: exp((l - mr) / T) times this
    const double coef = scale == 0.0 ? 0.0 : lost ? NAN : R == 0.0 ? 0.0 : scale * (exp(lqr) - pr) / R;
    a.stat[row] = make_float2(mr == -INFINITY ? 0.f : mr, (float)coef);
  }
  block_sums(kl, red + 3);
  if (tid == 0) {
    const double loss = bad ? NAN : none ? 0.0 : lost ? NAN : (double)a.T * (double)a.T * kl[0];
    if (bad) raise_error(a.err, DEV_BAD_TOKEN);
    if (row == 0 && odd_weights != 0.0) raise_error(a.err, DEV_BAD_PARAM);
    a.row_loss[row] = (float)loss;
    a.share[row] = w > 0.f ? (double)w / W * loss : 0.0;
  }
}

// (3) The gradient of one chunk of one row; the workgroup after the last chunk adds the losses.
// Bound by the bytes in and out: 240 rows of 151936 fp32 logits, 292 MB, 44.5 us, some of them from the
// caches that the first launch has filled.
template <typename LT>
__global__ __launch_bounds__(kDsThreads) void distill_grad_kernel(DistillArgs a, int chunks) {
  constexpr int N = RowVec<LT>::N, NV = kDsVecs<LT>;
  const int tid = threadIdx.x;
  __shared__ uint32_t bits[kDsChunk / 32];
  __shared__ float own[kDsChunk];
  __shared__ double red[kDsWaves];
  if ((int)blockIdx.x == chunks) {
    double s = 0.0;
    for (int r = tid; r < a.rows; r += kDsThreads) s += a.share[r];
    s = block_reduce_sum<kDsWaves>(s, red);
    if (tid == 0) *a.loss = (float)s;
    return;
  }
  const int row = blockIdx.x / a.nch, ch = blockIdx.x % a.nch;
  const uint32_t c0 = (uint32_t)ch * kDsChunk, V = a.V;
  const LT *lr = (const LT *)a.logits + (size_t)row * a.ld;
  LT *gr = (LT *)a.grad + (size_t)row * a.ld_grad;
  const size_t r0 = (size_t)row * a.k, i0 = r0 + min(tid, a.k - 1);
  int id = a.ids[i0];  // before the values: loads end in order
  float z = a.z[i0];
  const float2 st = a.stat[row];
  u32x4 x[NV];
  ds_load<LT>(lr, c0, V, x);
  if (tid < kDsChunk / 32) bits[tid] = 0;
  __syncthreads();
  for (int i = tid; i < a.k;) {
    const uint32_t at = (uint32_t)id - c0;
    if (at < kDsChunk) {
      atomicOr(&bits[at >> 5], 1u << (at & 31));
      own[at] = z;
    }
    i += kDsThreads;
    if (i < a.k) {
      id = a.ids[r0 + i];
      z = a.z[r0 + i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < NV; ++q) {
    const uint32_t at = (q * kDsThreads + tid) * N;
    const uint32_t mine = ds_bits<N>(bits, at);
    u32x4 y = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float v = order_val(RowVec<LT>::get(x[q], e));
      const float g = __builtin_amdgcn_exp2f((v - st.x) * a.c) * st.y;
      LT o;
      store_as(&o, st.y == 0.f ? 0.f : g);
      RowVec<LT>::set(y, e, o);
    }
    if (mine) {  // few lanes: the entries' own
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (mine >> e & 1) {
          LT o;
          store_as(&o, own[at + e]);
          RowVec<LT>::set(y, e, o);
        }
    }
    if (c0 + at + N <= V) {
      row_store(gr + c0 + at, y);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (c0 + at + e < V) gr[c0 + at + e] = RowVec<LT>::at(y, e);
    }
  }
}

// [error word, padded to 256][weights' sum, padded to 256][chunk pairs][entries: value, then gradient][rows: stat, share of the loss, loss]
DistillLayout distill_layout(int rows, int V, int k) {
  DistillLayout l;
  const size_t n = rows;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  l.nch = (int)(((long)V + kDsChunk - 1) / kDsChunk);
  l.wsum = 256;
  l.part = 512;
  l.z = l.part + up(n * l.nch * sizeof(float2));
  l.stat = l.z + up(n * k * sizeof(float));
  l.share = l.stat + up(n * sizeof(float2));
  l.row_loss = l.share + up(n * sizeof(double));
  l.bytes = l.row_loss + up(n * sizeof(float));
  return l;
}

void launch_distill(const DistillArgs &a, bool bf16, hipStream_t st) {
  const int chunks = a.rows * a.nch;
  auto go = [&](auto part, auto grad) {
    hipLaunchKernelGGL(part, dim3(chunks + 1), dim3(kDsThreads), 0, st, a, chunks);
    hipLaunchKernelGGL(distill_row_kernel, dim3(a.rows), dim3(kDsThreads), 0, st, a);
    const int n = a.grad ? chunks : 0;
    hipLaunchKernelGGL(grad, dim3(n + 1), dim3(kDsThreads), 0, st, a, n);
  };
  if (bf16) go(distill_part_kernel<bf16_t>, distill_grad_kernel<bf16_t>);
  else go(distill_part_kernel<float>, distill_grad_kernel<float>);
}

}  // namespace dk
