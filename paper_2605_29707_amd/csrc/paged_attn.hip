// Attention of new tokens over a cache of pages, and the weights that it gives to every slot.
//   o_r = sum_s p_rs v_s,  p_rs = exp(scale q_r k_s - lse_r) over the slots s that row r sees
// Rows are the new tokens of a sequence times the query heads of one kv head: row i G + h.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mfma.h"
#include "paged.h"

namespace dk {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef __attribute__((ext_vector_type(4))) short short4v;

DEVI float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// A tile's place (16, 32 or 128 rows, as planned): sequence, lengths, first row, what it sees.
struct Tile {
  int b, row0, rows, vis;  // rows: of the sequence; vis: no row of the tile sees a slot from here on
  SeqRange s;
};

// The tile-th tile of M rows over all sequences; false behind the last.  A sequence's last tiles come
// first: with causal rows they are the longest.  With `err`, sequences whose lengths disagree set it: one workgroup of a launch looks
// at all of them.
DEVI bool find_tile(const PagedAttnArgs &a, int tile, int M, int32_t *err, Tile &t) {
  const int lane = threadIdx.x & 63, G = a.nq / a.c.n_kv;
  int base = 0;
  bool found = false, down = false;  // down: from here on sequences are left out (starts_ascend)
  for (int s0 = 0; s0 < a.c.batch && (!found || err); s0 += 64) {
    SeqRange s{0, 0, 0};
    const int i = min(s0 + lane, a.c.batch - 1);
    const int lo = a.starts[i], hi = a.starts[i + 1], len = a.lens[i];
    bool live = check_range(lo, hi, len, a.tokens, a.max_new, a.max_len, err, s) && s0 + lane < a.c.batch;
    if (found) continue;
    const uint64_t drops = __ballot(hi < lo);
    live = live && !down && !(drops & ((1ull << lane) - 1));
    down |= drops != 0;
    // (a launch has fewer than 2^24 tiles, and `base` stays at most `tile`: nothing passes 32 bits)
    const int n = live ? min((int)(((int64_t)s.n * G + M - 1) / M), 1 << 24) : 0, upto = base + wave_running_sum(n);
    const uint64_t here = __ballot(upto > tile);
    if (here) {
      const int l = __ffsll((unsigned long long)here) - 1;
      t.b = s0 + l;
      t.s.start = __builtin_amdgcn_readlane(s.start, l);
      t.s.n = __builtin_amdgcn_readlane(s.n, l);
      t.s.len = __builtin_amdgcn_readlane(s.len, l);
      t.rows = t.s.n * G;
      // (tile - first tile of the sequence) counts from its last one
      t.row0 = ((t.rows + M - 1) / M - 1 - (tile - __builtin_amdgcn_readlane(upto - n, l))) * M;
      const int last = (min(t.row0 + M, t.rows) - 1) / G;
      t.vis = a.mask ? t.s.len : t.s.len - t.s.n + last + 1;
      found = true;
    } else {
      base = __builtin_amdgcn_readlane(upto, 63);
    }
  }
  return found;
}

// The length of a sequence's runs, a multiple of `whole` slots: the launch's, or shorter where the sequence is so much shorter than max_len that
// 2^run_shift runs of it (as many as give each CU two workgroups) are.  A caller that captures a graph gives the longest length that it will ever have.
DEVI int run_of(const PagedAttnArgs &a, int len, int run, int whole) {
  const int part = (len + (1 << a.run_shift) - 1) >> a.run_shift;  // (len < 2^30, run_shift at most 7)
  return min(run, (part + whole - 1) & ~(whole - 1));
}

// The run of the at-th workgroup of a kv head.  Tiles' first runs, the ones that short sequences have, are an odd number of workgroups
// apart: workgroups are handed to the CUs in turn, and 64 sequences of 2000 slots in a launch for 32768, 16 apart, took 249 us (130 so,
// 97 in a launch for 2000).
DEVI int split_of(int at, int tile, int splits) { return (splits & 1 ? at : at + tile) % splits; }

// Operands of the two products.  Scores: S^T = K Q^T in tiles of 16 slots x 16 rows, lane (g, r) = 16 g + r with
// the scores of row r and slots 4 g .. 4 g + 3.  That is the second operand of O^T = V^T P^T as it stands,
// if the slots of a step are taken in the order (4 g .. 4 g + 3, 16 + 4 g .. 16 + 4 g + 3).
template <typename T, int DH> struct Ops;

template <int DH> struct Ops<bf16_t, DH> {
  static constexpr int KST = DH / 32, OT = DH / 16;
  // lds: this wave's 32 rows of v, 32 bytes of padding each, so that the 16 rows that a transposed read takes lie
  // in different banks
  static constexpr int LDSROW = DH * 2 + 32, LDSBYTES = 32 * LDSROW, VN = DH / 16;
  DEVI static u32x4 row_frag(const char *row, int st, int g) { return *(const u32x4 *)(row + (st * 32 + g * 8) * 2); }
  DEVI static floatx4 score(const u32x4 (&k)[KST], const u32x4 (&q)[KST]) {
    floatx4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < KST; ++st)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[st]), __builtin_bit_cast(bf16x8, q[st]), s, 0, 0, 0);
    return s;
  }
  // v: VN 16-byte items of the 32 rows, item n of lane l at row n * (64 / LPR) + l / LPR
  static constexpr int LPR = DH / 8;
  DEVI static int v_row(int n, int lane) { return n * (64 / LPR) + lane / LPR; }
  DEVI static int v_col(int lane) { return (lane % LPR) * 16; }
  // Which of the 32 slots hold NaN or an infinity in v (the same in every lane); those values become 0.
  DEVI static uint32_t take_odd(u32x4 (&v)[VN], int lane) {
    uint32_t odd = 0;
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      bool mine = false;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool lo = (v[n][c] & 0x7f80u) == 0x7f80u, hi = (v[n][c] & 0x7f800000u) == 0x7f800000u;
        v[n][c] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
        mine |= lo || hi;
      }
      const uint64_t all = __ballot(mine);
#pragma unroll
      for (int y = 0; y < 64 / LPR; ++y)
        if (all >> (y * LPR) & ((1ull << LPR) - 1)) odd |= 1u << (n * (64 / LPR) + y);
    }
    return odd;
  }
  // p: weights of slots 16 tt + 4 g + e, as high and low bf16 parts: with one part the rounding of the weights
  // (2^-9 of each) would add as much error as the output's own
  DEVI static void add(char *lds, const float (&p)[8], floatx4 (&o)[OT], int lane) {
    const int g = lane >> 4, r = lane & 15;
    bf16x8 hi, lo;
    split8(p, hi, lo);
#pragma unroll
    for (int t = 0; t < OT; ++t) {
      typedef __attribute__((address_space(3))) short4v lds4;
      const char *at = lds + (4 * g + r / 4) * LDSROW + (16 * t + (r % 4) * 4) * 2;
      const short4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)at);
      const short4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 16 * LDSROW));
      typedef __attribute__((ext_vector_type(8))) short short8v;
      const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi, o[t], 0, 0, 0);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo, o[t], 0, 0, 0);
    }
  }
  // first column of the four that o[t] holds in lane group g
  DEVI static int out_col(int t, int g) { return 16 * t + 4 * g; }
  static constexpr int OSTEP = 1;  // and their distance
};

template <int DH> struct Ops<float, DH> {
  static constexpr int KST = DH / 16, OT = DH / 16;
  static constexpr int LDSROW = 0, LDSBYTES = 0, VN = DH / 8;
  DEVI static u32x4 row_frag(const char *row, int st, int g) { return *(const u32x4 *)(row + (st * 16 + g * 4) * 4); }
  DEVI static floatx4 score(const u32x4 (&k)[KST], const u32x4 (&q)[KST]) {
    floatx4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < KST; ++st)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[st][e]), __uint_as_float(q[st][e]), s, 0, 0, 0);
    return s;
  }
  // v: item n = (slot 16 tt + 4 g + e, 64 columns jj) as n = (tt * 4 + e) * (DH / 64) + jj: four columns 64 jj + 4 r
  static constexpr int JJ = DH / 64;
  DEVI static int v_col(int lane) { return (lane & 15) * 16; }
  DEVI static int v_row(int n, int lane) { return 16 * (n / JJ / 4) + 4 * (lane >> 4) + n / JJ % 4; }
  DEVI static uint32_t take_odd(u32x4 (&v)[VN], int lane) {
    uint32_t odd = 0;
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      bool mine = false;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bool bad = (v[n][c] & 0x7f800000u) == 0x7f800000u;
        v[n][c] = bad ? 0u : v[n][c];
        mine |= bad;
      }
      const uint64_t all = __ballot(mine);
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if (all >> (16 * y) & 0xffffull) odd |= 1u << (16 * (n / JJ / 4) + 4 * y + n / JJ % 4);
    }
    return odd;
  }
  DEVI static void add(const u32x4 (&v)[VN], const float (&p)[8], floatx4 (&o)[OT]) {
#pragma unroll
    for (int n = 0; n < VN; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        o[n % JJ * 4 + c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[n][c]), p[n / JJ], o[n % JJ * 4 + c], 0, 0, 0);
  }
  // o[jj * 4 + c], lane group g, element e: column 64 jj + 16 g + 4 e + c
  DEVI static int out_col(int t, int g) { return 64 * (t / 4) + 16 * g + t % 4; }
  static constexpr int OSTEP = 4;
};

// Scores of 32 slots and a tile of 16 rows: lane (g, r) gets row r's of slots 16 (e / 4) + 4 g + e % 4.  (Single values from
// here on: with elements of the product's vectors replaced under the branches of a mask, this compiler (ROCm 7.2) wrote one
// element over the other three.)
template <typename T, int DH>
DEVI void score8(const u32x4 (&k)[2][Ops<T, DH>::KST], const u32x4 (&q)[Ops<T, DH>::KST], float (&x)[8]) {
  const floatx4 s0 = Ops<T, DH>::score(k[0], q), s1 = Ops<T, DH>::score(k[1], q);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = s0[e];
    x[4 + e] = s1[e];
  }
}

// A slot that holds NaN or infinities in v, which the products took as 0: they go, weighted, to the rows that see it.
template <typename T, int DH>
DEVI void add_odd(const char *row, int slot, const float (&p)[8], uint32_t dark, floatx4 (&o)[Ops<T, DH>::OT], int lane) {
  using O = Ops<T, DH>;
  const int g = lane >> 4, src = 16 * (slot % 16 / 4) + (lane & 15), e = 4 * (slot / 16) + slot % 4;
  float w = 0.f;
#pragma unroll
  for (int x = 0; x < 8; ++x) w = x == e ? p[x] : w;
  w = __shfl(w, src, 64);
  const bool seen = !(__shfl(dark, src, 64) >> e & 1);
#pragma unroll
  for (int t = 0; t < O::OT; ++t)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float v = to_f32(((const T *)row)[O::out_col(t, g) + c * O::OSTEP]);
      const bool bad = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
      o[t][c] += bad && seen ? w * v : 0.f;
    }
}

// Where the scores (base 2) of 32 slots and a row of a sequence's kv head are kept: step by step, the rows' 128 bytes side by side.
DEVI float *scores_at(const PagedAttnArgs &a, int b, int kvh, int slot, int row) {
  return a.scores + (((int64_t)(b * a.c.n_kv + kvh) * a.scores_steps + slot / 32) * a.scores_rows + row) * 32;
}

constexpr int kPaThreads = 256, kPaWaves = 4, kPaStep = 32;

// A workgroup has a tile of 16 NT rows and a run of slots, a wave every fourth 32 slots of it; the waves' results are
// joined in LDS.  Bound by the cache's bytes where rows are few (64 sequences of 4096 to 16385 slots, 32 heads on 8: 500 us, 5.4 TB/s),
// by the products' rate with 32 fp32 rows.
template <typename T, int DH, int NT, bool MASKED, bool ONE_PAGE>
__global__ __launch_bounds__(kPaThreads) void paged_attn_kernel(PagedAttnArgs a, int splits, int run) {
  using O = Ops<T, DH>;
  constexpr int M = 16 * NT, ESZ = sizeof(T);
  constexpr int MERGE = kPaWaves * 16 * (DH + 4) * 4;
  constexpr int VBYTES = kPaWaves * O::LDSBYTES;
  __shared__ __align__(16) char lds[MERGE > VBYTES ? MERGE : VBYTES];
  __shared__ float s_m[kPaWaves][M], s_l[kPaWaves][M];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15;
  const int kvh = blockIdx.x % a.c.n_kv, tile = blockIdx.x / a.c.n_kv / splits, split = split_of(blockIdx.x / a.c.n_kv, tile, splits);
  Tile t;
  if (!find_tile(a, tile, M, blockIdx.x == gridDim.x - 1 ? a.err : nullptr, t)) return;
  run = run_of(a, t.s.len, run, kPaWaves * kPaStep);
  const int k0 = split * run, k1 = min(t.vis, k0 + run);
  if (k0 >= k1) return;
  const int G = a.nq / a.c.n_kv, n0 = t.s.len - t.s.n;

  u32x4 q[NT][O::KST];
  int lim[NT];  // the last slot that this lane's row sees, causally
  const uint8_t *mrow[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = t.row0 + 16 * nt + r, i = min(row, t.rows - 1) / G;
    lim[nt] = row < t.rows ? n0 + i : -1;
    if (MASKED) mrow[nt] = a.mask + (int64_t)(t.s.start + i) * a.mask_ld;
    const char *p = (const char *)a.q + ((int64_t)(t.s.start + i) * a.q_stride + (int64_t)(kvh * G + min(row, t.rows - 1) % G) * DH) * ESZ;
#pragma unroll
    for (int st = 0; st < O::KST; ++st) q[nt][st] = O::row_frag(p, st, g);
  }
  float m[NT], l[NT];
  floatx4 o[NT][O::OT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -INFINITY;
    l[nt] = 0.f;
#pragma unroll
    for (int x = 0; x < O::OT; ++x) o[nt][x] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float sc = a.scale * kLog2e;
  const char *kb = a.c.k + (a.layer * a.c.layer_stride + kvh * a.c.head_stride) * ESZ;
  const char *vb = a.c.v + (a.layer * a.c.layer_stride + kvh * a.c.head_stride) * ESZ;
  char *mylds = lds + wave * O::LDSBYTES;
  // A step's rows: ONE_PAGE, its 32 slots lie in one page (page_size >= 32), their address is a scalar and a lane's offset in the page
  // the same every step; else every lane looks up one slot and takes its rows' pages from the others.  The page's number is loaded
  // a step before the rows (and ahead of that step's: loads return in order), k's rows once the scores have used the last ones, v's once those are in LDS (or used): a wave has
  // one step's rows on their way all the time.
  const int near_k = r * (int)a.c.slot_stride * ESZ;
  int page = 0;
  bool lost = false;
  auto look = [&](int kt) {
    const int slot = ONE_PAGE ? kt : kt + (lane & 31);
    return a.c.table[(int64_t)t.b * a.c.max_pages + (min(slot, k1 - 1) >> a.c.page_shift)];
  };
  auto settle = [&](int p) {
    if (ONE_PAGE) p = __builtin_amdgcn_readfirstlane(p);
    if ((unsigned)p < (unsigned)a.c.n_pages) return p;
    lost = true;
    return 0;
  };
  auto row_at = [&](const char *base, int kt, int x) {
    return base + slot_offset(a.c, __shfl(page, x, 64), min(kt + x, k1 - 1)) * ESZ;
  };
  u32x4 k[2][O::KST], v[O::VN];
  auto load_k = [&](int kt) {
    if constexpr (ONE_PAGE) {
      const char *p = kb + slot_offset(a.c, page, kt) * ESZ;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int st = 0; st < O::KST; ++st) k[tt][st] = O::row_frag(p + tt * 16 * a.c.slot_stride * ESZ + near_k, st, g);
    } else {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const char *p = row_at(kb, kt, 16 * tt + r);
#pragma unroll
        for (int st = 0; st < O::KST; ++st) k[tt][st] = O::row_frag(p, st, g);
      }
    }
  };
  auto load_v = [&](int kt) {
    if constexpr (ONE_PAGE) {
      const char *p = vb + slot_offset(a.c, page, kt) * ESZ;
#pragma unroll
      for (int n = 0; n < O::VN; ++n) {
        const int col = ESZ == 2 ? O::v_col(lane) : O::v_col(lane) + n % (DH / 64) * 256;
        // (a lane's row: that of item 0, and the same distance further for all lanes)
        v[n] = *(const u32x4 *)(p + (O::v_row(n, lane) - O::v_row(0, lane)) * a.c.slot_stride * ESZ +
                                (O::v_row(0, lane) * (int)a.c.slot_stride * ESZ + col));
      }
    } else {
#pragma unroll
      for (int n = 0; n < O::VN; ++n) {
        const int col = ESZ == 2 ? O::v_col(lane) : O::v_col(lane) + n % (DH / 64) * 256;
        v[n] = *(const u32x4 *)(row_at(vb, kt, O::v_row(n, lane)) + col);
      }
    }
  };
  constexpr int STRIDE = kPaWaves * kPaStep;
  int kt = k0 + wave * kPaStep, ahead = 0;
  page = settle(look(kt));
  // q arrives with the page.  (Where it is only waited for in the loop, which a path without a step reaches too, that wait is one for
  // all of a step's loads: 59 sequences of 760 slots 30.3 us, 29.9 here.)
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int st = 0; st < O::KST; ++st) __asm__ volatile("" ::"v"(q[nt][st]));
  if (kt < k1) {
    ahead = look(kt + STRIDE);
    load_k(kt);
    load_v(kt);
  }
  auto step = [&](auto next) {  // next: loads for the step after this one go out
    constexpr bool more = decltype(next)::value;
    const int page_now = page;
    float sx[NT][8];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) score8<T, DH>(k, q[nt], sx[nt]);
    if (more) {
      page = settle(ahead);
      ahead = look(kt + 2 * STRIDE);
      load_k(kt + STRIDE);
    }
    // rows past the run's end are zeros: a weight of 0 times what lies there might be NaN
    if (kt + kPaStep > k1) {
#pragma unroll
      for (int n = 0; n < O::VN; ++n)
        if (kt + O::v_row(n, lane) >= k1) v[n] = u32x4{0, 0, 0, 0};
    }
    const bool whole = kt + kPaStep <= min(n0, k1);
    uint32_t odd = 0;  // slots of this step, some of them hidden from some row, whose v holds NaN or an infinity
    if (!whole) odd = O::take_odd(v, lane);
    if constexpr (ESZ == 2) {
#pragma unroll
      for (int n = 0; n < O::VN; ++n) *(u32x4 *)(mylds + O::v_row(n, lane) * O::LDSROW + O::v_col(lane)) = v[n];
      __builtin_amdgcn_wave_barrier();
      if (more) load_v(kt + STRIDE);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = sx[nt][e] * sc;
      uint32_t dark = 0;  // hidden among this lane's eight (a score of -inf hides nothing: 0 times NaN is NaN in whole steps too)
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int slot = kt + 16 * (e / 4) + 4 * g + e % 4;
          bool seen = slot <= lim[nt];
          if (MASKED) seen = (slot < n0) | (mrow[nt][max(0, min(slot, t.s.len - 1) - n0)] != 0);
          seen &= slot < k1;
          x[e] = seen ? x[e] : -INFINITY;
          dark |= seen ? 0u : 1u << e;
        }
      }
      // (Whole calls, 64 sequences' next tokens with their weights: 536 us without these stores, 540 with all of them to one place, 615 in earnest:
      // the 82 MB of writes between the reads.)
      if (NT == 1 && a.scores && t.row0 + r < t.rows) {
        float *to = scores_at(a, t.b, kvh, kt, r) + 4 * g;
        *(floatx4 *)to = floatx4{x[0], x[1], x[2], x[3]};
        *(floatx4 *)(to + 16) = floatx4{x[4], x[5], x[6], x[7]};
      }
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float mn = fmaxf(m[nt], top), ms = mn == -INFINITY ? 0.f : mn;
      const float alpha = fast_exp2(m[nt] - ms);
      m[nt] = mn;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = fast_exp2(x[e] - ms);
        sum += x[e];
      }
      l[nt] = l[nt] * alpha + sum;
#pragma unroll
      for (int y = 0; y < O::OT; ++y) o[nt][y] *= alpha;
      if constexpr (ESZ == 2) O::add(mylds, x, o[nt], lane);
      else O::add(v, x, o[nt]);
      if (odd) {
#pragma unroll 1
        for (int e = 0; e < 32; ++e)
          if (odd >> e & 1)
            add_odd<T, DH>(vb + slot_offset(a.c, __builtin_amdgcn_readlane(page_now, e), kt + e) * ESZ, e, x, dark, o[nt], lane);
      }
    }
    if constexpr (ESZ == 2) __builtin_amdgcn_wave_barrier();
    else if (more) load_v(kt + STRIDE);
  };
  for (; kt + STRIDE < k1; kt += STRIDE) step(std::true_type{});
  if (kt < k1) step(std::false_type{});
  if (lost) raise_error(a.err, DEV_BAD_PAGE);

  // the waves' maxima and sums, then their rows 16 at a time
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] += __shfl_xor(l[nt], 16, 64);
    l[nt] += __shfl_xor(l[nt], 32, 64);
    if (g == 0) {
      s_m[wave][16 * nt + r] = m[nt];
      s_l[wave][16 * nt + r] = l[nt];
    }
  }
  float *om = (float *)lds;
  constexpr int LD = DH + 4;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    __syncthreads();
#pragma unroll
    for (int x = 0; x < O::OT; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) om[(wave * 16 + r) * LD + O::out_col(x, g) + e * O::OSTEP] = o[nt][x][e];
    __syncthreads();
    // 16 threads a row
    const int rr = threadIdx.x / 16, c0 = threadIdx.x % 16, row = t.row0 + 16 * nt + rr;
    if (row >= t.rows) continue;
    float top = -INFINITY, sum = 0.f, f[kPaWaves];
#pragma unroll
    for (int w = 0; w < kPaWaves; ++w) top = fmaxf(top, s_m[w][16 * nt + rr]);
    const float ms = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < kPaWaves; ++w) {
      f[w] = fast_exp2(s_m[w][16 * nt + rr] - ms);
      sum += s_l[w][16 * nt + rr] * f[w];
    }
    const int tok = t.s.start + row / G, head = kvh * G + row % G;
    const int64_t at = ((int64_t)split * a.tokens + tok) * a.nq + head;
    const bool none = !a.part_o && sum == 0.f;  // no score above -inf: 0 whatever v holds
    const float inv = a.part_o ? 1.f : 1.f / sum;
#pragma unroll
    for (int cc = 0; cc < DH / 64; ++cc) {
      const int c = cc * 64 + c0 * 4;
      floatx4 y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kPaWaves; ++w) y += *(const floatx4 *)(om + (w * 16 + rr) * LD + c) * f[w];
      y = none ? floatx4{0.f, 0.f, 0.f, 0.f} : y * inv;
      if (a.part_o) {
        *(floatx4 *)(a.part_o + at * DH + c) = y;
      } else {
        T *dst = (T *)a.out + (int64_t)tok * a.o_stride + (int64_t)head * DH + c;
        if constexpr (ESZ == 2) {
          *(uint2 *)dst = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
        } else {
          *(floatx4 *)dst = y;
        }
      }
    }
    if (c0 == 0) {
      if (a.part_o) *(float2 *)(a.part_ml + at * 2) = make_float2(top, sum);
      else if (a.lse) a.lse[(int64_t)tok * a.nq + head] = (top + log2f(sum)) * kLn2;
    }
  }
}

// ---------------------------------------------------------------------------
// Chunks: a workgroup has 128 rows, 32 a wave, and goes over a run's slots 64 at a time through two LDS buffers.  The
// products are 32 x 32 x 16: scores S^T = K Q^T leave lane l = 32 h + r with row r's of slots 8 (e / 4) + 4 h + e % 4, which is
// again the second operand of O^T = V^T P^T for the slots of a step in the order (4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3).
// Weights are rounded to bf16 for that product (half a step of each, as far off as the output's own rounding).
// A wave reads every row of k and v from LDS once: as many bytes a clock as the products of 32 rows take.  In both
// buffers a row's 16-byte items are permuted by the row, so that neither read has bank conflicts: k's 16 rows of one item,
// v's eight rows of 32 bytes.
// Bound by the products: 4096 tokens after 12288, 32 heads on 8, 983 to 1069 us by the card, 0.90 to 0.98 PFLOP/s.
// ---------------------------------------------------------------------------
constexpr int kChunkRows = 128, kChunkStep = 64;
typedef float floatx16 __attribute__((ext_vector_type(16)));

// PAGES, how a step's 64 slots lie in pages: 3, in one; 2, in two of 32; 1, those of a wave's load (64 / (items a row) neighbours) in one; 0, anyhow.
template <int DH, bool MASKED, int PAGES>
__global__ __launch_bounds__(256, 2) void paged_chunk_kernel(PagedAttnArgs a, int splits, int run) {
  constexpr int RB = DH * 2, CH = RB / 16, KST = DH / 16, DT = DH / 32, LPT = kChunkStep * CH / 256, TILE = kChunkStep * RB;
  __shared__ __align__(16) char s_k[2][TILE], s_v[2][TILE];
  __shared__ uint64_t s_odd[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, r = lane & 31;
  const int kvh = blockIdx.x % a.c.n_kv, tile = blockIdx.x / a.c.n_kv / splits, split = split_of(blockIdx.x / a.c.n_kv, tile, splits);
  Tile t;
  if (!find_tile(a, tile, kChunkRows, blockIdx.x == gridDim.x - 1 ? a.err : nullptr, t)) return;
  run = run_of(a, t.s.len, run, kChunkStep);
  const int k0 = split * run, k1 = min(t.vis, k0 + run);
  if (k0 >= k1) return;
  const int G = a.nq / a.c.n_kv, n0 = t.s.len - t.s.n;
  // slots below this are seen by all rows of the workgroup
  const int clear = min(k1, MASKED ? n0 : n0 + t.row0 / G + 1);

  const int row = t.row0 + wave * 32 + r, row_in = min(row, t.rows - 1), tok = t.s.start + row_in / G;
  const int lim = row < t.rows ? n0 + row_in / G : -1;
  const uint8_t *mrow = MASKED ? a.mask + (int64_t)tok * a.mask_ld : nullptr;
  u32x4 q[KST];
  {
    const char *p = (const char *)a.q + ((int64_t)tok * a.q_stride + (int64_t)(kvh * G + row_in % G) * DH) * 2;
#pragma unroll
    for (int st = 0; st < KST; ++st) q[st] = *(const u32x4 *)(p + st * 32 + h * 16);
  }
  const float sc = a.scale * kLog2e;
  const int64_t head = a.layer * a.c.layer_stride + kvh * a.c.head_stride;
  const char *kb = a.c.k + head * 2, *vb = a.c.v + head * 2;

  // This thread's items of a step: 16 bytes of row (tid + 256 i) / CH.  Where a load's rows lie in one page its address is a scalar and
  // a lane's offset, and the page's number is loaded a step before the rows.
  constexpr int NEAR = 64 / CH, EACH = PAGES >= 2 ? (PAGES == 3 ? kChunkStep : 32) : 256 / CH, LOOKS = kChunkStep / EACH;  // rows a page number is for
  const int my_row = tid / CH, my_col = tid % CH;
  const uint32_t lane_at = PAGES ? (uint32_t)(PAGES >= 2 ? my_row : lane / CH) * (uint32_t)a.c.slot_stride * 2 + my_col * 16 : 0;
  bool lost = false;
  u32x4 kr[LPT], vr[LPT];
  int ahead[LOOKS];
  // the first slot of a load's rows; behind the run, of the last one
  auto first_of = [&](int kt, int i) {
    return PAGES >= 2 ? min(kt + i * EACH, (k1 - 1) & ~(EACH - 1)) : min(kt + wave * NEAR + i * EACH, (k1 - 1) & ~(NEAR - 1));
  };
  auto look = [&](int kt) {
    if constexpr (PAGES != 0) {
#pragma unroll
      for (int i = 0; i < LOOKS; ++i) ahead[i] = a.c.table[(int64_t)t.b * a.c.max_pages + (first_of(kt, i) >> a.c.page_shift)];
    }
  };
  auto load = [&](int kt) {
    const char *kp = nullptr, *vp = nullptr;
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
      if constexpr (PAGES != 0) {
        constexpr int LOADS = EACH / (256 / CH);  // with one page number
        if (i % LOADS == 0) {
          int page = __builtin_amdgcn_readfirstlane(ahead[i / LOADS]);
          if ((unsigned)page >= (unsigned)a.c.n_pages) {
            lost = true;
            page = 0;
          }
          const int64_t at = slot_offset(a.c, page, first_of(kt, i / LOADS)) * 2;
          kp = kb + at;
          vp = vb + at;
        }
        const int64_t more = (int64_t)(i % LOADS * (256 / CH)) * a.c.slot_stride * 2;
        kr[i] = *(const u32x4 *)(kp + more + lane_at);
        vr[i] = *(const u32x4 *)(vp + more + lane_at);
      } else {
        const int slot = min(kt + my_row + i * (256 / CH), k1 - 1);
        int page = page_of(a.c, t.b, slot);
        if (page < 0) {
          lost = true;
          page = 0;
        }
        const int64_t at = slot_offset(a.c, page, slot) * 2 + my_col * 16;
        kr[i] = *(const u32x4 *)(kb + at);
        vr[i] = *(const u32x4 *)(vb + at);
      }
    }
  };
  auto swz_k = [](int x) { return CH == 16 ? x & 15 : (x >> 1) & 7; };
  auto swz_v = [](int x) { return (CH == 16 ? (x & 3) << 2 : (x & 2) << 1) | ((x >> 1) & 2); };
  auto store = [&](int kt, int buf) {
    if (kt + kChunkStep > clear) {  // workgroup-uniform
      uint64_t odd = 0;
#pragma unroll
      for (int i = 0; i < LPT; ++i) {
        const int x = my_row + i * (256 / CH);
        bool mine = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const bool lo = (vr[i][c] & 0x7f80u) == 0x7f80u, hi = (vr[i][c] & 0x7f800000u) == 0x7f800000u;
          vr[i][c] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
          mine |= lo || hi;
        }
        // rows past the run's end count for nothing
        const uint64_t all = __ballot(mine && kt + x < k1);
#pragma unroll
        for (int y = 0; y < 64 / CH; ++y)
          if (all >> (y * CH) & ((1ull << CH) - 1)) odd |= 1ull << (wave * (64 / CH) + i * (256 / CH) + y);
      }
      if (lane == 0) s_odd[buf][wave] = odd;
    }
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
      const int x = my_row + i * (256 / CH);
      *(u32x4 *)(s_k[buf] + x * RB + (my_col ^ swz_k(x)) * 16) = kr[i];
      *(u32x4 *)(s_v[buf] + x * RB + (my_col ^ swz_v(x)) * 16) = vr[i];
    }
  };

  float m = -INFINITY, l = 0.f;
  floatx16 o[DT];
#pragma unroll
  for (int x = 0; x < DT; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[x][e] = 0.f;
  const int k_at = r * RB + (h ^ swz_k(r)) * 16;  // item 2 st + h: with the bits of st
  const int v_i = lane & 15, v_x = 4 * h + v_i / 4, v_half = (lane >> 4) & 1;

  look(k0);
  load(k0);
  look(k0 + kChunkStep);
  store(k0, 0);
  __syncthreads();
  int buf = 0;
  for (int kt = k0; kt < k1; kt += kChunkStep, buf ^= 1) {
    const bool more = kt + kChunkStep < k1;
    if (more) load(kt + kChunkStep);
    look(kt + 2 * kChunkStep);
    floatx16 s[2];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[y][e] = 0.f;
    // (the two sums take turns: a product waits for the one before it on the same sum)
#pragma unroll
    for (int st = 0; st < KST; ++st)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const u32x4 f = *(const u32x4 *)(s_k[buf] + y * 32 * RB + (k_at ^ (st * 32)));
        s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f), __builtin_bit_cast(bf16x8, q[st]), s[y], 0, 0, 0);
      }
    float x[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] = s[e / 16][e % 16];
    uint64_t odd = 0;
    uint32_t dark = 0;
    if (kt + kChunkStep > clear) {
#pragma unroll
      for (int w = 0; w < 4; ++w) odd |= s_odd[buf][w];
      // the mask of four neighbouring slots at a time, from a place in the row that keeps the load inside of it
      uint32_t four[8];
      if (MASKED && t.s.n >= 4) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int first = kt + 32 * (u / 4) + 8 * (u % 4) + 4 * h - n0, from = min(max(first, 0), t.s.n - 4);
          __builtin_memcpy(&four[u], mrow + from, 4);
          const int off = min(max(first - from, -4), 4) * 8;  // (bytes of slots before the new ones or behind the last are not looked at)
          four[u] = (uint32_t)(off < 0 ? (uint64_t)four[u] << -off : (uint64_t)four[u] >> off);
        }
      } else if (MASKED) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          four[u] = 0;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            four[u] |= (uint32_t)mrow[min(max(kt + 32 * (u / 4) + 8 * (u % 4) + 4 * h + c - n0, 0), t.s.n - 1)] << (8 * c);
        }
      }
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int slot = kt + 32 * (e / 16) + 8 * (e % 16 / 4) + 4 * h + e % 4;
        bool seen = slot <= lim;
        if (MASKED) seen = (slot < n0) | ((four[e / 4] >> (8 * (e % 4)) & 0xff) != 0);
        seen &= slot < k1;
        x[e] = seen ? x[e] : -INFINITY;
        dark |= seen ? 0u : 1u << e;
      }
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 32; ++e) top = fmaxf(top, x[e]);
    {
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * sc;
    }
    // the sums' common factor 2^-m moves only when a row's maximum passes it by 2^6: weights stay below 2^6, and most steps
    // leave the output as it is
    if (__ballot(top > m + 6.f)) {
      const float mn = fmaxf(m, top), alpha = fast_exp2(m - (mn == -INFINITY ? 0.f : mn));
      m = mn;
      l *= alpha;
#pragma unroll
      for (int y = 0; y < DT; ++y) o[y] *= alpha;
    }
    const float ms = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      x[e] = fast_exp2(fmaf(x[e], sc, -ms));
      sum += x[e];
    }
    l += sum;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      bf16x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = (__bf16)x[8 * u + e];
#pragma unroll
      for (int y = 0; y < DT; ++y) {
        typedef __attribute__((address_space(3))) short4v lds4;
        typedef __attribute__((ext_vector_type(8))) short short8v;
        const int c = (y * 4 + v_half * 2 + (v_i & 3) / 2) ^ swz_v(v_x);
        const char *at = s_v[buf] + (16 * u + v_x) * RB + c * 16 + (v_i & 1) * 8;
        const short4v v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)at);
        const short4v v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 8 * RB));
        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p, o[y], 0, 0, 0);
      }
    }
    if (odd) {  // values that the product took as 0 go, weighted, to the rows that see them
#pragma unroll 1
      for (int e = 0; e < kChunkStep; ++e) {
        if (!(odd >> e & 1)) continue;
        const int page = max(page_of(a.c, t.b, kt + e), 0);
        const uint16_t *vrow = (const uint16_t *)(vb + slot_offset(a.c, page, kt + e) * 2);
        const int src = 32 * ((e >> 2) & 1) + r, at = 16 * (e >> 5) + 4 * ((e >> 3) & 3) + (e & 3);
        float w = 0.f;
#pragma unroll
        for (int y = 0; y < 32; ++y) w = y == at ? x[y] : w;
        w = __shfl(w, src, 64);
        const bool seen = !(__shfl(dark, src, 64) >> at & 1);
#pragma unroll
        for (int y = 0; y < DT; ++y)
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float v = __uint_as_float((uint32_t)vrow[32 * y + 8 * (c / 4) + 4 * h + c % 4] << 16);
            const bool bad = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
            o[y][c] += bad && seen ? w * v : 0.f;
          }
      }
    }
    if (more) store(kt + kChunkStep, buf ^ 1);
    __syncthreads();
  }
  if (lost) raise_error(a.err, DEV_BAD_PAGE);
  {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  }
  if (row >= t.rows) return;
  const int qh = kvh * G + row % G;
  const int64_t at = ((int64_t)split * a.tokens + tok) * a.nq + qh;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (!a.part_o && l == 0.f) {  // no score above -inf: 0 whatever v holds
#pragma unroll
    for (int y = 0; y < DT; ++y)
#pragma unroll
      for (int c = 0; c < 16; ++c) o[y][c] = 0.f;
  }
#pragma unroll
  for (int y = 0; y < DT; ++y)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int col = 32 * y + 8 * c + 4 * h;
      if (a.part_o) {
        *(floatx4 *)(a.part_o + at * DH + col) = floatx4{o[y][4 * c], o[y][4 * c + 1], o[y][4 * c + 2], o[y][4 * c + 3]};
      } else {
        bf16_t *dst = (bf16_t *)a.out + (int64_t)tok * a.o_stride + (int64_t)qh * DH + col;
        *(uint2 *)dst = make_uint2(pack_bf16(o[y][4 * c] * inv, o[y][4 * c + 1] * inv),
                                   pack_bf16(o[y][4 * c + 2] * inv, o[y][4 * c + 3] * inv));
      }
    }
  if (h == 0) {
    if (a.part_o) *(float2 *)(a.part_ml + at * 2) = make_float2(m, l);
    else if (a.lse) a.lse[(int64_t)tok * a.nq + qh] = (m + log2f(l)) * kLn2;
  }
}

// Joins the runs of one row (a new token's query head): a wave takes every W-th run, eight at a time, and the row's W waves'
// sums meet in LDS.  One wave a row up to eight runs, which is one round trip; four above.
template <typename T, int DH, int W>
__global__ __launch_bounds__(256) void paged_attn_join_kernel(PagedAttnArgs a, int M, int run) {
  constexpr int E = DH / 64, U = 8;
  const int lane = threadIdx.x & 63, unit = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = unit % W;
  const int64_t at = (int64_t)blockIdx.x * (4 / W) + unit / W;
  if (at >= (int64_t)a.tokens * a.nq) return;
  const int tok = (int)(at / a.nq), head = (int)(at % a.nq), G = a.nq / a.c.n_kv;
  int b;
  SeqRange s;
  if (!seq_of_token(a.starts, a.lens, a.c.batch, tok, a.tokens, a.max_new, a.max_len, b, s)) return;
  run = run_of(a, s.len, run, M == kChunkRows ? kChunkStep : kPaWaves * kPaStep);
  const int row = (tok - s.start) * G + head % G, last = (min((row / M + 1) * M, s.n * G) - 1) / G;
  const int vis = a.mask ? s.len : s.len - s.n + last + 1, runs = (vis + run - 1) / run;
  const int64_t step = (int64_t)a.tokens * a.nq;
  const float *po = a.part_o + at * DH + lane * E, *pm = a.part_ml + at * 2;
  float m = -INFINITY, l = 0.f, y[E] = {};
  for (int x0 = wave; x0 < runs; x0 += W * U) {
    float2 ml[U];
    float v[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t x = min(x0 + W * u, runs - 1);
      ml[u] = *(const float2 *)(pm + x * step * 2);
#pragma unroll
      for (int e = 0; e < E; ++e) v[u][e] = po[x * step * DH + e];
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (x0 + W * u >= runs) ml[u].x = -INFINITY;
      top = fmaxf(top, ml[u].x);
    }
    const float ms = top == -INFINITY ? 0.f : top, f0 = fast_exp2(m - ms);
    m = top;
    l *= f0;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] *= f0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (x0 + W * u >= runs) break;  // wave-uniform
      const float f = fast_exp2(ml[u].x - ms);
      l += ml[u].y * f;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] += v[u][e] * f;
    }
  }
  float sum = l, top = m;
  if constexpr (W > 1) {
    __shared__ float s_m[W], s_l[W], s_y[W][DH];
    if (lane == 0) {
      s_m[wave] = m;
      s_l[wave] = l;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_y[wave][lane * E + e] = y[e];
    __syncthreads();
    if (wave != 0) return;
    sum = 0.f;
#pragma unroll
    for (int w = 1; w < W; ++w) top = fmaxf(top, s_m[w]);
    const float ms = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = fast_exp2(s_m[w] - ms);
      sum += s_l[w] * f;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] += s_y[w][lane * E + e] * f;
    }
  }
  const float inv = 1.f / sum;
  T *dst = (T *)a.out + (int64_t)tok * a.o_stride + (int64_t)head * DH + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) store_as(dst + e, sum == 0.f ? 0.f : y[e] * inv);  // (no score above -inf: 0 whatever v holds)
  if (lane == 0 && a.lse) a.lse[at] = (top + log2f(sum)) * kLn2;
}

// weights[slot] += the sum of p over the rows of a sequence's kv head, at most 16, whose scores (base 2) the attention left: four
// slots a thread.  Bound by their bytes, a few hundredths of k's, which the kernel below would read again.
__global__ __launch_bounds__(256) void paged_weights_of_scores_kernel(PagedAttnArgs a, int slabs) {
  const int kvh = blockIdx.x % a.c.n_kv, b = blockIdx.x / a.c.n_kv / slabs;
  const int slot = (blockIdx.x / a.c.n_kv % slabs * 256 + threadIdx.x) * 4;
  const bool ascend = starts_ascend(a.starts, b);
  SeqRange s;
  if (!seq_range(a.starts, a.lens, b, a.tokens, a.max_new, a.max_len, nullptr, s) || !ascend || slot >= s.len) return;
  const int G = a.nq / a.c.n_kv;
  floatx4 sum{0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < s.n; ++i)
    for (int h = 0; h < G; ++h) {
      const int64_t row = (int64_t)(s.start + i) * a.nq + kvh * G + h;
      const float ls = a.lse[row] * kLog2e;
      const floatx4 x = *(const floatx4 *)(scores_at(a, b, kvh, slot, i * G + h) + slot % 32);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += ls == -INFINITY || x[e] == -INFINITY ? 0.f : fast_exp2(x[e] - ls);  // (a hidden slot, also where lse is NaN)
    }
  if (a.c.page_shift >= 2 && slot + 4 <= s.len) {
    const int page = page_of(a.c, b, slot);
    if (page < 0) return;
    floatx4 *w = (floatx4 *)(a.c.weights + weight_offset(a.c, a.layer, page, kvh, slot));
    *w += sum;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (slot + e >= s.len) break;
      const int page = page_of(a.c, b, slot + e);
      if (page >= 0) a.c.weights[weight_offset(a.c, a.layer, page, kvh, slot + e)] += sum[e];
    }
  }
}

// weights[slot] += the sum over the call's rows of p, for fp32: a wave has 32 slots of one kv head and goes over every row that may
// see them, in order (so the sum is the same every time).  Bound by the products of few waves: 1024 tokens after 4096, 32 heads on 8, 625 us,
// 62 TFLOP/s, with 1280 waves on 1024 SIMDs.
template <int DH, bool MASKED>
__global__ __launch_bounds__(kPaThreads) void paged_weights_kernel(PagedAttnArgs a, int slabs) {
  using O = Ops<float, DH>;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int kvh = blockIdx.x % a.c.n_kv, b = blockIdx.x / a.c.n_kv / slabs;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kt = (blockIdx.x / a.c.n_kv % slabs * kPaWaves + wave) * kPaStep;
  const bool ascend = starts_ascend(a.starts, b);
  SeqRange s;
  if (!seq_range(a.starts, a.lens, b, a.tokens, a.max_new, a.max_len, nullptr, s) || !ascend || kt >= s.len) return;
  const int G = a.nq / a.c.n_kv, n0 = s.len - s.n, rows = s.n * G;
  const int page = page_of(a.c, b, min(kt + (lane & 31), s.len - 1));
  const char *kb = a.c.k + (a.layer * a.c.layer_stride + kvh * a.c.head_stride) * 4;
  u32x4 k[2][O::KST];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int x = 16 * tt + r;
    const char *p = kb + slot_offset(a.c, max(__shfl(page, x, 64), 0), min(kt + x, s.len - 1)) * 4;
#pragma unroll
    for (int st = 0; st < O::KST; ++st) k[tt][st] = O::row_frag(p, st, g);
  }
  const float sc = a.scale * kLog2e;
  float sum[8] = {};
  // the first row that sees slot kt
  const int first = MASKED ? 0 : max(0, kt - n0) * G / 16 * 16;
  for (int row0 = first; row0 < rows; row0 += 16) {
    const int row = min(row0 + r, rows - 1), i = row / G, head = kvh * G + row % G;
    const int64_t tok = s.start + i;
    const char *p = (const char *)a.q + (tok * a.q_stride + (int64_t)head * DH) * 4;
    u32x4 q[O::KST];
#pragma unroll
    for (int st = 0; st < O::KST; ++st) q[st] = O::row_frag(p, st, g);
    const float ls = a.lse[tok * a.nq + head] * kLog2e;
    const bool live = row0 + r < rows && ls != -INFINITY;
    float x[8];
    score8<float, DH>(k, q, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int slot = kt + 16 * (e / 4) + 4 * g + e % 4;
      bool seen = slot <= n0 + i;
      if (MASKED) seen = (slot < n0) | (a.mask[tok * a.mask_ld + max(0, min(slot, s.len - 1) - n0)] != 0);
      seen = seen & live & (slot < s.len);
      const float w = fast_exp2(x[e] * sc - ls);
      sum[e] += seen ? w : 0.f;
    }
  }
  // over the 16 rows of a lane group
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float v = sum[e];
    v += row_ror<8>(v);
    v += row_ror<4>(v);
    v += row_ror<2>(v);
    v += row_ror<1>(v);
    const int x = 16 * (e / 4) + 4 * g + e % 4, pg = __shfl(page, x, 64);
    if (r == 0 && kt + x < s.len && pg >= 0) a.c.weights[weight_offset(a.c, a.layer, pg, kvh, kt + x)] += v;
  }
}

// The same for bf16: a workgroup has 256 slots, 64 a wave, whose rows of k stay in registers; the call's rows pass through two LDS
// buffers 32 at a time (with their lse and the last slot that they see), in order.  Where the slots make few workgroups, `parts` of them
// share a slab's rows, every parts-th 32, and leave their sums to the next kernel.  Bound by the products and their exponentials: 4096 tokens
// after 12288 take 1664 to 1814 us in all by the card, 983 to 1069 without the weights (this kernel 682: 0.71 PFLOP/s).
constexpr int kWeightSlots = 256;

template <int DH, bool MASKED>
__global__ __launch_bounds__(256, 2) void paged_chunk_weights_kernel(PagedAttnArgs a, int slabs, int parts) {
  constexpr int RB = DH * 2, CH = RB / 16, KST = DH / 16, LPT = 32 * CH / 256;
  __shared__ __align__(16) char s_q[2][32 * RB];
  __shared__ float s_ls[2][32];
  __shared__ int s_lim[2][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, r = lane & 31;
  const int kvh = blockIdx.x % a.c.n_kv, part = blockIdx.x / a.c.n_kv % parts, rest = blockIdx.x / a.c.n_kv / parts;
  const int b = rest / slabs, slab = rest % slabs * kWeightSlots;
  SeqRange s;
  if (!seq_range(a.starts, a.lens, b, a.tokens, a.max_new, a.max_len, nullptr, s) || slab >= s.len || !starts_ascend(a.starts, b)) return;
  s.start = __builtin_amdgcn_readfirstlane(s.start);
  s.n = __builtin_amdgcn_readfirstlane(s.n);
  s.len = __builtin_amdgcn_readfirstlane(s.len);
  const int G = a.nq / a.c.n_kv, n0 = s.len - s.n, rows = s.n * G, kt = slab + wave * 64;
  const char *kb = a.c.k + (a.layer * a.c.layer_stride + kvh * a.c.head_stride) * 2;
  u32x4 k[2][KST];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int slot = min(kt + 32 * y + r, s.len - 1);
    const char *p = kb + slot_offset(a.c, max(page_of(a.c, b, slot), 0), slot) * 2;
#pragma unroll
    for (int st = 0; st < KST; ++st) k[y][st] = *(const u32x4 *)(p + st * 32 + h * 16);
  }
  const float sc = a.scale * kLog2e;
  const int my_row = tid / CH, my_col = tid % CH;
  u32x4 qr[LPT];
  float ls = 0.f;
  int lim = 0;
  auto load = [&](int row0) {
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
      const int row = min(row0 + my_row + i * (256 / CH), rows - 1);
      qr[i] = *(const u32x4 *)((const char *)a.q + ((int64_t)(s.start + row / G) * a.q_stride + (int64_t)(kvh * G + row % G) * DH) * 2 + my_col * 16);
    }
    if (tid < 32) {
      const int row = min(row0 + tid, rows - 1);
      lim = n0 + row / G;
      ls = a.lse[(int64_t)(s.start + row / G) * a.nq + kvh * G + row % G] * kLog2e;
      if (row0 + tid >= rows || ls == -INFINITY) ls = INFINITY;  // its weights are 0
    }
  };
  auto swz = [](int x) { return CH == 16 ? x & 15 : (x >> 1) & 7; };
  auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
      const int x = my_row + i * (256 / CH);
      *(u32x4 *)(s_q[buf] + x * RB + (my_col ^ swz(x)) * 16) = qr[i];
    }
    if (tid < 32) {
      s_ls[buf][tid] = ls;
      s_lim[buf][tid] = lim;
    }
  };
  float sum[32] = {};
  const int q_at = r * RB + (h ^ swz(r)) * 16;
  // the first tile with a row that sees slot `slab`
  const int first = (MASKED ? 0 : max(0, slab - n0) * G / 32 * 32) + 32 * part, ahead = 32 * parts;
  load(first);
  store(0);
  __syncthreads();
  int buf = 0;
  for (int row0 = first; row0 < rows; row0 += ahead, buf ^= 1) {
    const bool more = row0 + ahead < rows;
    if (more) load(row0 + ahead);
    floatx16 x[2];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[y][e] = 0.f;
#pragma unroll
    for (int st = 0; st < KST; ++st) {
      const u32x4 f = *(const u32x4 *)(s_q[buf] + (q_at ^ (st * 32)));
#pragma unroll
      for (int y = 0; y < 2; ++y)
        x[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k[y][st]), __builtin_bit_cast(bf16x8, f), x[y], 0, 0, 0);
    }
    const float ml = s_ls[buf][r];
    float w[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) w[e] = fast_exp2(fmaf(x[e / 16][e % 16], sc, -ml));
    if (kt + 64 > (MASKED ? n0 : n0 + row0 / G + 1) || row0 + 32 > rows) {
      const int last = s_lim[buf][r];
      const uint8_t *mrow = MASKED ? a.mask + (int64_t)(s.start + last - n0) * a.mask_ld : nullptr;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int slot = kt + 32 * (e / 16) + 8 * (e % 16 / 4) + 4 * h + e % 4;
        bool seen = slot <= last;
        if (MASKED) seen = (slot < n0) | (mrow[max(0, min(slot, s.len - 1) - n0)] != 0);
        seen &= (ml != INFINITY) & (slot < s.len);
        w[e] = seen ? w[e] : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) sum[e] += w[e];
    if (more) store(buf ^ 1);
    __syncthreads();
  }
  // over the 32 rows of a lane half; lane r then has the r-th of its half's 32 slots
  float mine = 0.f;
#pragma unroll
  for (int e = 0; e < 32; ++e) {
    float v = sum[e];
    v += row_ror<8>(v);
    v += row_ror<4>(v);
    v += row_ror<2>(v);
    v += row_ror<1>(v);
    v += __shfl_xor(v, 16, 64);
    mine = r == e ? v : mine;
  }
  const int slot = kt + 32 * (r / 16) + 8 * (r % 16 / 4) + 4 * h + r % 4;
  if (parts > 1) {
    a.part_w[((int64_t)(b * a.c.n_kv + kvh) * parts + part) * slabs * kWeightSlots + slot] = mine;
  } else if (slot < s.len) {
    const int page = page_of(a.c, b, slot);
    if (page >= 0) a.c.weights[weight_offset(a.c, a.layer, page, kvh, slot)] += mine;
  }
}

__global__ __launch_bounds__(kWeightSlots) void paged_weights_join_kernel(PagedAttnArgs a, int slabs, int parts) {
  const int kvh = blockIdx.x % a.c.n_kv, b = blockIdx.x / a.c.n_kv / slabs;
  const int slot = blockIdx.x / a.c.n_kv % slabs * kWeightSlots + threadIdx.x;
  const bool ascend = starts_ascend(a.starts, b);
  SeqRange s;
  if (!seq_range(a.starts, a.lens, b, a.tokens, a.max_new, a.max_len, nullptr, s) || !ascend || slot >= s.len) return;
  const int page = page_of(a.c, b, slot);
  if (page < 0) return;
  const float *p = a.part_w + (int64_t)(b * a.c.n_kv + kvh) * parts * slabs * kWeightSlots + slot;
  float sum = 0.f;
  for (int x = 0; x < parts; ++x) sum += p[(int64_t)x * slabs * kWeightSlots];
  a.c.weights[weight_offset(a.c, a.layer, page, kvh, slot)] += sum;
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
PagedAttnPlan plan_paged_attn(bool bf16, int tokens, int batch, int nq, int n_kv, int max_new, int max_len, bool accumulate) {
  const int G = nq / n_kv;
  PagedAttnPlan p;
  // Up to 16 rows a kernel whose waves take every fourth 32 slots; for bf16 above that the chunks' (at one row a head it takes
  // 634 us for 64 sequences of 4096 to 16384 slots, the first 500; one of 8192: 22.9 and 16.7.  At 32 rows two tiles of the first
  // take 74 us for 32 sequences of 2048, 70 the chunks').
  p.rows = (long)max_new * G <= 16 ? 16 : (bf16 ? kChunkRows : 32);
  // tiles of rows: at most one part-filled for each sequence, and no more than every sequence's longest
  const long busy = tokens < batch ? tokens : batch;
  p.tiles = std::min((long)tokens * G / p.rows + busy, busy * (((long)max_new * G + p.rows - 1) / p.rows));
  // Weights of few rows are summed from their scores (64 sequences of 8700 slots and 32 heads: 34 us for what takes 335 from q
  // and k), as long as those take at most 1 GB
  p.scores_rows = max_new * G;
  p.scores_steps = (max_len + 31) / 32;
  if (!accumulate || p.rows != 16 || (double)p.scores_steps * 128 * p.scores_rows * batch * n_kv > 1e9) p.scores_steps = 0;
  // else, for bf16, from k by workgroups of 256 slots: as many share a slab's rows as give each CU two
  const long slabs = ((long)max_len + kWeightSlots - 1) / kWeightSlots * batch * n_kv;
  p.parts = 1;
  if (accumulate && bf16 && !p.scores_steps && slabs < 512)
    p.parts = (int)std::min((511 + slabs) / slabs, std::min(16L, ((long)max_new * G + 63) / 64));
  p.part_w = p.parts > 1 ? slabs * kWeightSlots * p.parts : 0;
  // A sequence is cut into runs of whole steps (a workgroup's 128 slots or 64), as few as give each CU two workgroups (one where the
  // products of 32 fp32 rows bound them: a tree of 61 nodes over 4000 slots 54 us in 4 runs, 63 in 8).
  const long groups = p.tiles * n_kv, target = p.rows == 32 ? 256 : 512;
  const int whole = p.rows == kChunkRows ? kChunkStep : 128, pieces = (int)(((long)max_len + whole - 1) / whole);
  long want = std::min((target - 1 + groups) / groups, (long)pieces);
  if (p.rows == 16) {
    // The join takes 32 runs in one round (one sequence of 8000 slots 14.7 us in 32 runs, 17.8 in 63), and a wave's two or
    // four steps less than the join does (32 sequences of 250 slots 10.3 us, 14.1 in two runs).
    want = pieces <= (bf16 ? 4 : 2) ? 1 : std::min(want, 32L);
  } else {
    // Each run costs a row's fp32 sums, written and read (0.5 ns), a step 1.3 us (4 of fp32): together least at sqrt(steps x 2600 / rows) runs;
    // halved from `want` to within a factor of sqrt(2) of that, so that workgroups still fill the CUs evenly.  Two trees of 500 nodes
    // 21 us in one run, 44 in two; one of 61 over 4000 slots 26 in 8, 30 in 32.
    const double best = std::sqrt((bf16 ? 2600. : 8000.) * pieces / ((double)tokens * nq));
    while (want > 1 && want > 1.414 * best) want = (want + 1) / 2;
    if (want > 8 && want < 12) want = 8;  // (what a wave of the join takes in one round)
  }
  const long fill = want;
  // With few rows runs of more than 1024 are cut further, so that sequences of different
  // lengths end together (64 of 4096 to 16385 slots, weights and all: 622 us, 681 in runs of 8320).
  if (p.rows == 16) want = std::max(want, std::min((8191 + groups) / groups, (long)max_len / 1024));
  const int splits = (int)std::min(want, (long)std::min(pieces, 128));
  p.run = (pieces + splits - 1) / splits * whole;
  p.splits = (int)(((long)max_len + p.run - 1) / p.run);
  p.run_shift = 0;
  while ((2L << p.run_shift) <= std::min(fill, (long)p.splits)) ++p.run_shift;
  return p;
}

template <typename T, int DH, bool MASKED>
static void attn_of(const PagedAttnArgs &a, const PagedAttnPlan &p, hipStream_t st) {
  const dim3 grid((unsigned)(p.tiles * p.splits * a.c.n_kv)), block(kPaThreads);
  if constexpr (sizeof(T) == 2)
    if (p.rows == kChunkRows) {
      const bool small = a.c.slot_stride < (1 << 24);  // a row's offset in its page in 32 bits
      if (small && a.c.page_shift >= 6) hipLaunchKernelGGL((paged_chunk_kernel<DH, MASKED, 3>), grid, block, 0, st, a, p.splits, p.run);
      else if (small && a.c.page_shift == 5) hipLaunchKernelGGL((paged_chunk_kernel<DH, MASKED, 2>), grid, block, 0, st, a, p.splits, p.run);
      else if (small && a.c.page_shift >= 3) hipLaunchKernelGGL((paged_chunk_kernel<DH, MASKED, 1>), grid, block, 0, st, a, p.splits, p.run);
      else hipLaunchKernelGGL((paged_chunk_kernel<DH, MASKED, 0>), grid, block, 0, st, a, p.splits, p.run);
    }
  const bool one_page = a.c.page_shift >= 5 && a.c.slot_stride < (1 << 24);
  if (p.rows == 16 && one_page) hipLaunchKernelGGL((paged_attn_kernel<T, DH, 1, MASKED, true>), grid, block, 0, st, a, p.splits, p.run);
  else if (p.rows == 16) hipLaunchKernelGGL((paged_attn_kernel<T, DH, 1, MASKED, false>), grid, block, 0, st, a, p.splits, p.run);
  if constexpr (sizeof(T) == 4) {
    if (p.rows == 32 && one_page) hipLaunchKernelGGL((paged_attn_kernel<T, DH, 2, MASKED, true>), grid, block, 0, st, a, p.splits, p.run);
    else if (p.rows == 32) hipLaunchKernelGGL((paged_attn_kernel<T, DH, 2, MASKED, false>), grid, block, 0, st, a, p.splits, p.run);
  }
  // Four waves a row where rows are few beside the runs (one sequence's next token, 32 runs: 14.7 us, 21.5 with one wave a row; 64 of them, 15 runs:
  // 9.1 and 11.1; 6400 rows of a chunk in 12 runs 102 and 94).
  if (p.splits > 8 && (long)a.tokens * a.nq <= (p.rows == 16 ? 256L : 128L) * p.splits)
    hipLaunchKernelGGL((paged_attn_join_kernel<T, DH, 4>), dim3((unsigned)((long)a.tokens * a.nq)), block, 0, st, a, p.rows, p.run);
  else if (p.splits > 1)
    hipLaunchKernelGGL((paged_attn_join_kernel<T, DH, 1>), dim3((unsigned)(((long)a.tokens * a.nq + 3) / 4)), block, 0, st, a, p.rows, p.run);
  if (a.accumulate && a.scores) {
    const int slabs = (a.max_len + 1023) / 1024;
    hipLaunchKernelGGL(paged_weights_of_scores_kernel, dim3((unsigned)((long)slabs * a.c.batch * a.c.n_kv)), block, 0, st, a, slabs);
  } else if (a.accumulate) {
    const int each = sizeof(T) == 2 ? kWeightSlots : kPaWaves * kPaStep, slabs = (a.max_len + each - 1) / each;
    const dim3 all((unsigned)((long)slabs * a.c.batch * a.c.n_kv)), cut(all.x * p.parts);
    if constexpr (sizeof(T) == 2) {
      hipLaunchKernelGGL((paged_chunk_weights_kernel<DH, MASKED>), cut, block, 0, st, a, slabs, p.parts);
      if (p.parts > 1) hipLaunchKernelGGL(paged_weights_join_kernel, all, dim3(kWeightSlots), 0, st, a, slabs, p.parts);
    } else hipLaunchKernelGGL((paged_weights_kernel<DH, MASKED>), all, block, 0, st, a, slabs);
  }
}
template <typename T, int DH>
static void attn_masked(const PagedAttnArgs &a, const PagedAttnPlan &p, hipStream_t st) {
  a.mask ? attn_of<T, DH, true>(a, p, st) : attn_of<T, DH, false>(a, p, st);
}
void launch_paged_attn(const PagedAttnArgs &a, const PagedAttnPlan &p, hipStream_t st) {
  if (a.c.bf16) a.c.dh == 128 ? attn_masked<bf16_t, 128>(a, p, st) : attn_masked<bf16_t, 64>(a, p, st);
  else a.c.dh == 128 ? attn_masked<float, 128>(a, p, st) : attn_masked<float, 64>(a, p, st);
}

}  // namespace dk
