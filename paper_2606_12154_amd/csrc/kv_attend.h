// What the attention kernels of the quantized caches share: queries as fp16 terms,
// a wave's columns with their running softmax, split outputs and their joining.
//
// Operand columns are (row, query head of the kv head's group) pairs, row-major:
// column c of a sequence is row c / G, head c % G.
#pragma once

#include <cmath>

#include "kv_rows.h"

namespace hh {
namespace {

// Pages of a split, given the pages that a column tile attends to: whole steps of two.
__device__ __forceinline__ int split_pages(int np, int splits) {
  const int pairs = (np + 1) >> 1;
  return 2 * ((pairs + splits - 1) / splits);
}

// A weight as two fp16 terms: what its nearest fp16 number leaves goes into the second
// (two at once: two conversions of pairs and two mixed FMAs, where single
// conversions there and back take twice as many instructions).
__device__ __forceinline__ void split_weights(float a, float b, f16x2& h, f16x2& l) {
  h = f16x2{(_Float16)a, (_Float16)b};
  const unsigned w = __builtin_bit_cast(unsigned, h);
  float x, y;
  asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel_hi:[1,0,0]" : "=v"(x) : "v"(w), "v"(a));
  asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(w), "v"(b));
  l = f16x2{(_Float16)x, (_Float16)y};
}

__device__ __forceinline__ f16x8 join8(f16x4 a, f16x4 b) {
  return f16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// Weights are 2^(S qs - base): base puts a column's largest score so far at
// 2^kOffset, and is raised once a score passes 2^(kOffset + kSlack), which fp16
// still holds, so that a weight is off by 2^-37 of the row's largest at most (half
// of fp16's lowest step, 2^-25).  A higher offset would keep more and raise the base
// more often; with this one later scores of ordinary rows hardly pass the largest of a
// wave's first 32 by the slack's factor of 15, and the step needs no reductions across
// lanes (8,192-token prompt 513 us, as with an offset of 2^7 and a slack of 2^8).
constexpr float kOffset = 12.f, kSlack = 3.9f;

// A base decides a step's weights only as a number: it is found first, and then every
// weight's power is one rounding of S qs - base, the same for equal scores in whatever step they
// come.  From kLarge on the exact product's last bits would show in the weights, and S qs is
// rounded by itself.  Rounding may then lift a power past the slack, so that such bases are looked
// at in every step; from kWhole on a base is the largest score, since the offset would be rounded
// too.
constexpr float kLarge = 0x1p16f, kWhole = 0x1p22f;
__device__ __forceinline__ float base_for(float top) { return fabsf(top) < kWhole ? top - kOffset : top; }
__device__ __forceinline__ float rounded(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// Loads in flight need not land at this barrier: it orders LDS alone.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Where a wave stands: columns c0 .. c0 + 16 NQ - 1 of one (sequence, kv head).
struct Place {
  Seq s;
  int head, G, cols, c0;
  Div group;
};

// The query of the lane's column of a 16-column tile, 8 dimensions of each half:
// as loaded (with its rotation), and as operands.
struct RawQuery {
  RawRow row;
  f32x4 turn[4];
};
// QT: fp16 terms, two of fp32 and rotated queries, one of 16-bit ones that are not
// rotated.  Queries (but for fp16 ones of one term) are scaled by a power of two that puts
// a row's largest element into [2^13, 2^14), so that one term holds any 16-bit
// query and two hold 22 bits of an fp32 one.
// Scores' factor to powers of two is at most 2^80, so that they (sums below 2^37) are finite.
// Where it would be more, different scores lie 2^32 apart at least (queries and keys are
// multiples of 2^-24, whole ones in few columns on the 8-bit cache of 2^-20), and the largest takes all
// whatever the factor.
constexpr float kMostFactor = 0x1p80f;
template <int QT>
struct Query {
  f16x8 h[2], l[QT == 2 ? 2 : 1];
  float qs;  // scores to powers of two
};

// A lane's column in its tile of 16 / PACK.
template <int PACK>
__device__ __forceinline__ int column_of() { return threadIdx.x & (16 / PACK - 1); }
// Columns behind the last one repeat it (and are not written).
__device__ __forceinline__ int column_row(const Place& w, int c) { return (unsigned)min(c, w.cols - 1) / w.group; }

template <int QT, int PACK>
__device__ __forceinline__ void load_query(RawQuery& q, const Place& w, const Kv4Attend& A, int tile) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = w.c0 + 16 * tile + column_of<PACK>();
  const int rw = column_row(w, c), j = min(c, w.cols - 1) - rw * w.G;
  const size_t at = (size_t)(w.s.row0 + rw) * A.q_stride + (w.head * w.G + j) * 64 + 8 * g;
  load_raw(q.row, A.q, at, at + 32, A.q_type);
  if (QT == 2 && A.rope.at) {
    const int pos = min(max(w.s.first + rw, 0), A.rope.len - 1);
    const f32x4* cs = reinterpret_cast<const f32x4*>(A.rope.at + (size_t)pos * 32 + 8 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i) q.turn[i] = cs[i];
  }
}

template <int QT>
__device__ __forceinline__ Query<QT> make_query(const RawQuery& q, const Kv4Attend& A) {
  Query<QT> z;
  if (QT == 1 && A.q_type == kRowF16) {
    z.h[0] = __builtin_bit_cast(f16x8, q.row.w[0]);
    z.h[1] = __builtin_bit_cast(f16x8, q.row.w[1]);
    z.qs = __builtin_amdgcn_fmed3f(A.scale * 1.4426950408889634f, 1e-37f, kMostFactor);
    return z;
  }
  float x[16];
  raw_values(q.row, A.q_type, x);
  if (QT == 2 && A.rope.at) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = x[i], v = x[8 + i], co = q.turn[i >> 1][2 * (i & 1)], si = q.turn[i >> 1][2 * (i & 1) + 1];
      x[i] = u * co - v * si;
      x[8 + i] = v * co + u * si;
    }
  }
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
  top = rows_max(top);
  int e = 0;
  if (top > 0.f && top < INFINITY) e = 14 - __builtin_amdgcn_frexp_expf(top);
  z.qs = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(A.scale * 1.4426950408889634f, -e), 1e-37f, kMostFactor);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float y = __builtin_amdgcn_ldexpf(x[i], e);
    const _Float16 h = (_Float16)y;
    z.h[i >> 3][i & 7] = h;
    if constexpr (QT == 2) z.l[i >> 3][i & 7] = (_Float16)(y - (float)h);
  }
  return z;
}

// A wave's NQ tiles of 16 columns.
// PACK: of up to 8 columns, two copies stand side by side, the left one for the
// first page of a step, the right one for the second, each with zeros in the
// other's operands.  A lane then has four scores a step, not eight of which half
// are of no column, and the copies are joined at the end (32 sequences of 4,000
// positions 24.1 -> 22.2 us, one of 131,072 22.7 -> 21.8, of 300 5.0 -> 4.8).
template <int NQ, int QT, int PACK>
struct Columns {
  static_assert(PACK == 1 || NQ == 1);
  static constexpr int N = 8 / PACK;  // scores of a lane, step and tile
  Query<QT> q[NQ * PACK];
  int lim[NQ];  // keys that the column sees
  f32x4 o[NQ][4], sum[NQ];
  float base[NQ];
  bool first;
  // Bits of what a score has to pass, against its base, for bases to be looked at: kAny (-Inf) at
  // first, and once a base is large.
  static constexpr int kAny = (int)0xff800000, kSome = __builtin_bit_cast(int, kOffset + kSlack);
  int limit;

  __device__ __forceinline__ void start(const Place& w, int most) {
    first = true;
    limit = kAny;
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      base[t] = 0.f;
      lim[t] = min(max(w.s.first + column_row(w, w.c0 + 16 * t + column_of<PACK>()) + 1, 0), most);
    }
  }

  static __device__ __forceinline__ bool right() { return threadIdx.x & 8; }
  __device__ __forceinline__ void pack(const Query<QT>& z) {
    const f16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      q[k].qs = z.qs;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        q[k].h[i] = right() == k ? z.h[i] : zero;
        if constexpr (QT == 2) q[k].l[i] = right() == k ? z.l[i] : zero;
      }
    }
  }

  // A step takes two pages: their scores, the scores' weights, the weighted values.

  // kf[page][half of the dimensions].
  __device__ __forceinline__ void scores(const f16x8 (*kf)[2], f32x4 (*sc)[2]) const {
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x4& y = sc[t][PACK == 2 ? 0 : i];
        const Query<QT>& z = q[PACK == 2 ? i : t];
        if (PACK == 1 || i == 0) y = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (QT == 2) {
          y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][0], z.l[0], y, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][1], z.l[1], y, 0, 0, 0);
        }
        y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][0], z.h[0], y, 0, 0, 0);
        y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][1], z.h[1], y, 0, 0, 0);
      }
  }

  // MASK: slots past a column's keys (the pages' first positions are at0 and at1), and
  // bad ones (N bits), whose keys or values are NaN.  The check of all columns' largest scores
  // is the step's only branch, but for large bases.
  template <bool MASK>
  __device__ __forceinline__ void weights(f32x4 (*sc)[2], int at0, int at1, unsigned bad, f16x8* ph, f16x8* pl) {
    const int g = (threadIdx.x & 63) >> 4;
    float top[NQ], high = -INFINITY;
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      top[t] = -INFINITY;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (MASK) {
          if (bad >> i & 1u) sc[t][i >> 2][i & 3] = NAN;
          if (((PACK == 2 ? right() : i >> 2) ? at1 : at0) + 4 * g + (i & 3) >= lim[t]) sc[t][i >> 2][i & 3] = -INFINITY;
        }
        top[t] = fmaxf(top[t], sc[t][i >> 2][i & 3]);
      }
      high = fmaxf(high, fmaf(top[t], q[t].qs, -base[t]));
    }
    // A wave's first pages set the base: a column that sees none of them sees
    // none of the later ones either.
    if (__builtin_amdgcn_ballot_w64(high > __int_as_float(limit))) {
      bool is_large = false;
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        const float mx = rounded(rows_max(top[t]), q[t].qs);
        float to = mx > -INFINITY ? base_for(mx) : base[t];
        if (!first) to = fmaxf(to, base[t]);
        const float f = first ? 1.f : __builtin_amdgcn_exp2f(base[t] - to);
        base[t] = to;
        is_large = is_large || !(fabsf(to) < kLarge);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[t][j] *= f;
        sum[t] *= f;
      }
      limit = __builtin_amdgcn_ballot_w64(is_large) ? kAny : kSome;
    }
    first = false;
    if (limit == kAny) {
#pragma unroll
      for (int t = 0; t < NQ; ++t)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = sc[t][i >> 2][i & 3];
          sc[t][i >> 2][i & 3] = fabsf(base[t]) < kLarge ? fmaf(x, q[t].qs, -base[t]) : rounded(x, q[t].qs) - base[t];
        }
    } else {
#pragma unroll
      for (int t = 0; t < NQ; ++t)
#pragma unroll
        for (int i = 0; i < N; ++i) sc[t][i >> 2][i & 3] = fmaf(sc[t][i >> 2][i & 3], q[t].qs, -base[t]);
    }
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        f16x2 h, l;
        const float a = sc[t][i >> 2][i & 3], b = sc[t][(i + 1) >> 2][(i + 1) & 3];
        split_weights(__builtin_amdgcn_exp2f(a), __builtin_amdgcn_exp2f(b), h, l);
        ph[t][i] = h[0];
        ph[t][i + 1] = h[1];
        pl[t][i] = l[0];
        pl[t][i + 1] = l[1];
      }
    if constexpr (PACK == 2) {
      ph[0] = on_side(ph[0]);
      pl[0] = on_side(pl[0]);
    }
  }
  // A lane's four weights where its page's values are.
  static __device__ __forceinline__ f16x8 on_side(const f16x8& w) {
    const f16x4 zero = {0, 0, 0, 0}, x = {w[0], w[1], w[2], w[3]};
    return join8(right() ? zero : x, right() ? x : zero);
  }

  // vf[dimension of four].  Weights are summed as they enter the products.
  __device__ __forceinline__ void values(const f16x8* vf, const f16x8* ph, const f16x8* pl) {
    const f16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j], pl[t], o[t][j], 0, 0, 0);
      sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pl[t], sum[t], 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j], ph[t], o[t][j], 0, 0, 0);
      sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, ph[t], sum[t], 0, 0, 0);
    }
  }

  // Behind a wave's steps, the first of which began at position `from`.  An infinity in a query of
  // one term can make every score -Inf, which stands for hidden keys; the softmax of such is NaN.
  // (With two terms the second one is Inf - Inf.)
  __device__ __forceinline__ void finish(int from) {
    if constexpr (QT == 1) {
#pragma unroll
      for (int t = 0; t < NQ; ++t)
        if (sum[t][0] == 0.f && lim[t] > (PACK == 2 && right() ? from + kPage : from)) sum[t][0] = NAN;
    }
  }

  // A column that saw no key has no base.
  __device__ __forceinline__ float base_of(int t) const { return sum[t][0] == 0.f ? -INFINITY : base[t]; }
};

// N consecutive dimensions of column col, from d0 on: the output, or (joined)
// the split's part of it, with base m and sum of weights l.
template <int N>
__device__ __forceinline__ void put(const Kv4Rows& R, const Kv4Attend& A, const Place& w, int col, int d0, const float* x,
                                    float l, float m, bool joined, int split, int splits) {
  if (col >= w.cols) return;
  const int at_row = (unsigned)col / w.group;
  const int rw = w.s.row0 + at_row, hd = w.head * w.G + col - at_row * w.G;
  if (joined) {
    const size_t at = ((size_t)split * R.n_rows + rw) * A.hq + hd;
    float* dst = A.part + at * 64 + d0;
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *reinterpret_cast<f32x4*>(dst + 4 * i) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    if (d0 == 0) {
      float2* ml = reinterpret_cast<float2*>(A.part + (size_t)splits * R.n_rows * A.hq * 64) + at;
      *ml = make_float2(m, l);
    }
    return;
  }
  float y[N];
  const float inv = l == 0.f ? 0.f : 1.0f / l;  // nothing to attend to: 0
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = x[i] * inv;
  store_row<N>(A.out, (size_t)rw * A.out_stride + hd * 64 + d0, A.out_type, y);
}

// Splits that hold keys of column c's tile in a sequence (as the attention
// kernel cut them); 1: the attention kernel wrote the output.  (The joining kernels
// take `every` splits of a row where it is given.)
__device__ __forceinline__ int splits_of(const Kv4Pool& P, const Seq& s, int G, int c, int tile_cols, int splits) {
  const int cols = s.n * G, c0 = c / tile_cols * tile_cols;
  const int row_b = (min(c0 + tile_cols, cols) - 1) / G;
  const int some_see = min(max(s.first + row_b + 1, 0), P.max_pages * kPage);
  const int np = (some_see + kPage - 1) / kPage, per = split_pages(np, splits);
  return per >= np ? 1 : (np + per - 1) / per;
}

// Joins the splits of few (row, head)s, a workgroup each: lane l of wave w has
// dimensions 4 (l % 16) .. + 3 of splits 4 w + l / 16, + 16, ...: all loads are
// in flight at once.
__global__ __launch_bounds__(256) void k_kv_join(Kv4Pool P, Kv4Rows R, Kv4Attend A, int tile_cols, int splits,
                                                   int every) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned b = blockIdx.x, row = b / (unsigned)A.hq;
  const int hd = b - row * A.hq, i = row % (unsigned)R.max_rows;
  const Seq s = load_seq(P, R, R.seq0 + row / (unsigned)R.max_rows);
  if (i >= s.n) return;
  const int G = A.hq / P.hkv;
  const int n = every ? every : splits_of(P, s, G, i * G + hd % G, tile_cols, splits);
  if (n == 1) return;
  const size_t at = (size_t)(s.row0 + i) * A.hq + hd, step = (size_t)R.n_rows * A.hq;
  const float2* ml = reinterpret_cast<const float2*>(A.part + (size_t)splits * step * 64) + at;
  const float* part = A.part + at * 64 + 4 * (lane & 15);
  constexpr int N = kMaxSplits / 16;  // loads of a lane
  f32x4 y[N];
  float2 z[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int sp = k * 16 + wave * 4 + (lane >> 4);
    y[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    z[k] = make_float2(-INFINITY, 0.f);
    if (sp < n) {
      z[k] = ml[sp * step];
      y[k] = *reinterpret_cast<const f32x4*>(part + sp * step * 64);
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < N; ++k) m = fmaxf(m, z[k].x);
  m = rows_max(m);
  float x[5] = {0.f, 0.f, 0.f, 0.f, 0.f};  // 4 dimensions and the sum of weights, against m
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float f = z[k].x > -INFINITY ? __builtin_amdgcn_exp2f(z[k].x - m) : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += f * y[k][j];
    x[4] += f * z[k].y;
  }
#pragma unroll
  for (int j = 0; j < 5; ++j) x[j] = rows_sum(x[j]);
  __shared__ float xs[4][6][16];
  if (lane < 16) {
#pragma unroll
    for (int j = 0; j < 5; ++j) xs[wave][j][lane] = x[j];
    xs[wave][5][lane] = m;
  }
  __syncthreads();
  if (threadIdx.x >= 16) return;
  m = fmaxf(fmaxf(xs[0][5][lane], xs[1][5][lane]), fmaxf(xs[2][5][lane], xs[3][5][lane]));
#pragma unroll
  for (int j = 0; j < 5; ++j) x[j] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = xs[w][5][lane], f = mw > -INFINITY ? __builtin_amdgcn_exp2f(mw - m) : 0.f;
#pragma unroll
    for (int j = 0; j < 5; ++j) x[j] += f * xs[w][j][lane];
  }
  const float inv = x[4] == 0.f ? 0.f : 1.0f / x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] *= inv;
  store_row<4>(A.out, (size_t)(s.row0 + i) * A.out_stride + hd * 64 + 4 * lane, A.out_type, x);
}

// Up to 16 splits of many (row, head)s, 16 lanes each: lane l of them has
// split l's statistics and dimensions 4 l .. + 3.
__global__ __launch_bounds__(256) void k_kv_join_rows(Kv4Pool P, Kv4Rows R, Kv4Attend A, int tile_cols, int splits,
                                                        int every) {
  const int l16 = threadIdx.x & 15;
  const unsigned b = blockIdx.x * 16u + (threadIdx.x >> 4), row = b / (unsigned)A.hq;
  const int hd = b - row * A.hq, i = row % (unsigned)R.max_rows;
  const unsigned sq = row / (unsigned)R.max_rows;
  // (No early return: the lanes of a wave exchange below.)
  const bool in = sq < (unsigned)R.n_seqs;
  const Seq s = load_seq(P, R, R.seq0 + (in ? sq : 0));
  const int G = A.hq / P.hkv;
  const int n = in && i < s.n ? (every ? every : splits_of(P, s, G, i * G + hd % G, tile_cols, splits)) : 1;
  const size_t at = (size_t)(s.row0 + (n > 1 ? i : 0)) * A.hq + hd, step = (size_t)R.n_rows * A.hq;
  const float2* ml = reinterpret_cast<const float2*>(A.part + (size_t)splits * step * 64) + at;
  const float* part = A.part + at * 64 + 4 * l16;
  float2 z = make_float2(-INFINITY, 0.f);
  if (n > 1 && l16 < n) z = ml[l16 * step];
  const float m = row_max16(z.x);
  const float f = z.x > -INFINITY ? __builtin_amdgcn_exp2f(z.x - m) : 0.f;
  const float l = row_sum16(f * z.y);
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < splits; k0 += 4) {
    f32x4 y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      y[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (n > 1 && k0 + k < n) y[k] = *reinterpret_cast<const f32x4*>(part + (k0 + k) * step * 64);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float w = __shfl(f, (k0 + k) & 15, 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] += w * y[k][j];
    }
  }
  if (n == 1) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] *= inv;
  store_row<4>(A.out, (size_t)(s.row0 + i) * A.out_stride + hd * 64 + 4 * l16, A.out_type, x);
}

// The joining kernel's launch; `every`: splits of each row, 0 where they go by its keys.
// Five and more splits of few rows are read at once by a workgroup each (rows of 32
// heads at 3,000, with the attention: one, 16 splits, 8.2 us, by 16 lanes each 9.8; 16,
// 8 splits, 14.8 and 15.2); fewer splits or more rows want fewer workgroups (32 rows,
// 8 splits, 23.5 and 23.1; 64, 2 splits, 33.6 and 31.1).
hipError_t launch_join(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, int tile_cols, int splits,
                       int every) {
  const int64_t outs = (int64_t)R.n_seqs * R.max_rows * A.hq;
  if (splits > 16 || (splits > 4 && outs <= 512))
    return launch(k_kv_join, (unsigned)outs, 256, 0, st, P, R, A, tile_cols, splits, every);
  return launch(k_kv_join_rows, (unsigned)((outs + 15) / 16), 256, 0, st, P, R, A, tile_cols, splits, every);
}

}  // namespace
}  // namespace hh
