// Selecting blocks of an 8-bit cache by their mean keys (gfx950): for a row and kv head
// the n blocks whose summaries score highest with the group's added queries.
//
// Scores are whole numbers times powers of two: the query in 8 bits times a summary's
// 8-bit codes, sums below 2^20, times the summary's scale.  fp32 holds them exactly, so that
// which blocks are selected does not depend on an order of additions.  They are matrix
// products (mfma_i32_16x16x64_i8) of 16 blocks' summaries and 16 rows' queries (one row's
// sixteen times in decode steps), and go into LDS as integers of their order.
//
// Then a wave takes a row, each lane a run of its scores.  The n-th largest is found by
// counting those at or above a guess between the bounds so far, and near either bound by the next
// key there: 4 to 5 counts among 300 to 1,400 scores of ordinary spread, 11 at most (halving
// the integers takes 14, and 30 among equal scores).  What is above it is selected, and of what
// equals it the first blocks; a sum over lanes gives their places.
//
// What bounds it: 32 rows of 600 to 1,400 blocks take 19 us, 10 of them reading 32,000 x 8 lines of
// 128 bytes, of which 80 are used, 6 searching, by one wave of each workgroup alone.  4,000 prompt
// rows of 437 blocks: 44, of which the scores 25 (112 MB of lines out of L2), the search 15, places 4.
// Measured and not kept: a histogram of the scores in LDS before the first guess (2 counts, but 44 ->
// 56), 16 lanes a row (43), 32 rows a workgroup (49).
#include "kv_rows.h"

namespace hh {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ queries and scores

// A pair's rotation, x c - y s and y c + x s, in 64 bits: one product of each is rounded (and
// exact where a query is not the sum of several, 24 bits by 24), then the sum.
__device__ __forceinline__ void turn(double& x, double& y, float2 t) {
  const double c = t.x, s = t.y, u = fma(x, c, -(y * s));
  y = fma(y, c, x * s);
  x = u;
}

__device__ __forceinline__ void load_pair(const void* p, size_t at, int type, float* f) {
  if (type == kRowF32) {
    const float2 v = *reinterpret_cast<const float2*>(static_cast<const float*>(p) + at);
    f[0] = v.x;
    f[1] = v.y;
    return;
  }
  const unsigned w = *reinterpret_cast<const unsigned*>(static_cast<const unsigned short*>(p) + at);
  const f16x2 h = __builtin_bit_cast(f16x2, w);
  f[0] = type == kRowF16 ? (float)h[0] : __uint_as_float(w << 16);
  f[1] = type == kRowF16 ? (float)h[1] : __uint_as_float(w & 0xffff0000u);
}

// Bits of |x| in their order, in two words.
struct Magnitude {
  unsigned hi, lo;
};
__device__ __forceinline__ Magnitude magnitude64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return Magnitude{(unsigned)(u >> 32) & 0x7fffffffu, (unsigned)u};
}
// The least e with |x| <= 127 * 2^e for the upper word of the largest |x| and whether the
// largest has more: |x| = m 2^k, m below 2, and 127 is 2^6 (1 + 63 / 64).
__device__ __forceinline__ int query_exponent(unsigned hi, bool more) {
  const unsigned m = hi & 0xfffffu;
  return (int)(hi >> 20) - 1023 - (m > 0xfc000u || (m == 0xfc000u && more) ? 5 : 6);
}
constexpr unsigned kInf64 = 0x7ff00000u;  // upper words of infinities and NaN: from here on

// Four rows' queries, by a wave: the group's queries added and rotated in 64 bits, as whole
// numbers of at most 127: rint(Q 2^-e), e the least with max|Q| <= 127 2^e; zeros where
// an element is not finite.  Lane l works on row l % 4 of them, dimensions 2 k, 2 k + 1 and the
// same of the other half (k = l / 4).
__device__ __forceinline__ void four_queries(const Kv8Select& S, const Seq& s, int row, int head, int G, signed char (*codes)[64]) {
  const int lane = threadIdx.x & 63, k = lane >> 2;
  const size_t at = (size_t)(s.row0 + row) * S.q_stride + (size_t)head * G * 64 + 2 * k;
  float2 t[2];
  if (S.rope.at) {
    const f32x4 cs = *reinterpret_cast<const f32x4*>(S.rope.at + (size_t)min(max(s.first + row, 0), S.rope.len - 1) * 32 + 2 * k);
    t[0] = make_float2(cs[0], cs[1]);
    t[1] = make_float2(cs[2], cs[3]);
  }
  double x[4] = {0.0, 0.0, 0.0, 0.0};
  for (int j = 0; j < G; j += 4) {  // four heads' loads at once
    float f[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      load_pair(S.q, at + (size_t)min(j + u, G - 1) * 64, S.q_type, f[u]);
      load_pair(S.q, at + (size_t)min(j + u, G - 1) * 64 + 32, S.q_type, f[u] + 2);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] += j + u < G ? (double)f[u][i] : 0.0;
  }
  if (S.rope.at) {
    turn(x[0], x[2], t[0]);
    turn(x[1], x[3], t[1]);
  }
  // Over the 16 lanes of the row.
  auto over = [](unsigned v) { return rows_max(max_dpp<0x128>(max_dpp<0x124>(v))); };
  unsigned top = 0u, more = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, magnitude64(x[i]).hi);
  top = over(top);
#pragma unroll
  for (int i = 0; i < 4; ++i) more |= magnitude64(x[i]).hi == top ? magnitude64(x[i]).lo : 0u;
  more = over(more);
  const bool none = top >= kInf64 || top == 0u;  // (less than 2^-1022 counts as zero)
  const int e = query_exponent(top, more != 0u);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    codes[lane & 3][2 * k + (i & 1) + 16 * (i & 2)] = (signed char)(none ? 0 : (int)rint(__builtin_amdgcn_ldexp(x[i], -e)));
}
// The queries of a workgroup's rows as operands: lane l has row l % 16, dimensions 8 g .. + 7
// of each half (g = l / 16).
__device__ __forceinline__ i32x4 query_operand(const signed char (*codes)[64], int row) {
  const int g = (threadIdx.x & 63) >> 4;
  const u32x2 a = *reinterpret_cast<const u32x2*>(codes[row] + 8 * g), b = *reinterpret_cast<const u32x2*>(codes[row] + 8 * g + 32);
  return i32x4{(int)a[0], (int)a[1], (int)b[0], (int)b[1]};
}

// Where a workgroup stands: `rows` rows of a sequence from row0 on, one kv head.
struct Tile {
  Seq s;
  int row0, head, rows, nb;  // nb: blocks of the last row
};
__device__ __forceinline__ int blocks_of(const Kv4Pool& P, const Seq& s, int row) {
  return min((s.first + row) >> 4, P.max_pages - 1) + 1;
}
__device__ __forceinline__ bool tile_of(Tile& z, const Kv4Pool& P, const Kv4Rows& R, unsigned item, int rows, Div heads, Div tiles) {
  const unsigned b = item / heads, sq = b / tiles;
  z.head = item - b * heads.d;
  z.row0 = (b - sq * tiles.d) * rows;
  z.s = load_seq(P, R, R.seq0 + sq);
  z.rows = min(rows, z.s.n - z.row0);
  z.nb = blocks_of(P, z.s, z.row0 + z.rows - 1);
  return z.rows > 0;
}

// Scores of 64 blocks from 64 i on, i = i0, i0 + step, ... below (blocks + 63) / 64: those of row r to
// keys + r * pitch, as integers of their order (which are never 0), up to the end of the last 16.
// Lane l brings block 64 i + l's page id, a step ahead; the loads of four tiles of 16 blocks
// are in flight together.
__device__ __forceinline__ unsigned id_at(const Kv4Pool& P, const int* table, int i, int nb) {
  const unsigned x = (unsigned)table[min(64 * i + (int)(threadIdx.x & 63), nb - 1)];
  return x < (unsigned)P.n_pages ? x : 0u;  // an id outside the pool reads its first page
}
__device__ __forceinline__ void score_blocks(const Kv4Pool& P, const Tile& z, i32x4 q, unsigned first_id, int i0, int step,
                                             int end, unsigned* keys, int pitch) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int* table = P.table + (size_t)z.s.trow * P.max_pages;
  unsigned id = first_id;
  for (int i = i0; i < end; i += step) {
    const unsigned next = id_at(P, table, i + step, z.nb);
    i32x4 m[4];
    float scale[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const unsigned of = (unsigned)__shfl((int)id, 16 * u + r);
      const unsigned char* blk = P.pool + ((size_t)of * (unsigned)P.hkv + (unsigned)z.head) * kKv8Block;
      const u32x2 a = *reinterpret_cast<const u32x2*>(blk + kKv8Sums + 8 * g);
      const u32x2 b = *reinterpret_cast<const u32x2*>(blk + kKv8Sums + 8 * g + 32);
      m[u] = i32x4{(int)a[0], (int)a[1], (int)b[0], (int)b[1]};
      scale[u] = (float)*reinterpret_cast<const _Float16*>(blk + kKv8Scales + 8);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = 64 * i + 16 * u;
      const i32x4 d = __builtin_amdgcn_mfma_i32_16x16x64_i8(m[u], q, i32x4{0, 0, 0, 0}, 0, 0, 0);
      u32x4 k;
#pragma unroll
      for (int j = 0; j < 4; ++j)  // (+ 0: a negative zero counts as zero)
        k[j] = ordered_bits((float)d[j] * __shfl(scale[u], 4 * g + j) + 0.f);
      if (r < z.rows && at < z.nb) *reinterpret_cast<u32x4*>(keys + r * pitch + at + 4 * g) = k;
    }
    id = next;
  }
}

// The scores of 256 blocks of a row each, for k_kv8_select.
__global__ __launch_bounds__(256) void k_kv8_score(Kv4Pool P, Kv4Rows R, Kv8Select S, Div heads, Div tiles, Div chunks) {
  __shared__ __align__(16) signed char codes[4][64];
  const unsigned item = blockIdx.x / chunks;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), chunk = blockIdx.x - item * chunks.d, i0 = 4 * chunk + wave;
  Tile z;
  if (!tile_of(z, P, R, item, 1, heads, tiles) || z.nb <= S.n || 256 * chunk >= z.nb) return;
  const unsigned id = id_at(P, P.table + (size_t)z.s.trow * P.max_pages, i0, z.nb);
  if (wave == 0) four_queries(S, z.s, z.row0, z.head, S.hq / P.hkv, codes);
  __syncthreads();
  score_blocks(P, z, query_operand(codes, 0), id, i0, 4, min((z.nb + 63) >> 6, 4 * chunk + 4),
               S.keys + ((size_t)(z.s.row0 + z.row0) * P.hkv + z.head) * S.pitch, 0);
}

// ------------------------------------------------------------------ selection

__device__ __forceinline__ float key_value(unsigned k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// A guess between two bounds lo < hi (hi - lo > 1) of the want-th largest key, by the counts
// at_lo > want > at_hi of keys at or above them: in the middle between where the line
// between the counts meets `want`, which is too far for most distributions, and where the
// line between their logarithms does, which is not far enough.  Of eight guesses
// one halves the values and one the integers between, so that the search ends.
struct Bounds {
  unsigned lo, hi;
  float at_lo, at_hi, log_lo, log_hi;  // log_hi: of at_hi + 1/2
};
__device__ __forceinline__ unsigned guess(const Bounds& x, float want, float log_want, int turn) {
  const float a = key_value(x.lo), b = key_value(x.hi);
  const float line = (x.at_lo - want) * __builtin_amdgcn_rcpf(x.at_lo - x.at_hi);
  const float curve = (x.log_lo - log_want) * __builtin_amdgcn_rcpf(x.log_lo - x.log_hi);
  const float part = (turn & 7) == 5 ? 0.5f : 0.5f * (line + curve);
  const unsigned next = min(max(ordered_bits(fmaf(b - a, part, a)), x.lo + 1u), x.hi - 1u);
  return (turn & 7) == 7 ? x.lo + (x.hi - x.lo) / 2 : next;
}

__device__ __forceinline__ unsigned wave_top(unsigned x) {
  return rows_max(max_dpp<0x128>(max_dpp<0x124>(max_dpp<0x4E>(max_dpp<0xB1>(x)))));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned add_dpp(unsigned x) {
  return x + (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
}
// Sum over the lanes up to this one.
__device__ __forceinline__ unsigned scan64(unsigned x) {
  x = add_dpp<0x111, 0xF>(x);  // 1, 2, 4 and 8 lanes back in rows of 16
  x = add_dpp<0x112, 0xF>(x);
  x = add_dpp<0x114, 0xF>(x);
  x = add_dpp<0x118, 0xF>(x);
  x = add_dpp<0x142, 0xA>(x);  // the last lane of the row before, to rows 1 and 3
  return add_dpp<0x143, 0xC>(x);  // lane 31, to rows 2 and 3
}
__device__ __forceinline__ unsigned wave_total(unsigned x) {
  return (unsigned)__builtin_amdgcn_readlane((int)scan64(x), 63);
}

// A workgroup's waves have up to 16 rows and one kv head, TEAM: one row together.  A thread
// has up to E scores of a row, a run of `each` of them (an odd number: runs then start in
// different banks).  READ: the scores are k_kv8_score's.
template <int E, bool TEAM, bool READ>
__global__ __launch_bounds__(1024) void k_kv8_select(Kv4Pool P, Kv4Rows R, Kv8Select S, int rows, Div heads, Div tiles) {
  extern __shared__ __align__(16) unsigned keys[];
  __shared__ __align__(16) signed char codes[16][64];
  __shared__ unsigned counts[3];
  __shared__ uint2 parts[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  Tile z;
  if (!tile_of(z, P, R, blockIdx.x, rows, heads, tiles)) return;
  const int threads = TEAM ? blockDim.x : 64, place = TEAM ? threadIdx.x : lane;  // of a row
  int* outs = S.out + ((size_t)(z.s.row0 + z.row0) * P.hkv + z.head) * S.n;
  const int each = ((z.nb + threads - 1) / threads) | 1, pitch = each * threads;
  if (z.nb > S.n) {
    if constexpr (READ) {
      const u32x4* from = reinterpret_cast<const u32x4*>(S.keys + ((size_t)(z.s.row0 + z.row0) * P.hkv + z.head) * S.pitch);
      for (int i = threadIdx.x; i < (z.nb + 3) / 4; i += blockDim.x) reinterpret_cast<u32x4*>(keys)[i] = from[i];
    } else {
      const unsigned id = id_at(P, P.table + (size_t)z.s.trow * P.max_pages, wave, z.nb);
      for (int row = 4 * wave; row < z.rows; row += 4 * waves)
        four_queries(S, z.s, z.row0 + min(row + (lane & 3), z.rows - 1), z.head, S.hq / P.hkv, codes + row);
      __syncthreads();
      score_blocks(P, z, query_operand(codes, min(lane & 15, z.rows - 1)), id, wave, waves, (z.nb + 63) >> 6, keys, pitch);
    }
    if (threadIdx.x < 3) counts[threadIdx.x] = 0;
    __syncthreads();
  }
  for (int row = TEAM ? 0 : wave; row < z.rows; row += TEAM ? 1 : waves) {
    const int nb = blocks_of(P, z.s, z.row0 + row);
    int* out = outs + (size_t)row * P.hkv * S.n;
    if (nb <= S.n) {
      for (int i = place; i < S.n; i += threads) out[i] = i < nb ? i : -1;
      continue;
    }
    // The forced blocks at both ends are 0 .. S.first - 1 and tail ...
    const int tail = nb - S.last, want = S.n - S.first - S.last;
    for (int i = place; i < S.first; i += threads) out[i] = i;
    for (int i = place; i < S.last; i += threads) out[S.n - S.last + i] = tail + i;
    if (want == 0) continue;
    unsigned key[E], high = 0u, low = 0u;  // the largest, and the largest complement
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int b = place * each + i;
      key[i] = i < each && b >= S.first && b < tail ? keys[row * pitch + b] : 0u;
      high = max(high, key[i]);
      low = max(low, key[i] ? ~key[i] : 0u);
    }
    high = wave_top(high);
    low = wave_top(low);
    if constexpr (TEAM) {
      if (lane == 0) parts[wave] = make_uint2(high, low);
      __syncthreads();
      for (int v = 0; v < waves; ++v) {
        high = max(high, parts[v].x);
        low = max(low, parts[v].y);
      }
    }
    // Counts over several waves go through LDS, three places in turn.
    int turn = 0;
    auto count = [&](unsigned least) {
      unsigned n = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) n += key[i] >= least;
      n = wave_total(n);
      if constexpr (TEAM) {
        const int at = turn % 3;
        if (lane == 0) atomicAdd(&counts[at], n);
        __syncthreads();
        n = counts[at];
        if (threadIdx.x == 0) counts[at == 0 ? 2 : at - 1] = 0;
      }
      return (int)n;
    };
    // The want-th largest key is at least lo and below hi.
    Bounds x;
    x.lo = ~low;
    x.hi = high + 1u;
    x.at_lo = (float)(tail - S.first);
    x.at_hi = 0.f;
    x.log_lo = __builtin_amdgcn_logf(x.at_lo);
    x.log_hi = -1.f;
    const float wanted = (float)want, log_want = __builtin_amdgcn_logf(wanted);
    // Near either bound the next key there is the guess, so that equal ones end the search.
    auto over_all = [&](unsigned v) {
      v = wave_top(v);
      if constexpr (TEAM) {
        __syncthreads();
        if (lane == 0) parts[wave].x = v;
        __syncthreads();
        for (int w = 0; w < waves; ++w) v = max(v, parts[w].x);
      }
      return v;
    };
    while (x.hi - x.lo > 1u && x.at_lo > wanted) {
      unsigned next;
      const bool from_lo = x.at_lo - wanted <= 2.f, from_hi = !from_lo && wanted - x.at_hi <= 2.f;
      if (from_lo) {
        unsigned v = 0u;
#pragma unroll
        for (int i = 0; i < E; ++i) v = max(v, key[i] >= x.lo ? ~key[i] : 0u);
        next = ~over_all(v) + 1u;
      } else if (from_hi) {
        unsigned v = 0u;
#pragma unroll
        for (int i = 0; i < E; ++i) v = max(v, key[i] < x.hi ? key[i] : 0u);
        next = over_all(v);
      } else {
        next = guess(x, wanted, log_want, turn);
      }
      const int n = count(next);
      ++turn;
      if (n >= want) {
        x.lo = next;
        x.at_lo = (float)n;
        x.log_lo = __builtin_amdgcn_logf(x.at_lo);
        if (from_hi) x.hi = next + 1u;
      } else {
        x.hi = next;
        x.at_hi = (float)n;
        x.log_hi = __builtin_amdgcn_logf(x.at_hi + 0.5f);
        if (from_lo) x.lo = next - 1u;
      }
    }
    const unsigned lo = x.lo;
    // Keys above lo are all selected, and of those equal to it the first ones: the
    // numbers of both, in one word each 16 bits, of the threads before this one and of all.
    uint64_t above = 0, tie = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      above |= (uint64_t)(key[i] > lo) << i;
      tie |= (uint64_t)(key[i] == lo) << i;
    }
    const unsigned mine = (unsigned)__builtin_popcountll(above) | (unsigned)__builtin_popcountll(tie) << 16;
    const unsigned upto = scan64(mine);
    unsigned before = upto - mine, total = (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
    if constexpr (TEAM) {
      __syncthreads();
      if (lane == 0) parts[wave].x = total;
      __syncthreads();
      total = 0u;
      for (int v = 0; v < waves; ++v) {
        if (v < wave) before += parts[v].x;
        total += parts[v].x;
      }
    }
    const int spare = want - (int)(total & 0xffffu), equal = before >> 16;
    while (tie && equal + __builtin_popcountll(tie) > spare) tie &= ~(1ull << (63 - __builtin_clzll(tie)));
    above |= tie;
    int* to = out + S.first + (before & 0xffffu) + min(equal, spare);
    for (; above; above &= above - 1) *to++ = place * each + __builtin_ctzll(above);
  }
}

typedef void (*Select)(Kv4Pool, Kv4Rows, Kv8Select, int, Div, Div);

}  // namespace

hipError_t kv8_select(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv8Select& S, const Kv8SelectPlan& p) {
  const Select kernel = p.chunks       ? k_kv8_select<33, true, true>
                        : p.team       ? k_kv8_select<33, true, false>
                        : p.keys == 9  ? k_kv8_select<9, false, false>
                        : p.keys == 17 ? k_kv8_select<17, false, false>
                                       : k_kv8_select<33, false, false>;
  if (p.lds > 64 << 10) {
    // More LDS than a kernel may have unasked.  The limit is the process's, so that it is set to the
    // kernel's most: a call on another thread may have one of its own between this one's and its launch.
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(p.team ? kMostTeamLds : kMostRowsLds));
    if (e != hipSuccess) return e;
  }
  const int tiles = (R.max_rows + p.rows - 1) / p.rows;
  return by_sequences(R, p.threads, [&](const Kv4Rows& r) {
    const int64_t items = (int64_t)r.n_seqs * tiles * P.hkv;
    if (p.chunks) {
      const hipError_t e = launch(k_kv8_score, (unsigned)(items * p.chunks), 256, 0, st, P, r, S, div_by(P.hkv), div_by(tiles), div_by(p.chunks));
      if (e != hipSuccess) return e;
    }
    return launch(kernel, (unsigned)items, 64 * p.waves, p.lds, st, P, r, S, p.rows, div_by(P.hkv), div_by(tiles));
  });
}

}  // namespace hh
