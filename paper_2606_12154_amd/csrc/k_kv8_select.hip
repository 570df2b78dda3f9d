// Selecting blocks of an 8-bit cache by their mean keys (gfx950): for a row and kv head
// the n blocks whose summaries score highest with the group's added queries.
//
// Scores are whole numbers times powers of two: the query in 8 bits times a summary's
// 8-bit codes, sums below 2^20, times the summary's scale.  fp32 holds them exactly, so that
// which blocks are selected does not depend on an order of additions.
#include <type_traits>

#include "kv_rows.h"

namespace hh {
namespace {

__device__ __forceinline__ float query_at(const void* q, size_t at, int type) {
  if (type == kRowF32) return static_cast<const float*>(q)[at];
  const unsigned w = static_cast<const unsigned short*>(q)[at];
  return type == kRowF16 ? (float)__builtin_bit_cast(_Float16, (unsigned short)w) : __uint_as_float(w << 16);
}

// Dimension `lane` of the group's queries, added and rotated in 64 bits, as a whole number
// of at most 127: rint(Q 2^-e), e the least with max|Q| <= 127 2^e.  All zeros where an
// element is not finite.
__device__ __forceinline__ int query_code(const Kv8Select& S, const Seq& s, int row, int head, int G) {
  const int lane = threadIdx.x & 63;
  const size_t at = (size_t)(s.row0 + row) * S.q_stride + (size_t)head * G * 64 + lane;
  double x = 0.0;
  for (int j = 0; j < G; ++j) x += (double)query_at(S.q, at + (size_t)j * 64, S.q_type);
  if (S.rope.at) {
    const double y = __shfl_xor(x, 32);
    const float2 t = S.rope.at[(size_t)min(max(s.first + row, 0), S.rope.len - 1) * 32 + (lane & 31)];
    // Pairs (i, i + 32): a c - b s and b c + a s, each rounded once after its sum.
    const double c = t.x, sn = t.y;
    x = lane < 32 ? fma(x, c, -(y * sn)) : fma(x, c, y * sn);
  }
  const bool fine = fabs(x) < (double)INFINITY;
  double top = fabs(x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmax(top, __shfl_xor(top, o));
  if (__builtin_amdgcn_ballot_w64(!fine) || !(top > 0.0)) return 0;
  const int e = __builtin_amdgcn_frexp_exp(top) - (__builtin_amdgcn_frexp_mant(top) <= 127.0 / 128.0 ? 7 : 6);
  return (int)rint(__builtin_amdgcn_ldexp(x, -e));
}

// Lanes with `on` below this one.
__device__ __forceinline__ int below(uint64_t on) {
  return __builtin_amdgcn_mbcnt_hi((unsigned)(on >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)on, 0u));
}

// T threads have one (row, kv head): N scores each, as integers of their order, 0 where
// a block is none or forced.  Wave w of them has the blocks from 64 w `each` on, lane l those
// 64 i + l on from there.
template <int T, int N>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_kv8_select(Kv4Pool P, Kv4Rows R, Kv8Select S, Div heads, Div rows) {
  constexpr int W = T / 64, GROUPS = T < 256 ? 256 / T : 1;  // waves of an item, items of a workgroup
  const int lane = threadIdx.x & 63, in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = W == 1 ? 0 : in_group;
  const unsigned item = blockIdx.x * (unsigned)GROUPS + (W == 1 ? in_group : 0);
  const unsigned b = item / heads, sq = b / rows;
  const int head = item - b * heads.d, row = b - sq * rows.d;
  if (sq >= (unsigned)R.n_seqs) return;
  const Seq s = load_seq(P, R, R.seq0 + sq);
  if (row >= s.n) return;
  int* out = S.out + ((size_t)(s.row0 + row) * P.hkv + head) * S.n;
  // The row's blocks; the forced ones at both ends.
  const int nb = min((s.first + row) >> 4, P.max_pages - 1) + 1;
  if (nb <= S.n) {
    for (int i = wave * 64 + lane; i < S.n; i += T) out[i] = i < nb ? i : -1;
    return;
  }
  const int head_end = S.first, tail = nb - S.last, want = S.n - S.first - S.last;

  // Quarter lane % 4 of the query, for the block of 4 lanes.
  __shared__ __align__(16) signed char codes[GROUPS * W][64];
  codes[in_group][lane] = (signed char)query_code(S, s, row, head, S.hq / P.hkv);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  const u32x4 qc = *reinterpret_cast<const u32x4*>(&codes[in_group][16 * (lane & 3)]);

  const int each = (nb + T - 1) / T, base = 64 * wave * each;
  const int* table = P.table + (size_t)s.trow * P.max_pages;
  unsigned key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    key[i] = 0u;
    if (i < each) {
      const int blk = base + 64 * i + lane;
      const unsigned x = (unsigned)table[min(blk, nb - 1)];
      const unsigned id = x < (unsigned)P.n_pages ? x : 0u;  // an id outside the pool reads its first page
      const size_t pitch = (size_t)P.hkv * kKv8Block, lead = (size_t)head * kKv8Block;
      const unsigned short sc = *reinterpret_cast<const unsigned short*>(P.pool + id * pitch + lead + kKv8Scales + 8);
      int dot = 0;
      // Block U of the four lanes' own.
      auto block = [&](auto u) {
        constexpr int U = decltype(u)::value;
        const unsigned their = (unsigned)__builtin_amdgcn_update_dpp(0, (int)id, U * 0x55, 0xF, 0xF, false);
        const u32x4 m = *reinterpret_cast<const u32x4*>(P.pool + their * pitch + lead + kKv8Sums + 16 * (lane & 3));
        int d = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) d = __builtin_amdgcn_sdot4((int)m[j], (int)qc[j], d, false);
        d += __builtin_amdgcn_update_dpp(0, d, 0xB1, 0xF, 0xF, false);
        d += __builtin_amdgcn_update_dpp(0, d, 0x4E, 0xF, 0xF, false);
        dot = (lane & 3) == U ? d : dot;
      };
      block(std::integral_constant<int, 0>());
      block(std::integral_constant<int, 1>());
      block(std::integral_constant<int, 2>());
      block(std::integral_constant<int, 3>());
      const float score = (float)dot * (float)__builtin_bit_cast(_Float16, sc);
      // (A negative zero counts as zero.)
      if (blk >= head_end && blk < tail) key[i] = ordered_bits(score + 0.f);
    }
  }

  // The want-th largest key: bits from the top, as long as so many keys have them.  Counts
  // over several waves go through LDS, three buffers in turn.
  __shared__ int counts[W == 1 ? 1 : 3];
  __shared__ int2 parts[W];
  auto count = [&](unsigned least, int turn) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < each) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[i] >= least));
    if constexpr (W > 1) {
      if (lane == 0) atomicAdd(&counts[turn], n);
      __syncthreads();
      n = counts[turn];
      if (threadIdx.x == 0) counts[turn == 0 ? 2 : turn - 1] = 0;
    }
    return n;
  };
  if constexpr (W > 1) {
    if (threadIdx.x < 3) counts[threadIdx.x] = 0;
    __syncthreads();
  }
  unsigned least = 0u;
  int turn = 0;
  if (want > 0) {
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned next = least | 1u << bit;
      const int n = count(next, turn);
      turn = turn == 2 ? 0 : turn + 1;
      if (n < want) continue;
      least = next;
      if (n == want) break;
    }
  }
  // Keys above it are all selected, and of those equal to it the first ones.
  int more = 0, same = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < each) {
      more += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[i] > least));
      same += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[i] == least));
    }
  int more_all = more, more_before = 0, same_before = 0;
  if constexpr (W > 1) {
    if (lane == 0) parts[wave] = make_int2(more, same);
    __syncthreads();
    more_all = 0;
    for (int v = 0; v < W; ++v) {
      const int2 z = parts[v];
      if (v < wave) {
        more_before += z.x;
        same_before += z.y;
      }
      more_all += z.x;
    }
  }
  const int spare = want - more_all;
  if (want > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < each) {
        const bool high = key[i] > least, tie = key[i] == least;
        const uint64_t highs = __builtin_amdgcn_ballot_w64(high), ties = __builtin_amdgcn_ballot_w64(tie);
        const int ahead = more_before + below(highs), equal = same_before + below(ties);
        if (high || (tie && equal < spare)) out[S.first + ahead + min(equal, spare)] = base + 64 * i + lane;
        more_before += __builtin_popcountll(highs);
        same_before += __builtin_popcountll(ties);
      }
  }
  for (int i = wave * 64 + lane; i < S.first; i += T) out[i] = i;
  for (int i = wave * 64 + lane; i < S.last; i += T) out[S.n - S.last + i] = tail + i;
}

template <int T>
hipError_t launch_select(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv8Select& S, int keys) {
  const int64_t items = (int64_t)R.n_seqs * R.max_rows * P.hkv;
  const int threads = T < 256 ? 256 : T, each = threads / T;
  const auto kernel = keys == 4 ? k_kv8_select<T, 4> : keys == 16 ? k_kv8_select<T, 16> : k_kv8_select<T, 64>;
  return launch(kernel, (unsigned)((items + each - 1) / each), threads, 0, st, P, R, S, div_by(P.hkv), div_by(R.max_rows));
}

}  // namespace

hipError_t kv8_select(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv8Select& S, const Kv8SelectPlan& p) {
  return by_sequences(R, p.threads, [&](const Kv4Rows& r) {
    return p.lanes == 64    ? launch_select<64>(st, P, r, S, p.keys)
           : p.lanes == 256 ? launch_select<256>(st, P, r, S, p.keys)
                            : launch_select<1024>(st, P, r, S, p.keys);
  });
}

}  // namespace hh
