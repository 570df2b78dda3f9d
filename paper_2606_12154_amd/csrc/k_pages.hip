// Pages of a paged cache: copies between pages and compaction of a pool, in
// every layer at once.  Both only move bytes; a layer's pool holds its pages
// one after the other.
#include "hh_device.h"
#include "hh_kv.h"

#include <algorithm>

namespace hh {
namespace {

// Copies go in pieces of 2 KiB, one a wave (two 16-byte loads a lane in flight);
// pieces of a page are whole but for its last.  What bounds them is memory:
// written lines are not kept in the caches (63 copies of one 512 KiB page: 8.4 ->
// 7.1 us), and where pages are read once and are too many for the caches,
// neither are read ones (1,500 pages of 147 KB: 95.5 -> 92.6 us, 4.8 TB/s of
// reads and writes; a large plain copy reaches 5.0).  Pieces of 4 KiB took 0.8 us
// more, of 8 KiB half as long again.
constexpr int kPiece = 2048;
constexpr int64_t kCached = (int64_t)64 << 20;  // bytes that may still be in the caches

template <bool ONCE>
__device__ __forceinline__ void copy_piece(const unsigned char* __restrict__ src, unsigned char* __restrict__ dst,
                                           int64_t bytes, int piece) {
  const int lane = threadIdx.x & 63;
  const int64_t off = (int64_t)piece * kPiece + lane * 16;
  u32x4 v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (off + i * 1024 < bytes) {
      const u32x4* p = reinterpret_cast<const u32x4*>(src + off + i * 1024);
      v[i] = ONCE ? __builtin_nontemporal_load(p) : *p;
    }
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (off + i * 1024 < bytes) __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(dst + off + i * 1024));
}

// Pairs travel as kernel arguments (at most 4 KiB of them a launch).
constexpr int kPairs = 480;
struct PairArgs {
  int n;
  int src[kPairs], dst[kPairs];
};

template <bool ONCE>
__global__ __launch_bounds__(256) void k_copy_pages(PagePool P, int pieces, PairArgs a) {
  int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int piece = (int)(w % pieces);
  w /= pieces;
  const int pair = (int)(w % a.n), layer = (int)(w / a.n);
  if (layer >= P.n_layers) return;
  unsigned char* base = P.pool + layer * P.layer_stride;
  copy_piece<ONCE>(base + a.src[pair] * P.bytes, base + a.dst[pair] * P.bytes, P.bytes, piece);
}

// ------------------------------------------------------------------ compaction

constexpr int kPlanThreads = 1024;

// Sum of v over the threads before this one; total: over all of them.
__device__ __forceinline__ int exclusive_scan(int v, int* red, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) red[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before += red[w];
    total += red[w];
  }
  __syncthreads();
  return before + x - v;
}

// One workgroup finds the live pages (a bit each in LDS), their count, and the
// moves: live pages behind the count, in order, to the free ones before it.
// moves: [0] their number, then sources, destinations and the new id of every
// page that moves.
__global__ __launch_bounds__(kPlanThreads) void k_compact_plan(int n_pages, const int* __restrict__ table, int rows,
                                                               int max_pages, const int* __restrict__ lengths,
                                                               int* __restrict__ live, int* moves) {
  extern __shared__ unsigned bits[];
  __shared__ int red[kPlanThreads / 64];
  const int t = threadIdx.x, words = (n_pages + 31) / 32;
  for (int i = t; i < words; i += kPlanThreads) bits[i] = 0u;
  __syncthreads();
  const int wave = t >> 6, lane = t & 63;
  for (int r = wave; r < rows; r += kPlanThreads / 64) {
    const int held = min((max(lengths[r], 0) + (int64_t)kPage - 1) / kPage, (int64_t)max_pages);
    for (int i = lane; i < held; i += 64) {
      const int id = table[(size_t)r * max_pages + i];
      if ((unsigned)id < (unsigned)n_pages) atomicOr(&bits[id >> 5], 1u << (id & 31));
    }
  }
  __syncthreads();
  // Thread t has words w0 .. w1 - 1.
  const int per = (words + kPlanThreads - 1) / kPlanThreads;
  const int w0 = min(t * per, words), w1 = min(w0 + per, words);
  int mine = 0;
  for (int i = w0; i < w1; ++i) mine += __popc(bits[i]);
  int count, moved, holes;
  exclusive_scan(mine, red, count);
  // Bits of word i for the ids at or behind the count.
  auto behind = [&](int i) { return i * 32 >= count ? ~0u : i * 32 + 32 <= count ? 0u : ~0u << (count - i * 32); };
  int from = 0, to = 0;
  for (int i = w0; i < w1; ++i) {
    from += __popc(bits[i] & behind(i));
    to += __popc(~bits[i] & ~behind(i));
  }
  int a = exclusive_scan(from, red, moved), b = exclusive_scan(to, red, holes);
  int* src = moves + 1;
  int* dst = src + n_pages;
  int* to_id = dst + n_pages;
  for (int i = w0; i < w1; ++i) {
    for (unsigned m = bits[i] & behind(i); m; m &= m - 1) src[a++] = i * 32 + __ffs(m) - 1;
    for (unsigned m = ~bits[i] & ~behind(i); m; m &= m - 1) dst[b++] = i * 32 + __ffs(m) - 1;
  }
  __threadfence_block();
  __syncthreads();
  for (int i = t; i < moved; i += kPlanThreads) to_id[src[i]] = dst[i];
  if (t == 0) {
    moves[0] = moved;
    *live = count;
  }
}

// The first move_groups workgroups copy, the others rewrite the page tables.
template <bool ONCE>
__global__ __launch_bounds__(256) void k_compact_move(PagePool P, int pieces, const int* __restrict__ moves,
                                                      int move_groups, int* __restrict__ table, int rows,
                                                      int max_pages, const int* __restrict__ lengths,
                                                      const int* __restrict__ live) {
  const int* src = moves + 1;
  const int* dst = src + P.n_pages;
  const int* to_id = dst + P.n_pages;
  if ((int)blockIdx.x < move_groups) {
    const int n = moves[0];
    const int64_t all = (int64_t)n * pieces * P.n_layers;
    for (int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < all;
         w += (int64_t)move_groups * 4) {
      const int64_t rest = w / pieces;
      const int i = (int)(rest % n), layer = (int)(rest / n);
      unsigned char* base = P.pool + layer * P.layer_stride;
      copy_piece<ONCE>(base + src[i] * P.bytes, base + dst[i] * P.bytes, P.bytes, (int)(w % pieces));
    }
    return;
  }
  const int count = *live;
  const int group = blockIdx.x - move_groups, groups = gridDim.x - move_groups;
  for (int r = group; r < rows; r += groups) {
    const int held = min((max(lengths[r], 0) + (int64_t)kPage - 1) / kPage, (int64_t)max_pages);
    for (int i = threadIdx.x; i < held; i += 256) {
      const size_t at = (size_t)r * max_pages + i;
      const int id = table[at];
      if (id >= count && id < P.n_pages) table[at] = to_id[id];
    }
  }
}

// ------------------------------------------------------------------ streams

struct ForkArgs {
  int n, has_last;
  int ids[kForks], last[kForks];
};

// One row of workgroups a fork; nothing that it reads does it write.
__global__ __launch_bounds__(256) void k_fork_streams(int src, int len, int max_ctx, int max_pages, ForkArgs a,
                                                      int* __restrict__ table, int* __restrict__ pos,
                                                      int* __restrict__ pending, unsigned long long* __restrict__ slot,
                                                      int* __restrict__ hist) {
  const int s = a.ids[blockIdx.y], full = len / kPage;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < len) hist[(size_t)s * max_ctx + i] = hist[(size_t)src * max_ctx + i];
  if (i < full) table[(size_t)s * max_pages + i] = table[(size_t)src * max_pages + i];
  if (i == 0) {
    if (a.has_last) table[(size_t)s * max_pages + full] = a.last[blockIdx.y];
    pos[s] = len;
    pending[s] = pending[src];
    slot[s] = 0ull;
  }
}

__global__ void k_truncate_stream(int s, int len, int max_ctx, int* __restrict__ pos, int* __restrict__ pending,
                                  const int* __restrict__ hist, int* __restrict__ entry, int page) {
  if (entry) *entry = page;
  pos[s] = len;
  pending[s] = hist[(size_t)s * max_ctx + len - 1];
}

__global__ __launch_bounds__(256) void k_zero_floats(float* __restrict__ p, size_t n) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i + 4 <= n) {
    *reinterpret_cast<f32x4*>(p + i) = f32x4{0.f, 0.f, 0.f, 0.f};
  } else {
    for (size_t j = i; j < n; ++j) p[j] = 0.f;
  }
}

int pieces_of(const PagePool& P) { return (int)((P.bytes + kPiece - 1) / kPiece); }

}  // namespace

hipError_t copy_pages(hipStream_t st, const PagePool& P, int n, const int* src, const int* dst, bool once) {
  once = once && n * P.bytes * P.n_layers > kCached;
  const int pieces = pieces_of(P);
  // Layers and pairs of a launch, which has fewer than 2^32 threads.
  constexpr int64_t kWaves = 1 << 25;
  const int layers = (int)std::min<int64_t>(P.n_layers, kWaves / pieces);  // (a page has 2^15 pieces at most)
  const int most = (int)std::min<int64_t>(kPairs, kWaves / pieces / layers);
  for (int l = 0; l < P.n_layers; l += layers) {
    PagePool Q = P;
    Q.pool += l * P.layer_stride;
    Q.n_layers = std::min(layers, P.n_layers - l);
    for (int o = 0; o < n; o += most) {
      PairArgs a;
      a.n = std::min(most, n - o);
      for (int i = 0; i < a.n; ++i) {
        a.src[i] = src[o + i];
        a.dst[i] = dst[o + i];
      }
      const unsigned groups = (unsigned)(((int64_t)a.n * pieces * Q.n_layers + 3) / 4);
      const hipError_t e = launch(once ? k_copy_pages<true> : k_copy_pages<false>, groups, 256, 0, st, Q, pieces, a);
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

size_t compact_workspace(int n_pages) { return ((size_t)1 + 3 * (size_t)n_pages) * sizeof(int); }

hipError_t compact_pages(hipStream_t st, const PagePool& P, int* table, int table_rows, int max_pages,
                         const int* lengths, int* live, void* ws) {
  int* moves = static_cast<int*>(ws);
  const size_t lds = (size_t)(P.n_pages + 31) / 32 * 4;
  static_assert(kMaxCompactPages / 8 + 1024 <= 160 * 1024, "LDS");
  if (lds > 48 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_compact_plan),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, kMaxCompactPages / 8);
    if (e != hipSuccess) return e;
  }
  const hipError_t e =
      launch(k_compact_plan, 1, kPlanThreads, lds, st, P.n_pages, table, table_rows, max_pages, lengths, live, moves);
  if (e != hipSuccess) return e;
  const int pieces = pieces_of(P);
  // At most half the pool moves; the loop takes what is left beyond 2,048 workgroups.
  const int64_t most = ((int64_t)P.n_pages / 2 + 1) * pieces * P.n_layers;
  const int move_groups = (int)std::min<int64_t>((most + 3) / 4, 2048);
  const int table_groups = std::min(table_rows, 256);
  const unsigned all = move_groups + table_groups;
  // (Their number is known to the device alone: half of the pool at most.)
  const bool once = P.n_pages / 2 * P.bytes * P.n_layers > kCached;
  return launch(once ? k_compact_move<true> : k_compact_move<false>, all, 256, 0, st, P, pieces, moves, move_groups, table,
                table_rows, max_pages, lengths, live);
}

hipError_t fork_streams(hipStream_t st, int src, int n, const int* ids, const int* last, int len, int max_ctx,
                        int max_pages, int* table, int* pos, int* pending, unsigned long long* slot, int* hist) {
  ForkArgs a{};
  a.n = n;
  a.has_last = last != nullptr;
  for (int i = 0; i < n; ++i) {
    a.ids[i] = ids[i];
    a.last[i] = last ? last[i] : 0;
  }
  const dim3 grid((unsigned)std::max(1, (len + 255) / 256), (unsigned)n);
  return launch(k_fork_streams, grid, 256, 0, st, src, len, max_ctx, max_pages, a, table, pos, pending, slot, hist);
}

hipError_t truncate_stream(hipStream_t st, int s, int len, int max_ctx, int* pos, int* pending, const int* hist,
                           int* entry, int page) {
  return launch(k_truncate_stream, 1, 1, 0, st, s, len, max_ctx, pos, pending, hist, entry, page);
}

void zero_floats(hipStream_t st, float* p, size_t n) {
  if (n > 0) k_zero_floats<<<(unsigned)((n + 1023) / 1024), 256, 0, st>>>(p, n);
}

}  // namespace hh
