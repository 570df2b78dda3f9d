// Launchers of the quantized paged caches' kernels (4 bits: k_kv4.hip; 8 bits:
// k_kv8.hip, k_kv8_select.hip) and of the page kernels (k_pages.hip); arguments have
// been checked by the callers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kv4_plan.h"
#include "kv8_plan.h"

namespace hh {

constexpr int kKv4Block = 1152;  // bytes of one (page, kv head): codes 512 + 512, scales 64 + 64

enum RowType { kRowF32 = 0, kRowBF16 = 1, kRowF16 = 2 };

struct Kv4Pool {
  unsigned char* pool;
  const int* table;
  int n_pages, hkv, max_pages, table_rows;
};

// row_start and table_row may be null: one row each, table row s.
struct Kv4Rows {
  const int* row_start;
  const int* first_pos;
  const int* table_row;
  int n_seqs, n_rows, max_rows;
  int seq0 = 0;  // a launch's first sequence
};

// fp32 (cos, sin) at [position][pair], or null.
struct RopeTable {
  const float2* at;
  int len;
};

struct Kv4Attend {
  const void* q;
  void* out;
  int64_t q_stride, out_stride;
  int q_type, out_type, hq;
  float scale;
  RopeTable rope;
  float* part;  // workspace: split outputs and statistics
};

// These three return their launches' own status.  Callers refuse sequences whose grid
// has more than kMaxThreads.
constexpr int64_t kMaxThreads = UINT32_MAX;
hipError_t kv4_append(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const void* k, const void* v, int type,
                      int64_t k_stride, int64_t v_stride, RopeTable rope);
hipError_t kv4_read(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, void* k, void* v, int type, int64_t k_stride,
                    int64_t v_stride);
int64_t kv4_row_threads(const Kv4Pool& P, const Kv4Rows& R);  // of a sequence, append and read

// pages: a bound of the pages that a sequence holds.
inline Kv4Plan kv4_plan(const Kv4Pool& P, const Kv4Rows& R, int hq, int pages) {
  return kv4_plan(Kv4Sizes{R.n_seqs, R.n_rows, R.max_rows, hq, P.hkv, pages});
}
hipError_t kv4_attend(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv4Plan& p);

// ---- the 8-bit cache: blocks of another size, descriptions alike
constexpr int kKv8Block = 2176;  // codes 1024 + 1024, summary 64, scales and marks 16 (of 64)
constexpr int kKv8Values = 1024, kKv8Sums = 2048, kKv8Scales = 2112;  // byte offsets
constexpr int kKv8Low = -20, kKv8High = 9;                            // exponents of scales

hipError_t kv8_append(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const void* k, const void* v, int type,
                      int64_t k_stride, int64_t v_stride, RopeTable rope);
hipError_t kv8_read(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, void* k, void* v, int type, int64_t k_stride,
                    int64_t v_stride);
int64_t kv8_row_threads(const Kv4Pool& P, const Kv4Rows& R);

inline Kv8Plan kv8_plan(const Kv4Pool& P, const Kv4Rows& R, int hq, int pages) {
  return kv8_plan(Kv4Sizes{R.n_seqs, R.n_rows, R.max_rows, hq, P.hkv, pages});
}
// (Keys enter the products as a sixteenth: A.scale is the softmax's times this.)
constexpr float kKv8ScoreScale = 16.f;
hipError_t kv8_attend(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv8Plan& p);

// Listed blocks: device [n_rows][hkv][n].
struct Kv8List {
  const int* blocks;
  int n;
};
inline Kv8ListPlan kv8_list_plan(const Kv4Pool& P, const Kv4Rows& R, int hq, int n) {
  return kv8_list_plan(Kv4Sizes{R.n_seqs, R.n_rows, R.max_rows, hq, P.hkv, P.max_pages}, n);
}
hipError_t kv8_attend_list(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv8List& list,
                           const Kv8ListPlan& p);

struct Kv8Select {
  const void* q;
  int64_t q_stride;
  int q_type, hq;
  RopeTable rope;
  int n, first, last;  // blocks a row, forced ones at both ends
  int* out;            // [n_rows][hkv][n]
  unsigned* keys;      // workspace, `pitch` scores a (row, kv head), see Kv8SelectPlan
  int pitch;
};
inline Kv8SelectPlan kv8_select_plan(const Kv4Pool& P, const Kv4Rows& R) {
  return kv8_select_plan(Kv4Sizes{R.n_seqs, R.n_rows, R.max_rows, P.hkv, P.hkv, P.max_pages});
}
hipError_t kv8_select(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv8Select& S, const Kv8SelectPlan& p);

// n_layers pools of pages of `bytes` (a multiple of 16), layer_stride bytes apart.
struct PagePool {
  unsigned char* pool;
  int64_t layer_stride, bytes;
  int n_layers, n_pages;
};
// These return their launches' own status. once: no page is the source of two copies.
hipError_t copy_pages(hipStream_t st, const PagePool& P, int n, const int* src, const int* dst, bool once);
constexpr int kMaxCompactPages = 1 << 20;  // one bit each in LDS: 128 KiB
size_t compact_workspace(int n_pages);
hipError_t compact_pages(hipStream_t st, const PagePool& P, int* table, int table_rows, int max_pages,
                         const int* lengths, int* live, void* ws);

// ---- a context's streams (hh_fork, hh_truncate)
// Streams ids[0 .. n) become the first len positions of stream src: page-table
// entries of its full pages, then last[i] (where given) for the partly filled one;
// position, pending token and argmax history.  One launch, n at most kForks.
constexpr int kForks = 62;
hipError_t fork_streams(hipStream_t st, int src, int n, const int* ids, const int* last, int len, int max_ctx,
                        int max_pages, int* table, int* pos, int* pending, unsigned long long* slot, int* hist);
// Stream s ends at len > 0: its pending token is the argmax of position len - 1, and
// `entry` (where given) of its page table is `page`.
hipError_t truncate_stream(hipStream_t st, int s, int len, int max_ctx, int* pos, int* pending, const int* hist,
                           int* entry, int page);
// p[0 .. n) = 0, as a kernel (a graph's replays may clear memory only so).
void zero_floats(hipStream_t st, float* p, size_t n);

}  // namespace hh
