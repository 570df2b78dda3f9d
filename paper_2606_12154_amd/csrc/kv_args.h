// What the C entry points of the paged caches check of their arguments.
#pragma once

#include <hip/hip_runtime.h>

#include "hh.h"
#include "hh_kv.h"

namespace hh {
namespace {

bool aligned(const void* p, size_t a) { return p && reinterpret_cast<uintptr_t>(p) % a == 0; }

hh_status from_hip(hipError_t e) { return e == hipSuccess ? HH_OK : HH_ERR_HIP; }

bool row_type(int32_t t, int* type, int64_t* size) {
  if (t != HH_F32 && t != HH_BF16 && t != HH_F16) return false;
  *type = t == HH_F32 ? kRowF32 : t == HH_BF16 ? kRowBF16 : kRowF16;
  *size = t == HH_F32 ? 4 : 2;
  return true;
}

// Rows of n elements, `stride` apart, in 16-byte steps.
bool row_stride(int64_t stride, int64_t n, int64_t size) {
  return stride >= n && stride <= ((int64_t)1 << 40) && stride * size % 16 == 0;
}

// Sizes alone (the workspace query), then the pointers too.
bool sizes(const hh_kv4_pool* p, const hh_kv4_rows* r) {
  return p && r && p->n_pages >= 1 && p->n_kv_heads >= 1 && p->n_kv_heads <= 1024 && p->max_pages >= 1 &&
         p->max_pages <= 1 << 26 && p->table_rows >= 1 && r->n_seqs >= 1 && r->n_rows >= 1 && r->max_rows >= 1 &&
         r->n_rows < 1 << 30 && r->max_rows < 1 << 30;
}

bool describe(const hh_kv4_pool* p, const hh_kv4_rows* r, Kv4Pool* P, Kv4Rows* R) {
  if (!sizes(p, r)) return false;
  if (!r->row_start && r->n_rows < r->n_seqs) return false;
  *P = Kv4Pool{static_cast<unsigned char*>(p->pool), p->page_table, p->n_pages, p->n_kv_heads, p->max_pages, p->table_rows};
  *R = Kv4Rows{r->row_start, r->first_pos, r->table_row, r->n_seqs, r->n_rows, r->max_rows};
  return true;
}

bool pointers(const hh_kv4_pool* p, const hh_kv4_rows* r) {
  return aligned(p->pool, 16) && aligned(p->page_table, 4) && aligned(r->first_pos, 4) &&
         (!r->row_start || aligned(r->row_start, 4)) && (!r->table_row || aligned(r->table_row, 4));
}

bool rope_table(const float* rope, int32_t len, RopeTable* t) {
  *t = RopeTable{reinterpret_cast<const float2*>(rope), rope ? len : 0};
  return !rope || (aligned(rope, 16) && len >= 1);
}

}  // namespace
}  // namespace hh
