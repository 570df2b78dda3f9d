// C entry points of the 4-bit paged cache's operators and of the page
// operators (include/hh.h): argument checks, then the launchers of hh_kv.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>
#include <vector>

#include "kv_args.h"

using namespace hh;

namespace {

static_assert(kKv4Workspace == HH_KV4_WORKSPACE_MOST, "the header's bound");

bool page_pool(void* pool, int32_t n_layers, int64_t layer_stride, int64_t page_bytes, int32_t n_pages, PagePool* P) {
  if (!aligned(pool, 16) || n_layers < 1 || n_layers > 1 << 16 || n_pages < 1 || page_bytes < 16 ||
      page_bytes > (int64_t)1 << 26 || page_bytes % 16 != 0 || (double)page_bytes * n_pages * n_layers > 0x1p60)
    return false;
  if (n_layers > 1 && (layer_stride % 16 != 0 || layer_stride < page_bytes * n_pages)) return false;
  *P = PagePool{static_cast<unsigned char*>(pool), n_layers > 1 ? layer_stride : 0, page_bytes, n_layers, n_pages};
  return true;
}

}  // namespace

extern "C" {

hh_status hh_kv4_append(const hh_kv4_pool* pool, const hh_kv4_rows* rows, const void* k, const void* v, int32_t dtype,
                        int64_t k_stride, int64_t v_stride, const float* rope, int32_t rope_len, void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  RopeTable T;
  int type;
  int64_t size;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows) || !row_type(dtype, &type, &size)) return HH_ERR_INVALID_ARG;
  const int64_t n = (int64_t)P.hkv * 64;
  if (!aligned(k, 16) || !aligned(v, 16) || !row_stride(k_stride, n, size) || !row_stride(v_stride, n, size) ||
      !rope_table(rope, rope_len, &T))
    return HH_ERR_INVALID_ARG;
  if (kv4_row_threads(P, R) > kMaxThreads) return HH_ERR_UNSUPPORTED;
  return from_hip(kv4_append(static_cast<hipStream_t>(hip_stream), P, R, k, v, type, k_stride, v_stride, T));
}

hh_status hh_kv4_read(const hh_kv4_pool* pool, const hh_kv4_rows* rows, void* k, void* v, int32_t dtype,
                      int64_t k_stride, int64_t v_stride, void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  int type;
  int64_t size;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows) || !row_type(dtype, &type, &size)) return HH_ERR_INVALID_ARG;
  const int64_t n = (int64_t)P.hkv * 64;
  if (!aligned(k, 16) || !aligned(v, 16) || !row_stride(k_stride, n, size) || !row_stride(v_stride, n, size))
    return HH_ERR_INVALID_ARG;
  if (kv4_row_threads(P, R) > kMaxThreads) return HH_ERR_UNSUPPORTED;
  return from_hip(kv4_read(static_cast<hipStream_t>(hip_stream), P, R, k, v, type, k_stride, v_stride));
}

hh_status hh_kv4_attention_workspace(const hh_kv4_pool* pool, const hh_kv4_rows* rows, int32_t n_heads, size_t* bytes) {
  Kv4Pool P;
  Kv4Rows R;
  if (!bytes || !describe(pool, rows, &P, &R) || n_heads < 1 || n_heads % P.hkv != 0) return HH_ERR_INVALID_ARG;
  const Kv4Plan plan = kv4_plan(P, R, n_heads, P.max_pages);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  *bytes = plan.workspace;
  return HH_OK;
}

hh_status hh_kv4_attention(const hh_kv4_pool* pool, const hh_kv4_rows* rows, const void* q, int32_t q_dtype,
                           int64_t q_stride, int32_t n_heads, float scale, const float* rope, int32_t rope_len,
                           void* out, int32_t out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  Kv4Attend A;
  int64_t q_size, out_size;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows) || !row_type(q_dtype, &A.q_type, &q_size) ||
      !row_type(out_dtype, &A.out_type, &out_size) || n_heads < 1 || n_heads % P.hkv != 0 ||
      !rope_table(rope, rope_len, &A.rope))
    return HH_ERR_INVALID_ARG;
  const int64_t n = (int64_t)n_heads * 64;
  if (!aligned(q, 16) || !aligned(out, 16) || !row_stride(q_stride, n, q_size) || !row_stride(out_stride, n, out_size) ||
      !(scale > 0.f) || !std::isfinite(scale))
    return HH_ERR_INVALID_ARG;
  const Kv4Plan plan = kv4_plan(P, R, n_heads, P.max_pages);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  if (plan.workspace && (!aligned(workspace, 256) || workspace_bytes < plan.workspace)) return HH_ERR_INVALID_ARG;
  A.q = q;
  A.out = out;
  A.q_stride = q_stride;
  A.out_stride = out_stride;
  A.hq = n_heads;
  A.scale = scale;
  A.part = static_cast<float*>(workspace);
  return from_hip(kv4_attend(static_cast<hipStream_t>(hip_stream), P, R, A, plan));
}

hh_status hh_kv_copy_pages(void* pool, int32_t n_layers, int64_t layer_stride, int64_t page_bytes, int32_t n_pages,
                           int32_t n, const int32_t* src, const int32_t* dst, void* hip_stream) {
  PagePool P;
  if (!page_pool(pool, n_layers, layer_stride, page_bytes, n_pages, &P) || n < 0 || (n > 0 && (!src || !dst)))
    return HH_ERR_INVALID_ARG;
  // A page that is written is written once, and read by no copy of the call.
  std::vector<unsigned char> seen;
  try {
    seen.assign(n_pages, 0);
  } catch (const std::bad_alloc&) {
    return HH_ERR_OOM;
  }
  for (int32_t i = 0; i < n; ++i) {
    if (src[i] < 0 || src[i] >= n_pages || dst[i] < 0 || dst[i] >= n_pages) return HH_ERR_INVALID_ARG;
    if (seen[dst[i]]) return HH_ERR_INVALID_ARG;
    seen[dst[i]] = 1;
  }
  bool once = true;
  for (int32_t i = 0; i < n; ++i) {
    if (seen[src[i]] == 1) return HH_ERR_INVALID_ARG;
    once = once && seen[src[i]] == 0;
    seen[src[i]] = 2;
  }
  if (n == 0) return HH_OK;
  return from_hip(copy_pages(static_cast<hipStream_t>(hip_stream), P, n, src, dst, once));
}

hh_status hh_kv_compact_workspace(int32_t n_pages, size_t* bytes) {
  if (!bytes || n_pages < 1) return HH_ERR_INVALID_ARG;
  if (n_pages > kMaxCompactPages) return HH_ERR_UNSUPPORTED;
  *bytes = compact_workspace(n_pages);
  return HH_OK;
}

hh_status hh_kv_compact(void* pool, int32_t n_layers, int64_t layer_stride, int64_t page_bytes, int32_t n_pages,
                        int32_t* page_table, int32_t table_rows, int32_t max_pages, const int32_t* lengths,
                        int32_t* live, void* workspace, size_t workspace_bytes, void* hip_stream) {
  PagePool P;
  if (!page_pool(pool, n_layers, layer_stride, page_bytes, n_pages, &P) || !aligned(page_table, 4) || table_rows < 1 ||
      max_pages < 1 || max_pages > 1 << 26 || !aligned(lengths, 4) || !aligned(live, 4))
    return HH_ERR_INVALID_ARG;
  if (n_pages > kMaxCompactPages) return HH_ERR_UNSUPPORTED;
  if (!aligned(workspace, 256) || workspace_bytes < compact_workspace(n_pages)) return HH_ERR_INVALID_ARG;
  return from_hip(compact_pages(static_cast<hipStream_t>(hip_stream), P, page_table, table_rows, max_pages, lengths,
                                live, workspace));
}

}  // extern "C"
