// C entry points of the 8-bit paged cache's operators (include/hh.h): argument
// checks, then the launchers of hh_kv.h.
#include "kv_args.h"

using namespace hh;

static_assert(kKv8Block == HH_KV8_BLOCK, "the header's block");

namespace {

// Queries, or outputs, of n_heads heads of 64.
bool head_rows(const void* p, int32_t dtype, int64_t stride, int32_t n_heads, int* type) {
  int64_t size;
  return aligned(p, 16) && row_type(dtype, type, &size) && row_stride(stride, (int64_t)n_heads * 64, size);
}
bool heads_fit(const Kv4Pool& P, int32_t n_heads) { return n_heads >= 1 && n_heads % P.hkv == 0; }
bool space(const void* workspace, size_t have, size_t need) { return !need || (aligned(workspace, 256) && have >= need); }
bool scale_fits(float scale) { return scale > 0.f && scale <= 0x1p100f; }

// Everything of an attention but its keys.
hh_status attend_args(const Kv4Pool& P, const void* q, int32_t q_dtype, int64_t q_stride, int32_t n_heads, float scale,
                      const float* rope, int32_t rope_len, void* out, int32_t out_dtype, int64_t out_stride,
                      void* workspace, Kv4Attend* A) {
  if (!heads_fit(P, n_heads) || !head_rows(q, q_dtype, q_stride, n_heads, &A->q_type) ||
      !head_rows(out, out_dtype, out_stride, n_heads, &A->out_type) || !rope_table(rope, rope_len, &A->rope) ||
      !scale_fits(scale))
    return HH_ERR_INVALID_ARG;
  A->q = q;
  A->out = out;
  A->q_stride = q_stride;
  A->out_stride = out_stride;
  A->hq = n_heads;
  A->scale = scale * kKv8ScoreScale;
  A->part = static_cast<float*>(workspace);
  return HH_OK;
}

}  // namespace

extern "C" {

hh_status hh_kv8_append(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const void* k, const void* v, int32_t dtype,
                        int64_t k_stride, int64_t v_stride, const float* rope, int32_t rope_len, void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  RopeTable T;
  int type;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows) || !head_rows(k, dtype, k_stride, P.hkv, &type) ||
      !head_rows(v, dtype, v_stride, P.hkv, &type) || !rope_table(rope, rope_len, &T))
    return HH_ERR_INVALID_ARG;
  if (kv8_row_threads(P, R) > kMaxThreads) return HH_ERR_UNSUPPORTED;
  return from_hip(kv8_append(static_cast<hipStream_t>(hip_stream), P, R, k, v, type, k_stride, v_stride, T));
}

hh_status hh_kv8_read(const hh_kv8_pool* pool, const hh_kv8_rows* rows, void* k, void* v, int32_t dtype,
                      int64_t k_stride, int64_t v_stride, void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  int type;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows) || !head_rows(k, dtype, k_stride, P.hkv, &type) ||
      !head_rows(v, dtype, v_stride, P.hkv, &type))
    return HH_ERR_INVALID_ARG;
  if (kv8_row_threads(P, R) > kMaxThreads) return HH_ERR_UNSUPPORTED;
  return from_hip(kv8_read(static_cast<hipStream_t>(hip_stream), P, R, k, v, type, k_stride, v_stride));
}

hh_status hh_kv8_attention_workspace(const hh_kv8_pool* pool, const hh_kv8_rows* rows, int32_t n_heads, size_t* bytes) {
  Kv4Pool P;
  Kv4Rows R;
  if (!bytes || !describe(pool, rows, &P, &R) || !heads_fit(P, n_heads)) return HH_ERR_INVALID_ARG;
  const Kv8Plan plan = kv8_plan(P, R, n_heads, P.max_pages);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  *bytes = plan.workspace;
  return HH_OK;
}

hh_status hh_kv8_attention(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const void* q, int32_t q_dtype,
                           int64_t q_stride, int32_t n_heads, float scale, const float* rope, int32_t rope_len,
                           void* out, int32_t out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  Kv4Attend A;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows)) return HH_ERR_INVALID_ARG;
  const hh_status s = attend_args(P, q, q_dtype, q_stride, n_heads, scale, rope, rope_len, out, out_dtype, out_stride, workspace, &A);
  if (s != HH_OK) return s;
  const Kv8Plan plan = kv8_plan(P, R, n_heads, P.max_pages);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  if (!space(workspace, workspace_bytes, plan.workspace)) return HH_ERR_INVALID_ARG;
  return from_hip(kv8_attend(static_cast<hipStream_t>(hip_stream), P, R, A, plan));
}

hh_status hh_kv8_select_workspace(const hh_kv8_pool* pool, const hh_kv8_rows* rows, int32_t n_heads, int32_t n_blocks,
                                  size_t* bytes) {
  Kv4Pool P;
  Kv4Rows R;
  if (!bytes || !describe(pool, rows, &P, &R) || !heads_fit(P, n_heads) || n_blocks < 1) return HH_ERR_INVALID_ARG;
  if (n_blocks > HH_KV8_MOST_BLOCKS || P.max_pages > kMaxSelectPages) return HH_ERR_UNSUPPORTED;
  const Kv8SelectPlan plan = kv8_select_plan(P, R);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  *bytes = plan.workspace;
  return HH_OK;
}

hh_status hh_kv8_select(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const void* q, int32_t q_dtype,
                        int64_t q_stride, int32_t n_heads, const float* rope, int32_t rope_len, int32_t n_blocks,
                        int32_t keep_first, int32_t keep_last, int32_t* blocks, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  Kv8Select S;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows) || !heads_fit(P, n_heads) ||
      !head_rows(q, q_dtype, q_stride, n_heads, &S.q_type) || !rope_table(rope, rope_len, &S.rope) || n_blocks < 1 ||
      keep_first < 0 || keep_last < 1 || (int64_t)keep_first + keep_last > n_blocks || !aligned(blocks, 4))
    return HH_ERR_INVALID_ARG;
  if (n_blocks > HH_KV8_MOST_BLOCKS || P.max_pages > kMaxSelectPages) return HH_ERR_UNSUPPORTED;
  const Kv8SelectPlan plan = kv8_select_plan(P, R);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  if (!space(workspace, workspace_bytes, plan.workspace)) return HH_ERR_INVALID_ARG;
  S.q = q;
  S.q_stride = q_stride;
  S.hq = n_heads;
  S.n = n_blocks;
  S.first = keep_first;
  S.last = keep_last;
  S.out = blocks;
  S.keys = static_cast<unsigned*>(workspace);
  S.pitch = kv8_score_pitch(P.max_pages);
  return from_hip(kv8_select(static_cast<hipStream_t>(hip_stream), P, R, S, plan));
}

hh_status hh_kv8_attention_blocks_workspace(const hh_kv8_pool* pool, const hh_kv8_rows* rows, int32_t n_heads,
                                            int32_t n_blocks, size_t* bytes) {
  Kv4Pool P;
  Kv4Rows R;
  if (!bytes || !describe(pool, rows, &P, &R) || !heads_fit(P, n_heads) || n_blocks < 1) return HH_ERR_INVALID_ARG;
  if (n_blocks > HH_KV8_MOST_BLOCKS) return HH_ERR_UNSUPPORTED;
  const Kv8ListPlan plan = kv8_list_plan(P, R, n_heads, n_blocks);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  *bytes = plan.workspace;
  return HH_OK;
}

hh_status hh_kv8_attention_blocks(const hh_kv8_pool* pool, const hh_kv8_rows* rows, const int32_t* blocks,
                                  int32_t n_blocks, const void* q, int32_t q_dtype, int64_t q_stride, int32_t n_heads,
                                  float scale, const float* rope, int32_t rope_len, void* out, int32_t out_dtype,
                                  int64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  Kv4Pool P;
  Kv4Rows R;
  Kv4Attend A;
  if (!describe(pool, rows, &P, &R) || !pointers(pool, rows) || !aligned(blocks, 4) || n_blocks < 1)
    return HH_ERR_INVALID_ARG;
  const hh_status s = attend_args(P, q, q_dtype, q_stride, n_heads, scale, rope, rope_len, out, out_dtype, out_stride, workspace, &A);
  if (s != HH_OK) return s;
  if (n_blocks > HH_KV8_MOST_BLOCKS) return HH_ERR_UNSUPPORTED;
  const Kv8ListPlan plan = kv8_list_plan(P, R, n_heads, n_blocks);
  if (plan.threads > kMaxThreads) return HH_ERR_UNSUPPORTED;
  if (!space(workspace, workspace_bytes, plan.workspace)) return HH_ERR_INVALID_ARG;
  return from_hip(kv8_attend_list(static_cast<hipStream_t>(hip_stream), P, R, A, Kv8List{blocks, n_blocks}, plan));
}

}  // extern "C"
