// Entry points of the paged key-value cache: argument checks on the host, then the launches.  None of
// them allocates, waits or keeps anything between calls.
#include <climits>
#include <cmath>

#include "af_paged.h"

using namespace af;

namespace {

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

af_status refuse(af_status code, const char* what, const char* why) {
  set_error("%s: %s", what, why);
  return code;
}

// Checks the cache and the step's sizes and fills c.
af_status check_cache(const char* me, const af_paged_kv* kv, int32_t M, int32_t n_heads, PagedCache* c) {
  const auto invalid = [me](const char* why) { return refuse(AF_ERR_INVALID_ARG, me, why); };
  const auto unsupported = [me](const char* why) { return refuse(AF_ERR_UNSUPPORTED, me, why); };
  if (!kv) return invalid("kv must be non-NULL");
  if (kv->dtype != AF_BF16 && kv->dtype != AF_F32) return invalid("dtype must be AF_BF16 or AF_F32");
  if (kv->reserved != 0) return invalid("reserved must be 0");
  if (!kv->k || !kv->v || !kv->page_table || !kv->kv_lens) return invalid("k, v, page_table and kv_lens must be non-NULL");
  if (kv->n_pages <= 0 || kv->page_size <= 0 || kv->n_kv_heads <= 0 || kv->n_seq <= 0 || kv->max_pages <= 0 || M <= 0 || n_heads <= 0)
    return invalid("n_pages, page_size, n_kv_heads, n_seq, max_pages, M and n_heads must be positive");
  if (n_heads % kv->n_kv_heads != 0) return invalid("n_heads must be a multiple of n_kv_heads");
  if (!kv->q_starts && M != kv->n_seq) return invalid("without q_starts M must be n_seq");
  if (!aligned(kv->page_table, 4) || !aligned(kv->kv_lens, 4) || !aligned(kv->q_starts, 4))
    return invalid("a pointer is not aligned to its element type");
  if (kv->head_dim != 64 && kv->head_dim != 128) return unsupported("need head_dim 64 or 128");
  if (kv->page_size < PAGED_MIN_PAGE || (kv->page_size & (kv->page_size - 1)) != 0)
    return unsupported("need a page_size that is a power of two, 8 or more");
  const int64_t cap = (int64_t)kv->max_pages * kv->page_size;
  if (cap > PAGED_MAX_KEYS) return unsupported("a request's pages hold more than 2^30 keys");
  if ((int64_t)M * n_heads >= 1 << 30) return unsupported("M * n_heads is 2^30 or more");
  // (single rows count tiles of 32 keys, up to three a request beside the table's, and the end of the last of 512 shares)
  if (kv->n_seq * (cap / 32 + 8) > INT_MAX - 512) return unsupported("n_seq * max_pages * page_size / 32 is near 2^31 or past it");
  if (!aligned(kv->k, 16) || !aligned(kv->v, 16)) return unsupported("need 16-byte aligned k and v");
  *c = PagedCache{kv->k, kv->v, kv->page_table, kv->kv_lens, kv->q_starts, kv->n_pages, __builtin_ctz(kv->page_size),
                  kv->n_kv_heads, kv->n_seq, kv->max_pages, (int)cap, M};
  return AF_OK;
}

// Rows of n_heads heads, `stride` elements apart.
af_status check_rows(const char* me, const char* name, const af_paged_kv* kv, const void* p, int64_t stride, int32_t n_heads) {
  if (!p) {
    set_error("%s: %s must be non-NULL", me, name);
    return AF_ERR_INVALID_ARG;
  }
  if (stride < (int64_t)n_heads * kv->head_dim || stride > (int64_t)1 << 31) {
    set_error("%s: rows of %s are %lld elements apart, need %lld to 2^31", me, name, (long long)stride, (long long)n_heads * kv->head_dim);
    return AF_ERR_INVALID_ARG;
  }
  if (!aligned(p, 16) || stride * dtype_size(kv->dtype) % 16 != 0) {
    set_error("%s: need 16-byte aligned rows of %s", me, name);
    return AF_ERR_UNSUPPORTED;
  }
  return AF_OK;
}

af_status too_many(const char* me) { return refuse(AF_ERR_UNSUPPORTED, me, "more workgroups than a launch takes"); }

}  // namespace

extern "C" af_status af_op_rope_append_paged(const af_paged_kv* kv, const void* q, int64_t q_stride, const void* k,
                                             int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                                             const int32_t* sections, int32_t n_axes, float theta, void* q_out,
                                             int64_t q_out_stride, int32_t M, int32_t n_heads, void* hip_stream) {
  clear_error();
  const char* me = "af_op_rope_append_paged";
  AppendArgs a{};
  AF_TRY(check_cache(me, kv, M, n_heads, &a.c));
  AF_TRY(check_rows(me, "q", kv, q, q_stride, n_heads));
  AF_TRY(check_rows(me, "k", kv, k, k_stride, kv->n_kv_heads));
  AF_TRY(check_rows(me, "v", kv, v, v_stride, kv->n_kv_heads));
  AF_TRY(check_rows(me, "q_out", kv, q_out, q_out_stride, n_heads));
  if (n_axes < 1 || n_axes > PAGED_MAX_AXES) return refuse(AF_ERR_INVALID_ARG, me, "n_axes must be 1, 2 or 3");
  if (n_axes > 1 && (!positions || !sections))
    return refuse(AF_ERR_INVALID_ARG, me, "several axes need positions and sections");
  if (!aligned(positions, 4)) return refuse(AF_ERR_INVALID_ARG, me, "a pointer is not aligned to its element type");
  if (!(theta > 0.f) || std::isinf(theta)) return refuse(AF_ERR_INVALID_ARG, me, "theta must be positive and finite");
  if (M >= 1 << 24) return refuse(AF_ERR_UNSUPPORTED, me, "M is 2^24 or more");
  const int half = kv->head_dim / 2;
  int sum = 0;
  for (int i = 0; i < PAGED_MAX_AXES; ++i) {
    const int n = !sections ? (i == 0 ? half : 0) : i < n_axes ? sections[i] : 0;
    if (n < 0 || n > half) return refuse(AF_ERR_INVALID_ARG, me, "sections must be pairs of a head, head_dim / 2 in all");
    a.axis_end[i] = sum += n;
  }
  if (sum != half) return refuse(AF_ERR_INVALID_ARG, me, "sections must be pairs of a head, head_dim / 2 in all");
  a.q = q, a.k = k, a.v = v, a.q_out = q_out;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.q_out_stride = q_out_stride;
  a.positions = positions, a.n_axes = n_axes, a.n_heads = n_heads;
  // a product of two powers each: 16 calls of pow instead of 64, which took longer than the launch
  double low[8], high[8];
  for (int j = 0; j < 8; ++j) {
    low[j] = std::pow((double)theta, -2.0 * j / kv->head_dim) / 6.283185307179586476925;
    high[j] = std::pow((double)theta, -16.0 * j / kv->head_dim);
  }
  for (int j = 0; j < half; ++j) a.turns[j] = low[j % 8] * high[j / 8];
  AF_HIP(launch_rope_append(kv->dtype, kv->head_dim, a, (hipStream_t)hip_stream));
  return AF_OK;
}

extern "C" af_status af_attention_paged_workspace(const af_paged_kv* kv, int32_t M, int32_t n_heads, size_t* bytes) {
  clear_error();
  const char* me = "af_attention_paged_workspace";
  if (!bytes) return refuse(AF_ERR_INVALID_ARG, me, "bytes must be non-NULL");
  PagedCache c;
  long floats;
  AF_TRY(check_cache(me, kv, M, n_heads, &c));
  if (!paged_workspace(kv->dtype, kv->head_dim, c.n_kv_heads, n_heads, c.n_seq, !c.starts, M, c.cap, &floats)) return too_many(me);
  *bytes = (size_t)floats * sizeof(float);
  return AF_OK;
}

extern "C" af_status af_op_attention_paged(const af_paged_kv* kv, const void* q, int64_t q_stride, void* o, int64_t o_stride,
                                           float* lse, int32_t M, int32_t n_heads, float scale, int32_t window,
                                           int32_t n_sink, void* workspace, size_t workspace_bytes, void* hip_stream) {
  clear_error();
  const char* me = "af_op_attention_paged";
  PagedAttnArgs a{};
  PagedPlan p;
  AF_TRY(check_cache(me, kv, M, n_heads, &a.c));
  AF_TRY(check_rows(me, "q", kv, q, q_stride, n_heads));
  AF_TRY(check_rows(me, "o", kv, o, o_stride, n_heads));
  if (window < 0 || n_sink < 0) return refuse(AF_ERR_INVALID_ARG, me, "window and n_sink must be 0 or more");
  const float scale_log2 = (float)(scale * 1.4426950408889634);
  if (!std::isfinite(scale_log2)) return refuse(AF_ERR_INVALID_ARG, me, "scale must be finite, and below 2^127");
  if (!aligned(lse, 4)) return refuse(AF_ERR_INVALID_ARG, me, "a pointer is not aligned to its element type");
  if (!paged_plan(kv->dtype, kv->head_dim, kv->n_kv_heads, n_heads, kv->n_seq, !kv->q_starts, M, a.c.cap, &p)) return too_many(me);
  const size_t need = (size_t)p.floats * sizeof(float);
  if (need > 0 && (!workspace || workspace_bytes < need)) {
    set_error("%s: the workspace has %zu bytes, need %zu", me, workspace ? workspace_bytes : 0, need);
    return AF_ERR_INVALID_ARG;
  }
  if (!aligned(workspace, 16)) return refuse(AF_ERR_INVALID_ARG, me, "the workspace must be 16-byte aligned");
  a.q = q, a.o = o, a.lse = lse, a.q_stride = q_stride, a.o_stride = o_stride;
  a.n_heads = n_heads, a.group = divisor(n_heads / kv->n_kv_heads), a.n_kv_heads = divisor(kv->n_kv_heads);
  a.scale_log2 = scale_log2;
  a.window = window ? window : INT_MAX, a.sinks = window ? n_sink : 0;
  a.parts = (float*)workspace, a.parts_at = p.parts_at, a.rows_at = p.rows_at;
  a.shares = p.shares, a.single_waves = p.single_waves, a.row_parts = p.row_grid / kv->n_kv_heads;
  AF_HIP(launch_attention_paged(kv->dtype, kv->head_dim, a, p, (hipStream_t)hip_stream));
  return AF_OK;
}
