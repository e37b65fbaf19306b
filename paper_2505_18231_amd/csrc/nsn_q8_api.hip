// extern "C" boundary of the 8-bit cache: argument validation and dispatch only.
#include "nsn_host.h"
#include "nsn_q8.h"

namespace nsn {
namespace q8 {

static int check_shape(const nsn_q8_shape* s) {
  if (!s) {
    set_error("q8: shape is NULL");
    return NSN_ERR_INVALID_ARG;
  }
  if ((s->head_dim != 64 && s->head_dim != 128) || (s->code_type != NSN_Q8_INT8 && s->code_type != NSN_Q8_E4M3) ||
      (s->io_type != NSN_FP16 && s->io_type != NSN_BF16)) {
    set_error("q8: unsupported shape: head_dim=%d (64 or 128), code_type=%d, io_type=%d", s->head_dim, s->code_type, s->io_type);
    return NSN_ERR_UNSUPPORTED;
  }
  // (a launch has at most 65535 workgroups in its second dimension: an append needs two per kv head)
  if (s->n_kv_heads <= 0 || s->n_q_heads <= 0 || s->n_q_heads % s->n_kv_heads != 0 || s->n_q_heads > 65535 || s->n_kv_heads > 32767) {
    set_error("q8: n_q_heads=%d (at most 65535) must be a positive multiple of n_kv_heads=%d (at most 32767)", s->n_q_heads, s->n_kv_heads);
    return NSN_ERR_INVALID_ARG;
  }
  if (s->max_len <= 0 || s->max_len % kBlock != 0 || s->max_len > 1 << 30) {
    set_error("q8: max_len=%d must be a positive multiple of 64, at most 2^30", s->max_len);
    return NSN_ERR_INVALID_ARG;
  }
  if (s->page_size < 0 || s->page_size % kBlock != 0 || (s->page_size > 0 && (s->max_len % s->page_size != 0 || s->n_pages <= 0))) {
    set_error("q8: page_size=%d must be 0 or a multiple of 64 dividing max_len=%d, with n_pages=%d > 0", s->page_size, s->max_len,
              s->n_pages);
    return NSN_ERR_INVALID_ARG;
  }
  return NSN_OK;
}

static int check_cache(const nsn_q8_shape* s, const nsn_q8_cache* c, const char* name) {
  if (!c || !c->codes || !c->scales || (reinterpret_cast<uintptr_t>(c->codes) & 15) != 0 ||
      (reinterpret_cast<uintptr_t>(c->scales) & 3) != 0) {
    set_error("q8: %s cache: codes (16-byte aligned) and scales are needed", name);
    return NSN_ERR_INVALID_ARG;
  }
  if (s->page_size > 0 && (!c->block_table || (reinterpret_cast<uintptr_t>(c->block_table) & 3) != 0)) {
    set_error("q8: %s cache: paged layout needs a block_table", name);
    return NSN_ERR_INVALID_ARG;
  }
  return NSN_OK;
}

static int check_rows(const nsn_rows* r, const char* name) {
  if (!r || !r->data || (reinterpret_cast<uintptr_t>(r->data) & 15) != 0 || r->batch_stride % 8 != 0 || r->head_stride % 8 != 0 ||
      r->token_stride % 8 != 0) {
    set_error("q8: %s rows: 16-byte aligned data and strides that are multiples of 8 elements are needed", name);
    return NSN_ERR_INVALID_ARG;
  }
  return NSN_OK;
}

static bool meet(const void* p, const void* q, uintptr_t bytes) {  // two buffers of that size
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return (a < b ? b - a : a - b) < bytes;
}

// whether two caches share memory: contiguous ones by their extent; paged ones where the same pages go under the same table (which
// pages two tables name, the host does not see)
static bool overlap(const nsn_q8_shape& s, const nsn_q8_cache& x, const nsn_q8_cache& y, int batch) {
  if (s.page_size > 0) return (x.codes == y.codes || x.scales == y.scales) && x.block_table == y.block_table;
  const uintptr_t tokens = (uintptr_t)batch * s.n_kv_heads * s.max_len;
  return meet(x.codes, y.codes, tokens * s.head_dim) || meet(x.scales, y.scales, tokens / kBlock * sizeof(float));
}

static uintptr_t weights_bytes(const nsn_q8_shape& s, int batch) {
  return (uintptr_t)batch * s.n_kv_heads * s.max_len * sizeof(float);
}

// the addresses that rows reach
struct Span {
  uintptr_t begin, end;
};
static Span span_of(const nsn_rows& r, int batch, int heads, int tokens, int d) {
  Span s = {reinterpret_cast<uintptr_t>(r.data), reinterpret_cast<uintptr_t>(r.data) + (uintptr_t)d * 2};
  const int64_t reach[3] = {(batch - 1) * r.batch_stride * 2, (heads - 1) * r.head_stride * 2, (tokens - 1) * r.token_stride * 2};
  for (int64_t x : reach) (x < 0 ? s.begin : s.end) += (uintptr_t)x;
  return s;
}

static int launched(int rc, const char* what) {
  if (rc == NSN_ERR_HIP) set_error("%s: launch failed: %s", what, hipGetErrorString(hipGetLastError()));
  return rc;
}

}  // namespace q8
}  // namespace nsn

using namespace nsn;
using q8::check_cache;
using q8::check_rows;
using q8::check_shape;

extern "C" {

int64_t nsn_q8_k_code_offset(const nsn_q8_shape* shape, int64_t t, int c) {
  if (check_shape(shape) != NSN_OK) return -1;
  return (t < 0 || c < 0 || c >= shape->head_dim) ? -1 : t * shape->head_dim + c;
}
int64_t nsn_q8_v_code_offset(const nsn_q8_shape* shape, int64_t t, int c) {
  if (check_shape(shape) != NSN_OK) return -1;
  return (t < 0 || c < 0 || c >= shape->head_dim) ? -1 : q8::v_offset(shape->head_dim, t, c);
}

size_t nsn_q8_workspace_bytes(const nsn_q8_shape* shape, int op, int batch, int n, int max_seq_len, int n_splits) {
  if (check_shape(shape) != NSN_OK || batch <= 0 || batch > 65535 || n <= 0 || max_seq_len < 0 || max_seq_len > shape->max_len ||
      n_splits < 0)
    return 0;
  if (op == NSN_OP_Q8_ATTENTION) return q8::attention_workspace_bytes(*shape, batch, n, max_seq_len, n_splits);
  return 0;  // (an eviction needs none)
}

int nsn_q8_append(const nsn_q8_shape* shape, const nsn_rows* k, const nsn_rows* v, int max_new, const int32_t* seq_start_dev,
                  const int32_t* n_new_dev, int batch, const nsn_q8_cache* k_cache, const nsn_q8_cache* v_cache, void* stream) {
  int rc = check_shape(shape);
  if (rc != NSN_OK) return rc;
  if ((rc = check_cache(shape, k_cache, "K")) != NSN_OK) return rc;
  if ((rc = check_cache(shape, v_cache, "V")) != NSN_OK) return rc;
  if (!seq_start_dev || !n_new_dev || batch < 0 || batch > 65535 || max_new < 0) {
    set_error("q8_append: null pointer, negative size, or batch=%d beyond 65535", batch);
    return NSN_ERR_INVALID_ARG;
  }
  if (batch == 0 || max_new == 0) return NSN_OK;
  if ((rc = check_rows(k, "K")) != NSN_OK) return rc;
  if ((rc = check_rows(v, "V")) != NSN_OK) return rc;
  if (q8::overlap(*shape, *k_cache, *v_cache, batch)) {
    set_error("q8_append: the K and V caches share memory");
    return NSN_ERR_INVALID_ARG;
  }
  return q8::launched(q8::append_launch(*shape, *k, *v, max_new, seq_start_dev, n_new_dev, batch, *k_cache, *v_cache,
                                        static_cast<hipStream_t>(stream)), "q8_append");
}

int nsn_q8_attention(const nsn_q8_shape* shape, const nsn_rows* q, int n_q, const int32_t* q_lens_dev, const nsn_q8_cache* k_cache,
                     const nsn_q8_cache* v_cache, const int32_t* seq_lens_dev, int batch, int max_seq_len, float softmax_scale,
                     int causal, const float* weights_in, float* weights_out, int n_splits, void* out, float* lse, void* workspace,
                     size_t workspace_bytes, void* stream) {
  int rc = check_shape(shape);
  if (rc != NSN_OK) return rc;
  if ((rc = check_cache(shape, k_cache, "K")) != NSN_OK) return rc;
  if ((rc = check_cache(shape, v_cache, "V")) != NSN_OK) return rc;
  if (!seq_lens_dev || !out || (reinterpret_cast<uintptr_t>(out) & 15) != 0 || batch < 0 || batch > 65535 || n_q < 0 || n_splits < 0 ||
      max_seq_len < 0 || max_seq_len > shape->max_len) {
    set_error("q8_attention: null pointer, out not 16-byte aligned, negative size, batch=%d beyond 65535, or max_seq_len=%d beyond "
              "max_len=%d", batch, max_seq_len, shape->max_len);
    return NSN_ERR_INVALID_ARG;
  }
  if (!(softmax_scale > -INFINITY && softmax_scale < INFINITY)) {
    set_error("q8_attention: softmax_scale must be finite");
    return NSN_ERR_INVALID_ARG;
  }
  if (weights_in && !weights_out) {
    set_error("q8_attention: weights_in without weights_out");
    return NSN_ERR_INVALID_ARG;
  }
  if (weights_in && weights_in != weights_out && q8::meet(weights_in, weights_out, q8::weights_bytes(*shape, batch))) {
    set_error("q8_attention: weights_in and weights_out overlap without being the same");
    return NSN_ERR_INVALID_ARG;
  }
  if (batch == 0 || n_q == 0) {
    if (batch > 0 && weights_out && weights_in != weights_out) {
      set_error("q8_attention: weights of a call without queries");
      return NSN_ERR_INVALID_ARG;
    }
    return NSN_OK;
  }
  if ((rc = check_rows(q, "query")) != NSN_OK) return rc;
  if ((int64_t)n_q * (shape->n_q_heads / shape->n_kv_heads) > 1 << 24) {
    set_error("q8_attention: n_q=%d times %d query heads per kv head is beyond 2^24", n_q, shape->n_q_heads / shape->n_kv_heads);
    return NSN_ERR_UNSUPPORTED;
  }
  const size_t need = q8::attention_workspace_bytes(*shape, batch, n_q, max_seq_len, n_splits);
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15) != 0)) {
    set_error("q8_attention: a workspace of %zu bytes, 16-byte aligned, is needed", need);
    return NSN_ERR_WORKSPACE;
  }
  // (rows are read by several workgroups, and again for the weights)
  const q8::Span rows = q8::span_of(*q, batch, shape->n_q_heads, n_q, shape->head_dim);
  const uintptr_t to = reinterpret_cast<uintptr_t>(out);
  if (to < rows.end && rows.begin < to + (uintptr_t)batch * n_q * shape->n_q_heads * shape->head_dim * 2) {
    set_error("q8_attention: out lies among the query rows");
    return NSN_ERR_INVALID_ARG;
  }
  const q8::AttentionCall c = {*shape, *q, n_q, q_lens_dev, *k_cache, *v_cache, seq_lens_dev, batch, max_seq_len, softmax_scale,
                               causal != 0, weights_in, weights_out, n_splits, out, lse, workspace, static_cast<hipStream_t>(stream)};
  return q8::launched(q8::attention_launch(c), "q8_attention");
}

int nsn_q8_evict(const nsn_q8_shape* shape, const float* weights, const int32_t* seq_lens_dev, int batch, int max_seq_len, int keep,
                 int first, int recent, const nsn_q8_cache* k_cache, const nsn_q8_cache* v_cache, const nsn_q8_cache* k_out,
                 const nsn_q8_cache* v_out, int32_t* kept, int32_t* new_lens, float* weights_out, void*,
                 size_t, void* stream) {
  int rc = check_shape(shape);
  if (rc != NSN_OK) return rc;
  if ((rc = check_cache(shape, k_cache, "K")) != NSN_OK) return rc;
  if ((rc = check_cache(shape, v_cache, "V")) != NSN_OK) return rc;
  if ((rc = check_cache(shape, k_out, "K output")) != NSN_OK) return rc;
  if ((rc = check_cache(shape, v_out, "V output")) != NSN_OK) return rc;
  if (!weights || (reinterpret_cast<uintptr_t>(weights) & 15) != 0 || !seq_lens_dev || !kept || !new_lens || batch < 0 ||
      batch > 65535 || max_seq_len < 0 || max_seq_len > shape->max_len) {
    set_error("q8_evict: null pointer, weights not 16-byte aligned, negative size, batch=%d beyond 65535, or max_seq_len=%d beyond "
              "max_len=%d", batch, max_seq_len, shape->max_len);
    return NSN_ERR_INVALID_ARG;
  }
  if (keep < 1 || keep > shape->max_len || first < 0 || recent < 0 || (int64_t)first + recent > keep) {
    set_error("q8_evict: keep=%d must lie in 1 .. max_len=%d and hold first=%d and recent=%d (both >= 0)", keep, shape->max_len, first,
              recent);
    return NSN_ERR_INVALID_ARG;
  }
  if (weights_out && q8::meet(weights_out, weights, q8::weights_bytes(*shape, batch))) {
    set_error("q8_evict: weights_out lies in the buffer of weights");
    return NSN_ERR_INVALID_ARG;
  }
  const nsn_q8_cache* outs[2] = {k_out, v_out};
  for (int i = 0; i < 2; ++i) {
    if (q8::overlap(*shape, *outs[i], *k_cache, batch) || q8::overlap(*shape, *outs[i], *v_cache, batch) ||
        (i == 0 && q8::overlap(*shape, *k_out, *v_out, batch))) {
      set_error("q8_evict: an output lies in a cache that is read, or in the other output");
      return NSN_ERR_INVALID_ARG;
    }
  }
  if (q8::meet(new_lens, seq_lens_dev, (uintptr_t)batch * sizeof(int32_t))) {  // (every head reads the lengths)
    set_error("q8_evict: new_lens lies in the buffer of seq_lens");
    return NSN_ERR_INVALID_ARG;
  }
  if (batch == 0) return NSN_OK;
  const q8::EvictCall c = {*shape, weights, seq_lens_dev, batch, max_seq_len, keep, first, recent, *k_cache, *v_cache, *k_out, *v_out,
                           kept, new_lens, weights_out, static_cast<hipStream_t>(stream)};
  return q8::launched(q8::evict_launch(c), "q8_evict");
}

}  // extern "C"
