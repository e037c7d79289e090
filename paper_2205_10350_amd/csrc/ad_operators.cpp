// The operators behind the C ABI that need no context: 8-bit key/value caches, the acceptance of sampled blocks, and truncated distributions.
// Arguments are checked here; the kernels hold device tables to what the host arguments say.
#include <hip/hip_runtime.h>
#include <stdio.h>

#include <algorithm>

#include "ad_accept.h"
#include "ad_internal.h"
#include "ad_kv8.h"
#include "ad_truncate.h"

using namespace ad;

static int refuse(const char* msg) {
  set_global_error(msg);
  return AD_EINVAL;
}
static int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return AD_OK;
  char msg[200];
  snprintf(msg, sizeof(msg), "%.60s: %.120s", what, hipGetErrorString(e));
  set_global_error(msg);
  return AD_EDEVICE;
}
static bool off16(const void* p, int64_t stride) { return ((uintptr_t)p & 15) || stride % 8; }

extern "C" {

int ad_kv8_check(const ad_kv8_config* c) {
  if (!c) return refuse("null cache description");
  if (c->n_seq < 1 || c->n_seq > 4096) return refuse("ad_kv8: n_seq outside [1, 4096]");
  if (c->n_heads < 1 || c->n_heads > 256) return refuse("ad_kv8: n_heads outside [1, 256]");
  if (c->head_width != 32 && c->head_width != 64 && c->head_width != 128) return refuse("ad_kv8: head_width must be 32, 64 or 128");
  if (c->capacity < 1 || c->capacity > (1 << 24)) return refuse("ad_kv8: capacity outside [1, 2^24]");
  if (c->closed != 0 && c->closed != 1) return refuse("ad_kv8: closed must be 0 or 1");
  if (!c->closed && (c->k_max < 1 || c->k_max > 65536)) return refuse("ad_kv8: k_max outside [1, 65536]");
  if (c->format != AD_KV_E4M3 && c->format != AD_KV_I8) return refuse("ad_kv8: format must be AD_KV_E4M3 or AD_KV_I8");
  return AD_OK;
}
size_t ad_kv8_bytes(const ad_kv8_config* c) { return ad_kv8_check(c) == AD_OK ? kv8_dims(*c).bytes : 0; }

static int kv8_common(const ad_kv8_config* c, const void* cache, const int32_t* row_start, const int32_t* base, int32_t rows, int32_t max_rows) {
  const int rc = ad_kv8_check(c);
  if (rc != AD_OK) return rc;
  if (!cache || !row_start || !base) return refuse("ad_kv8: null buffer");
  if ((uintptr_t)cache & 255) return refuse("ad_kv8: the cache must be 256-byte aligned");
  if (rows < 0 || max_rows < 0 || max_rows > rows) return refuse("ad_kv8: rows < 0 or max_rows outside [0, rows]");
  return AD_OK;
}

int ad_kv8_append(const ad_kv8_config* c, void* cache, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  const int32_t* row_start, const int32_t* length, int32_t rows, int32_t max_rows, void* hip_stream) {
  const int rc = kv8_common(c, cache, row_start, length, rows, max_rows);
  if (rc != AD_OK) return rc;
  if (max_rows == 0) return AD_OK;
  if (!k || !v) return refuse("ad_kv8_append: null buffer");
  const int64_t width = (int64_t)c->n_heads * c->head_width;
  if (k_stride < width || v_stride < width || off16(k, k_stride) || off16(v, v_stride))
    return refuse("ad_kv8_append: k and v must be 16-byte aligned, their row strides multiples of 8 and at least n_heads * head_width");
  const Kv8Dims d = kv8_dims(*c);
  if (max_rows > d.k_max) return refuse(c->closed ? "ad_kv8_append: max_rows above the capacity" : "ad_kv8_append: max_rows above k_max");
  launch_kv8_append(d, cache, k, v, (size_t)k_stride, (size_t)v_stride, Kv8Rows{row_start, nullptr, length, 1, rows, max_rows, c->n_seq}, (hipStream_t)hip_stream);
  return launched("ad_kv8_append");
}

int ad_kv8_read(const ad_kv8_config* c, const void* cache, const int32_t* row_start, const int32_t* begin, const int32_t* length,
                int32_t rows, int32_t max_rows, int32_t dtype, void* k_out, void* v_out, void* hip_stream) {
  const int rc = kv8_common(c, cache, row_start, begin, rows, max_rows);
  if (rc != AD_OK) return rc;
  if (dtype != AD_F32 && dtype != AD_BF16) return refuse("ad_kv8_read: dtype must be AD_F32 or AD_BF16");
  if (max_rows == 0) return AD_OK;
  if (!length || !k_out || !v_out) return refuse("ad_kv8_read: null buffer");
  if (((uintptr_t)k_out | (uintptr_t)v_out) & 15) return refuse("ad_kv8_read: outputs must be 16-byte aligned");
  const Kv8Dims d = kv8_dims(*c);
  launch_kv8_read(d, cache, Kv8Rows{row_start, nullptr, begin, 1, rows, std::min(max_rows, d.capacity), c->n_seq}, length, dtype, k_out, v_out, (hipStream_t)hip_stream);
  return launched("ad_kv8_read");
}

size_t ad_kv8_attend_bytes(const ad_kv8_config* c, int32_t q_heads, int32_t rows, int32_t max_keys) {
  if (ad_kv8_check(c) != AD_OK || q_heads < 1 || rows < 1 || max_keys < 0) return 0;
  return kv8_attend_bytes(kv8_dims(*c), q_heads, rows, max_keys);
}

int ad_kv8_attend(const ad_kv8_config* c, const void* cache, const void* q, int64_t q_stride, int32_t q_heads,
                  const int32_t* row_start, const int32_t* length, int32_t rows, int32_t max_rows, int32_t max_keys, float scale,
                  void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = kv8_common(c, cache, row_start, length, rows, max_rows);
  if (rc != AD_OK) return rc;
  if (q_heads < c->n_heads || q_heads % c->n_heads || q_heads / c->n_heads > 256) return refuse("ad_kv8_attend: q_heads must be a multiple of n_heads, at most 256 times it");
  if (!(scale > -INFINITY && scale < INFINITY)) return refuse("ad_kv8_attend: scale must be finite");
  if (max_keys < 0) return refuse("ad_kv8_attend: max_keys < 0");
  if (max_rows == 0) return AD_OK;
  if (!q || !out) return refuse("ad_kv8_attend: null buffer");
  const int64_t width = (int64_t)q_heads * c->head_width;
  if (q_stride < width || out_stride < width || off16(q, q_stride) || off16(out, out_stride))
    return refuse("ad_kv8_attend: q and out must be 16-byte aligned, their row strides multiples of 8 and at least q_heads * head_width");
  const Kv8Dims d = kv8_dims(*c);
  if (!c->closed && max_rows > d.k_max) return refuse("ad_kv8_attend: max_rows above k_max");
  const size_t need = kv8_attend_bytes(d, q_heads, rows, max_keys);
  if (need && (!workspace || ((uintptr_t)workspace & 255))) return refuse("ad_kv8_attend: the workspace must be 256-byte aligned device memory");
  if (workspace_bytes < need) { set_global_error("ad_kv8_attend: workspace smaller than ad_kv8_attend_bytes()"); return AD_ENOMEM; }
  const Kv8Rows r{row_start, nullptr, length, 1, rows, max_rows, c->n_seq};
  if (!kv8_attend_fits(d, r, q_heads, max_keys)) return refuse("ad_kv8_attend: more workgroups than a launch takes (sequences x heads x rows x keys)");
  launch_kv8_attend(d, cache, q, (size_t)q_stride, out, (size_t)out_stride, q_heads, r, max_keys, scale, workspace, (hipStream_t)hip_stream);
  return launched("ad_kv8_attend");
}

size_t ad_kv8_attend_shared_bytes(const ad_kv8_config* c, const ad_kv8_config* texts, int32_t q_heads, int32_t rows, int32_t max_keys, int32_t max_shared_keys) {
  if (ad_kv8_check(c) != AD_OK || ad_kv8_check(texts) != AD_OK || q_heads < c->n_heads || rows < 1 || max_keys < 0 || max_shared_keys < 0) return 0;
  return kv8_attend_shared_bytes(kv8_dims(*c), kv8_dims(*texts), q_heads, rows, max_keys, max_shared_keys);
}

int ad_kv8_attend_shared(const ad_kv8_config* c, const void* cache, const ad_kv8_config* texts, const void* text_cache, const void* q, int64_t q_stride, int32_t q_heads,
                         const int32_t* row_start, const int32_t* length, const int32_t* seq_start, const int32_t* shared_length, int32_t rows, int32_t max_rows,
                         int32_t max_keys, int32_t max_shared_rows, int32_t max_shared_keys, float scale, void* out, int64_t out_stride, void* workspace,
                         size_t workspace_bytes, void* hip_stream) {
  int rc = kv8_common(c, cache, row_start, length, rows, max_rows);
  if (rc == AD_OK) rc = kv8_common(texts, text_cache, seq_start, shared_length, rows, max_shared_rows);
  if (rc != AD_OK) return rc;
  if (c->closed) return refuse("ad_kv8_attend_shared: the sequences' own cache must be a growing one");
  if (texts->n_heads != c->n_heads || texts->head_width != c->head_width || texts->format != c->format)
    return refuse("ad_kv8_attend_shared: both caches must have the same heads, head width and format");
  if (q_heads < c->n_heads || q_heads % c->n_heads || q_heads / c->n_heads > 256) return refuse("ad_kv8_attend_shared: q_heads must be a multiple of n_heads, at most 256 times it");
  if (!(scale > -INFINITY && scale < INFINITY)) return refuse("ad_kv8_attend_shared: scale must be finite");
  if (max_keys < 0 || max_shared_keys < 0) return refuse("ad_kv8_attend_shared: max_keys or max_shared_keys < 0");
  if (max_rows == 0) return AD_OK;
  if (!q || !out) return refuse("ad_kv8_attend_shared: null buffer");
  const int64_t width = (int64_t)q_heads * c->head_width;
  if (q_stride < width || out_stride < width || off16(q, q_stride) || off16(out, out_stride))
    return refuse("ad_kv8_attend_shared: q and out must be 16-byte aligned, their row strides multiples of 8 and at least q_heads * head_width");
  const Kv8Dims d = kv8_dims(*c), t = kv8_dims(*texts);
  if (max_rows > d.k_max) return refuse("ad_kv8_attend_shared: max_rows above k_max");
  const size_t need = kv8_attend_shared_bytes(d, t, q_heads, rows, max_keys, max_shared_keys);
  if (need && (!workspace || ((uintptr_t)workspace & 255))) return refuse("ad_kv8_attend_shared: the workspace must be 256-byte aligned device memory");
  if (workspace_bytes < need) { set_global_error("ad_kv8_attend_shared: workspace smaller than ad_kv8_attend_shared_bytes()"); return AD_ENOMEM; }
  const Kv8Rows r{row_start, nullptr, length, 1, rows, max_rows, c->n_seq};
  const Kv8Texts x{seq_start, shared_length, texts->n_seq, max_shared_rows};
  if (!kv8_attend_shared_fits(d, t, r, x, q_heads, max_keys, max_shared_keys)) return refuse("ad_kv8_attend_shared: more workgroups than a launch takes (sequences x heads x rows x keys)");
  launch_kv8_attend_shared(d, cache, t, text_cache, q, (size_t)q_stride, out, (size_t)out_stride, q_heads, r, x, max_keys, max_shared_keys, scale, workspace, (hipStream_t)hip_stream);
  return launched("ad_kv8_attend_shared");
}

int ad_kv8_copy(const ad_kv8_config* from, const void* origin, const ad_kv8_config* c, void* cache, const int32_t* source, const int32_t* place, const int32_t* begin,
                const int32_t* end, int32_t n, int32_t max_tokens, void* hip_stream) {
  int rc = ad_kv8_check(from);
  if (rc == AD_OK) rc = ad_kv8_check(c);
  if (rc != AD_OK) return rc;
  if (!origin || !cache) return refuse("ad_kv8_copy: null buffer");
  if (((uintptr_t)origin | (uintptr_t)cache) & 255) return refuse("ad_kv8_copy: the caches must be 256-byte aligned");
  if (from->n_heads != c->n_heads || from->head_width != c->head_width || from->format != c->format || from->closed != c->closed)
    return refuse("ad_kv8_copy: both caches must have the same heads, head width and format, and both grow or both be closed");
  const Kv8Dims d = kv8_dims(*from), t = kv8_dims(*c);
  if (origin == cache) {
    if (d.n_seq != t.n_seq || d.capacity != t.capacity || d.k_max != t.k_max) return refuse("ad_kv8_copy: two descriptions of one cache");
    if (begin) return refuse("ad_kv8_copy: within a cache sequences are copied from their first token on (begin must be null)");
  } else if ((uintptr_t)origin < (uintptr_t)cache + t.bytes && (uintptr_t)cache < (uintptr_t)origin + d.bytes) {
    return refuse("ad_kv8_copy: the caches overlap");
  }
  if (n < 0 || n > c->n_seq || max_tokens < 0) return refuse("ad_kv8_copy: n outside [0, n_seq] or max_tokens < 0");
  if (n == 0 || max_tokens == 0) return AD_OK;
  if (!source || !place || !end) return refuse("ad_kv8_copy: null buffer");
  if (!kv8_copy_fits(d, t, n, max_tokens)) return refuse("ad_kv8_copy: more workgroups than a launch takes (entries x tokens)");
  launch_kv8_copy(d, origin, t, cache, Kv8Moves{source, place, begin, end, n, max_tokens}, (hipStream_t)hip_stream);
  return launched("ad_kv8_copy");
}

size_t ad_accept_sampled_bytes(int32_t n_seq, int32_t rows, int32_t vocab) {
  return n_seq < 1 || rows < 1 || vocab < 1 ? 0 : accept_bytes(n_seq, rows, vocab);
}

int ad_accept_sampled(const void* logits, int32_t dtype, int64_t logits_stride, int32_t vocab, const int32_t* draft,
                      const float* draft_probs, int64_t probs_stride, const float* temperature, const float* accept_u, const float* pick_u,
                      const int32_t* row_start, int32_t n_seq, int32_t rows, int32_t max_rows, int32_t* n_accept, int32_t* tokens,
                      void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (dtype != AD_F32 && dtype != AD_BF16) return refuse("ad_accept_sampled: dtype must be AD_F32 or AD_BF16");
  if (vocab < 1 || vocab > (1 << 24)) return refuse("ad_accept_sampled: vocab outside [1, 2^24]");
  if (n_seq < 1 || n_seq > 4096) return refuse("ad_accept_sampled: n_seq outside [1, 4096]");
  if (rows < 0 || max_rows > rows || max_rows < (rows ? 1 : 0)) return refuse("ad_accept_sampled: rows < 0 or max_rows outside [1, rows]");
  if (!pick_u || !row_start || !n_accept) return refuse("ad_accept_sampled: null buffer");
  if (rows == 0) {   // (no sequence has a row: counts of 0)
    AcceptArgs a{};
    a.pick_u = pick_u; a.row_start = row_start; a.vocab = vocab; a.n_seq = n_seq; a.n_accept = n_accept;
    launch_accept_nothing(a, (hipStream_t)hip_stream);
    return launched("ad_accept_sampled");
  }
  if (!accept_packed(n_seq, rows, max_rows) && max_rows > 65535)
    return refuse("ad_accept_sampled: max_rows above 65535 (taken only where n_seq * max_rows > 4 * rows)");
  if (!logits || !draft || !accept_u || !tokens || !workspace) return refuse("ad_accept_sampled: null buffer");
  if (logits_stride < vocab || (draft_probs && probs_stride < vocab)) return refuse("ad_accept_sampled: row stride below vocab");
  if ((uintptr_t)logits & (dtype == AD_F32 ? 3 : 1)) return refuse("ad_accept_sampled: logits not aligned to their type");
  if ((uintptr_t)workspace & 255) return refuse("ad_accept_sampled: the workspace must be 256-byte aligned");
  if (workspace_bytes < accept_bytes(n_seq, rows, vocab)) { set_global_error("ad_accept_sampled: workspace smaller than ad_accept_sampled_bytes()"); return AD_ENOMEM; }
  AcceptArgs a{};
  a.logits = logits; a.stride = (size_t)logits_stride; a.draft = draft; a.probs = draft_probs; a.probs_stride = (size_t)probs_stride;
  a.temperature = temperature; a.accept_u = accept_u; a.pick_u = pick_u; a.row_start = row_start;
  a.vocab = vocab; a.n_seq = n_seq; a.rows = rows; a.max_rows = max_rows; a.n_accept = n_accept; a.tokens = tokens; a.keep = 0;
  launch_accept_sampled(dtype, a, workspace, (hipStream_t)hip_stream);
  return launched("ad_accept_sampled");
}

static int truncate_common(const char* what, const void* logits, int32_t dtype, int64_t stride, int32_t vocab, const int32_t* row_start, int32_t n_seq, int32_t rows) {
  auto no = [&](const char* why) {
    char msg[200];
    snprintf(msg, sizeof(msg), "%s: %s", what, why);
    return refuse(msg);
  };
  if (dtype != AD_F32 && dtype != AD_BF16) return no("dtype must be AD_F32 or AD_BF16");
  if (vocab < 1 || vocab > (1 << 20)) return no("vocab outside [1, 2^20]");   // (beyond it the weights' rounding could be seen in fp32 settings)
  if (rows < 0 || rows >= (1 << 22)) return no("rows outside [0, 2^22)");
  if (row_start ? n_seq < 1 || n_seq > 4096 : n_seq != rows) return no("n_seq outside [1, 4096], or without row_start not the rows");
  if (rows == 0) return AD_OK;
  if (!logits) return no("null buffer");
  if (stride < vocab) return no("row stride below vocab");
  if ((uintptr_t)logits & (dtype == AD_F32 ? 3 : 1)) return no("scores not aligned to their type");
  return AD_OK;
}

int ad_sample_tokens(const void* logits, int32_t dtype, int64_t logits_stride, int32_t vocab, const float* temperature, const int32_t* top_k, const float* top_p,
                     const float* min_p, const int32_t* row_start, int32_t n_seq, const float* u, int32_t rows, int32_t* tokens, float* log_probs, void* hip_stream) {
  const int rc = truncate_common("ad_sample_tokens", logits, dtype, logits_stride, vocab, row_start, n_seq, rows);
  if (rc != AD_OK || rows == 0) return rc;
  if (!u || !tokens) return refuse("ad_sample_tokens: null buffer");
  TruncateArgs a{};
  a.x = logits; a.stride = (size_t)logits_stride; a.vocab = vocab; a.n_seq = n_seq; a.rows = rows; a.row_start = row_start;
  a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = u; a.tokens = tokens; a.log_probs = log_probs;
  launch_sample(dtype, a, (hipStream_t)hip_stream);
  return launched("ad_sample_tokens");
}

int ad_truncate_scores(const void* logits, int32_t dtype, int64_t logits_stride, int32_t vocab, const float* temperature, const int32_t* top_k, const float* top_p,
                       const float* min_p, const int32_t* row_start, int32_t n_seq, int32_t rows, void* out, int64_t out_stride, void* hip_stream) {
  const int rc = truncate_common("ad_truncate_scores", logits, dtype, logits_stride, vocab, row_start, n_seq, rows);
  if (rc != AD_OK || rows == 0) return rc;
  if (!out) return refuse("ad_truncate_scores: null buffer");
  if (out_stride < vocab) return refuse("ad_truncate_scores: row stride below vocab");
  const size_t size = dtype == AD_F32 ? 4 : 2;
  if ((uintptr_t)out & (size - 1)) return refuse("ad_truncate_scores: out not aligned to its type");
  // rows that lie between the scores' rows overlap them nowhere
  const int64_t apart = (int64_t)(((intptr_t)out - (intptr_t)logits) / (intptr_t)size), between = logits_stride ? (apart % logits_stride + logits_stride) % logits_stride : 0;
  const bool interleaved = out_stride == logits_stride && between >= vocab && between + vocab <= logits_stride;
  if (out == logits ? out_stride != logits_stride && rows > 1
                    : !interleaved && (uintptr_t)out < (uintptr_t)logits + ((size_t)logits_stride * (rows - 1) + vocab) * size && (uintptr_t)logits < (uintptr_t)out + ((size_t)out_stride * (rows - 1) + vocab) * size)
    return refuse("ad_truncate_scores: out must be the scores themselves, with their stride, or not overlap them");
  TruncateArgs a{};
  a.x = logits; a.stride = (size_t)logits_stride; a.vocab = vocab; a.n_seq = n_seq; a.rows = rows; a.row_start = row_start;
  a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.out = out; a.out_stride = (size_t)out_stride;
  launch_truncate(dtype, a, (hipStream_t)hip_stream);
  return launched("ad_truncate_scores");
}

}  // extern "C"
