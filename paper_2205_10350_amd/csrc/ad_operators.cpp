// The operators behind the C ABI that need no context: 8-bit key/value caches and the acceptance of sampled blocks.
// Arguments are checked here; the kernels hold device tables to what the host arguments say.
#include <hip/hip_runtime.h>
#include <stdio.h>

#include <algorithm>

#include "ad_accept.h"
#include "ad_internal.h"
#include "ad_kv8.h"

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

}  // extern "C"
