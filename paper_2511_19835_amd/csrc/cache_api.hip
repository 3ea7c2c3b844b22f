// C-ABI entry points of the 8-bit key/value cache: host-side validation and launches.
#include <math.h>

#include "cache_checks.hpp"

extern "C" {

int rsa_cache_bytes(const rsa_cache* cache, size_t* code_bytes, size_t* scale_bytes, size_t* mean_bytes) {
  CacheDims c;
  const int rc = make_cache(cache, false, &c);
  if (rc != RSA_OK) return rc;
  const size_t records = (size_t)c.pages * c.heads_kv;
  if (code_bytes) *code_bytes = records * c.blk * c.d;
  if (scale_bytes) *scale_bytes = records * 4 * sizeof(float);
  if (mean_bytes) *mean_bytes = records * c.d;
  return RSA_OK;
}

int rsa_cache_workspace_bytes(const rsa_cache* cache, const rsa_rows* rows, int group, size_t* select_ws_bytes,
                              size_t* attn_ws_bytes) {
  CacheDims c;
  RowDims r;
  int rc = make_cache(cache, false, &c);
  if (rc != RSA_OK) return rc;
  rc = make_rows(rows, c, true, &r);
  if (rc != RSA_OK) return rc;
  if (group < 0) return RSA_E_RANGE;
  if (select_ws_bytes) *select_ws_bytes = rsa::cache_select_ws_bytes(c, r, group);
  if (attn_ws_bytes) *attn_ws_bytes = rsa::cache_attn_parts_bytes(c, r, group, 0);
  return RSA_OK;
}

int rsa_cache_write(const rsa_cache* cache, const rsa_rows* rows, const void* K, const void* V, const int32_t* start,
                    const int32_t* count, void* stream) {
  CacheDims c;
  RowDims r;
  const int rc = check_page_call(cache, rows, K, V, start, &c, &r);
  if (rc != RSA_OK) return rc;
  const rsa::CacheWriteArgs a = {(const uint16_t*)K, (const uint16_t*)V, start, count};
  return rsa::launch_cache_write(c, r, a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

int rsa_cache_read(const rsa_cache* cache, const rsa_rows* rows, const int32_t* start, const int32_t* count, void* K,
                   void* V, void* stream) {
  CacheDims c;
  RowDims r;
  const int rc = check_page_call(cache, rows, K, V, start, &c, &r);
  if (rc != RSA_OK) return rc;
  if (K == V) return RSA_E_RANGE;
  const rsa::CacheReadArgs a = {start, count, (uint16_t*)K, (uint16_t*)V};
  return rsa::launch_cache_read(c, r, a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

int rsa_cache_select(const rsa_cache* cache, const rsa_rows* rows, const void* Q, const int32_t* kv_len,
                     const int32_t* q_len, int group, int keep, int first, int last, int flags, int32_t* block_idx,
                     int32_t* kept, int list_len, void* ws, size_t ws_bytes, void* stream) {
  CacheDims c;
  RowDims r;
  int rc = make_cache(cache, true, &c);
  if (rc != RSA_OK) return rc;
  rc = make_rows(rows, c, true, &r);
  if (rc != RSA_OK) return rc;
  if (!Q || !kv_len || !block_idx || !kept) return RSA_E_NULL;
  if (misaligned(Q, 16)) return RSA_E_SHAPE;
  if (c.max_blocks > RSA_CACHE_MAX_SELECT) return RSA_E_UNSUPPORTED;
  if (group < 1 || keep < 1 || first < 0 || last < 0 || list_len < 1 || (flags & ~RSA_CACHE_CAUSAL)) return RSA_E_RANGE;
  int64_t need = (int64_t)first + last + (group - 1) / c.blk + 2;
  if (need < keep) need = keep;
  if (need > c.max_blocks) need = c.max_blocks;
  if (list_len < need) return RSA_E_RANGE;
  // (sixteen waves to a workgroup)
  if (((int64_t)(r.t - 1) / group + 1) * c.batch * c.heads_kv > kMostWorkgroups / 4) return RSA_E_UNSUPPORTED;
  if (ws && (misaligned(ws, 256) || ws_bytes < rsa::cache_select_ws_bytes(c, r, group))) return RSA_E_WORKSPACE;
  rsa::CacheSelectArgs a = {};
  a.Q = (const uint16_t*)Q;
  a.kv_len = kv_len;
  a.q_len = q_len;
  a.group = group < r.t ? group : r.t;
  a.groups = (int)(((int64_t)r.t + a.group - 1) / a.group);
  a.keep = keep;
  a.first = first;
  a.last = last;
  a.list_len = list_len;
  a.causal = flags & RSA_CACHE_CAUSAL;
  a.block_idx = block_idx;
  a.kept = kept;
  a.ws = ws;
  return rsa::launch_cache_select(c, r, a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

int rsa_cache_attn(const rsa_cache* cache, const rsa_rows* rows, const void* Q, const int32_t* kv_len,
                   const int32_t* q_len, float scale, int flags, const int32_t* block_idx, const int32_t* kept, int group,
                   int list_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  CacheDims c;
  RowDims r;
  rsa::CacheAttnArgs a;
  const int rc = check_attn_call(cache, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, list_len, O, lse, &c, &r, &a);
  if (rc != RSA_OK) return rc;
  if (rsa::cache_attn_workgroups(c, r, block_idx ? a.group : 0, a.list_len) > kMostWorkgroups) return RSA_E_UNSUPPORTED;
  if (ws) {
    const size_t need = rsa::cache_attn_parts_bytes(c, r, block_idx ? a.group : 0, a.list_len);
    if (ws_bytes < need || misaligned(ws, 256)) return RSA_E_WORKSPACE;
    a.parts = need ? (float*)ws : nullptr;
  }
  return rsa::launch_cache_attn(c, r, a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

}  // extern "C"
