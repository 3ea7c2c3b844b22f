// C-ABI entry points of the 4-bit key/value cache, of page assignment and of rotary positions: host-side validation and launches.
#include <math.h>

#include "cache_checks.hpp"
#include "fourbit_common.hpp"
#include "serve_common.hpp"

extern "C" {

int rsa_fourbit_bytes(const rsa_cache* cache, size_t* k_bytes, size_t* v_bytes, size_t* scale_bytes, size_t* mean_bytes) {
  CacheDims c;
  const int rc = make_cache(cache, false, &c);
  if (rc != RSA_OK) return rc;
  const size_t records = (size_t)c.pages * c.heads_kv;
  if (k_bytes) *k_bytes = records * (c.blk / 64) * rsa::fourbit_k_record(c.d);
  if (v_bytes) *v_bytes = records * (c.blk / 64) * rsa::fourbit_v_record(c.d);
  if (scale_bytes) *scale_bytes = records * 4 * sizeof(float);
  if (mean_bytes) *mean_bytes = records * c.d;
  return RSA_OK;
}

int rsa_fourbit_workspace_bytes(const rsa_cache* cache, const rsa_rows* rows, int group, size_t* attn_ws_bytes) {
  CacheDims c;
  RowDims r;
  int rc = make_cache(cache, false, &c);
  if (rc != RSA_OK) return rc;
  rc = make_rows(rows, c, true, &r);
  if (rc != RSA_OK) return rc;
  if (group < 0) return RSA_E_RANGE;
  if (attn_ws_bytes) *attn_ws_bytes = rsa::fourbit_attn_parts_bytes(c, r, group, 0);
  return RSA_OK;
}

int rsa_fourbit_write(const rsa_cache* cache, const rsa_rows* rows, const void* K, const void* V, const int32_t* start,
                      const int32_t* count, void* stream) {
  CacheDims c;
  RowDims r;
  const int rc = check_page_call(cache, rows, K, V, start, &c, &r);
  if (rc != RSA_OK) return rc;
  const rsa::CacheWriteArgs a = {(const uint16_t*)K, (const uint16_t*)V, start, count};
  return rsa::launch_fourbit_write(c, r, a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

int rsa_fourbit_read(const rsa_cache* cache, const rsa_rows* rows, const int32_t* start, const int32_t* count, void* K,
                     void* V, void* stream) {
  CacheDims c;
  RowDims r;
  const int rc = check_page_call(cache, rows, K, V, start, &c, &r);
  if (rc != RSA_OK) return rc;
  if (K == V) return RSA_E_RANGE;
  const rsa::CacheReadArgs a = {start, count, (uint16_t*)K, (uint16_t*)V};
  return rsa::launch_fourbit_read(c, r, a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

int rsa_fourbit_attn(const rsa_cache* cache, const rsa_rows* rows, const void* Q, const int32_t* kv_len,
                     const int32_t* q_len, float scale, int flags, const int32_t* block_idx, const int32_t* kept, int group,
                     int list_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  CacheDims c;
  RowDims r;
  rsa::CacheAttnArgs a;
  const int rc = check_attn_call(cache, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, list_len, O, lse, &c, &r, &a);
  if (rc != RSA_OK) return rc;
  const int grouped = block_idx ? a.group : 0;
  if (rsa::fourbit_attn_workgroups(c, r, grouped, a.list_len) > kMostWorkgroups) return RSA_E_UNSUPPORTED;
  if (ws) {
    const size_t need = rsa::fourbit_attn_parts_bytes(c, r, grouped, a.list_len);
    if (ws_bytes < need || misaligned(ws, 256)) return RSA_E_WORKSPACE;
    a.parts = need ? (float*)ws : nullptr;
  }
  return rsa::launch_fourbit_attn(c, r, a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

int rsa_cache_assign(const rsa_pages* pages, int t, const int32_t* kv_len, const int32_t* add, int32_t* shared,
                     const int32_t* free_count, int32_t* kv_new, int32_t* free_left, int32_t* start, int32_t* count,
                     int32_t* positions, int64_t* slots, void* stream) {
  if (!pages) return RSA_E_NULL;
  if (pages->batch < 1 || pages->max_blocks < 1 || pages->block < 1 || pages->pages < 1 || t < 1) return RSA_E_SHAPE;
  if (pages->batch > 65535 || pages->pages >= ((int64_t)1 << 31)) return RSA_E_UNSUPPORTED;
  if ((int64_t)pages->max_blocks * pages->block >= ((int64_t)1 << 31)) return RSA_E_UNSUPPORTED;    // positions are int32
  if ((int64_t)pages->batch * t >= ((int64_t)1 << 28) || (int64_t)pages->batch * pages->max_blocks >= ((int64_t)1 << 31)) return RSA_E_UNSUPPORTED;
  if (!pages->table || !pages->free_pages || !kv_len || !add || !free_count || !kv_new || !free_left || !start || !count) return RSA_E_NULL;
  const void* small[] = {pages->table, pages->free_pages, kv_len, add, shared, free_count, kv_new, free_left, start, count, positions};
  for (const void* p : small)
    if (misaligned(p, 4)) return RSA_E_SHAPE;
  if (misaligned(slots, 8)) return RSA_E_SHAPE;
  // (in place: kv_new over kv_len, free_left over free_count; anything else would be read after it was written)
  const void* out[] = {pages->table, pages->free_pages, kv_new, free_left, start, count, shared};
  for (size_t i = 0; i < sizeof out / sizeof *out; ++i) {
    if (!out[i]) continue;
    for (size_t j = 0; j < i; ++j)
      if (out[i] == out[j]) return RSA_E_RANGE;
    if (out[i] == add || out[i] == positions || out[i] == slots || (out[i] == kv_len && out[i] != kv_new) || (out[i] == free_count && out[i] != free_left))
      return RSA_E_RANGE;
  }
  for (const void* p : {(const void*)kv_len, (const void*)add, (const void*)free_count})
    if (p == positions || p == slots) return RSA_E_RANGE;
  if (positions && (const void*)positions == (const void*)slots) return RSA_E_RANGE;
  rsa::AssignArgs a = {};
  a.batch = pages->batch;
  a.max_blocks = pages->max_blocks;
  a.block = pages->block;
  a.t = t;
  a.pages = pages->pages;
  a.table = pages->table;
  a.free_pages = pages->free_pages;
  a.kv_len = kv_len;
  a.add = add;
  a.shared = shared;
  a.free_count = free_count;
  a.kv_new = kv_new;
  a.free_left = free_left;
  a.start = start;
  a.count = count;
  a.positions = positions;
  a.slots = slots;
  return rsa::launch_assign(a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

int rsa_rotary_frequencies(int pairs, double base, int scaling, double stretch, double old_len, double turns_few,
                           double turns_many, double* freq, float* factor) {
  if (!freq || !factor) return RSA_E_NULL;
  if (pairs < 1 || pairs > 512) return RSA_E_SHAPE;
  if (!(base > 1.0) || !isfinite(base) || scaling < RSA_ROTARY_PLAIN || scaling > RSA_ROTARY_PARTS) return RSA_E_RANGE;
  if (scaling != RSA_ROTARY_PLAIN && (!(stretch >= 1.0) || !isfinite(stretch))) return RSA_E_RANGE;
  if (scaling == RSA_ROTARY_PARTS && (!(old_len > 0.0) || !isfinite(old_len) || !(turns_few >= 0.0) || !(turns_many > turns_few) || !isfinite(turns_many)))
    return RSA_E_RANGE;
  if (scaling == RSA_ROTARY_BASE && pairs > 1) base *= pow(stretch, (double)pairs / (pairs - 1));
  if (!isfinite(base)) return RSA_E_RANGE;
  for (int j = 0; j < pairs; ++j) {
    double f = pow(base, -(double)j / pairs);
    if (scaling == RSA_ROTARY_LINEAR) f /= stretch;
    if (scaling == RSA_ROTARY_PARTS) {
      double keep = (old_len * f / 6.283185307179586 - turns_few) / (turns_many - turns_few);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f *= keep + (1.0 - keep) / stretch;
    }
    freq[j] = f;
  }
  *factor = scaling == RSA_ROTARY_PARTS ? (float)(0.1 * log(stretch) + 1.0) : 1.f;
  return RSA_OK;
}

int rsa_rotary_apply(const rsa_rotary* rotary, int batch, const rsa_rows* rows_q, const void* Q, void* Qr, const rsa_rows* rows_k,
                     const void* K, void* Kr, const int32_t* positions, const int32_t* start, const int32_t* count, int flags,
                     void* stream) {
  if (!rotary || !rows_q) return RSA_E_NULL;
  const rsa_rotary& p = *rotary;
  if (p.head_dim < 8 || p.head_dim % 8 || p.pairs < 1 || p.pairs > p.head_dim / 2) return RSA_E_SHAPE;
  if (p.head_dim > 1024) return RSA_E_UNSUPPORTED;
  if (p.axes < 1 || p.axes > 3) return RSA_E_SHAPE;
  int64_t sum = 0;
  for (int i = 0; i < p.axes; ++i) {
    if (p.axis_pairs[i] < 0) return RSA_E_SHAPE;
    sum += p.axis_pairs[i];
  }
  if (sum != p.pairs || batch < 1) return RSA_E_SHAPE;
  if (!(p.factor >= 0.f) || !isfinite(p.factor) || (flags & ~RSA_ROTARY_INVERSE)) return RSA_E_RANGE;
  if (!p.freq || !Q || !Qr || (rows_k && (!K || !Kr)) || (p.axes > 1 && !positions)) return RSA_E_NULL;
  if (misaligned(p.freq, 8) || misaligned(positions, 4) || misaligned(start, 4) || misaligned(count, 4)) return RSA_E_SHAPE;
  rsa::RotaryArgs a = {};
  a.batch = batch;
  a.t = rows_q->t;
  a.head_dim = p.head_dim;
  a.pairs = p.pairs;
  for (int i = 0, end = 0; i < 3; ++i) a.ends[i] = end += i < p.axes ? p.axis_pairs[i] : p.pairs;
  if (p.axes == 1) a.ends[0] = p.pairs;
  a.interleaved = p.interleaved != 0;
  a.inverse = flags & RSA_ROTARY_INVERSE;
  a.factor = p.factor == 0.f ? 1.f : p.factor;
  a.freq = p.freq;
  a.positions = positions;
  a.start = start;
  a.count = count;
  const rsa_rows* rows[2] = {rows_q, rows_k};
  const void* in[2] = {Q, K};
  void* out[2] = {Qr, Kr};
  int64_t heads = 0;
  for (int i = 0; i < 2; ++i) {
    if (!rows[i]) continue;
    const rsa_rows& r = *rows[i];
    if (r.heads < 1 || r.t < 1 || r.t != rows_q->t || r.stride_t < p.head_dim || r.stride_b < 1 || r.stride_h < 1) return RSA_E_SHAPE;
    if ((r.stride_t % 8) || (r.stride_b % 8) || (r.stride_h % 8) || misaligned(in[i], 16) || misaligned(out[i], 16)) return RSA_E_SHAPE;
    if ((int64_t)r.t * r.heads * batch >= ((int64_t)1 << 28)) return RSA_E_UNSUPPORTED;
    a.x[i] = {r.heads, r.stride_b, r.stride_h, r.stride_t, (const uint16_t*)in[i], (uint16_t*)out[i]};
    heads += r.heads;
  }
  if (rows_k && (Kr == Qr || Kr == Q || Qr == K)) return RSA_E_RANGE;
  // (64 pieces of at least eight channels to a workgroup)
  if ((int64_t)batch * a.t * (p.head_dim / 8 + 2) / 64 >= kMostWorkgroups || heads > 65535) return RSA_E_UNSUPPORTED;
  return rsa::launch_rotary(a, (hipStream_t)stream) == hipSuccess ? RSA_OK : RSA_E_LAUNCH;
}

}  // extern "C"
