// Host-side checks of the records that the calls on both caches (8 and 4 bits) take.
#pragma once

#include <math.h>

#include "cache_common.hpp"

namespace {

using rsa::CacheDims;
using rsa::RowDims;

constexpr int64_t kMostWorkgroups = (int64_t)1 << 23;       // of 256 threads

bool misaligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

int make_cache(const rsa_cache* in, bool pointers, CacheDims* out) {
  if (!in) return RSA_E_NULL;
  if (in->batch < 1 || in->heads_kv < 1 || in->max_blocks < 1 || in->pages < 1) return RSA_E_SHAPE;
  if (in->head_dim != 64 && in->head_dim != 128) return RSA_E_UNSUPPORTED;
  if (in->block != 64 && in->block != 128) return RSA_E_UNSUPPORTED;
  if ((int64_t)in->batch * in->heads_kv > 65535 || in->pages >= ((int64_t)1 << 31)) return RSA_E_UNSUPPORTED;
  if ((int64_t)in->max_blocks * in->block >= ((int64_t)1 << 31)) return RSA_E_UNSUPPORTED;   // positions are int32
  if (pointers) {
    if (!in->k_codes || !in->v_codes || !in->scales || !in->k_mean || !in->table) return RSA_E_NULL;
    if (misaligned(in->k_codes, 16) || misaligned(in->v_codes, 16) || misaligned(in->scales, 16) || misaligned(in->k_mean, 16) ||
        misaligned(in->table, 4))
      return RSA_E_SHAPE;
  }
  out->batch = in->batch;
  out->heads_kv = in->heads_kv;
  out->d = in->head_dim;
  out->blk = in->block;
  out->max_blocks = in->max_blocks;
  out->pages = in->pages;
  out->k = (uint8_t*)in->k_codes;
  out->v = (uint8_t*)in->v_codes;
  out->scales = in->scales;
  out->mean = in->k_mean;
  out->table = in->table;
  return RSA_OK;
}

// `queries`: rows of Q and O, whose heads may be several to a key/value head.
int make_rows(const rsa_rows* in, const CacheDims& c, bool queries, RowDims* out) {
  if (!in) return RSA_E_NULL;
  if (in->heads < 1 || in->t < 1) return RSA_E_SHAPE;
  if (queries ? in->heads % c.heads_kv != 0 : in->heads != c.heads_kv) return RSA_E_SHAPE;
  if (in->stride_t < c.d || in->stride_b < 1 || in->stride_h < 1) return RSA_E_SHAPE;
  if ((in->stride_t % 8) || (in->stride_b % 8) || (in->stride_h % 8)) return RSA_E_SHAPE;
  // a grid has less than 2^32 threads (a workgroup for 64 tokens of a key/value head, and two more; queries: see kMostWorkgroups)
  if ((int64_t)in->t * in->heads * c.batch >= ((int64_t)1 << 28) ||
      (!queries && ((int64_t)in->t / 64 + 2) * c.batch * c.heads_kv > kMostWorkgroups))
    return RSA_E_UNSUPPORTED;
  out->heads = in->heads;
  out->t = in->t;
  out->sb = in->stride_b;
  out->sh = in->stride_h;
  out->st = in->stride_t;
  return RSA_OK;
}

int check_page_call(const rsa_cache* cache, const rsa_rows* rows, const void* K, const void* V, const int32_t* start, CacheDims* c,
                    RowDims* r) {
  int rc = make_cache(cache, true, c);
  if (rc != RSA_OK) return rc;
  rc = make_rows(rows, *c, false, r);
  if (rc != RSA_OK) return rc;
  if (!K || !V || !start) return RSA_E_NULL;
  if (misaligned(K, 16) || misaligned(V, 16)) return RSA_E_SHAPE;
  return RSA_OK;
}

int check_attn_call(const rsa_cache* cache, const rsa_rows* rows, const void* Q, const int32_t* kv_len, const int32_t* q_len, float scale,
                    int flags, const int32_t* block_idx, const int32_t* kept, int group, int list_len, void* O, float* lse, CacheDims* c,
                    RowDims* r, rsa::CacheAttnArgs* out) {
  int rc = make_cache(cache, true, c);
  if (rc != RSA_OK) return rc;
  rc = make_rows(rows, *c, true, r);
  if (rc != RSA_OK) return rc;
  if (!Q || !kv_len || !O || !block_idx != !kept) return RSA_E_NULL;
  if (misaligned(Q, 16) || misaligned(O, 16)) return RSA_E_SHAPE;
  if (flags & ~RSA_CACHE_CAUSAL) return RSA_E_RANGE;
  const float scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf((float)c->d)) * 1.4426950408889634f;
  if (!(scale >= 0.f) || !isfinite(scale_log2e)) return RSA_E_RANGE;
  if (block_idx && (group < 1 || list_len < 1)) return RSA_E_RANGE;
  *out = {};
  rsa::CacheAttnArgs& a = *out;
  a.Q = (const uint16_t*)Q;
  a.kv_len = kv_len;
  a.q_len = q_len;
  a.block_idx = block_idx;
  a.kept = kept;
  a.group = block_idx && group < r->t ? group : r->t;
  a.groups = (int)(((int64_t)r->t + a.group - 1) / a.group);
  a.list_len = block_idx ? list_len : 0;
  a.causal = flags & RSA_CACHE_CAUSAL;
  a.scale_log2e = scale_log2e;
  a.O = (uint16_t*)O;
  a.lse = lse;
  return RSA_OK;
}

}  // namespace
