// Shared declarations of the translation units of the 8-bit key/value cache (gfx950 only).
//
// A page holds one block of BLK tokens of every key/value head. Inside (page, head) the e4m3 codes stand in the order in
// which the 16x16x32 matrix instructions of cache_attn_kernels.hip take them, so that a wave loads 1 KB in one piece and
// lane L finds its operands in its 16 bytes:
//   K  [BLK/16][d/64][g 0..3][key 0..15][16 channels]     lane 16 g + key: row `key`, channels 16 g .. 16 g + 15 of 64
//   V  [BLK/64][d/16][g 0..3][channel 0..15][t 0..3][i 0..3]  lane 16 g + channel: keys 16 t + 4 g + i of 64
// After S^T = K Q^T lane 16 g + q holds the scores of keys 4 g + i of every tile t of 16 keys: with this order of V those
// are its operand of O^T += V^T P^T, and nothing has to be moved between lanes.
#pragma once

#include "rsa_common.hpp"

namespace rsa {

struct CacheDims {
  int batch, heads_kv, d, blk;
  int max_blocks;            // entries of a row of the table
  int64_t pages;
  uint8_t *k, *v;            // [pages][heads_kv][blk*d]
  float* scales;             // [pages][heads_kv][4]: 2^eK, 2^eV, 2^em of the mean, 0
  int8_t* mean;              // [pages][heads_kv][d]
  const int32_t* table;      // [batch][max_blocks]
};
struct RowDims {
  int heads, t;
  int64_t sb, sh, st;
};

// Page of block `blk` of sequence b, or -1 where there is none (behind the table, or an entry that is no page).
__device__ __forceinline__ int cache_page(const CacheDims& c, int b, int blk) {
  if (blk < 0 || blk >= c.max_blocks) return -1;
  const int p = c.table[(int64_t)b * c.max_blocks + blk];
  return (p < 0 || p >= c.pages) ? -1 : p;
}
__device__ __forceinline__ float exp2_int(int e) {          // 2^e, -126 <= e <= 127
  return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ int exponent_of(float two_to_e) {  // of a power of two; within [-127, 128] whatever the bits
  return (int)((__builtin_bit_cast(uint32_t, two_to_e) >> 23) & 255u) - 127;
}
// Byte offset of (token, channel) among the codes of a page's keys / values of one head.
template <int D>
__device__ __forceinline__ int k_code_offset(int t, int ch) {
  return ((((t >> 4) * (D / 64) + (ch >> 6)) * 4 + ((ch & 63) >> 4)) * 16 + (t & 15)) * 16 + (ch & 15);
}
template <int D>
__device__ __forceinline__ int v_code_offset(int t, int ch) {
  return ((((t >> 6) * (D / 16) + (ch >> 4)) * 4 + ((t & 15) >> 2)) * 16 + (ch & 15)) * 16 + ((t & 63) >> 4) * 4 + (t & 3);
}

struct CacheWriteArgs {
  const uint16_t *K, *V;
  const int32_t *start, *count;   // [batch]; count may be NULL (all t)
};
hipError_t launch_cache_write(const CacheDims& c, const RowDims& r, const CacheWriteArgs& a, hipStream_t s);

struct CacheReadArgs {
  const int32_t *start, *count;
  uint16_t *K, *V;
};
hipError_t launch_cache_read(const CacheDims& c, const RowDims& r, const CacheReadArgs& a, hipStream_t s);

struct CacheSelectArgs {
  const uint16_t* Q;
  const int32_t *kv_len, *q_len;  // [batch]; q_len may be NULL (all t)
  int group, groups, keep, first, last, list_len;
  bool causal;
  int32_t *block_idx, *kept;
  void* ws;
};
hipError_t launch_cache_select(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, hipStream_t s);

struct CacheAttnArgs {
  const uint16_t* Q;
  const int32_t *kv_len, *q_len;
  const int32_t *block_idx, *kept;   // NULL: every block
  int group, groups, list_len;       // without lists one group of all t tokens
  bool causal;
  float scale_log2e;
  uint16_t* O;
  float* lse;
  float* parts;                      // NULL: the key axis is not split
};
// Bytes of `parts` that a call with lists of at most `list_len` blocks (0: no lists) takes.
size_t cache_attn_parts_bytes(const CacheDims& c, const RowDims& r, int group, int list_len);
hipError_t launch_cache_attn(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, hipStream_t s);

}  // namespace rsa
