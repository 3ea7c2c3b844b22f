// Shared declarations of the translation units of the key/value cache (gfx950 only): records, pages, spans and lane exchanges of the caches of 8 and of 4
// bits, launchers of the first (those of the second and the order of its pages are in fourbit_common.hpp).
//
// A page holds one block of BLK tokens of every key/value head. In 8 bits, inside (page, head) the e4m3 codes stand in the order in
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

struct BlockSpan {
  int64_t first;   // token (in the new rows) of the block's slot 0; negative where older tokens precede
  int lo, hi;      // slots that get a new token
  int page;        // -1: none
};
// The jth block that tokens [start, start + count) of sequence b touch; false: there is none.
template <int BLK>
__device__ __forceinline__ bool touched_block(const CacheDims& c, int t, const int32_t* start, const int32_t* count, int b, int j, BlockSpan* out) {
  const int64_t s = start[b];
  int64_t n = count ? count[b] : t;
  if (n > t) n = t;
  if (s < 0 || n <= 0) return false;
  const int64_t blk = s / BLK + j, at = blk * BLK;
  if (at >= s + n || blk >= c.max_blocks) return false;
  out->page = cache_page(c, b, (int)blk);
  out->first = at - s;
  out->lo = s > at ? (int)(s - at) : 0;
  out->hi = s + n - at < BLK ? (int)(s + n - at) : BLK;
  return true;
}

// Workgroups go round the eight XCDs in turn; numbered like this, those of an XCD take numbers that follow one another, so
// that what neighbours share (a sequence's heads the lines of scales, a head's groups means and codes) is in one L2.
__device__ __forceinline__ int xcd_run(int id, int all) {
  const int x = id % 8, per = all / 8, more = all % 8;
  return x * per + min(x, more) + id / 8;
}

// Values of other lanes by the vector ALU alone (through LDS, as __shfl does it, each exchange waits some 100 cycles, and
// the small calls of the cache are little else). Lanes of a row of 16, by control word:
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kFlip8 = 0x141 /* lane i and i ^ 7 */, kFlip16 = 0x140 /* i ^ 15 */, kXor8 = 0x128;
template <int CTRL>
__device__ __forceinline__ int row_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
// op of a value with that of lane ^ 16 / lane ^ 32.
template <class Op>
__device__ __forceinline__ int with_xor16(int x, Op op) {
  const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
  return op((int)r[0], (int)r[1]);
}
template <class Op>
__device__ __forceinline__ int with_xor32(int x, Op op) {
  const auto r = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
  return op((int)r[0], (int)r[1]);
}
// op over all lanes of a row of 16 / of the wave, in every lane (op is commutative and associative).
template <class Op>
__device__ __forceinline__ int over_row(int x, Op op) {
  x = op(x, row_lane<kXor1>(x));
  x = op(x, row_lane<kXor2>(x));
  x = op(x, row_lane<kFlip8>(x));
  return op(x, row_lane<kFlip16>(x));
}
template <class Op>
__device__ __forceinline__ int over_wave(int x, Op op) { return with_xor32(with_xor16(over_row(x, op), op), op); }
struct AddInt { __device__ __forceinline__ int operator()(int a, int b) const { return a + b; } };
struct MaxU32 { __device__ __forceinline__ int operator()(int a, int b) const { return (int)max((uint32_t)a, (uint32_t)b); } };
struct AddF32 {
  __device__ __forceinline__ int operator()(int a, int b) const {
    return __builtin_bit_cast(int, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
  }
};
struct MaxF32 {
  __device__ __forceinline__ int operator()(int a, int b) const {
    return __builtin_bit_cast(int, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  }
};

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
  void* ws;                       // NULL: scores and choice in one launch
};
// Bytes of `ws` (0: none is used).
size_t cache_select_ws_bytes(const CacheDims& c, const RowDims& r, int group);
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
// Workgroups, and bytes of `parts`, that a call with lists of `list_len` blocks (0: no lists) takes; no more bytes than without
// a limit on the lists.
int64_t cache_attn_workgroups(const CacheDims& c, const RowDims& r, int group, int list_len);
size_t cache_attn_parts_bytes(const CacheDims& c, const RowDims& r, int group, int list_len);
hipError_t launch_cache_attn(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, hipStream_t s);

}  // namespace rsa
