// Shared declarations of the translation units of the 4-bit key/value cache (gfx950 only).
//
// A page holds one block of BLK tokens of every key/value head, as BLK / 64 records of 64 tokens each, codes first and scales behind
// them, so that a step of 64 keys is one run of memory. Codes are e2m1, two to a byte, the lower half byte first, in the order in
// which the 16x16x32 matrix instructions of fourbit_attn_kernels.hip take them once they are widened to bf16:
//   K  [tile 0..3][run d/32][key 0..15][32 channels]      at d = 128 lane 16 run + key reads 16 bytes, at d = 64 lane 16 g + key the
//                                                         8 bytes of channels 16 g .. 16 g + 15
//      [run d/32][key 0..15][tile 0..3]                   exponents + 127 of (key, run of 32 channels), a dword to a lane; 255: NaN
//   V  [32 channels: d/32][g 0..3][channel 0..15][half 0..1][t 0..3][i 0..3]   lane 16 g + channel: keys 16 t + 4 g + i of channels
//                                                         c and 16 + c
//      [g 0..3][t 0..3][i 0..3]                           scales of the keys in bf16 (a power of two, or NaN)
// After S^T = K Q^T lane 16 g + q holds the scores of keys 4 g + i of every tile t: with this order of V those are its operand of
// O^T += V^T P^T. A key's scale goes into the widening (it runs along the channels that are summed), a value's into the weight
// of its token, which is why values have one scale to a token and keys one to 32 channels.
#pragma once

#include "cache_common.hpp"

namespace rsa {

// Bytes of a record of 64 tokens.
__host__ __device__ constexpr int fourbit_k_record(int d) { return 64 * (d / 2 + d / 32); }
__host__ __device__ constexpr int fourbit_v_record(int d) { return 64 * (d / 2 + 2); }

constexpr int kLeastExponent = -124;           // what is widened to bf16 stays a normal number
constexpr uint32_t kNanScale = 255;            // of a run of keys that held an infinity or NaN

hipError_t launch_fourbit_write(const CacheDims& c, const RowDims& r, const CacheWriteArgs& a, hipStream_t s);
hipError_t launch_fourbit_read(const CacheDims& c, const RowDims& r, const CacheReadArgs& a, hipStream_t s);
int64_t fourbit_attn_workgroups(const CacheDims& c, const RowDims& r, int group, int list_len);
size_t fourbit_attn_parts_bytes(const CacheDims& c, const RowDims& r, int group, int list_len);
hipError_t launch_fourbit_attn(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, hipStream_t s);

}  // namespace rsa
