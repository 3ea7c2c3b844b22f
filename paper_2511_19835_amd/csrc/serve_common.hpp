// Shared declarations of what stands between request lengths and a cache's calls: pages of new tokens, rotary positions.
#pragma once

#include "rsa_common.hpp"

namespace rsa {

struct AssignArgs {
  int batch, max_blocks, block, t;
  int64_t pages;
  int32_t *table, *free_pages;
  const int32_t *kv_len, *add, *free_count;
  int32_t *kv_new, *free_left, *start, *count;
  int32_t* shared;                                     // may be NULL (0)
  int32_t* positions;                                  // may be NULL
  int64_t* slots;                                      // may be NULL
};
hipError_t launch_assign(const AssignArgs& a, hipStream_t s);

struct RotaryArgs {
  int batch, t, head_dim, pairs;
  int ends[3];                     // first pair behind each axis
  bool interleaved, inverse;
  float factor;
  const double* freq;              // [pairs]
  const int32_t *positions, *start, *count;   // [axes][batch][t], or NULL: start[b] + i
  struct Rows {
    int heads;
    int64_t sb, sh, st;
    const uint16_t* in;
    uint16_t* out;
  } x[2];                          // heads = 0: none
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s);

}  // namespace rsa
