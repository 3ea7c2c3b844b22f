// The cheap score of the blocks of an 8-bit cache and the choice of those that a group of query tokens reads.
//
// score(j) = q8 . k8_j * 2^em_j with q8 the group's summed queries and k8_j the mean key of block j, both in 8 bits with a
// power-of-two scale (that of q8 is common to a row and left out). The dot product is integer work and the scale moves no
// bit, so a score is exact, equal scores are equal, and the choice does not depend on an order of sums.
//
// One workgroup per (sequence, key/value head, group): sum of the queries (fp64: exact for bf16 terms within 40 binades of
// each other), scores of all blocks into LDS as order-preserving keys, the threshold key by four passes over eight bits
// each, and the kept blocks in ascending order.
#include "cache_common.hpp"

namespace rsa {
namespace {

__device__ __forceinline__ uint32_t ordered_key(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ double finite_or_zero(uint32_t bits16) {
  return (bits16 & 0x7f80u) == 0x7f80u ? 0.0 : (double)bf16_bits_to_float(bits16);
}
constexpr uint32_t kUnseen = 0u, kForced = 0xffffffffu;   // below and above every score

// Sum of an int over the workgroup's threads before this one, and over all of them; `red`: 4 ints.
__device__ __forceinline__ int scan_threads(int v, int* red, int* all) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  int in = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(in, o);
    if (lane >= o) in += up;
  }
  __syncthreads();
  if (lane == 63) red[wave] = in;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += red[w];
    total += red[w];
  }
  *all = total;
  return before + in - v;
}

template <int D>
__global__ __launch_bounds__(256) void cache_select_kernel(CacheDims c, RowDims r, CacheSelectArgs a) {
  constexpr int CPR = D / 8, STRIPES = 256 / CPR;
  extern __shared__ uint32_t keys[];               // [max_blocks]
  __shared__ double qs[STRIPES][D];
  __shared__ __align__(16) int8_t q8[D];
  __shared__ uint32_t hist[256];
  __shared__ int red[4];
  __shared__ uint32_t pick[2];
  const int tid = threadIdx.x;
  const int grp = blockIdx.x % a.groups, bh = blockIdx.x / a.groups;
  const int b = bh / c.heads_kv, hk = bh % c.heads_kv, G = r.heads / c.heads_kv;
  const int64_t row = (int64_t)bh * a.groups + grp;
  int32_t* list = a.block_idx + row * a.list_len;

  int64_t kv = a.kv_len[b];
  int64_t ql = a.q_len ? a.q_len[b] : r.t;
  if (ql > r.t) ql = r.t;
  const int64_t t0 = (int64_t)grp * a.group, t1 = min(t0 + a.group, ql);   // tokens of the group
  const int64_t p0 = kv - ql + t0, p1 = kv - ql + t1 - 1;                  // their positions
  int64_t seen64 = a.causal ? (p1 < 0 ? 0 : p1 / c.blk + 1) : (kv + c.blk - 1) / c.blk;
  if (t1 <= t0 || kv <= 0) seen64 = 0;
  const int seen = (int)min(seen64, (int64_t)c.max_blocks);
  if (seen <= 0) {                                 // nothing to choose from (the whole workgroup)
    for (int i = tid; i < a.list_len; i += 256) list[i] = -1;
    if (tid == 0) a.kept[row] = 0;
    return;
  }

  // the group's query, in 8 bits
  {
    const int cc = tid % CPR, stripe = tid / CPR;
    double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int rows = (int)(t1 - t0) * G;
    for (int i = stripe; i < rows; i += STRIPES) {
      const uint4 v = *reinterpret_cast<const uint4*>(a.Q + (int64_t)b * r.sb + (int64_t)(hk * G + i % G) * r.sh + (t0 + i / G) * r.st + cc * 8);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[2 * e] += finite_or_zero(w[e] & 0xffffu);
        acc[2 * e + 1] += finite_or_zero(w[e] >> 16);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) qs[stripe][cc * 8 + e] = acc[e];
    __syncthreads();
    if (tid < D) {
      double s = 0;
      for (int i = 0; i < STRIPES; ++i) s += qs[i][tid];
      qs[0][tid] = s;
    }
    __syncthreads();
    if (tid < 64) {
      double most = 0;
      for (int ch = tid; ch < D; ch += 64) most = fmax(most, fabs(qs[0][ch]));
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) most = fmax(most, __shfl_xor(most, o));
      int e = -100;
      if (most > 0) {
        int xp;
        const double m = frexp(most, &xp);
        e = max(xp - 7 + (m > 127.0 / 128.0 ? 1 : 0), -100);
      }
      for (int ch = tid; ch < D; ch += 64) q8[ch] = (int8_t)(int)rint(ldexp(qs[0][ch], -e));
    }
    __syncthreads();
  }

  // keys of the blocks
  const int lo_forced = a.last > 0 ? (int)max((int64_t)0, p0 / c.blk - (p0 < 0 && p0 % c.blk ? 1 : 0) - a.last + 1) : 0x7fffffff;
  const int hi_forced = a.last > 0 && p1 >= 0 ? (int)(p1 / c.blk) : -1;
  int n_seen = 0, n_forced = 0;
  {
    constexpr int LPB = D / 16;                    // lanes to a block: 16 channels each
    const int part = tid % LPB;
    const int4 q = *reinterpret_cast<const int4*>(&q8[part * 16]);
    for (int m0 = 0; m0 < seen; m0 += 256 / LPB) {
      const int m = m0 + tid / LPB;
      const int page = m < seen ? cache_page(c, b, m) : -1;
      int dot = 0;
      float scale = 0.f;
      if (page >= 0) {
        const int64_t rec = (int64_t)page * c.heads_kv + hk;
        const int4 k = *reinterpret_cast<const int4*>(c.mean + rec * D + part * 16);
        scale = c.scales[rec * 4 + 2];
        dot = __builtin_amdgcn_sdot4(q.x, k.x, dot, false);
        dot = __builtin_amdgcn_sdot4(q.y, k.y, dot, false);
        dot = __builtin_amdgcn_sdot4(q.z, k.z, dot, false);
        dot = __builtin_amdgcn_sdot4(q.w, k.w, dot, false);
      }
#pragma unroll
      for (int o = 1; o < LPB; o <<= 1) dot += __shfl_xor(dot, o);
      if (part == 0 && m < seen) {
        // 2^-22 keeps the largest scale finite; the product is exact (|dot| < 2^21)
        uint32_t key = ordered_key((float)dot * 0x1p-22f * scale);
        const bool forced = m < a.first || (m >= lo_forced && m <= hi_forced);
        if (forced) key = kForced;
        key = page < 0 ? kUnseen : max(key, kUnseen + 1);
        keys[m] = key;
        n_seen += page >= 0;
        n_forced += page >= 0 && forced;
      }
    }
  }
  int all_seen, all_forced;
  scan_threads(n_seen, red, &all_seen);
  scan_threads(n_forced, red, &all_forced);        // (its barriers also publish the keys)
  const int want = min(min(max(a.keep, all_forced), all_seen), a.list_len);

  // the want-th largest key, eight bits at a time
  uint32_t tau = 0;
  int left = want;                                 // how many of the keys with the prefix found so far are wanted
  for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int m = tid; m < seen; m += 256) {
      const uint32_t k = keys[m];
      if (shift == 24 || (k >> (shift + 8)) == (tau >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    int all;
    const int mine = (int)hist[255 - tid];         // thread i: digit 255 - i
    const int above = scan_threads(mine, red, &all);
    if (above < left && above + mine >= left) {
      pick[0] = 255 - tid;
      pick[1] = above;
    }
    __syncthreads();
    tau |= pick[0] << shift;
    left -= (int)pick[1];
    __syncthreads();
  }
  // now `left` of the blocks equal to tau are kept, the lowest; thread i owns a run of blocks
  const int run = (seen + 255) / 256;
  const int m0 = min(tid * run, seen), m1 = min(m0 + run, seen);
  int n_eq = 0, all;
  for (int m = m0; m < m1; ++m) n_eq += keys[m] == tau;
  int eq_before = scan_threads(n_eq, red, &all);
  int n_out = 0;
  {
    int eq = eq_before;
    for (int m = m0; m < m1; ++m) {
      const uint32_t k = keys[m];
      n_out += want > 0 && k != kUnseen && (k > tau || (k == tau && eq++ < left));
    }
  }
  int at = scan_threads(n_out, red, &all);
  for (int m = m0; m < m1; ++m) {
    const uint32_t k = keys[m];
    if (want > 0 && k != kUnseen && (k > tau || (k == tau && eq_before++ < left))) list[at++] = m;
  }
  for (int i = want + tid; i < a.list_len; i += 256) list[i] = -1;
  if (tid == 0) a.kept[row] = want;
}

}  // namespace

hipError_t launch_cache_select(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, hipStream_t s) {
  const dim3 grid(a.groups * c.batch * c.heads_kv);
  const size_t lds = (size_t)c.max_blocks * sizeof(uint32_t);
  if (c.d == 128) hipLaunchKernelGGL((cache_select_kernel<128>), grid, dim3(256), lds, s, c, r, a);
  else hipLaunchKernelGGL((cache_select_kernel<64>), grid, dim3(256), lds, s, c, r, a);
  return hipGetLastError();
}

}  // namespace rsa
