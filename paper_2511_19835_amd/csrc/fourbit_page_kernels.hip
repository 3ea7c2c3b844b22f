// The 4-bit key/value cache as it is written and read back.
//
// Every token has its own scales (a power of two for each 32 channels of the key and for the value row), so that a write touches
// no older token: no code is ever rounded twice, and pages are the same bits however calls are cut. Only a block's mean key, for the
// selection, is made anew from all of its tokens: sums of code * 2^e in 64 bits, which are exact unless scales of a channel lie 2^40 apart.
//
// One workgroup per (block of tokens that the call touches, sequence, key/value head), for K and V. A thread holds runs of four tokens
// by eight channels: eight codes of a key are a dword of its page, and of the values four tokens of a channel are 16 bits, which is
// the order that the attention's products take them in (fourbit_common.hpp). Codes go through LDS and leave in 16-byte pieces; rows
// of 16 pieces are 272 bytes apart there, so that the lanes of a write fall on different banks. Only runs with a new token are coded.
//
// Many tokens are bound by memory: 24 heads of 119 056 tokens, d = 128, 1.85 GB each way, written in 365 to 404 us and read in 362 to 392 (4.6 to
// 5.1 TB/s; a copy 5.17). Few by latency: a token of 8 sequences, 8 heads, 6.4 and 3.5 us (length, page, codes of the block for its mean, LDS,
// mean), of 48 sequences, 24 heads, blocks of 128, 14.8 and 5.0 (19.7 and 6.5 with every run coded and two workgroups to a head).
#include "fourbit_common.hpp"

namespace rsa {
namespace {

typedef uint16_t ushortx2 __attribute__((ext_vector_type(2)));
constexpr int kRow = 272;                          // bytes of 16 pieces in LDS

// Largest magnitude of the eight bf16 of a chunk, as bits (above those of infinity: NaN).
__device__ __forceinline__ uint32_t largest8(const uint4& v) {
  auto mag = [](uint32_t w) __attribute__((always_inline)) { return __builtin_bit_cast(ushortx2, w & 0x7fff7fffu); };
  const ushortx2 a = __builtin_elementwise_max(__builtin_elementwise_max(mag(v.x), mag(v.y)), __builtin_elementwise_max(mag(v.z), mag(v.w)));
  return max((uint32_t)a[0], (uint32_t)a[1]);
}
// The least e >= kLeastExponent with amax <= 6 * 2^e = 1.5 * 2^(2 + e), amax given as bf16 bits; 128 where it is not finite.
__device__ __forceinline__ int fourbit_exponent(uint32_t bits) {
  const int e = (int)(bits >> 7) - 127 - 2 + ((bits & 127u) > 64u ? 1 : 0);
  return bits >= 0x7f80u ? 128 : max(e, kLeastExponent);
}
// Eight bf16 over 2^e as e2m1 (nearest, ties to even); zeros for e = 128.
__device__ __forceinline__ uint32_t to_codes(const uint4& v, int e) {
  const float scale = exp2_int(e == 128 ? 0 : e);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v.x), scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v.y), scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v.z), scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, v.w), scale, 3);
  return e == 128 ? 0 : w;
}
// Eight codes times 2^e in bf16 (exact).
__device__ __forceinline__ uint4 from_codes(uint32_t w, float scale) {
  uint4 v;
  v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return v;
}
// Four tokens by eight channels: w[i] holds the eight channels of token i; h[0] the four tokens of channels 0 and 2 in 16 bits each,
// h[1] those of 4 and 6, h[2] of 1 and 3, h[3] of 5 and 7.
constexpr uint32_t kLow = 0x0f0f0f0fu;
__device__ __forceinline__ void tokens_to_channels(const uint32_t (&w)[4], uint32_t (&h)[4]) {
  const uint32_t a = (w[0] & kLow) | ((w[1] & kLow) << 4), b = ((w[0] >> 4) & kLow) | (w[1] & ~kLow);
  const uint32_t c = (w[2] & kLow) | ((w[3] & kLow) << 4), d = ((w[2] >> 4) & kLow) | (w[3] & ~kLow);
  h[0] = __builtin_amdgcn_perm(c, a, 0x05010400u);
  h[1] = __builtin_amdgcn_perm(c, a, 0x07030602u);
  h[2] = __builtin_amdgcn_perm(d, b, 0x05010400u);
  h[3] = __builtin_amdgcn_perm(d, b, 0x07030602u);
}
// From the 16 bits of each channel.
__device__ __forceinline__ void channels_to_tokens(const uint32_t (&u)[8], uint32_t (&w)[4]) {
  const uint32_t p = __builtin_amdgcn_perm(u[2], u[0], 0x05010400u), q = __builtin_amdgcn_perm(u[6], u[4], 0x05010400u);
  const uint32_t r = __builtin_amdgcn_perm(u[3], u[1], 0x05010400u), s = __builtin_amdgcn_perm(u[7], u[5], 0x05010400u);
  const uint32_t a = __builtin_amdgcn_perm(q, p, 0x05040100u), c = __builtin_amdgcn_perm(q, p, 0x07060302u);
  const uint32_t b = __builtin_amdgcn_perm(s, r, 0x05040100u), d = __builtin_amdgcn_perm(s, r, 0x07060302u);
  w[0] = (a & kLow) | ((b & kLow) << 4);
  w[1] = ((a >> 4) & kLow) | (b & ~kLow);
  w[2] = (c & kLow) | ((d & kLow) << 4);
  w[3] = ((c >> 4) & kLow) | (d & ~kLow);
}

__device__ __forceinline__ double from_halves(int lo, int hi) { return __hiloint2double(hi, lo); }
template <int CTRL>
__device__ __forceinline__ double row_lane64(double x) { return from_halves(row_lane<CTRL>(__double2loint(x)), row_lane<CTRL>(__double2hiint(x))); }
template <class Op>
__device__ __forceinline__ double with_xor16_64(double x, Op op) {
  const uint32_t l = (uint32_t)__double2loint(x), h = (uint32_t)__double2hiint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(l, l, false, false), b = __builtin_amdgcn_permlane16_swap(h, h, false, false);
  return op(from_halves((int)a[0], (int)b[0]), from_halves((int)a[1], (int)b[1]));
}
template <class Op>
__device__ __forceinline__ double with_xor32_64(double x, Op op) {
  const uint32_t l = (uint32_t)__double2loint(x), h = (uint32_t)__double2hiint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(l, l, false, false), b = __builtin_amdgcn_permlane32_swap(h, h, false, false);
  return op(from_halves((int)a[0], (int)b[0]), from_halves((int)a[1], (int)b[1]));
}
struct AddF64 { __device__ __forceinline__ double operator()(double a, double b) const { return a + b; } };
struct MaxF64 { __device__ __forceinline__ double operator()(double a, double b) const { return fmax(a, b); } };

// Offsets in a record of 64 tokens / in its image in LDS.
template <int D>
struct At {
  // codes of a key: row (tile, run) of 16 pieces, piece = key; eight channels of a chunk are a dword
  static __device__ __forceinline__ int k_row(int u, int cc) { return u / 16 * (D / 32) + cc / 4; }
  static __device__ __forceinline__ int k_scale(int u, int run) { return (run * 16 + u % 16) * 4 + u / 16; }
  // codes of four values: row (32 channels, g) of 16 pieces, piece = channel of 16
  static __device__ __forceinline__ int v_row(int u, int ch) { return ch / 32 * 4 + u % 16 / 4; }
  static __device__ __forceinline__ int v_in_row(int u, int ch) { return ch % 16 * 16 + ch % 32 / 16 * 8 + u / 16 * 2; }
  static __device__ __forceinline__ int v_scale(int u) { return u % 16 / 4 * 16 + u / 16 * 4 + u % 4; }   // in bf16
};
// Whether some token lo <= slot < hi lies in group g (tokens 16 t + 4 g + i) of 64 tokens `s`.
__device__ __forceinline__ bool group_touched(int s, int g, int lo, int hi) {
  bool any = false;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int first = s * 64 + 16 * t + 4 * g;
    any |= first < hi && first + 4 > lo;
  }
  return any;
}

template <int D, int BLK>
__global__ __launch_bounds__(256) void fourbit_write_kernel(CacheDims c, RowDims r, CacheWriteArgs a, int blocks) {
  constexpr int CPR = D / 8;                       // chunks of eight channels
  constexpr int QUADS = 256 / CPR;                 // runs of four tokens in flight
  constexpr int NP = BLK / (4 * QUADS) > 0 ? BLK / (4 * QUADS) : 1;
  constexpr int SPB = BLK / 64, ROWS = D / 8;      // rows of 16 pieces of a record's codes, K or V
  constexpr int KR = fourbit_k_record(D), VR = fourbit_v_record(D);
  __shared__ __align__(16) uint8_t img_k[SPB][ROWS][kRow], img_v[SPB][ROWS][kRow];
  __shared__ __align__(16) uint8_t img_ks[SPB][2 * D];
  __shared__ __align__(16) uint16_t img_vs[SPB][64];
  __shared__ double sums[4][D];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  // (the heads of a block follow one another: their rows are neighbours in [token, head] order, their pages in memory)
  const int h = blockIdx.x % c.heads_kv, bj = blockIdx.x / c.heads_kv;
  const int b = bj / blocks, j = bj % blocks;
  BlockSpan sp;
  if (!touched_block<BLK>(c, r.t, a.start, a.count, b, j, &sp)) return;   // the whole workgroup

  // new rows (requested while the page is looked up)
  const int cc = tid % CPR, quad = tid / CPR;
  const bool mine = quad * 4 < BLK;
  const int64_t base = (int64_t)b * r.sb + (int64_t)h * r.sh + sp.first * r.st + cc * 8;
  uint4 x[2][NP][4];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const uint16_t* X = (w == 0 ? a.K : a.V) + base;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int slot = (p * QUADS + quad) * 4 + i;
        x[w][p][i] = make_uint4(0, 0, 0, 0);
        if (mine && slot >= sp.lo && slot < sp.hi) x[w][p][i] = *reinterpret_cast<const uint4*>(X + slot * r.st);
      }
  }
  if (sp.page < 0) return;                         // (the whole workgroup)
  const int64_t rec = ((int64_t)sp.page * c.heads_kv + h) * SPB;
  uint8_t *pk = c.k + rec * KR, *pv = c.v + rec * VR;
  const bool whole = sp.lo == 0 && sp.hi == BLK;

  // what the block holds already: the keys' codes for the mean, and the pieces of values that new tokens share with others
  uint32_t kd[NP][4];
  int ke[NP][4];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = (p * QUADS + quad) * 4 + i, u = slot % 64;
      kd[p][i] = 0;
      ke[p][i] = 128;
      if (mine && slot < sp.lo) {
        const uint8_t* src = pk + slot / 64 * KR;
        kd[p][i] = *reinterpret_cast<const uint32_t*>(src + (At<D>::k_row(u, cc) * 16 + u % 16) * 16 + cc % 4 * 4);
        const int byte = src[32 * D + At<D>::k_scale(u, cc / 4)];
        ke[p][i] = byte == (int)kNanScale ? 128 : min(max(byte, 1), 254) - 127;
        if (ke[p][i] == 128) kd[p][i] = 0;
      }
    }
  if (!whole) {
    for (int pc = tid; pc < SPB * ROWS * 16; pc += 256) {
      const int s = pc / (ROWS * 16), row = pc / 16 % ROWS;
      if (group_touched(s, row % 4, sp.lo, sp.hi))
        *reinterpret_cast<uint4*>(&img_v[s][row][pc % 16 * 16]) = *reinterpret_cast<const uint4*>(pv + s * VR + pc % (ROWS * 16) * 16);
    }
    __syncthreads();
  }

  double part[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (mine) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int slot0 = (p * QUADS + quad) * 4, u0 = slot0 % 64, s = slot0 / 64;
      if (slot0 < sp.hi) {
        if (slot0 + 4 > sp.lo) {                   // a new token (the lanes of a run of tokens go the same way)
          uint32_t vw[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int slot = slot0 + i, u = u0 + i;
            const bool is = slot >= sp.lo && slot < sp.hi;
            int most = (int)largest8(x[0][p][i]);     // over the 32 channels of the run
            most = MaxU32()(most, row_lane<kXor1>(most));
            most = MaxU32()(most, row_lane<kXor2>(most));
            const int e = fourbit_exponent((uint32_t)most);
            const uint32_t w = to_codes(x[0][p][i], e);
            if (is) {
              kd[p][i] = w;
              ke[p][i] = e;
              *reinterpret_cast<uint32_t*>(&img_k[s][At<D>::k_row(u, cc)][u % 16 * 16 + cc % 4 * 4]) = w;
              if (cc % 4 == 0) img_ks[s][At<D>::k_scale(u, cc / 4)] = (uint8_t)(e + 127);
            }
            int mv = (int)largest8(x[1][p][i]);       // over the row
            mv = MaxU32()(mv, row_lane<kXor1>(mv));
            mv = MaxU32()(mv, row_lane<kXor2>(mv));
            mv = MaxU32()(mv, row_lane<kFlip8>(mv));
            if (D == 128) mv = MaxU32()(mv, row_lane<kFlip16>(mv));
            const int ev = fourbit_exponent((uint32_t)mv);
            vw[i] = to_codes(x[1][p][i], ev);
            if (is && cc == 0) img_vs[s][At<D>::v_scale(u)] = ev == 128 ? 0x7fc0u : (uint16_t)((ev + 127) << 7);
          }
          uint32_t hw[4], fresh = 0xffffu;         // half bytes of the four tokens that are new
          tokens_to_channels(vw, hw);
          if (sp.lo > slot0) fresh &= 0xffffu << (4 * (sp.lo - slot0));
          if (sp.hi < slot0 + 4) fresh &= 0xffffu >> (4 * (slot0 + 4 - sp.hi));
#pragma unroll
          for (int ch = 0; ch < 8; ++ch) {
            const int pair = ch % 2 * 2 + ch / 4;
            const uint32_t z = ch / 2 % 2 ? hw[pair] >> 16 : hw[pair] & 0xffffu;
            uint16_t* dst = reinterpret_cast<uint16_t*>(&img_v[s][At<D>::v_row(u0, cc * 8 + ch)][At<D>::v_in_row(u0, cc * 8 + ch)]);
            *dst = (uint16_t)(fresh == 0xffffu ? z : (z & fresh) | (*dst & ~fresh));
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float scale = exp2_int(ke[p][i] == 128 ? 0 : ke[p][i]);
          // (4 * 2^126 is an infinity in bf16 and fp32: not counted, like any other)
          if (ke[p][i] == 126) kd[p][i] &= ~((kd[p][i] >> 1 & kd[p][i] >> 2 & 0x11111111u) * 15u);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            floatx2 f;
            if (q == 0) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(kd[p][i], scale, 0);
            else if (q == 1) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(kd[p][i], scale, 1);
            else if (q == 2) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(kd[p][i], scale, 2);
            else f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(kd[p][i], scale, 3);
            part[2 * q] += (double)f[0];
            part[2 * q + 1] += (double)f[1];
          }
        }
      }
    }
  }
#pragma unroll
  for (int ch = 0; ch < 8; ++ch) {                  // over the runs of tokens of this wave
    if (CPR == 8) part[ch] += row_lane64<kXor8>(part[ch]);
    part[ch] = with_xor32_64(with_xor16_64(part[ch], AddF64()), AddF64());
    if (lane < CPR) sums[wave][cc * 8 + ch] = part[ch];
  }
  __syncthreads();

  // pieces out
  for (int pc = tid; pc < SPB * ROWS * 16; pc += 256) {
    const int s = pc / (ROWS * 16), row = pc / 16 % ROWS, n = pc % 16, off = pc % (ROWS * 16) * 16;
    const int slot = s * 64 + row / (D / 32) * 16 + n;
    if (slot >= sp.lo && slot < sp.hi) *reinterpret_cast<uint4*>(pk + s * KR + off) = *reinterpret_cast<const uint4*>(&img_k[s][row][n * 16]);
    if (whole || group_touched(s, row % 4, sp.lo, sp.hi))
      *reinterpret_cast<uint4*>(pv + s * VR + off) = *reinterpret_cast<const uint4*>(&img_v[s][row][n * 16]);
  }
  if (whole) {
    constexpr int KP = 2 * D / 16, VP = 8;          // pieces of scales in a record
    for (int pc = tid; pc < SPB * (KP + VP); pc += 256) {
      const int s = pc / (KP + VP), q = pc % (KP + VP);
      if (q < KP) *reinterpret_cast<uint4*>(pk + s * KR + 32 * D + q * 16) = *reinterpret_cast<const uint4*>(&img_ks[s][q * 16]);
      else *reinterpret_cast<uint4*>(pv + s * VR + 32 * D + (q - KP) * 16) = *reinterpret_cast<const uint4*>(&img_vs[s][(q - KP) * 8]);
    }
  } else {
    for (int w = tid; w < (sp.hi - sp.lo) * (D / 32); w += 256) {
      const int slot = sp.lo + w / (D / 32), at = At<D>::k_scale(slot % 64, w % (D / 32));
      pk[slot / 64 * KR + 32 * D + at] = img_ks[slot / 64][at];
    }
    for (int w = tid; w < sp.hi - sp.lo; w += 256) {
      const int slot = sp.lo + w, at = At<D>::v_scale(slot % 64);
      reinterpret_cast<uint16_t*>(pv + slot / 64 * VR + 32 * D)[at] = img_vs[slot / 64][at];
    }
  }

  // the mean of the block's keys in 8 bits
  if (tid < D) {
    const double n = (double)sp.hi;
    auto sum = [&](int ch) __attribute__((always_inline)) { return (sums[0][ch] + sums[1][ch]) + (sums[2][ch] + sums[3][ch]); };
    const double own = sum(tid) / n;
    double most = fabs(sum(lane));
    if (D == 128) most = fmax(most, fabs(sum(lane + 64)));
    most = fmax(most, row_lane64<kXor1>(most));
    most = fmax(most, row_lane64<kXor2>(most));
    most = fmax(most, row_lane64<kFlip8>(most));
    most = fmax(most, row_lane64<kFlip16>(most));
    most = with_xor32_64(with_xor16_64(most, MaxF64()), MaxF64());
    most /= n;                                     // (the largest mean: a division keeps the order)
    int em = -100;
    if (most > 0) {
      int xp;
      const double f = frexp(most, &xp);
      em = max(xp - 7 + (f > 127.0 / 128.0 ? 1 : 0), -100);
    }
    c.mean[((int64_t)sp.page * c.heads_kv + h) * D + tid] = (int8_t)(int)rint(ldexp(own, -em));
    if (tid == 0) *reinterpret_cast<float4*>(c.scales + ((int64_t)sp.page * c.heads_kv + h) * 4) = make_float4(0.f, 0.f, exp2_int(em), 0.f);
  }
}

// Codes back into token rows.
template <int D, int BLK>
__global__ __launch_bounds__(256) void fourbit_read_kernel(CacheDims c, RowDims r, CacheReadArgs a, int blocks) {
  constexpr int CPR = D / 8, SPB = BLK / 64, ROWS = D / 8;
  constexpr int KR = fourbit_k_record(D), VR = fourbit_v_record(D);
  __shared__ __align__(16) uint8_t img_v[SPB][ROWS][kRow];
  const int tid = threadIdx.x;
  const int j = blockIdx.x % blocks, bh = blockIdx.x / blocks;
  const int b = bh / c.heads_kv, h = bh % c.heads_kv;
  BlockSpan sp;
  if (!touched_block<BLK>(c, r.t, a.start, a.count, b, j, &sp) || sp.page < 0) return;
  const int64_t rec = ((int64_t)sp.page * c.heads_kv + h) * SPB;
  const uint8_t *pk = c.k + rec * KR, *pv = c.v + rec * VR;
  const int64_t base = (int64_t)b * r.sb + (int64_t)h * r.sh + sp.first * r.st;
  for (int pc = tid; pc < SPB * ROWS * 16; pc += 256) {
    const int s = pc / (ROWS * 16), row = pc / 16 % ROWS;
    if (group_touched(s, row % 4, sp.lo, sp.hi))
      *reinterpret_cast<uint4*>(&img_v[s][row][pc % 16 * 16]) = *reinterpret_cast<const uint4*>(pv + s * VR + pc % (ROWS * 16) * 16);
  }
  for (int w = sp.lo * CPR + tid; w < sp.hi * CPR; w += 256) {
    const int slot = w / CPR, cc = w % CPR, u = slot % 64;
    const uint8_t* src = pk + slot / 64 * KR;
    const uint32_t code = *reinterpret_cast<const uint32_t*>(src + (At<D>::k_row(u, cc) * 16 + u % 16) * 16 + cc % 4 * 4);
    const uint32_t byte = src[32 * D + At<D>::k_scale(u, cc / 4)];
    const float scale = byte == kNanScale ? __builtin_nanf("") : __builtin_bit_cast(float, byte << 23);
    *reinterpret_cast<uint4*>(a.K + base + slot * r.st + cc * 8) = from_codes(code, scale);
  }
  __syncthreads();
  for (int w = sp.lo / 4 * CPR + tid; w < (sp.hi + 3) / 4 * CPR; w += 256) {
    const int slot0 = w / CPR * 4, cc = w % CPR, u0 = slot0 % 64, s = slot0 / 64;
    uint32_t u[8], code[4];
#pragma unroll
    for (int ch = 0; ch < 8; ++ch) u[ch] = *reinterpret_cast<const uint16_t*>(&img_v[s][At<D>::v_row(u0, cc * 8 + ch)][At<D>::v_in_row(u0, cc * 8 + ch)]);
    channels_to_tokens(u, code);
    const uint2 sc = *reinterpret_cast<const uint2*>(pv + s * VR + 32 * D + At<D>::v_scale(u0) * 2);      // of the four tokens
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t half = i < 2 ? sc.x : sc.y;
      const float scale = __builtin_bit_cast(float, i % 2 ? half & 0xffff0000u : half << 16);
      if (slot0 + i >= sp.lo && slot0 + i < sp.hi) *reinterpret_cast<uint4*>(a.V + base + (slot0 + i) * r.st + cc * 8) = from_codes(code[i], scale);
    }
  }
}

template <int D, int BLK>
hipError_t launch_write_t(const CacheDims& c, const RowDims& r, const CacheWriteArgs& a, hipStream_t s) {
  const int blocks = (r.t + BLK - 2) / BLK + 1;    // a run of t tokens touches at most these
  hipLaunchKernelGGL((fourbit_write_kernel<D, BLK>), dim3(blocks * c.batch * c.heads_kv), dim3(256), 0, s, c, r, a, blocks);
  return hipGetLastError();
}
template <int D, int BLK>
hipError_t launch_read_t(const CacheDims& c, const RowDims& r, const CacheReadArgs& a, hipStream_t s) {
  const int blocks = (r.t + BLK - 2) / BLK + 1;
  hipLaunchKernelGGL((fourbit_read_kernel<D, BLK>), dim3(blocks * c.batch * c.heads_kv), dim3(256), 0, s, c, r, a, blocks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fourbit_write(const CacheDims& c, const RowDims& r, const CacheWriteArgs& a, hipStream_t s) {
  if (c.d == 128) return c.blk == 128 ? launch_write_t<128, 128>(c, r, a, s) : launch_write_t<128, 64>(c, r, a, s);
  return c.blk == 128 ? launch_write_t<64, 128>(c, r, a, s) : launch_write_t<64, 64>(c, r, a, s);
}
hipError_t launch_fourbit_read(const CacheDims& c, const RowDims& r, const CacheReadArgs& a, hipStream_t s) {
  if (c.d == 128) return c.blk == 128 ? launch_read_t<128, 128>(c, r, a, s) : launch_read_t<128, 64>(c, r, a, s);
  return c.blk == 128 ? launch_read_t<64, 128>(c, r, a, s) : launch_read_t<64, 64>(c, r, a, s);
}

}  // namespace rsa
