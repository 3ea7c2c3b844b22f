// The 8-bit key/value cache as it is written and read back.
//
// Scales are powers of two. For a floating code that costs nothing (an element keeps its four significant bits wherever the
// block's largest lies between two powers), and it makes every step but the rounding to four bits exact: x * 2^-e, codes
// moved to a larger scale when a later token asks for one (only what becomes subnormal is rounded again), and the way back,
// code * 2^e in bf16.
//
// One workgroup per (block of tokens that the call touches, sequence, key/value head), for K and V: the largest magnitude of
// the new tokens decides the two exponents, so all rows of the block are in registers before the first code is made. The
// codes go through LDS, where they are put in page order (cache_common.hpp), and leave in 16-byte pieces.
//
// Long writes and reads are bound by memory: 119 056 tokens of 24 heads of 128 written in 451 us (2.20 GB, 4.9 TB/s), 20 280 read in
// 80 (0.37 GB, 4.6 TB/s); a copy of 1 GiB makes 5.2. One token is bound by latency, 7.6 us for eight of eight heads: a page's scales and codes,
// the maximum, the codes in LDS, the mean, each waiting for the one before; so pieces stay in registers and sums go by lane
// exchanges (11.0 us with exchanges through LDS and integer divisions).
#include <type_traits>

#include "cache_common.hpp"

namespace rsa {
namespace {

// Largest finite magnitude of the eight bf16 of a chunk, as bits; `a` is the largest so far.
__device__ __forceinline__ uint32_t finite_max(uint32_t a, const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    a = max(a, lo < 0x7f80u ? lo : 0u);
    a = max(a, hi < 0x7f80u ? hi : 0u);
  }
  return a;
}
// The least e >= -126 with amax <= 448 * 2^e = 1.75 * 2^(8 + e), amax given as bf16 bits.
__device__ __forceinline__ int code_exponent(uint32_t bits) {
  const int e = (int)(bits >> 7) - 127 - 8 + ((bits & 127u) > 0x60u ? 1 : 0);
  return e < -126 ? -126 : e;
}
// Four values over 2^e as e4m3 (nearest, ties to even), byte i = x[i]; |x| <= 448, or not finite: NaN.
__device__ __forceinline__ uint32_t to_codes(const float (&x)[4]) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = fabsf(x[i]) <= 448.f ? x[i] : __builtin_nanf("");
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
  return (uint32_t)r;
}
__device__ __forceinline__ void from_codes(uint32_t c, float (&x)[4]) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
  const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
}
__device__ __forceinline__ bool code_is_nan(uint32_t byte) { return (byte & 127u) == 127u; }
// The value of a code in units of 2^-9; NaN counts as 0. At most 448 * 512 < 2^18: sums over a block are exact in 32 bits.
__device__ __forceinline__ int code_units(float x) { return x == x ? (int)(x * 512.f) : 0; }

template <int D, int BLK>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheDims c, RowDims r, CacheWriteArgs a, int blocks) {
  constexpr int CPR = D / 8;                       // chunks of eight channels
  constexpr int QUADS = 256 / CPR;                 // runs of four tokens in flight
  constexpr int NP = BLK / (4 * QUADS) > 0 ? BLK / (4 * QUADS) : 1;
  constexpr int PIECES = BLK * D / 16;             // 16-byte pieces of a page's codes
  __shared__ __align__(16) uint8_t codes[2][BLK * D];
  __shared__ int sums[D];
  __shared__ uint32_t red[2][4];
  const int tid = threadIdx.x;
  const int j = blockIdx.x % blocks, bh = blockIdx.x / blocks;
  const int b = bh / c.heads_kv, h = bh % c.heads_kv;
  BlockSpan sp;
  if (!touched_block<BLK>(c, r.t, a.start, a.count, b, j, &sp)) return;   // the whole workgroup

  // new rows (requested while the page is looked up)
  const int cc = tid % CPR, quad = tid / CPR;
  const bool mine = quad * 4 < BLK;
  const int64_t base = (int64_t)b * r.sb + (int64_t)h * r.sh + sp.first * r.st + cc * 8;
  uint4 x[2][NP][4];
  uint32_t big[2] = {0, 0};
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
  const int64_t rec = (int64_t)sp.page * c.heads_kv + h;

  // what the block holds already (its first `lo` slots): 16-byte pieces tid, tid + 256, ...
  constexpr int PPT = PIECES / 256 > 0 ? PIECES / 256 : 1;
  const int prow = tid % 16, pg = tid / 16 % 4;    // of all pieces of a thread: key of 16 (K) or channel of 16 (V), and g
  uint4 was[2][PPT];
  float held_scale[2] = {1.f, 1.f};
  if (sp.lo > 0) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      held_scale[w] = c.scales[rec * 4 + w];
      const uint8_t* src = (w == 0 ? c.k : c.v) + rec * (BLK * D);
#pragma unroll
      for (int u = 0; u < PPT; ++u) {
        const int pc = tid + u * 256;
        const int first = w == 0 ? pc / D * 16 + prow : pc / (4 * D) * 64 + 4 * pg;   // its lowest token
        was[w][u] = make_uint4(0, 0, 0, 0);
        if (pc < PIECES && first < sp.lo) was[w][u] = *reinterpret_cast<const uint4*>(src + pc * 16);
      }
    }
  }
  if (tid < D) sums[tid] = 0;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) big[w] = finite_max(big[w], x[w][p][i]);
    big[w] = (uint32_t)over_wave((int)big[w], MaxU32());
    if (tid % 64 == 0) red[w][tid / 64] = big[w];
  }
  __syncthreads();
  int e[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) e[w] = code_exponent(max(max(red[w][0], red[w][1]), max(red[w][2], red[w][3])));

  // the older tokens, moved to the larger scale where the new ones ask for it
  if (sp.lo > 0) {
    int part[16] = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};      // K: sums of 16 channels (the same for all pieces of a thread)
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const int held = min(max(exponent_of(held_scale[w]), -126), 120);
      const float down = exp2_int(max(held - max(held, e[w]), -126));
      e[w] = max(e[w], held);
#pragma unroll
      for (int u = 0; u < PPT; ++u) {
        const int pc = tid + u * 256;
        uint32_t q[4] = {was[w][u].x, was[w][u].y, was[w][u].z, was[w][u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (w == 1) {                                                  // dword i: keys t64 + 16 i + 4 g .. + 3 of a channel
            const int old = sp.lo - (pc / (4 * D) * 64 + 16 * i + 4 * pg);
            q[i] &= old <= 0 ? 0u : old >= 4 ? 0xffffffffu : 0xffffffffu >> (32 - 8 * old);
          }
          if (down != 1.f) {
            float f[4];
            from_codes(q[i], f);
#pragma unroll
            for (int x = 0; x < 4; ++x) f[x] *= down;
            q[i] = to_codes(f);
          }
          if (w == 0) {
            float f[4];
            from_codes(q[i], f);
#pragma unroll
            for (int x = 0; x < 4; ++x) part[4 * i + x] += code_units(f[x]);
          }
        }
        if (pc < PIECES) *reinterpret_cast<uint4*>(&codes[w][pc * 16]) = make_uint4(q[0], q[1], q[2], q[3]);
      }
    }
    // over the 16 keys that the lanes of a row hold: each exchange halves the channels that a lane is left with
    auto halve = [&](auto ctrl, int o) __attribute__((always_inline)) {
      const bool up = (prow & o) != 0;
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (x < o) {
          const int keep = up ? part[x + o] : part[x], give = up ? part[x] : part[x + o];
          part[x] = keep + row_lane<decltype(ctrl)::value>(give);
        }
    };
    halve(std::integral_constant<int, kXor8>{}, 8);
    halve(std::integral_constant<int, kFlip8>{}, 4);
    halve(std::integral_constant<int, kXor2>{}, 2);
    halve(std::integral_constant<int, kXor1>{}, 1);
    if (tid < PIECES) atomicAdd(&sums[tid / 64 % (D / 64) * 64 + pg * 16 + prow], part[0]);
    __syncthreads();
  }

  // codes of the new tokens, four keys of a channel at a time
  if (mine) {
    int part[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float inv = exp2_int(-e[w]);
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int slot0 = (p * QUADS + quad) * 4;
        // (a block begun before has its zeros and older codes in place: one token costs one wave its conversion, not all)
        if (sp.lo > 0 && (slot0 >= sp.hi || slot0 + 4 <= sp.lo)) continue;
        uint32_t cd[8];                             // by channel: byte i = token slot0 + i
#pragma unroll
        for (int q = 0; q < 4; ++q) {               // channels 2 q, 2 q + 1
          float lo[4], hi[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4& v = x[w][p][i];
            const uint32_t word = q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w;
            lo[i] = bf16_bits_to_float(word & 0xffffu) * inv;
            hi[i] = bf16_bits_to_float(word >> 16) * inv;
          }
          cd[2 * q] = to_codes(lo);
          cd[2 * q + 1] = to_codes(hi);
        }
        if (w == 0) {
#pragma unroll
          for (int ch = 0; ch < 8; ++ch) {
            float f[4];
            from_codes(cd[ch], f);
#pragma unroll
            for (int i = 0; i < 4; ++i) part[ch] += code_units(f[i]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {             // eight channels of a key are eight bytes in a row
            uint32_t lo = 0, hi = 0;
#pragma unroll
            for (int ch = 0; ch < 4; ++ch) {
              lo |= ((cd[ch] >> (8 * i)) & 255u) << (8 * ch);
              hi |= ((cd[ch + 4] >> (8 * i)) & 255u) << (8 * ch);
            }
            if (slot0 + i >= sp.lo) *reinterpret_cast<uint2*>(&codes[0][k_code_offset<D>(slot0 + i, cc * 8)]) = make_uint2(lo, hi);
          }
        } else {
          const int old = sp.lo - slot0;            // older tokens among the four
          if (old < 4) {
            const uint32_t hold = old <= 0 ? 0u : 0xffffffffu >> (32 - 8 * old);
#pragma unroll
            for (int ch = 0; ch < 8; ++ch) {
              uint32_t* dst = reinterpret_cast<uint32_t*>(&codes[1][v_code_offset<D>(slot0, cc * 8 + ch)]);
              if (hold) atomicOr(dst, cd[ch] & ~hold);                     // the others are zero; a read would wait for LDS
              else *dst = cd[ch];
            }
          }
        }
      }
    }
#pragma unroll
    for (int ch = 0; ch < 8; ++ch) {                // over the runs of tokens of this wave
      if (CPR == 8) part[ch] += row_lane<kXor8>(part[ch]);
      part[ch] = with_xor32(with_xor16(part[ch], AddInt()), AddInt());
      if (tid % 64 < CPR && part[ch]) atomicAdd(&sums[cc * 8 + ch], part[ch]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    uint8_t* dst = (w == 0 ? c.k : c.v) + rec * (BLK * D);
    for (int pc = tid; pc < PIECES; pc += 256) *reinterpret_cast<uint4*>(dst + pc * 16) = *reinterpret_cast<const uint4*>(&codes[w][pc * 16]);
  }

  // the mean of the block's keys in 8 bits: sums are exact, the division is the one rounding before the code's own
  if (tid < D) {
    uint32_t most = 0;                              // of all channels, in each wave
#pragma unroll
    for (int ch = tid % 64; ch < D; ch += 64) most = max(most, (uint32_t)abs(sums[ch]));
    most = (uint32_t)over_wave((int)most, MaxU32());
    const double n = (double)sp.hi;
    int em = -100;
    if (most) {
      int xp;
      const double m = frexp((double)most / n, &xp);
      em = max(xp - 7 + (m > 127.0 / 128.0 ? 1 : 0) + e[0] - 9, -100);
    }
    c.mean[rec * D + tid] = (int8_t)(int)rint(ldexp((double)sums[tid] / n, e[0] - 9 - em));
    if (tid == 0) *reinterpret_cast<float4*>(c.scales + rec * 4) = make_float4(exp2_int(e[0]), exp2_int(e[1]), exp2_int(em), 0.f);
  }
}

// Codes back into token rows: pieces in, through LDS as rows of bf16, rows out.
template <int D, int BLK>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheDims c, RowDims r, CacheReadArgs a, int blocks) {
  constexpr int PIECES = BLK * D / 16;
  constexpr int ROW = D + 8;
  __shared__ __align__(16) uint16_t rows[BLK * ROW];
  const int tid = threadIdx.x;
  const int j = blockIdx.x % blocks, bh = blockIdx.x / blocks;
  const int b = bh / c.heads_kv, h = bh % c.heads_kv;
  BlockSpan sp;
  if (!touched_block<BLK>(c, r.t, a.start, a.count, b, j, &sp) || sp.page < 0) return;
  const int64_t rec = (int64_t)sp.page * c.heads_kv + h;
  for (int w = 0; w < 2; ++w) {
    const uint8_t* src = (w == 0 ? c.k : c.v) + rec * (BLK * D);
    const float scale = c.scales[rec * 4 + w];
    for (int pc = tid; pc < PIECES; pc += 256) {
      const uint4 v = *reinterpret_cast<const uint4*>(src + pc * 16);
      const uint32_t q[4] = {v.x, v.y, v.z, v.w};
      const int row = pc % 16, g = pc / 16 % 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[4];
        from_codes(q[i], f);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int key = w == 0 ? pc / D * 16 + row : pc / (4 * D) * 64 + 16 * i + 4 * g + u;
          const int ch = w == 0 ? pc / 64 % (D / 64) * 64 + g * 16 + i * 4 + u : pc / 64 % (D / 16) * 16 + row;
          rows[key * ROW + ch] = to_bf16_bits(f[u] * scale);
        }
      }
    }
    __syncthreads();
    uint16_t* X = (w == 0 ? a.K : a.V) + (int64_t)b * r.sb + (int64_t)h * r.sh + sp.first * r.st;
    for (int u = tid; u < BLK * (D / 8); u += 256) {
      const int slot = u / (D / 8), ch = u % (D / 8) * 8;
      if (slot >= sp.lo && slot < sp.hi) *reinterpret_cast<uint4*>(X + slot * r.st + ch) = *reinterpret_cast<const uint4*>(&rows[slot * ROW + ch]);
    }
    __syncthreads();
  }
}

template <int D, int BLK>
hipError_t launch_write_t(const CacheDims& c, const RowDims& r, const CacheWriteArgs& a, hipStream_t s) {
  const int blocks = (r.t - 1) / BLK + 2;          // a run of t tokens touches at most these
  hipLaunchKernelGGL((cache_write_kernel<D, BLK>), dim3(blocks * c.batch * c.heads_kv), dim3(256), 0, s, c, r, a, blocks);
  return hipGetLastError();
}
template <int D, int BLK>
hipError_t launch_read_t(const CacheDims& c, const RowDims& r, const CacheReadArgs& a, hipStream_t s) {
  const int blocks = (r.t - 1) / BLK + 2;
  hipLaunchKernelGGL((cache_read_kernel<D, BLK>), dim3(blocks * c.batch * c.heads_kv), dim3(256), 0, s, c, r, a, blocks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheDims& c, const RowDims& r, const CacheWriteArgs& a, hipStream_t s) {
  if (c.d == 128) return c.blk == 128 ? launch_write_t<128, 128>(c, r, a, s) : launch_write_t<128, 64>(c, r, a, s);
  return c.blk == 128 ? launch_write_t<64, 128>(c, r, a, s) : launch_write_t<64, 64>(c, r, a, s);
}
hipError_t launch_cache_read(const CacheDims& c, const RowDims& r, const CacheReadArgs& a, hipStream_t s) {
  if (c.d == 128) return c.blk == 128 ? launch_read_t<128, 128>(c, r, a, s) : launch_read_t<128, 64>(c, r, a, s);
  return c.blk == 128 ? launch_read_t<64, 128>(c, r, a, s) : launch_read_t<64, 64>(c, r, a, s);
}

}  // namespace rsa
