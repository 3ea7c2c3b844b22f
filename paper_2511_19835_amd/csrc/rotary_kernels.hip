// Rotary positions: each pair of channels turned by position * frequency, or (the gradient) turned back.
//     y1 = f (x1 cos - x2 sin),  y2 = f (x1 sin + x2 cos)
// The angle is taken as turns, position * frequency / 2 pi, in fp64, with what the two products round away added to what is left of a whole turn:
// 2^-26 of a turn up to 2^80 (in fp64 alone a position of 2^31 at a radian each leaves 2^-22 radians, in fp32 one of 2^20 2^-4). Only what is
// left of a quarter goes on in fp32. sine and cosine are the Taylor series on an eighth of a turn to each side of the next quarter, off by less than
// 2^-23 (9.2e-8 over four million angles on the host).
//
// A workgroup has 64 pieces, eight pairs of one token each: its four waves compute a quarter of the angles each, which go through LDS,
// and then take every fourth head. Bound by memory: two bytes of each channel in and two out.
// 48 heads of 119 056 tokens along three axes 528 us (2.93 GB, 5.5 TB/s); a token of 32 sequences, 40 heads, 3.4 us.
#include <type_traits>

#include "serve_common.hpp"

namespace rsa {
namespace {

// cos and sin of pos * freq. (No contraction: a product that goes into a multiply-add brings along what `rest` adds.)
__device__ __forceinline__ void turn(double pos, double freq, float& co, float& si) {
#pragma clang fp contract(off)
  constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;      // 1 / 2 pi in two parts
  const double angle = pos * freq, angle_rest = fma(pos, freq, -angle);
  const double turns = angle * kTurn, rest = fma(angle, kTurn, -turns) + fma(angle, kTurnRest, angle_rest * kTurn);
  const double f = (turns - rint(turns)) + rest, q = rint(4. * f);
  const float y = (float)(fma(-0.25, q, f) * 6.283185307179586), z = y * y;      // |y| <= pi / 4
  const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int k = (int)q & 3;                        // quarters
  co = k & 1 ? s : c;
  si = k & 1 ? c : s;
  if (k == 1 || k == 2) co = -co;
  if (k >= 2) si = -si;
}

// Where a thread's pairs are: kHalf: pairs 8 u .. of (channel j, channel pairs + j), pairs a multiple of 8; kInterleaved: channels 16 u ..
// 16 u + 15; kOdd: as kHalf for any number of pairs, 16 bytes at a time from any channel on. There the last piece, if it is not a whole one, takes
// the eight pairs (or copied channels) up to the end and stores only its own, so that no thread reads what another writes and uses it.
// 24 + 24 heads of 119 056 tokens, 55 pairs of 128 channels: 873 us (element by element 3354; 56 pairs 544).
enum Form { kHalf, kInterleaved, kOdd };

// (the compiler takes pointers that are chosen by an index for generic ones otherwise)
typedef __attribute__((address_space(1))) const uint16_t* In;
typedef __attribute__((address_space(1))) uint16_t* Out;
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
// Vectors at addresses of whole channels.
typedef uintx4 __attribute__((aligned(2))) uintx4_any;
typedef uintx2 __attribute__((aligned(2))) uintx2_any;
typedef uint32_t __attribute__((aligned(2))) uint_any;

__device__ __forceinline__ uintx4 load8(In src) {
  return *(const __attribute__((address_space(1))) uintx4_any*)src;
}
// The last n channels of eight.
__device__ __forceinline__ void store_last(Out dst, const uintx4& v, int n) {
  if (n == 8) *(__attribute__((address_space(1))) uintx4_any*)dst = v;
  if (n & 4) *(__attribute__((address_space(1))) uintx2_any*)(dst + 4) = uintx2{v[2], v[3]};
  if (n & 2) *(__attribute__((address_space(1))) uint_any*)(dst + (n & 4 ? 2 : 6)) = n & 4 ? v[1] : v[3];
  if (n & 1) dst[8 - n] = (uint16_t)((n == 7 ? v[0] : n == 5 ? v[1] : n == 3 ? v[2] : v[3]) >> 16);    // channel 1, 3, 5, 7
}

// HEADS: heads of a wave that are in flight together. 48 heads of 119 056 tokens: 4, 6, 8, 12 at once 583, 564, 550, 528 us (5.5 TB/s); 24 of 6231
// tokens of 64 channels, in two groups: 2, 4, 12 at once 7.0, 6.9, 8.6 (the registers of twelve cost more than they bring there).
template <Form F, int HEADS>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int units, int heads_per) {
  __shared__ float2 cs[8][64];
  const int turning = (a.pairs + 7) / 8;           // units that turn; behind them 16 channels each are copied
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t id = (int64_t)blockIdx.x * 64 + lane;
  const int64_t row = id / units;
  const int u = (int)(id % units);
  const int b = (int)(row / a.t), i = (int)(row % a.t);
  // its first pair; kOdd: of the last eight, if there are so many
  const int j0 = F == kOdd && a.pairs >= 8 ? min(8 * u, a.pairs - 8) : 8 * u;
  const bool is = row < (int64_t)a.batch * a.t && !(a.count && i >= a.count[b]);
  if (is && u < turning) {
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int e = 2 * wave + z, j = j0 + e;
      float co = 1.f, si = 0.f;
      if (j < a.pairs) {
        double pos = (double)(a.start ? a.start[b] : 0) + i;
        if (a.positions) {
          const int axis = (j >= a.ends[0]) + (j >= a.ends[1]);
          pos = a.positions[((int64_t)axis * a.batch + b) * a.t + i];
        }
        turn(pos, a.freq[j], co, si);
        co *= a.factor;
        si *= a.inverse ? -a.factor : a.factor;
      }
      cs[e][lane] = make_float2(co, si);
    }
  }
  __syncthreads();
  if (!is) return;
  float co[8], si[8];
  if (u < turning) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 z = cs[e][lane];
      co[e] = z.x;
      si[e] = z.y;
    }
  }
  const int h1 = min((int)(blockIdx.y + 1) * heads_per, a.x[0].heads + a.x[1].heads);
  // two chunks of eight channels, of which the last n0 and n1 are the thread's own
  int c0, c1, n0 = 8, n1 = 8;
  if (F == kInterleaved) {
    c0 = 16 * u;
    c1 = c0 + 8;
  } else if (u < turning) {
    c0 = j0;
    c1 = a.pairs + j0;
    if (F == kOdd) n0 = n1 = min(a.pairs - 8 * u, 8);
  } else {
    c0 = 2 * a.pairs + (u - turning) * 16;
    c1 = c0 + 8;
    if (F == kOdd) {
      n0 = min(a.head_dim - c0, 8);
      n1 = min(a.head_dim - c1, 8);
      c0 = min(c0, a.head_dim - 8);
      c1 = n1 > 0 ? min(c1, a.head_dim - 8) : a.head_dim;
    }
  }
  const bool both = c1 < a.head_dim;
  auto place = [&](int h, In& in, Out& out) __attribute__((always_inline)) {
    const bool second = h >= a.x[0].heads;
    const RotaryArgs::Rows& x = a.x[second];
    const int64_t at = (int64_t)b * x.sb + (int64_t)(second ? h - a.x[0].heads : h) * x.sh + (int64_t)i * x.st;
    in = (In)x.in + at;
    out = (Out)x.out + at;
  };
  if (F == kOdd && a.pairs < 8 && u < turning) {   // fewer than eight pairs: one by one
    for (int h = blockIdx.y * heads_per + wave; h < h1; h += 4) {
      In in;
      Out out;
      place(h, in, out);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < a.pairs) {
          const float p = bf16_bits_to_float(in[e]), q = bf16_bits_to_float(in[a.pairs + e]);
          out[e] = to_bf16_bits(p * co[e] - q * si[e]);
          out[a.pairs + e] = to_bf16_bits(p * si[e] + q * co[e]);
        }
    }
    return;
  }
  for (int first = blockIdx.y * heads_per + wave; first < h1; first += 4 * HEADS) {
    uintx4 v[HEADS], w[HEADS];
    Out out[HEADS];
    bool skip[HEADS];
#pragma unroll
    for (int z = 0; z < HEADS; ++z) {
      skip[z] = first + 4 * z >= h1;
      if (skip[z]) continue;
      In in;
      place(first + 4 * z, in, out[z]);
      skip[z] = u >= turning && in == out[z];
      w[z] = uintx4{0, 0, 0, 0};
      if (F == kOdd) {
        v[z] = load8(in + c0);
        if (both) w[z] = load8(in + c1);
      } else {
        v[z] = *(const __attribute__((address_space(1))) uintx4*)(in + c0);
        if (both) w[z] = *(const __attribute__((address_space(1))) uintx4*)(in + c1);
      }
    }
#pragma unroll
    for (int z = 0; z < HEADS; ++z) {
      if (skip[z]) continue;
      if (u < turning) {
        uint32_t p[4] = {v[z][0], v[z][1], v[z][2], v[z][3]}, q[4] = {w[z][0], w[z][1], w[z][2], w[z][3]};
        if (F != kInterleaved) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p0 = bf16_bits_to_float(p[e] & 0xffffu), p1 = __builtin_bit_cast(float, p[e] & 0xffff0000u);
            const float q0 = bf16_bits_to_float(q[e] & 0xffffu), q1 = __builtin_bit_cast(float, q[e] & 0xffff0000u);
            p[e] = pack_bf16x2(p0 * co[2 * e] - q0 * si[2 * e], p1 * co[2 * e + 1] - q1 * si[2 * e + 1]);
            q[e] = pack_bf16x2(p0 * si[2 * e] + q0 * co[2 * e], p1 * si[2 * e + 1] + q1 * co[2 * e + 1]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            uint32_t& x = e < 4 ? p[e] : q[e - 4];
            const float z0 = bf16_bits_to_float(x & 0xffffu), z1 = __builtin_bit_cast(float, x & 0xffff0000u);
            const uint32_t y = pack_bf16x2(z0 * co[e] - z1 * si[e], z0 * si[e] + z1 * co[e]);
            x = 8 * u + e < a.pairs ? y : x;       // (a channel behind the pairs is no product: 0 * infinity)
          }
        }
        v[z] = uintx4{p[0], p[1], p[2], p[3]};
        w[z] = uintx4{q[0], q[1], q[2], q[3]};
      }
      if (F == kOdd) {
        store_last(out[z] + c0, v[z], n0);
        if (both) store_last(out[z] + c1, w[z], n1);
      } else {
        *(__attribute__((address_space(1))) uintx4*)(out[z] + c0) = v[z];
        if (both) *(__attribute__((address_space(1))) uintx4*)(out[z] + c1) = w[z];
      }
    }
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s) {
  const int turning = (a.pairs + 7) / 8, rest = a.head_dim - 2 * a.pairs;
  const int units = a.interleaved ? (a.head_dim + 15) / 16 : turning + (rest + 15) / 16;
  const int64_t pieces = ((int64_t)a.batch * a.t * units + 63) / 64;
  const int heads = a.x[0].heads + a.x[1].heads;
  // Heads are shared out over workgroups too where there would be few: two to a compute unit (four: 6.9 us for the 6231 tokens, two 6.8, eight 7.7).
  int64_t groups = (512 + pieces - 1) / pieces;
  const int64_t most = (heads + 3) / 4;
  groups = groups > most ? most : groups;
  const int per = (int)((most + groups - 1) / groups * 4);
  const dim3 grid((uint32_t)pieces, (uint32_t)((heads + per - 1) / per));
  const int of_wave = per / 4;
  const dim3 block(256);
  auto launch = [&](auto form) {
    constexpr Form F = decltype(form)::value;
    if (of_wave <= 4) hipLaunchKernelGGL((rotary_kernel<F, 4>), grid, block, 0, s, a, units, per);
    else if (of_wave <= 8) hipLaunchKernelGGL((rotary_kernel<F, 8>), grid, block, 0, s, a, units, per);
    else hipLaunchKernelGGL((rotary_kernel<F, 12>), grid, block, 0, s, a, units, per);
  };
  if (a.interleaved) launch(std::integral_constant<Form, kInterleaved>{});
  else if (a.pairs % 8 == 0) launch(std::integral_constant<Form, kHalf>{});
  else launch(std::integral_constant<Form, kOdd>{});
  return hipGetLastError();
}

}  // namespace rsa
