// Rotary positions: each pair of channels turned by position * frequency, or (the gradient) turned back.
//     y1 = f (x1 cos - x2 sin),  y2 = f (x1 sin + x2 cos)
// The angle is taken in fp64 as turns, position * frequency / 2 pi, and only what is left of a whole turn goes on in fp32: far
// positions lose nothing (in fp32 a position of 2^20 leaves 2^-4 radians). sine and cosine are the Taylor series on an eighth of a turn
// to each side of the next quarter, off by less than 2^-23.
//
// A thread has eight pairs of one token, so that the angles are computed once, and walks a run of heads with them. Bound by memory:
// two bytes of each channel in and two out.
#include "serve_common.hpp"

namespace rsa {
namespace {

// cos and sin of 2 pi * turns.
__device__ __forceinline__ void turn(double turns, float& co, float& si) {
  const float f = (float)(turns - rint(turns));    // [-1/2, 1/2]
  const float q = rintf(4.f * f);
  const float y = (f - 0.25f * q) * 6.283185307179586f, z = y * y;      // |y| <= pi / 4; the difference is exact
  const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int k = (int)q & 3;                        // quarters
  co = k & 1 ? s : c;
  si = k & 1 ? c : s;
  if (k == 1 || k == 2) co = -co;
  if (k >= 2) si = -si;
}

// Where a thread's pairs are: kHalf: pairs 8 u .. of (channel j, channel pairs + j), pairs a multiple of 8; kInterleaved: channels 16 u ..
// 16 u + 15; kOdd: as kHalf for any number of pairs, element by element.
enum Form { kHalf, kInterleaved, kOdd };

template <Form F>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int units, int heads_per) {
  const int turning = (a.pairs + 7) / 8;           // units that turn; behind them 16 channels each are copied
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = id / units;
  const int u = (int)(id % units);
  if (row >= (int64_t)a.batch * a.t) return;
  const int b = (int)(row / a.t), i = (int)(row % a.t);
  if (a.count && i >= a.count[b]) return;
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, a.x[0].heads + a.x[1].heads);

  float co[8], si[8];
  if (u < turning) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = 8 * u + e;
      co[e] = 1.f;
      si[e] = 0.f;
      if (j < a.pairs) {
        double pos = (double)(a.start ? a.start[b] : 0) + i;
        if (a.positions) {
          const int axis = (j >= a.ends[0]) + (j >= a.ends[1]);
          pos = a.positions[((int64_t)axis * a.batch + b) * a.t + i];
        }
        turn(pos * a.freq[j] * 0.15915494309189535, co[e], si[e]);
        co[e] *= a.factor;
        si[e] *= a.inverse ? -a.factor : a.factor;
      }
    }
  }
  for (int h = h0; h < h1; ++h) {
    const bool second = h >= a.x[0].heads;
    const RotaryArgs::Rows& x = a.x[second];
    const int64_t at = (int64_t)b * x.sb + (int64_t)(second ? h - a.x[0].heads : h) * x.sh + (int64_t)i * x.st;
    const uint16_t* in = x.in + at;
    uint16_t* out = x.out + at;
    if (u >= turning && in == out) continue;
    if (F == kOdd) {
      if (u < turning) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = 8 * u + e;
          if (j < a.pairs) {
            const float p = bf16_bits_to_float(in[j]), q = bf16_bits_to_float(in[a.pairs + j]);
            out[j] = to_bf16_bits(p * co[e] - q * si[e]);
            out[a.pairs + j] = to_bf16_bits(p * si[e] + q * co[e]);
          }
        }
      } else {
        for (int ch = 2 * a.pairs + (u - turning) * 16, n = 0; n < 16 && ch < a.head_dim; ++n, ++ch) out[ch] = in[ch];
      }
      continue;
    }
    // two chunks of eight channels
    int c0, c1;
    if (F == kInterleaved) {
      c0 = 16 * u;
      c1 = c0 + 8;
    } else if (u < turning) {
      c0 = 8 * u;
      c1 = a.pairs + 8 * u;
    } else {
      c0 = 2 * a.pairs + (u - turning) * 16;
      c1 = c0 + 8;
    }
    const bool both = c1 < a.head_dim;
    uint4 v = *reinterpret_cast<const uint4*>(in + c0), w = make_uint4(0, 0, 0, 0);
    if (both) w = *reinterpret_cast<const uint4*>(in + c1);
    if (u < turning) {
      uint32_t p[4] = {v.x, v.y, v.z, v.w}, q[4] = {w.x, w.y, w.z, w.w};
      if (F == kHalf) {
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
          uint32_t& z = e < 4 ? p[e] : q[e - 4];
          const float z0 = bf16_bits_to_float(z & 0xffffu), z1 = __builtin_bit_cast(float, z & 0xffff0000u);
          const uint32_t t = pack_bf16x2(z0 * co[e] - z1 * si[e], z0 * si[e] + z1 * co[e]);
          z = 8 * u + e < a.pairs ? t : z;         // (a channel behind the pairs is no product: 0 * infinity)
        }
      }
      v = make_uint4(p[0], p[1], p[2], p[3]);
      w = make_uint4(q[0], q[1], q[2], q[3]);
    }
    *reinterpret_cast<uint4*>(out + c0) = v;
    if (both) *reinterpret_cast<uint4*>(out + c1) = w;
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s) {
  const int turning = (a.pairs + 7) / 8, rest = a.head_dim - 2 * a.pairs;
  const int units = a.interleaved ? (a.head_dim + 15) / 16 : turning + (rest + 15) / 16;
  const int64_t threads = (int64_t)a.batch * a.t * units;
  const int heads = a.x[0].heads + a.x[1].heads;
  // workgroups for every compute unit several times over, and as many heads to a thread as that leaves
  const int64_t wgs = (threads + 255) / 256;
  int64_t per = heads * wgs / 4096;
  per = per < 1 ? 1 : per > heads ? heads : per;
  const dim3 grid((uint32_t)wgs, (uint32_t)((heads + per - 1) / per));
  if (a.interleaved) hipLaunchKernelGGL(rotary_kernel<kInterleaved>, grid, dim3(256), 0, s, a, units, (int)per);
  else if (a.pairs % 8 == 0) hipLaunchKernelGGL(rotary_kernel<kHalf>, grid, dim3(256), 0, s, a, units, (int)per);
  else hipLaunchKernelGGL(rotary_kernel<kOdd>, grid, dim3(256), 0, s, a, units, (int)per);
  return hipGetLastError();
}

}  // namespace rsa
