// Attention of new queries over the 8-bit key/value cache, over all blocks or over listed ones.
//
// A tile is 16 QT query rows of one (sequence, key/value head): rows are (token, query head of the key/value head), token
// by token, so that one pass over the keys serves all heads that share them. Each wave computes, with 16x16x32 products,
//     S^T = K Q^T      (M = key, N = query, k = channel; e4m3 -> bf16, exact)
//     O^T += V^T P^T   (M = channel, N = query, k = key; e4m3 -> fp16, exact)
// with the softmax between them lane-local: codes lie in the page in operand order (cache_common.hpp), so the loop needs
// neither LDS nor a barrier; the codes go from memory into the registers that the products read. The scale of a block's
// keys goes into the scores, that of its values into the exponent of P (below).
//
// P is rounded to fp16 (11 bits; V has 4): half a step is 2^-11 of p, against the output's own 2^-8 in bf16. Range: the
// running reference m of a row follows its maximum lazily (only when a score passes it by more than 8 in log2), so p <= 2^8. A
// row's O is held over 2^eo; where eo is up to kAbove below the exponent ev of a block's values, P takes 2^(ev - eo) with it: at
// most 2^15, and never less than p, so that a weight of 2^-14 keeps its 11 bits beside a block of larger values too (of 2^-21 where
// no block's are larger). Its sum gives the sum of the weights back exactly. Other blocks move eo first (follow_values), as far as
// O keeps all of its bits; what is then still outside (a block that is nothing beside the row's O, or whose weights are) is summed apart.
//
// The four waves of a workgroup take every fourth step of 64 keys and are joined in LDS; where there are few tiles the key
// axis is also split over workgroups, whose normalised parts (fp32) cache_join_kernel adds in a fixed order.
// Bound by memory: one token of 32 sequences of up to 32 768 tokens (8 heads of 128) 241 us at 5.7 TB/s, of one of 237 600 (24 heads)
// 246 us at 5.9, from lists of 64 blocks (268 MB) 52 us at 5.1; reading 1.46 GB in long pieces makes 6.1, a copy of 1 GiB 5.2.
#include "cache_attn_common.hpp"

namespace rsa {
namespace {

constexpr int kAbove = 7;
// Sixteen codes as the bf16 / fp16 operands of two products (bytes 0-7 and 8-15).
__device__ __forceinline__ void widen(const uint4& v, bf16x8 (&o)[2]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true);
    o[i / 2][i % 2 * 4 + 0] = lo[0]; o[i / 2][i % 2 * 4 + 1] = lo[1];
    o[i / 2][i % 2 * 4 + 2] = hi[0]; o[i / 2][i % 2 * 4 + 3] = hi[1];
  }
}
__device__ __forceinline__ void widen(const uint4& v, halfx8 (&o)[2]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const halfx2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false);
    const halfx2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true);
    o[i / 2][i % 2 * 4 + 0] = lo[0]; o[i / 2][i % 2 * 4 + 1] = lo[1];
    o[i / 2][i % 2 * 4 + 2] = hi[0]; o[i / 2][i % 2 * 4 + 3] = hi[1];
  }
}
// 0xff in every byte that holds the code of NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t top = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (top >> 7) * 255u;
}

// o * f * 2^e.
__device__ __forceinline__ floatx4 scaled(const floatx4& o, float f, int e) {
  floatx4 z;
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = ldexpf(o[i] * f, e);
  return z;
}
// No block was seen yet: the first decides, there is nothing to move.
constexpr int kNoScale = -512;
template <int QT>
__device__ __forceinline__ void begin_values(int ev, int (&eo)[QT], int& lo, int& hi) {
  if (lo != kNoScale) return;
  lo = hi = ev - kAbove;
#pragma unroll
  for (int x = 0; x < QT; ++x) eo[x] = lo;
}
// A block with values over 2^ev is outside some column's window: each column's eo goes to ev - kAbove, but only so far that its largest |o| stays
// within 2^-90 .. 2^100 (no bit of it is lost, and what the keys still add is at most 2^55), and then as far up as the block's own
// weights, the largest of them 2^(most - m), ask for. The columns' lowest and highest eo are left in lo and hi, the same in every lane.
// Rare: scales of 2^3 apart cost nothing; a frame on 20 280 keys with every second block 2^10 times larger takes 490 us instead of 383.
template <int QT, int VC>
__device__ __forceinline__ void follow_values(int ev, const float (&most)[QT], const float (&m)[QT], int (&eo)[QT], floatx4 (&o)[QT][VC], int& lo, int& hi) {
  uint32_t low = 0, high = 0;                      // eo < 512
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    float big = 0.f, top = most[x];
#pragma unroll
    for (int v = 0; v < VC; ++v)
#pragma unroll
      for (int e = 0; e < 4; ++e) big = fmaxf(big, fabsf(o[x][v][e]));
    big = __builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, big), MaxF32()), MaxF32()));
    top = __builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, top), MaxF32()), MaxF32()));
    const int aim = ev - kAbove;
    int to = aim;
    if (big > 0.f) {
      const int at = exponent_of(big), weight = fabsf(m[x]) < kWhole ? (int)ceilf(fminf(fmaxf(top - m[x], -1000.f), 0.f)) : 0;
      to = max(min(max(aim, eo[x] - max(100 - at, 0)), eo[x] + max(at + 90, 0)), aim + weight);
    }
#pragma unroll
    for (int v = 0; v < VC; ++v)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[x][v][e] = ldexpf(o[x][v][e], eo[x] - to);
    eo[x] = to;
    low = max(low, (uint32_t)(512 - to));
    high = max(high, (uint32_t)(512 + to));
  }
  lo = 512 - __builtin_amdgcn_readfirstlane(over_row((int)low, MaxU32()));
  hi = __builtin_amdgcn_readfirstlane(over_row((int)high, MaxU32())) - 512;
}

// One run of 16 value codes of a lane (channel tile v): where NaN stands under a key that a column sees (the first left[x] of
// the 64), the column's output becomes NaN.
template <int QT, int VC>
__device__ __forceinline__ void mark_nan(const uint4& w, const int (&left)[QT], int g, int v, floatx4 (&o)[QT][VC]) {
  halfx8 is[2];                                    // 1.0 for a NaN
  widen(make_uint4(nan_bytes(w.x) & 0x38383838u, nan_bytes(w.y) & 0x38383838u, nan_bytes(w.z) & 0x38383838u, nan_bytes(w.w) & 0x38383838u), is);
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    halfx8 see[2];
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e) see[y / 2][y % 2 * 4 + e] = 16 * y + 4 * g + e < left[x] ? (_Float16)1.f : (_Float16)0.f;
    floatx4 hit = {0.f, 0.f, 0.f, 0.f};
    hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(is[0], see[0], hit, 0, 0, 0);
    hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(is[1], see[1], hit, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (hit[e] > 0.f) o[x][v][e] = __builtin_nanf("");
  }
}

template <int D, int BLK, int QT>
__global__ __launch_bounds__(256, QT == 1 ? 2 : 1) void cache_attn_kernel(CacheDims c, RowDims r, CacheAttnArgs a, TileGrid tg) {
  constexpr int KC = D / 64, VC = D / 16;          // 16-byte loads of a lane for 16 keys / for 64 keys
  constexpr int SPB = BLK / 64;                    // steps of 64 keys in a block
  constexpr int PITCH = D + 4;                     // floats of a row in the joining buffer
  __shared__ __align__(16) float join[4][16][PITCH];
  __shared__ float join_m[4][16], join_l[4][16];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int g = lane / 16, n = lane % 16;
  const int split = blockIdx.x % tg.splits;
  const int64_t id = blockIdx.x / tg.splits;
  const Tile t = tile_of(c, r, a, tg, id);
  const int G = r.heads / c.heads_kv;

  // queries of this lane's columns, as operands, and how many keys each sees
  bf16x8 q[QT][2 * KC];
  int seen[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int row = t.row0 + 16 * x + n, tok = t.t0 + row / G;
    const bool is = row < t.rows && tok < t.ql;
    seen[x] = !is ? 0 : visible_keys(c, a, t, tok);
    const uint16_t* src = a.Q + (int64_t)t.b * r.sb + (int64_t)(t.hk * G + row % G) * r.sh + (int64_t)tok * r.st;
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (is) v = *reinterpret_cast<const uint4*>(src + k * 64 + g * 16 + hf * 8);
        q[x][2 * k + hf] = __builtin_bit_cast(bf16x8, v);
      }
  }
  floatx4 o[QT][VC];
  float m[QT], l[QT], lazy = kLazy;
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    m[x] = kNoReference;
    l[x] = 0.f;
#pragma unroll
    for (int v = 0; v < VC; ++v) o[x][v] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  int eo[QT], lo = kNoScale, hi = kNoScale;                // o is held over 2^eo; the lowest and the highest of the wave's columns
#pragma unroll
  for (int x = 0; x < QT; ++x) eo[x] = kNoScale;

  const int u0 = (int)((int64_t)t.units * split / tg.splits), u1 = (int)((int64_t)t.units * (split + 1) / tg.splits);
  const int steps = (u1 - u0) * SPB;
  // this wave's steps are wave, wave + 4, ...; lane i looks up the i-th of the next 64
  for (int base = wave; base < steps; base += 256) {
    int my_blk = -1, my_page = -1;
    float my_k = 0.f, my_v = 0.f;
    const int my_step = base + lane * 4;
    if (my_step < steps) {
      my_blk = u0 + my_step / SPB;
      if (a.block_idx) my_blk = a.block_idx[(int64_t)t.lrow * a.list_len + my_blk];
      if (my_blk < t.blocks) my_page = cache_page(c, t.b, my_blk);
      if (my_page >= 0) {
        const float2 sc = *reinterpret_cast<const float2*>(c.scales + ((int64_t)my_page * c.heads_kv + t.hk) * 4);
        my_k = sc.x;
        my_v = sc.y;
      }
    }
    unsigned long long todo = __ballot(my_page >= 0);
    uint4 kc[4 * KC], vc[VC];
    auto load_k = [&](int i) __attribute__((always_inline)) {
      const int64_t rec = (int64_t)__builtin_amdgcn_readlane(my_page, i) * c.heads_kv + t.hk;
      const uint8_t* p = c.k + rec * (BLK * D) + ((base + i * 4) % SPB) * (64 * D) + lane * 16;
#pragma unroll
      for (int x = 0; x < 4 * KC; ++x) kc[x] = *reinterpret_cast<const uint4*>(p + x * 1024);
    };
    auto load_v = [&](int i) __attribute__((always_inline)) {
      const int64_t rec = (int64_t)__builtin_amdgcn_readlane(my_page, i) * c.heads_kv + t.hk;
      const uint8_t* p = c.v + rec * (BLK * D) + ((base + i * 4) % SPB) * (64 * D) + lane * 16;
#pragma unroll
      for (int x = 0; x < VC; ++x) vc[x] = *reinterpret_cast<const uint4*>(p + x * 1024);
    };
    int i = todo ? __builtin_ctzll(todo) : -1;
    if (i >= 0) {
      load_k(i);
      load_v(i);
      begin_values<QT>(exponent_of(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_v), i))), eo, lo, hi);
    }
    while (i >= 0) {
      todo &= todo - 1;
      const int next = todo ? __builtin_ctzll(todo) : -1;
      const int key0 = __builtin_amdgcn_readlane(my_blk, i) * BLK + ((base + i * 4) % SPB) * 64;
      const float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_k), i)) * a.scale_log2e;
      const int ev = exponent_of(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_v), i)));

      floatx4 s[QT][4];
#pragma unroll
      for (int x = 0; x < QT; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) s[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          bf16x8 op[2];
          widen(kc[y * KC + k], op);
#pragma unroll
          for (int x = 0; x < QT; ++x) {
            s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[0], q[x][2 * k], s[x][y], 0, 0, 0);
            s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[1], q[x][2 * k + 1], s[x][y], 0, 0, 0);
          }
        }
      if (next >= 0) load_k(next);

      // scores; keys that a row does not see leave its softmax
      const bool partly = key0 + 64 > t.lo_seen;
      bool over = false;
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const int left = seen[x] - key0;             // of the 64
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float z = s[x][y][e] * ks;
            if (partly) z = 16 * y + 4 * g + e < left ? z : -INFINITY;
            s[x][y][e] = z;
            over |= z > m[x] + lazy;
          }
      }
      if (__any(over)) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          float mx = kNoReference;
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[x][y][e]);
          mx = __builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, mx), MaxF32()), MaxF32()));
          if (mx > m[x] + lazy) {                  // the same in the four lanes of a column
            mx = floorf(mx);                       // (whole, so that what is taken from it and what it rescales stays exact)
            const float down = exp2f(m[x] - mx);
            m[x] = mx;
            l[x] *= down;
#pragma unroll
            for (int v = 0; v < VC; ++v) o[x][v] *= down;
          }
        }
        if (far_from_zero<QT>(m)) lazy = 0.f;
      }
      bool apart = false;
      if (ev < hi || ev > lo + kAbove) {
        float most[QT];
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          most[x] = -INFINITY;
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) most[x] = fmaxf(most[x], s[x][y][e]);
        }
        follow_values<QT, VC>(ev, most, m, eo, o, lo, hi);
        apart = ev < hi || ev > lo + kAbove;
        if (apart) {
#pragma unroll
          for (int x = 0; x < QT; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
              for (int e = 0; e < 4; ++e) l[x] += __builtin_amdgcn_exp2f(s[x][y][e] - m[x]);
        }
      }
      halfx8 p[QT][2];
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const int back = eo[x] - ev;               // P takes 2^(ev - eo) with it, so that it goes with o
        const float ref = m[x] + (float)back;
        float sum = 0.f;
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float w = __builtin_amdgcn_exp2f(s[x][y][e] - ref);
            sum += w;
            p[x][y / 2][y % 2 * 4 + e] = (_Float16)w;
          }
        l[x] += apart ? 0.f : ldexpf(sum, back);
      }

      // a value that is NaN under a key that a row does not see must not reach it through 0 * NaN
      bool odd = false;
      if (partly) {
        uint32_t bad = 0;
#pragma unroll
        for (int v = 0; v < VC; ++v) bad |= nan_bytes(vc[v].x) | nan_bytes(vc[v].y) | nan_bytes(vc[v].z) | nan_bytes(vc[v].w);
        odd = __any(bad != 0);
      }
      if (odd) {
        int left[QT];
#pragma unroll
        for (int x = 0; x < QT; ++x) left[x] = seen[x] - key0;
#pragma unroll
        for (int v = 0; v < VC; ++v) {
          const uint4 w = vc[v];
          mark_nan<QT, VC>(w, left, g, v, o);
          vc[v] = make_uint4(w.x & ~nan_bytes(w.x), w.y & ~nan_bytes(w.y), w.z & ~nan_bytes(w.z), w.w & ~nan_bytes(w.w));
        }
      }
#pragma unroll
      for (int v = 0; v < VC; ++v) {
        halfx8 op[2];
        widen(vc[v], op);
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          o[x][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op[0], p[x][0], o[x][v], 0, 0, 0);
          o[x][v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op[1], p[x][1], o[x][v], 0, 0, 0);
        }
      }
      if (next >= 0) load_v(next);
      i = next;
    }
  }

  // join the four waves, 16 rows at a time
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const float sum = __builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, l[x]), AddF32()), AddF32()));
    if (x > 0) __syncthreads();
    if (g == 0) {
      join_m[wave][n] = m[x];
      join_l[wave][n] = sum;
    }
    __syncthreads();
    float most = join_m[0][n];
#pragma unroll
    for (int w = 1; w < 4; ++w) most = fmaxf(most, join_m[w][n]);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) total += join_l[w][n] * exp2f(join_m[w][n] - most);
    const float f = total == 0.f ? 0.f : exp2f(m[x] - most) / total;
#pragma unroll
    for (int v = 0; v < VC; ++v) *reinterpret_cast<floatx4*>(&join[wave][n][16 * v + 4 * g]) = scaled(o[x][v], f, eo[x]);
    __syncthreads();
    constexpr int CPR = D / 8;
    for (int u = tid; u < 16 * CPR; u += 256) {
      const int rr = u / CPR, ch = u % CPR * 8, row = t.row0 + 16 * x + rr, tok = t.t0 + row / G;
      if (row >= t.rows || tok >= t.ql) continue;
      float z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = (join[0][rr][ch + e] + join[1][rr][ch + e]) + (join[2][rr][ch + e] + join[3][rr][ch + e]);
      if (tg.splits == 1) {
        uint4 v = make_uint4(pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3]), pack_bf16x2(z[4], z[5]), pack_bf16x2(z[6], z[7]));
        *reinterpret_cast<uint4*>(a.O + (int64_t)t.b * r.sb + (int64_t)(t.hk * G + row % G) * r.sh + (int64_t)tok * r.st + ch) = v;
      } else {
        float* dst = a.parts + ((int64_t)blockIdx.x * tg.stored + 16 * x + rr) * D + ch;
        *reinterpret_cast<float4*>(dst) = make_float4(z[0], z[1], z[2], z[3]);
        *reinterpret_cast<float4*>(dst + 4) = make_float4(z[4], z[5], z[6], z[7]);
      }
    }
    const int row = t.row0 + 16 * x + n, tok = t.t0 + row / G;
    if (tid < 16 && row < t.rows && tok < t.ql) {
      const float lse2 = total == 0.f ? -INFINITY : most + log2f(total);
      if (tg.splits > 1) (a.parts + (int64_t)gridDim.x * tg.stored * D)[(int64_t)blockIdx.x * tg.stored + 16 * x + n] = lse2;
      else if (a.lse) a.lse[((int64_t)t.b * r.heads + t.hk * G + row % G) * r.t + tok] = lse2 * kLn2;
    }
  }
}

// The same for many query rows, bound by the matrix pipe and the vector ALU beside it. 64 QT rows to a workgroup, 16 QT to
// a wave: every wave needs all codes, so they are widened once for the workgroup, a quarter by each wave, into LDS in the
// order of the operands (each 1 KB that a wave reads is lanes times 16 bytes: no conflicts, no address work). Two buffers, one
// barrier a step of 64 keys: while a step is computed the codes of the next are widened and those of the one after are on
// their way. 64 KB of LDS at d = 128, so that two workgroups share a compute unit and the softmax of one can run beside the
// products of the other. 1560 queries of 24 heads over 20 280 keys: 382 us, 1020 TFLOP/s; the matrix pipe is busy 45 % of the time, the
// vector ALU 53 and LDS 42. Codes are widened and written between the softmax and the values' products, and operands read four ahead of their
// products (when that was chosen, on a slower box: 393 us; widened in front of the scores 427, behind the values' products 411; eight ahead 396).
constexpr int kAhead = 256;                        // steps that are looked up together
template <int D, int BLK, int QT>
__global__ __launch_bounds__(256, 2) void cache_tile_kernel(CacheDims c, RowDims r, CacheAttnArgs a, TileGrid tg) {
  constexpr int KC = D / 64, VC = D / 16, VW = VC / 4;   // VW: 1 KB pieces of values that a wave widens (of keys: KC)
  constexpr int SPB = BLK / 64;
  constexpr int KBYTES = 4 * KC * 2048, BYTES = KBYTES + VC * 2048;       // of a buffer: keys, then values
  __shared__ __align__(16) uint8_t lds_k[2][KBYTES], lds_v[2][BYTES - KBYTES];
  __shared__ int4 look[kAhead];                    // page, first key, scale of the keys, scale of the values
  __shared__ __align__(16) int odd[2][4];
  __shared__ int n_valid[4];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int g = lane / 16, n = lane % 16;
  // tiles of one key/value head that walk the same part of the keys follow one another on an XCD
  const int inner = tg.per_group * a.groups;
  const int id = xcd_run(blockIdx.x, gridDim.x);
  const int split = id / inner % tg.splits;
  const int64_t tile = (int64_t)(id / inner / tg.splits) * inner + (tg.last_first ? inner - 1 - id % inner : id % inner);
  const Tile t = tile_of(c, r, a, tg, tile);
  const int G = r.heads / c.heads_kv;

  bf16x8 q[QT][2 * KC];
  int seen[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int row = t.row0 + (wave * QT + x) * 16 + n, tok = t.t0 + row / G;
    const bool is = row < t.rows && tok < t.ql;
    seen[x] = !is ? 0 : visible_keys(c, a, t, tok);
    const uint16_t* src = a.Q + (int64_t)t.b * r.sb + (int64_t)(t.hk * G + row % G) * r.sh + (int64_t)tok * r.st;
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (is) v = *reinterpret_cast<const uint4*>(src + k * 64 + g * 16 + hf * 8);
        q[x][2 * k + hf] = __builtin_bit_cast(bf16x8, v);
      }
  }
  // the queries are here before the loop: a wait for them inside it would be one for every load in flight
#pragma unroll
  for (int x = 0; x < QT; ++x)
#pragma unroll
    for (int k = 0; k < 2 * KC; ++k) asm volatile("" : "+v"(q[x][k]));
  floatx4 o[QT][VC];
  float m[QT], l[QT], lazy = kLazy;
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    m[x] = kNoReference;
    l[x] = 0.f;
#pragma unroll
    for (int v = 0; v < VC; ++v) o[x][v] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  int eo[QT], lo = kNoScale, hi = kNoScale;
#pragma unroll
  for (int x = 0; x < QT; ++x) eo[x] = kNoScale;

  const int u0 = (int)((int64_t)t.units * split / tg.splits), u1 = (int)((int64_t)t.units * (split + 1) / tg.splits);
  const int steps = (u1 - u0) * SPB;
  for (int base = 0; base < steps; base += kAhead) {
    // the next steps: those with a page, put together in order (one look-up for the workgroup, so that its waves walk the
    // same steps whatever happens to the table meanwhile)
    __syncthreads();
    {
      const int s = base + tid;
      int blk = -1, page = -1;
      if (s < steps) {
        blk = u0 + s / SPB;
        if (a.block_idx) blk = a.block_idx[(int64_t)t.lrow * a.list_len + blk];
        if (blk < t.blocks) page = cache_page(c, t.b, blk);
      }
      const unsigned long long all = __ballot(page >= 0);
      if (lane == 0) n_valid[wave] = __popcll(all);
      __syncthreads();
      int at = __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
      for (int w = 0; w < wave; ++w) at += n_valid[w];
      if (page >= 0) {
        const uint2 sc = *reinterpret_cast<const uint2*>(c.scales + ((int64_t)page * c.heads_kv + t.hk) * 4);
        look[at] = make_int4(page, blk * BLK + s % SPB * 64, (int)sc.x, (int)sc.y);
      }
      __syncthreads();
    }
    const int count = __builtin_amdgcn_readfirstlane(n_valid[0] + n_valid[1] + n_valid[2] + n_valid[3]);
    if (count == 0) continue;
    // what a step is, the same in every lane
    struct Step { int page, key; float ks; int ev; };
    auto entry = [&](int i) __attribute__((always_inline)) { return look[min(i, count - 1)]; };
    auto step_of = [&](const int4& v) __attribute__((always_inline)) {
      Step z;
      z.page = __builtin_amdgcn_readfirstlane(v.x);
      z.key = __builtin_amdgcn_readfirstlane(v.y);
      // (above 0, so that a masked score stays -inf)
      z.ks = fmaxf(__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(v.z)) * a.scale_log2e, 0x1p-149f);
      z.ev = exponent_of(__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(v.w)));
      return z;
    };
    uint4 raw_k[KC], raw_v[VW];
    auto request = [&](const Step& z, uint4* raw, const uint8_t* codes, int pieces) __attribute__((always_inline)) {
      const uint8_t* src = codes + ((int64_t)z.page * c.heads_kv + t.hk) * (BLK * D) + z.key % BLK * D;
#pragma unroll
      for (int x = 0; x < pieces; ++x) raw[x] = *reinterpret_cast<const uint4*>(src + ((wave * pieces + x) * 1024 + lane * 16));
    };
    // a row of the tile does not see all keys of the step: no NaN into 0 * NaN
    auto clear_nan = [&](int buf) __attribute__((always_inline)) {
      uint32_t bad = 0;
#pragma unroll
      for (int x = 0; x < VW; ++x) {
        uint4& w = raw_v[x];
        const uint4 nb = make_uint4(nan_bytes(w.x), nan_bytes(w.y), nan_bytes(w.z), nan_bytes(w.w));
        bad |= nb.x | nb.y | nb.z | nb.w;
        w = make_uint4(w.x & ~nb.x, w.y & ~nb.y, w.z & ~nb.z, w.w & ~nb.w);
      }
      const bool any = __any(bad != 0);
      if (lane == 0) odd[buf][wave] = any;
    };
    auto store_k = [&](int buf) __attribute__((always_inline)) {
      uint8_t* to = lds_k[buf] + lane * 16;
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        bf16x8 op[2];
        widen(raw_k[x], op);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) *reinterpret_cast<bf16x8*>(to + (wave * KC + x) * 2048 + hf * 1024) = op[hf];
      }
    };
    auto store_v = [&](int buf) __attribute__((always_inline)) {
      uint8_t* to = lds_v[buf] + lane * 16;
#pragma unroll
      for (int x = 0; x < VW; ++x) {
        halfx8 op[2];
        widen(raw_v[x], op);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) *reinterpret_cast<halfx8*>(to + (wave * VW + x) * 2048 + hf * 1024) = op[hf];
      }
    };
    auto scores = [&](const uint8_t* buf, floatx4 (&s)[QT][4]) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < QT; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) s[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 2 * KC; ++k)
#pragma unroll
        for (int y = 0; y < 4; ++y) {              // (a sum is touched again 4 QT products later)
          const bf16x8 op = *reinterpret_cast<const bf16x8*>(buf + (y * 2 * KC + k) * 1024);
#pragma unroll
          for (int x = 0; x < QT; ++x) s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op, q[x][k], s[x][y], 0, 0, 0);
        }
    };

    Step now = step_of(entry(0)), next = step_of(entry(1));
    begin_values<QT>(now.ev, eo, lo, hi);
    request(now, raw_k, c.k, KC);
    request(now, raw_v, c.v, VW);
    if (now.key + 64 > t.lo_seen) clear_nan(0);
    store_k(0);
    store_v(0);
    request(next, raw_k, c.k, KC);
    request(next, raw_v, c.v, VW);
    for (int i = 0; i < count; ++i) {
      __syncthreads();
      if (next.key + 64 > t.lo_seen) clear_nan((i + 1) & 1);
      const int4 ahead = entry(i + 2);
      const bool partly = now.key + 64 > t.lo_seen;
      if (partly) {
        const int4 f = *reinterpret_cast<const int4*>(odd[i & 1]);
        if (__builtin_amdgcn_readfirstlane(f.x | f.y | f.z | f.w)) {
          const int64_t at = ((int64_t)now.page * c.heads_kv + t.hk) * (BLK * D) + now.key % BLK * D + lane * 16;
          int left[QT];
#pragma unroll
          for (int x = 0; x < QT; ++x) left[x] = seen[x] - now.key;
#pragma unroll
          for (int v = 0; v < VC; ++v) mark_nan<QT, VC>(*reinterpret_cast<const uint4*>(c.v + at + v * 1024), left, g, v, o);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      floatx4 s[QT][4];
      scores(lds_k[i & 1] + lane * 16, s);
#pragma unroll
      for (int u = 0; u < 4; ++u) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
      for (int u = 0; u < 8 * KC - 4; ++u) {
        __builtin_amdgcn_sched_group_barrier(0x008, QT, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, QT * 4, 0);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      if (partly) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const int left = seen[x] - now.key;
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[x][y][e] = 16 * y + 4 * g + e < left ? s[x][y][e] : -INFINITY;
        }
      }
      float most[QT];
      bool over = false;
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        most[x] = -INFINITY;
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int e = 0; e < 4; e += 2) most[x] = fmaxf(fmaxf(most[x], s[x][y][e]), s[x][y][e + 1]);
        most[x] *= now.ks;
        over |= most[x] > m[x] + lazy;
      }
      if (__any(over)) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const float mx = __builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, most[x]), MaxF32()), MaxF32()));
          const float to = mx > m[x] + lazy ? floorf(mx) : m[x];    // the same in the four lanes of a column; whole, as above
          const float down = __builtin_amdgcn_exp2f(m[x] - to);
          m[x] = to;
          l[x] *= down;
#pragma unroll
          for (int v = 0; v < VC; ++v) o[x][v] *= down;
        }
        if (far_from_zero<QT>(m)) lazy = 0.f;
      }
      // Far from zero the multiply-add below would leave a product's own rounding, which may be 2^8 and more: rounded products, as m is one
      float ks = now.ks;
      if (__builtin_expect(lazy == 0.f, 0)) {
        ks = 1.f;
#pragma unroll
        for (int x = 0; x < QT; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) s[x][y] *= now.ks;
      }
      bool apart = false;
      if (__builtin_expect(now.ev < hi || now.ev > lo + kAbove, 0)) {
        follow_values<QT, VC>(now.ev, most, m, eo, o, lo, hi);
        apart = now.ev < hi || now.ev > lo + kAbove;
        if (apart) {
#pragma unroll
          for (int x = 0; x < QT; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
              for (int e = 0; e < 4; ++e) l[x] += __builtin_amdgcn_exp2f(fmaf(s[x][y][e], ks, -m[x]));
        }
      }
      halfx8 p[QT][2];
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const int back = eo[x] - now.ev;
        const float ref = m[x] + (float)back;
        float sum = 0.f;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          float w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] = __builtin_amdgcn_exp2f(fmaf(s[x][y][e], ks, -ref));
            sum += w[e];
          }
          const halfx2 lo2 = __builtin_convertvector(floatx2{w[0], w[1]}, halfx2), hi2 = __builtin_convertvector(floatx2{w[2], w[3]}, halfx2);
          p[x][y / 2][y % 2 * 4 + 0] = lo2[0]; p[x][y / 2][y % 2 * 4 + 1] = lo2[1];
          p[x][y / 2][y % 2 * 4 + 2] = hi2[0]; p[x][y / 2][y % 2 * 4 + 3] = hi2[1];
        }
        l[x] += apart ? 0.f : ldexpf(sum, back);
      }
      __builtin_amdgcn_sched_barrier(0);
      store_k((i + 1) & 1);
      store_v((i + 1) & 1);
      const Step later = step_of(ahead);
      request(later, raw_k, c.k, KC);
      request(later, raw_v, c.v, VW);
      __builtin_amdgcn_s_setprio(1);
      const uint8_t* buf = lds_v[i & 1] + lane * 16;
#pragma unroll
      for (int v = 0; v < VC; v += 2)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int vv = v; vv < v + 2; ++vv) {
            const halfx8 op = *reinterpret_cast<const halfx8*>(buf + (vv * 2 + hf) * 1024);
#pragma unroll
            for (int x = 0; x < QT; ++x) o[x][vv] = __builtin_amdgcn_mfma_f32_16x16x32_f16(op, p[x][hf], o[x][vv], 0, 0, 0);
          }
#pragma unroll
      for (int u = 0; u < 4; ++u) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
#pragma unroll
      for (int u = 0; u < 2 * VC - 4; ++u) {
        __builtin_amdgcn_sched_group_barrier(0x008, QT, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, QT * 4, 1);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
      now = next;
      next = later;
    }
  }

  // rows out: normalised, turned through the wave's share of a buffer
  constexpr int PITCH = D + 8;                     // bf16 of a row
  static_assert(4 * 16 * PITCH * 2 <= 2 * KBYTES, "rows of a wave do not fit");
  uint16_t* turn = reinterpret_cast<uint16_t*>(&lds_k[0][0]) + wave * 16 * PITCH;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const float total = __builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, l[x]), AddF32()), AddF32()));
    const float f = total == 0.f ? 0.f : 1.f / total;
    const int first = (wave * QT + x) * 16, row = t.row0 + first + n, tok = t.t0 + row / G;
    const float lse2 = total == 0.f ? -INFINITY : m[x] + log2f(total);
    const bool is = row < t.rows && tok < t.ql;
    if (tg.splits > 1) {
      const int64_t at = (tile * tg.splits + split) * tg.stored + first + n;
      if (is) {
#pragma unroll
        for (int v = 0; v < VC; ++v) *reinterpret_cast<floatx4*>(a.parts + at * D + 16 * v + 4 * g) = scaled(o[x][v], f, eo[x]);
        if (g == 0) (a.parts + (int64_t)gridDim.x * tg.stored * D)[at] = lse2;
      }
      continue;
    }
    if (is && g == 0 && a.lse) a.lse[((int64_t)t.b * r.heads + t.hk * G + row % G) * r.t + tok] = lse2 * kLn2;
#pragma unroll
    for (int v = 0; v < VC; ++v) {
      const floatx4 z = scaled(o[x][v], f, eo[x]);
      *reinterpret_cast<uint2*>(turn + n * PITCH + 16 * v + 4 * g) = make_uint2(pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3]));
    }
    __builtin_amdgcn_wave_barrier();               // (the wave's own rows: LDS keeps a wave's order)
#pragma unroll
    for (int u = lane; u < 16 * (D / 8); u += 64) {
      const int rr = u / (D / 8), ch = u % (D / 8) * 8, orow = t.row0 + first + rr, otok = t.t0 + orow / G;
      if (orow < t.rows && otok < t.ql)
        *reinterpret_cast<uint4*>(a.O + (int64_t)t.b * r.sb + (int64_t)(t.hk * G + orow % G) * r.sh + (int64_t)otok * r.st + ch) =
            *reinterpret_cast<const uint4*>(turn + rr * PITCH + ch);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <int D, int BLK>
hipError_t launch_t(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, Plan p, hipStream_t s) {
  const dim3 grid((uint32_t)(p.tiles * p.grid.splits)), block(256);
  // Where there are several rounds of tiles and the last tokens see the most keys, these go first, so that the launch ends with short
  // tiles: prompts of 4096 and 16 384 tokens, 32 heads over 8: 187 -> 163, 2013 -> 1867 us.
  p.grid.last_first = a.causal && p.tiles * p.grid.splits > 2 * kCus;
  if (p.tiled && p.qt == 1) hipLaunchKernelGGL((cache_tile_kernel<D, BLK, 1>), grid, block, 0, s, c, r, a, p.grid);
  else if (p.tiled) hipLaunchKernelGGL((cache_tile_kernel<D, BLK, 2>), grid, block, 0, s, c, r, a, p.grid);
  else if (p.qt == 1) hipLaunchKernelGGL((cache_attn_kernel<D, BLK, 1>), grid, block, 0, s, c, r, a, p.grid);
  else hipLaunchKernelGGL((cache_attn_kernel<D, BLK, 2>), grid, block, 0, s, c, r, a, p.grid);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_join<D>(c, r, a, p, s);
}

}  // namespace

int64_t cache_attn_workgroups(const CacheDims& c, const RowDims& r, int group, int list_len) {
  const Plan p = plan_of(c, r, group, list_len);
  return p.tiles * p.grid.splits;
}

size_t cache_attn_parts_bytes(const CacheDims& c, const RowDims& r, int group, int list_len) {
  const Plan p = plan_of(c, r, group, list_len);
  return p.grid.splits == 1 ? 0 : (size_t)p.tiles * p.grid.splits * p.grid.stored * (c.d + 1) * sizeof(float);
}

hipError_t launch_cache_attn(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, hipStream_t s) {
  Plan p = plan_of(c, r, a.block_idx ? a.group : 0, a.block_idx ? a.list_len : 0);
  if (!a.parts) p.grid.splits = 1;
  if (c.d == 128) return c.blk == 128 ? launch_t<128, 128>(c, r, a, p, s) : launch_t<128, 64>(c, r, a, p, s);
  return c.blk == 128 ? launch_t<64, 128>(c, r, a, p, s) : launch_t<64, 64>(c, r, a, p, s);
}

}  // namespace rsa
