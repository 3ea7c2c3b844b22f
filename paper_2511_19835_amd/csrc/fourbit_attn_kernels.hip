// Attention of new queries over the 4-bit key/value cache, over all blocks or over listed ones.
//
// Tiles, splits and joins are those of the 8-bit cache (cache_attn_common.hpp): a tile is 16 QT rows of one (sequence, key/value
// head), and each wave computes, with 16x16x32 products of bf16,
//     S^T = K Q^T      (M = key, N = query, k = channel)
//     O^T += V^T P^T   (M = channel, N = query, k = key)
// with the softmax between them lane-local. A code times its key's scale is exact in bf16, so the scores are those of the stored
// keys, summed in fp32; a value's code is widened alone, and its token's scale goes into P.
//
// P in bf16: half a step is 2^-8 of a weight, and a scale only moves its exponent, whatever the scales of the tokens are to each other, so no
// running scale of the outputs is needed. Few rows, which wait for memory, take what the rounding leaves of it as a second product (2^-15 of a weight
// remains at most). The running reference m of a row is moved only when a lane's 16 weights of a step have become large beside it, so most steps take no
// maximum.
#include "fourbit_common.hpp"

#include "cache_attn_common.hpp"

namespace rsa {
namespace {

// Eight codes as bf16, times `scale` (a power of two: exact).
__device__ __forceinline__ bf16x8 widen8(uint32_t w, float scale) {
  bf16x8 o;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  o[0] = a[0]; o[1] = a[1]; o[2] = b[0]; o[3] = b[1];
  o[4] = c[0]; o[5] = c[1]; o[6] = d[0]; o[7] = d[1];
  return o;
}
// Byte t of a lane's exponents as a scale: 2^(byte - 127), NaN for 255 (whose bits are infinity: times 0 that is NaN).
__device__ __forceinline__ float key_scale(uint32_t w, int t) {
  const float s = __builtin_bit_cast(float, (w >> (8 * t) & 255u) << 23);
  return __builtin_fmaf(s, 0.f, s);
}
// Scales of keys 16 t + 4 g + i of 64 from a lane's 32 bytes.
__device__ __forceinline__ void value_scales(const uint4 (&w)[2], float (&s)[4][4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint32_t lo = t % 2 ? w[t / 2].z : w[t / 2].x, hi = t % 2 ? w[t / 2].w : w[t / 2].y;
    s[t][0] = bf16_bits_to_float(lo & 0xffffu);
    s[t][1] = __builtin_bit_cast(float, lo & 0xffff0000u);
    s[t][2] = bf16_bits_to_float(hi & 0xffffu);
    s[t][3] = __builtin_bit_cast(float, hi & 0xffff0000u);
  }
}

// Weights are made 2^kBias too large, so that a token's scale comes in by a subtraction of exponents (16 bits, two at once; below 0 it stays 0):
// bits of the scale taken from those of 2^kBias say by how much. Scales above 2^kBias (values above 768) and NaN go the long
// way (1000 rows of 4 x 8 heads on 32 768 keys 469 us, all of them the long way 689; 16 rows 32 and 33). The exponent of a weight within 2 of the reference stays below 8: its rounding is 2^-22, which is what a log-sum-exp of one key is off by (2^-18 with a kBias of 90).
constexpr float kBias = 7.f;
constexpr uint32_t kMostScale = 0x43004300u;     // 2^7 in bf16, twice
typedef uint16_t ushortx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t less_than_most(uint32_t w) {      // (its own inverse)
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(ushortx2, kMostScale) - __builtin_bit_cast(ushortx2, w));
}
__device__ __forceinline__ bf16x2 scaled2(uint32_t w, uint32_t less) {
  return __builtin_bit_cast(bf16x2, __builtin_elementwise_sub_sat(__builtin_bit_cast(ushortx2, w), __builtin_bit_cast(ushortx2, less)));
}

// The upper half of two weights, and what it leaves of one (exact).
__device__ __forceinline__ uint32_t cut_bf16x2(float a, float b) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
}
__device__ __forceinline__ float behind_bf16(float a) { return a - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) & 0xffff0000u); }
// Weights of a lane's 16 scores of a row (times `ks`), 2^kBias too large, over the reference: their sum, and P, the weights in bf16 with their tokens'
// scales taken in; FINE: cut to bf16, and what that leaves of them. -> whether the reference has to follow: it is moved only when the sum is more than
// 2^8 (bf16 and fp32 have the range), so that no maximum is taken otherwise; then they are made once more, over the new one at most 1.
template <bool FINE>
__device__ __forceinline__ bool weigh_row(const floatx4 (&s)[4], float ks, float m, const uint4 (&less)[2], float& sum, bf16x8 (&p)[2], bf16x8 (&rest)[2]) {
  const float ref = m - kBias;
  sum = 0.f;
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    float w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = __builtin_amdgcn_exp2f(fmaf(s[y][e], ks, -ref));
      sum += w[e];
    }
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const uint4 d = less[y / 2];
      const uint32_t of = y % 2 ? e ? d.w : d.z : e ? d.y : d.x;
      const bf16x2 z = scaled2(FINE ? cut_bf16x2(w[e], w[e + 1]) : pack_bf16x2(w[e], w[e + 1]), of);
      p[y / 2][y % 2 * 4 + e] = z[0];
      p[y / 2][y % 2 * 4 + e + 1] = z[1];
      if constexpr (FINE) {
        const bf16x2 r = scaled2(pack_bf16x2(behind_bf16(w[e]), behind_bf16(w[e + 1])), of);
        rest[y / 2][y % 2 * 4 + e] = r[0];
        rest[y / 2][y % 2 * 4 + e + 1] = r[1];
      }
    }
  }
  asm volatile("" : "+v"(p[0]), "+v"(p[1]));       // (made here, not behind the branches)
  if constexpr (FINE) asm volatile("" : "+v"(rest[0]), "+v"(rest[1]));
  return sum > 0x1p15f;                            // 2^(8 + kBias)
}
// The reference goes up to the row's largest score, where that is larger -> what is to be taken of what was summed over the old one (0 from 2^-126
// down). The same in the four lanes of a column. (The score itself, so that the weight of the key that moves it is 1, exact in bf16; one that outweighs the
// others by less than it takes to move the reference is rounded like any other.)
__device__ __forceinline__ float move_row(const floatx4 (&s)[4], float ks, float& m) {
  float mx = -INFINITY;
#pragma unroll
  for (int y = 0; y < 4; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[y][e]);
  mx = __builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, mx), MaxF32()), MaxF32())) * ks;
  const float to = mx > m ? mx : m;
  const float down = __builtin_amdgcn_exp2f(m - to);
  m = to;
  return down;
}
// Far from zero a multiply-add would leave a product's own rounding, which may be 2^8 and more, and the reference has no bits for kBias:
// there it follows each step's largest score, and the scores become rounded products less the reference.
__device__ __forceinline__ void from_reference(floatx4 (&s)[4], float ks, float m) {
#pragma clang fp contract(off)
#pragma unroll
  for (int y = 0; y < 4; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float product = s[y][e] * ks;
      s[y][e] = product - m;
    }
}
// P of tokens with a scale above 2^kBias or NaN, by products; no NaN of a token that the row does not see into 0 * NaN.
template <bool FINE>
__device__ __forceinline__ void odd_row(const floatx4 (&s)[4], float ks, float m, const uint4 (&less)[2], bf16x8 (&p)[2], bf16x8 (&rest)[2]) {
  uint4 w[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) w[x] = make_uint4(less_than_most(less[x].x), less_than_most(less[x].y), less_than_most(less[x].z), less_than_most(less[x].w));
  float vs[4][4];
  value_scales(w, vs);
#pragma unroll
  for (int y = 0; y < 4; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float z = __builtin_amdgcn_exp2f(fmaf(s[y][e], ks, -m)) * vs[y][e];
      const float w = s[y][e] == -INFINITY ? 0.f : z;
      if constexpr (FINE) {
        p[y / 2][y % 2 * 4 + e] = (__bf16)(w - behind_bf16(w));
        rest[y / 2][y % 2 * 4 + e] = (__bf16)behind_bf16(w);
      } else {
        p[y / 2][y % 2 * 4 + e] = (__bf16)w;
      }
    }
}

// What a lane loads for a step of 64 keys.
template <int D>
struct Step64 {
  uint32_t k[4][D / 32];       // codes of 16 keys: D / 4 channels of one key
  uint32_t ks;                 // exponents of this lane's run of channels, key n of each tile
  uint4 v[D / 32];
  uint4 vs[2];
};

// Few rows: a wave's steps go from memory to registers to products, no barrier until the end. Bound by memory: a token of 32 sequences of up to 32 768
// keys, 32 heads over 8 (0.72 GB), 136 us and 6 of joining; all of them full 172 us, 6.5 TB/s (170 with P rounded once: the second product costs 1 to 3 %,
// d = 64 up to 12 %). 17 to 32 rows by the vector ALU (4 x 8 heads on 32 768 keys 40 us, 36 with P rounded once).
// 3 rows of 2 heads on 1088 keys 7.2 us: lengths, pages, codes, products and the join one after the other.
template <int D, int BLK, int QT, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void fourbit_attn_kernel(CacheDims c, RowDims r, CacheAttnArgs a, TileGrid tg) {
  constexpr int KM = D / 32, VC = D / 16;          // products of a tile of 16 keys / channel tiles
  constexpr int SPB = BLK / 64;                    // steps of 64 keys in a block
  constexpr int KR = fourbit_k_record(D), VR = fourbit_v_record(D);
  constexpr int PITCH = D + 4;                     // floats of a row in the joining buffer
  __shared__ __align__(16) float join[NW][16][PITCH];
  __shared__ float join_m[NW][16], join_l[NW][16];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int g = lane / 16, n = lane % 16;
  const int split = blockIdx.x % tg.splits;
  const int64_t id = blockIdx.x / tg.splits;
  const Tile t = tile_of(c, r, a, tg, id);
  const int G = r.heads / c.heads_kv;

  // queries of this lane's columns, as operands (channels (D / 4) g + 8 m ..), and how many keys each sees
  bf16x8 q[QT][KM];
  int seen[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int row = t.row0 + 16 * x + n, tok = t.t0 + row / G;
    const bool is = row < t.rows && tok < t.ql;
    seen[x] = !is ? 0 : visible_keys(c, a, t, tok);
    const uint16_t* src = a.Q + (int64_t)t.b * r.sb + (int64_t)(t.hk * G + row % G) * r.sh + (int64_t)tok * r.st + g * (D / 4);
#pragma unroll
    for (int k = 0; k < KM; ++k) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (is) v = *reinterpret_cast<const uint4*>(src + k * 8);
      q[x][k] = __builtin_bit_cast(bf16x8, v);
    }
  }
  floatx4 o[QT][VC];
  float m[QT], l[QT];                              // reference, sum of the weights
  bool far = false;                                // a reference is 2^23 and more
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    m[x] = kNoReference;
    l[x] = 0.f;
#pragma unroll
    for (int v = 0; v < VC; ++v) o[x][v] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  const float all_ks = fmaxf(a.scale_log2e, 0x1p-149f);      // (above 0, so that a masked score stays -inf)

  const int u0 = (int)((int64_t)t.units * split / tg.splits), u1 = (int)((int64_t)t.units * (split + 1) / tg.splits);
  const int steps = (u1 - u0) * SPB;
  // this wave's steps are wave, wave + NW, ...; lane i looks up the i-th of the next 64
  for (int base = wave; base < steps; base += 64 * NW) {
    int my_blk = -1, my_page = -1;
    const int my_step = base + lane * NW;
    if (my_step < steps) {
      my_blk = u0 + my_step / SPB;
      if (a.block_idx) my_blk = a.block_idx[(int64_t)t.lrow * a.list_len + my_blk];
      if (my_blk < t.blocks) my_page = cache_page(c, t.b, my_blk);
    }
    unsigned long long todo = __ballot(my_page >= 0);
    // Two steps are in registers, one used and one on its way; where two tiles of rows leave no room, one, loaded again as it is used up.
    constexpr int SETS = QT == 1 ? 2 : 1;
    Step64<D> at[SETS];
    auto load_k = [&](Step64<D>& z, int i) __attribute__((always_inline)) {
      const int64_t rec = ((int64_t)__builtin_amdgcn_readlane(my_page, i) * c.heads_kv + t.hk) * SPB + (base + i * NW) % SPB;
      const uint8_t* pk = c.k + rec * KR;
      z.ks = *reinterpret_cast<const uint32_t*>(pk + 32 * D + (D == 128 ? lane : (g / 2) * 16 + n) * 4);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if constexpr (D == 128) {
          const uint4 w = *reinterpret_cast<const uint4*>(pk + y * 1024 + lane * 16);
          z.k[y][0] = w.x; z.k[y][1] = w.y; z.k[y][2] = w.z; z.k[y][3] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(pk + y * 512 + ((g / 2) * 16 + n) * 16 + (g % 2) * 8);
          z.k[y][0] = w.x; z.k[y][1] = w.y;
        }
      }
    };
    auto load_v = [&](Step64<D>& z, int i) __attribute__((always_inline)) {
      const int64_t rec = ((int64_t)__builtin_amdgcn_readlane(my_page, i) * c.heads_kv + t.hk) * SPB + (base + i * NW) % SPB;
      const uint8_t* pv = c.v + rec * VR;
#pragma unroll
      for (int x = 0; x < 2; ++x) z.vs[x] = *reinterpret_cast<const uint4*>(pv + 32 * D + g * 32 + x * 16);
#pragma unroll
      for (int x = 0; x < D / 32; ++x) z.v[x] = *reinterpret_cast<const uint4*>(pv + x * 1024 + lane * 16);
    };
    auto compute = [&](Step64<D>& z, int i, int again) __attribute__((always_inline)) {
      const int key0 = __builtin_amdgcn_readlane(my_blk, i) * BLK + ((base + i * NW) % SPB) * 64;
      floatx4 s[QT][4];
#pragma unroll
      for (int x = 0; x < QT; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) s[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float sc = key_scale(z.ks, y);
#pragma unroll
        for (int k = 0; k < KM; ++k) {
          const bf16x8 op = widen8(z.k[y][k], sc);
#pragma unroll
          for (int x = 0; x < QT; ++x) s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op, q[x][k], s[x][y], 0, 0, 0);
        }
      }
      if (SETS == 1) load_k(z, again);
      if (key0 + 64 > t.lo_seen) {                 // keys that a row does not see leave its softmax
        asm volatile("");                          // (a branch, no selects)
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const int left = seen[x] - key0;         // of the 64
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[x][y][e] = 16 * y + 4 * g + e < left ? s[x][y][e] : -INFINITY;
        }
      }
      uint4 less[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) less[x] = make_uint4(less_than_most(z.vs[x].x), less_than_most(z.vs[x].y), less_than_most(z.vs[x].z), less_than_most(z.vs[x].w));
      bf16x8 p[QT][2], rest[QT][2];
      float sum[QT];
      auto weigh = [&](float ks) __attribute__((always_inline)) {
        bool over = false;
#pragma unroll
        for (int x = 0; x < QT; ++x) over |= weigh_row<true>(s[x], ks, far ? 0.f : m[x], less, sum[x], p[x], rest[x]);
        return over;
      };
      auto move = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const float down = move_row(s[x], all_ks, m[x]);
          l[x] *= down;
#pragma unroll
          for (int v = 0; v < VC; ++v) o[x][v] *= down;
        }
      };
      if (far) {
        asm volatile("");
        move();
#pragma unroll
        for (int x = 0; x < QT; ++x) from_reference(s[x], all_ks, m[x]);
      }
      if (__any(weigh(far ? 1.f : all_ks))) {
        move();
        if (far_from_zero<QT>(m)) {
          far = true;
#pragma unroll
          for (int x = 0; x < QT; ++x) from_reference(s[x], all_ks, m[x]);
        }
        weigh(far ? 1.f : all_ks);
      }
#pragma unroll
      for (int x = 0; x < QT; ++x) l[x] += sum[x];
      const uint32_t any_odd = (less[0].x | less[0].y | less[0].z | less[0].w | less[1].x | less[1].y | less[1].z | less[1].w) & 0x80008000u;
      if (__any(any_odd != 0)) {
        asm volatile("");
#pragma unroll
        for (int x = 0; x < QT; ++x) odd_row<true>(s[x], far ? 1.f : all_ks, far ? 0.f : m[x], less, p[x], rest[x]);
      }
#pragma unroll
      for (int v = 0; v < VC; ++v) {
        const uint4 w = z.v[v / 2];
        const bf16x8 lo = widen8(v % 2 ? w.z : w.x, 1.f), hi = widen8(v % 2 ? w.w : w.y, 1.f);
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          o[x][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, p[x][0], o[x][v], 0, 0, 0);
          o[x][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, p[x][1], o[x][v], 0, 0, 0);
          o[x][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, rest[x][0], o[x][v], 0, 0, 0);
          o[x][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, rest[x][1], o[x][v], 0, 0, 0);
        }
      }
      if (SETS == 1) load_v(z, again);
    };
    auto take = [&]() __attribute__((always_inline)) {
      const int i = todo ? __builtin_ctzll(todo) : -1;
      todo &= todo - 1;
      return i;
    };
    int i = take();
    if (i >= 0) {
      load_k(at[0], i);
      load_v(at[0], i);
    }
    while (i >= 0) {
      const int j = take();
      if constexpr (SETS == 1) {
        compute(at[0], i, j < 0 ? i : j);
        i = j;
      } else {
        if (j >= 0) {
          load_k(at[1], j);
          load_v(at[1], j);
        }
        compute(at[0], i, i);
        if (j < 0) break;
        i = take();
        if (i >= 0) {
          load_k(at[0], i);
          load_v(at[0], i);
        }
        compute(at[1], j, j);
      }
    }
  }

  // join the waves, 16 rows at a time
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const float sum = ldexpf(__builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, l[x]), AddF32()), AddF32())), -(int)kBias);
    if (x > 0) __syncthreads();
    if (g == 0) {
      join_m[wave][n] = m[x];
      join_l[wave][n] = sum;
    }
    __syncthreads();
    float most = join_m[0][n];
#pragma unroll
    for (int w = 1; w < NW; ++w) most = fmaxf(most, join_m[w][n]);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) total += join_l[w][n] * exp2f(join_m[w][n] - most);
    const float f = total == 0.f ? 0.f : exp2f(m[x] - most) / total;
#pragma unroll
    for (int v = 0; v < VC; ++v) *reinterpret_cast<floatx4*>(&join[wave][n][16 * v + 4 * g]) = o[x][v] * f;
    __syncthreads();
    constexpr int CPR = D / 8;
    for (int u = tid; u < 16 * CPR; u += 64 * NW) {
      const int rr = u / CPR, ch = u % CPR * 8, row = t.row0 + 16 * x + rr, tok = t.t0 + row / G;
      if (row >= t.rows || tok >= t.ql) continue;
      float z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[e] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; w += 2) z[e] += join[w][rr][ch + e] + join[w + 1][rr][ch + e];
      }
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

// The same for many query rows. 64 QT rows to a workgroup, 16 QT to a wave: every wave needs all codes, so they are widened once for
// the workgroup, a quarter by each wave, into LDS in the order of the operands. Two buffers, one barrier a step of 64 keys; codes are requested
// two steps ahead and widened between the softmax and the products of the values.
// 24 heads, 1560 tokens on 20 280 keys, repeated: 360 us and 12.6 of joining, 1040 TFLOP/s (a library product 1219; on another box 1056 and 1404, and 897
// after a pause of 0.2 s); the matrix pipe is busy 50 % of the time, the vector ALU 58 %, LDS 40 %. Scores of the next step beside this one's weights 456 us, each wave widening for itself without LDS
// 417, two groups of waves a phase apart 486, products of 32x32x16 421 (against 383 to 392 of the form of the day).
// 64 rows (56 us where 32 rows take 36): neither half the LDS reads, nor eight waves, nor four steps ahead are faster.
// Three workgroups to a compute unit at d = 64, two at d = 128. us with two and three:
// 128 rows of 16 x 8 heads on 8192 keys 63, 58; 1000 rows 343, 310 (866 TFLOP/s); 1000 rows of 12 heads on 30 000 keys 137, 124 (743 TFLOP/s); the
// last two on another box 323 and 139.
constexpr int kAhead = 256;                        // steps that are looked up together
template <int D, int BLK, int QT>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void fourbit_tile_kernel(CacheDims c, RowDims r, CacheAttnArgs a, TileGrid tg) {
  constexpr int KM = D / 32, VC = D / 16, VW = VC / 4;   // VW: channel tiles that a wave widens
  constexpr int SPB = BLK / 64;
  constexpr int KR = fourbit_k_record(D), VR = fourbit_v_record(D);
  constexpr int KBYTES = 4 * KM * 1024, VBYTES = VC * 2048;
  __shared__ __align__(16) uint8_t lds_k[2][KBYTES], lds_v[2][VBYTES];
  __shared__ __align__(16) uint32_t lds_s[2][32];  // scales of the values
  __shared__ int2 look[kAhead];                    // page, first key
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

  bf16x8 q[QT][KM];
  int seen[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int row = t.row0 + (wave * QT + x) * 16 + n, tok = t.t0 + row / G;
    const bool is = row < t.rows && tok < t.ql;
    seen[x] = !is ? 0 : visible_keys(c, a, t, tok);
    const uint16_t* src = a.Q + (int64_t)t.b * r.sb + (int64_t)(t.hk * G + row % G) * r.sh + (int64_t)tok * r.st + g * (D / 4);
#pragma unroll
    for (int k = 0; k < KM; ++k) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (is) v = *reinterpret_cast<const uint4*>(src + k * 8);
      q[x][k] = __builtin_bit_cast(bf16x8, v);
    }
  }
  // the queries are here before the loop: a wait for them inside it would be one for every load in flight
#pragma unroll
  for (int x = 0; x < QT; ++x)
#pragma unroll
    for (int k = 0; k < KM; ++k) asm volatile("" : "+v"(q[x][k]));
  floatx4 o[QT][VC];
  float m[QT], l[QT];
  bool far = false;                                // a reference is 2^23 and more
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    m[x] = kNoReference;
    l[x] = 0.f;
#pragma unroll
    for (int v = 0; v < VC; ++v) o[x][v] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float all_ks = fmaxf(a.scale_log2e, 0x1p-149f);      // (above 0, so that a masked score stays -inf)

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
      if (page >= 0) look[at] = make_int2(page, blk * BLK + s % SPB * 64);
      __syncthreads();
    }
    const int count = __builtin_amdgcn_readfirstlane(n_valid[0] + n_valid[1] + n_valid[2] + n_valid[3]);
    if (count == 0) continue;
    struct Step { int page, key; };                // the same in every lane
    auto entry = [&](int i) __attribute__((always_inline)) { return look[min(i, count - 1)]; };
    auto step_of = [&](const int2& v) __attribute__((always_inline)) {
      return Step{__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y)};
    };
    struct Raw { uint32_t k[KM], v[2 * VW], ks, vs; } ra, rb;      // of the next step and of the one behind it
    auto request = [&](const Step& z, Raw& raw) __attribute__((always_inline)) {
      const int64_t rec = ((int64_t)z.page * c.heads_kv + t.hk) * SPB + z.key % BLK / 64;
      const uint8_t *pk = c.k + rec * KR, *pv = c.v + rec * VR;
      raw.ks = *reinterpret_cast<const uint32_t*>(pk + 32 * D + (D == 128 ? lane : (g / 2) * 16 + n) * 4);
      raw.vs = *reinterpret_cast<const uint32_t*>(pv + 32 * D + (lane % 32) * 4);
      if constexpr (D == 128) {
        const uint4 k = *reinterpret_cast<const uint4*>(pk + wave * 1024 + lane * 16);
        raw.k[0] = k.x; raw.k[1] = k.y; raw.k[2] = k.z; raw.k[3] = k.w;
        const uint4 v = *reinterpret_cast<const uint4*>(pv + wave * 1024 + lane * 16);
        raw.v[0] = v.x; raw.v[1] = v.y; raw.v[2] = v.z; raw.v[3] = v.w;
      } else {
        const uint2 k = *reinterpret_cast<const uint2*>(pk + wave * 512 + ((g / 2) * 16 + n) * 16 + (g % 2) * 8);
        raw.k[0] = k.x; raw.k[1] = k.y;
        const uint2 v = *reinterpret_cast<const uint2*>(pv + wave / 2 * 1024 + lane * 16 + wave % 2 * 8);
        raw.v[0] = v.x; raw.v[1] = v.y;
      }
    };
    auto store = [&](int buf, const Raw& raw) __attribute__((always_inline)) {
      const float sc = key_scale(raw.ks, wave);
#pragma unroll
      for (int k = 0; k < KM; ++k) *reinterpret_cast<bf16x8*>(lds_k[buf] + (wave * KM + k) * 1024 + lane * 16) = widen8(raw.k[k], sc);
#pragma unroll
      for (int x = 0; x < 2 * VW; ++x) *reinterpret_cast<bf16x8*>(lds_v[buf] + (wave * 2 * VW + x) * 1024 + lane * 16) = widen8(raw.v[x], 1.f);
      if (tid < 32) lds_s[buf][tid] = less_than_most(raw.vs);
      return __any((raw.vs & 0x7fffu) > (kMostScale & 0xffffu) || (raw.vs >> 16 & 0x7fffu) > (kMostScale & 0xffffu)) != 0;
    };

    Step now = step_of(entry(0)), next = step_of(entry(1)), third = step_of(entry(2));
    request(now, rb);
    request(next, ra);
    bool odd = store(0, rb);                       // of the step `now`
    request(third, rb);
    auto step = [&](int i, Raw& raw) __attribute__((always_inline)) {
      __syncthreads();
      const int2 ahead = entry(i + 3);
      const bool partly = now.key + 64 > t.lo_seen;
      uint4 less[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) less[x] = *reinterpret_cast<const uint4*>(&lds_s[i & 1][g * 8 + x * 4]);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      floatx4 s[QT][4];
#pragma unroll
      for (int x = 0; x < QT; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) s[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};
      {
        const uint8_t* buf = lds_k[i & 1] + lane * 16;
#pragma unroll
        for (int k = 0; k < KM; ++k)
#pragma unroll
          for (int y = 0; y < 4; ++y) {            // (a sum is touched again 4 QT products later)
            const bf16x8 op = *reinterpret_cast<const bf16x8*>(buf + (y * KM + k) * 1024);
#pragma unroll
            for (int x = 0; x < QT; ++x) s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op, q[x][k], s[x][y], 0, 0, 0);
          }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
      for (int u = 0; u < 4 * KM - 4; ++u) {
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
      bf16x8 p[QT][2], none[2];
      float sum[QT];
      auto weigh = [&](float ks) __attribute__((always_inline)) {
        bool over = false;
#pragma unroll
        for (int x = 0; x < QT; ++x) over |= weigh_row<false>(s[x], ks, far ? 0.f : m[x], less, sum[x], p[x], none);
        return over;
      };
      auto move = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const float down = move_row(s[x], all_ks, m[x]);
          l[x] *= down;
#pragma unroll
          for (int v = 0; v < VC; ++v) o[x][v] *= down;
        }
      };
      if (far) {
        asm volatile("");
        move();
#pragma unroll
        for (int x = 0; x < QT; ++x) from_reference(s[x], all_ks, m[x]);
      }
      if (__any(weigh(far ? 1.f : all_ks))) {
        move();
        if (far_from_zero<QT>(m)) {
          far = true;
#pragma unroll
          for (int x = 0; x < QT; ++x) from_reference(s[x], all_ks, m[x]);
        }
        weigh(far ? 1.f : all_ks);
      }
#pragma unroll
      for (int x = 0; x < QT; ++x) l[x] += sum[x];
      if (odd) {                                   // rare
        asm volatile("");
#pragma unroll
        for (int x = 0; x < QT; ++x) odd_row<false>(s[x], far ? 1.f : all_ks, far ? 0.f : m[x], less, p[x], none);
      }
      __builtin_amdgcn_sched_barrier(0);
      odd = store((i + 1) & 1, raw);
      const Step later = step_of(ahead);
      request(later, raw);
      __builtin_amdgcn_s_setprio(1);
      const uint8_t* buf = lds_v[i & 1] + lane * 16;
#pragma unroll
      for (int v = 0; v < VC; v += 2)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int vv = v; vv < v + 2; ++vv) {
            const bf16x8 op = *reinterpret_cast<const bf16x8*>(buf + (vv * 2 + hf) * 1024);
#pragma unroll
            for (int x = 0; x < QT; ++x) o[x][vv] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op, p[x][hf], o[x][vv], 0, 0, 0);
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
      next = third;
      third = later;
    };
    for (int i = 0; i < count; i += 2) {
      step(i, ra);
      if (i + 1 >= count) break;
      step(i + 1, rb);
    }
  }

  // rows out: normalised, turned through the wave's share of a buffer
  constexpr int PITCH = D + 8;                     // bf16 of a row
  static_assert(4 * 16 * PITCH * 2 <= 2 * KBYTES, "rows of a wave do not fit");
  uint16_t* turn = reinterpret_cast<uint16_t*>(&lds_k[0][0]) + wave * 16 * PITCH;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const float total = ldexpf(__builtin_bit_cast(float, with_xor32(with_xor16(__builtin_bit_cast(int, l[x]), AddF32()), AddF32())), -(int)kBias);
    const float f = total == 0.f ? 0.f : 1.f / total;
    const int first = (wave * QT + x) * 16, row = t.row0 + first + n, tok = t.t0 + row / G;
    const float lse2 = total == 0.f ? -INFINITY : m[x] + log2f(total);
    const bool is = row < t.rows && tok < t.ql;
    if (tg.splits > 1) {
      const int64_t at = (tile * tg.splits + split) * tg.stored + first + n;
      if (is) {
#pragma unroll
        for (int v = 0; v < VC; ++v) *reinterpret_cast<floatx4*>(a.parts + at * D + 16 * v + 4 * g) = o[x][v] * f;
        if (g == 0) (a.parts + (int64_t)gridDim.x * tg.stored * D)[at] = lse2;
      }
      continue;
    }
    if (is && g == 0 && a.lse) a.lse[((int64_t)t.b * r.heads + t.hk * G + row % G) * r.t + tok] = lse2 * kLn2;
#pragma unroll
    for (int v = 0; v < VC; ++v) {
      const floatx4 z = o[x][v] * f;
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

constexpr int kShortFew = 16;                      // steps up to which more than 32 rows go in tiles of 32 (plan_of)
template <int D, int BLK>
hipError_t launch_t(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, Plan p, hipStream_t s) {
  const dim3 grid((uint32_t)(p.tiles * p.grid.splits)), block(256);
  // Where there are several rounds of tiles and the last tokens see the most keys, these go first, so that the launch ends with short tiles.
  p.grid.last_first = a.causal && p.tiles * p.grid.splits > 2 * kCus;
  if (p.tiled && p.qt == 1) hipLaunchKernelGGL((fourbit_tile_kernel<D, BLK, 1>), grid, block, 0, s, c, r, a, p.grid);
  else if (p.tiled) hipLaunchKernelGGL((fourbit_tile_kernel<D, BLK, 2>), grid, block, 0, s, c, r, a, p.grid);
  // A tile to a compute unit and less, in one launch: eight waves share its keys (3 rows of 2 heads on 1088 keys: 8.7 us with four, 8.0).
  else if (p.qt == 1 && p.grid.splits == 1 && p.tiles <= kCus) hipLaunchKernelGGL((fourbit_attn_kernel<D, BLK, 1, 8>), grid, dim3(512), 0, s, c, r, a, p.grid);
  else if (p.qt == 1) hipLaunchKernelGGL((fourbit_attn_kernel<D, BLK, 1, 4>), grid, block, 0, s, c, r, a, p.grid);
  else hipLaunchKernelGGL((fourbit_attn_kernel<D, BLK, 2, 4>), grid, block, 0, s, c, r, a, p.grid);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_join<D>(c, r, a, p, s);
}

}  // namespace

int64_t fourbit_attn_workgroups(const CacheDims& c, const RowDims& r, int group, int list_len) {
  const Plan p = plan_of(c, r, group, list_len, kShortFew);
  return p.tiles * p.grid.splits;
}

size_t fourbit_attn_parts_bytes(const CacheDims& c, const RowDims& r, int group, int list_len) {
  const Plan p = plan_of(c, r, group, list_len, kShortFew);
  return p.grid.splits == 1 ? 0 : (size_t)p.tiles * p.grid.splits * p.grid.stored * (c.d + 1) * sizeof(float);
}

hipError_t launch_fourbit_attn(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, hipStream_t s) {
  Plan p = plan_of(c, r, a.block_idx ? a.group : 0, a.block_idx ? a.list_len : 0, kShortFew);
  if (!a.parts) p.grid.splits = 1;
  if (c.d == 128) return c.blk == 128 ? launch_t<128, 128>(c, r, a, p, s) : launch_t<128, 64>(c, r, a, p, s);
  return c.blk == 128 ? launch_t<64, 128>(c, r, a, p, s) : launch_t<64, 64>(c, r, a, p, s);
}

}  // namespace rsa
