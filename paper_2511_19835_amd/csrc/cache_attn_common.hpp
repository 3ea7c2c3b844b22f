// What the attention kernels over both caches (8 and 4 bits) share: which rows and keys a tile has, how the work is split, and how
// the parts of a split key axis are joined.
#pragma once

#include "cache_common.hpp"

namespace rsa {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNoReference = -3.0e38f;     // of a row that has seen no key; finite, so that differences stay defined
constexpr float kLazy = 8.f;
// From scores of kWhole on a difference of a few is rounded: there a reference follows its maximum at once, which keeps P in range.
constexpr float kWhole = 0x1p23f;
template <int QT>
__device__ __forceinline__ bool far_from_zero(const float (&m)[QT]) {   // of any column of the wave
  bool far = false;
#pragma unroll
  for (int x = 0; x < QT; ++x) far |= fabsf(m[x]) >= kWhole && m[x] != kNoReference;
  return __any(far);
}
constexpr int kCus = 256;                    // compute units of an MI355X
// Parts that a tile's keys are split into at most, for the few tiles of a long cache. us with 64, 128 and 256: a token of 32 heads on one
// key/value head, 131 072 keys, 29, 23, 23; of 8 heads on 65 536 keys 16, 14, 17; 64 tokens of 8 heads on 131 072 keys 63, 55, 55 (16 parts: 187).
constexpr int kMostParts = 128;

// What a tile is, the same in every lane.
struct Tile {
  int b, hk;            // sequence, key/value head
  int t0;               // first token of its group
  int row0, rows;       // first row among the group's (token, head) rows, and how many the group has
  int lrow;             // row of the lists (also without lists: the row of partial results)
  int64_t kv;           // tokens in the cache
  int ql;               // query tokens of the sequence
  int units;            // blocks to walk: listed ones, or all that any row of the tile sees
  int blocks;           // blocks that hold a visible key
  int lo_seen;          // keys that every row of the tile sees
};
struct TileGrid {
  int rows_per_tile;    // 16 QT
  int per_group;        // tiles of a group
  int splits;
  int stored;           // rows of a partial result: min(16 QT, rows of a group)
  bool last_first;      // cache_tile_kernel: a sequence's last tokens go first
};

// Keys that query token `tok` of the tile's sequence sees.
__device__ __forceinline__ int visible_keys(const CacheDims& c, const CacheAttnArgs& a, const Tile& t, int tok) {
  const int64_t n = a.causal ? min(max(t.kv - t.ql + tok + 1, (int64_t)0), t.kv) : t.kv;
  return (int)min(n, (int64_t)c.max_blocks * c.blk);
}
__device__ __forceinline__ Tile tile_of(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, const TileGrid& tg, int64_t id) {
  Tile t;
  const int G = r.heads / c.heads_kv;
  const int k = (int)(id % tg.per_group);
  t.lrow = (int)(id / tg.per_group);
  const int bh = t.lrow / a.groups, grp = t.lrow % a.groups;
  t.b = bh / c.heads_kv;
  t.hk = bh % c.heads_kv;
  t.t0 = grp * a.group;
  t.rows = min(a.group, r.t - t.t0) * G;
  t.row0 = k * tg.rows_per_tile;
  t.kv = max(a.kv_len[t.b], 0);
  t.ql = a.q_len ? min(a.q_len[t.b], r.t) : r.t;
  const int last_row = min(t.row0 + tg.rows_per_tile, t.rows) - 1;
  const int first_tok = t.t0 + t.row0 / G, last_tok = min(t.t0 + last_row / G, t.ql - 1);
  int hi = 0;
  t.lo_seen = 0;
  if (t.row0 < t.rows && first_tok < t.ql) {       // some row of the tile is a query
    t.lo_seen = visible_keys(c, a, t, first_tok);
    hi = visible_keys(c, a, t, last_tok);
  }
  t.blocks = (int)(((int64_t)hi + c.blk - 1) >> (c.blk == 128 ? 7 : 6));
  t.units = t.blocks;
  if (a.block_idx) t.units = t.blocks > 0 ? min(max(a.kept[t.lrow], 0), a.list_len) : 0;
  return t;
}

// Parts of a tile's rows, weighted by their share of the softmax denominator and added in the order of the keys. A row
// takes `lanes` (a power of two) threads to each chunk of eight channels, which share its parts, each over its own largest
// log-sum-exp: one thread alone waits for one part after another (24 rows of 43 parts: 28.8 us with one, 5.1 with sixteen).
template <int D>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheDims c, RowDims r, CacheAttnArgs a, TileGrid tg, int64_t tiles, int lanes) {
  constexpr int CPR = D / 8;
  __shared__ float add[256][10];
  const int G = r.heads / c.heads_kv;
  const int tid = threadIdx.x, ch = tid % CPR * 8, sl = tid / CPR % lanes;
  const int64_t u = (int64_t)blockIdx.x * (256 / CPR / lanes) + tid / CPR / lanes;
  const int rr = (int)(u % tg.stored);
  const int64_t id = u / tg.stored;
  const int lrow = (int)(id / tg.per_group), k = (int)(id % tg.per_group);
  const int bh = lrow / a.groups, grp = lrow % a.groups, b = bh / c.heads_kv, hk = bh % c.heads_kv;
  const int t0 = grp * a.group, row = k * tg.rows_per_tile + rr, tok = t0 + row / G;
  bool is = id < tiles && row < min(a.group, r.t - t0) * G;
  if (is) is = tok < (a.q_len ? min(a.q_len[b], r.t) : r.t);
  float most = -INFINITY, z[8] = {0, 0, 0, 0, 0, 0, 0, 0}, total = 0.f;
  if (is) {
    const int64_t first = id * tg.splits;
    const float* part_lse = a.parts + tiles * tg.splits * tg.stored * D;
#pragma unroll 4
    for (int s = sl; s < tg.splits; s += lanes) most = fmaxf(most, part_lse[(first + s) * tg.stored + rr]);
#pragma unroll 4
    for (int s = sl; s < tg.splits; s += lanes) {
      const float p = part_lse[(first + s) * tg.stored + rr];
      const float w = p == -INFINITY ? 0.f : exp2f(p - most);
      const float* src = a.parts + ((first + s) * tg.stored + rr) * D + ch;
      const float4 lo = *reinterpret_cast<const float4*>(src), hi = *reinterpret_cast<const float4*>(src + 4);
      total += w;
      z[0] += w * lo.x; z[1] += w * lo.y; z[2] += w * lo.z; z[3] += w * lo.w;
      z[4] += w * hi.x; z[5] += w * hi.y; z[6] += w * hi.z; z[7] += w * hi.w;
    }
  }
  if (lanes > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) add[tid][e] = z[e];
    add[tid][8] = total;
    add[tid][9] = most;
    __syncthreads();
    if (sl > 0) return;
    for (int x = 1; x < lanes; ++x) most = fmaxf(most, add[tid + x * CPR][9]);
    total = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = 0.f;
    for (int x = 0; x < lanes; ++x) {
      const float* part = add[tid + x * CPR];
      const float w = part[9] == -INFINITY ? 0.f : exp2f(part[9] - most);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] += w * part[e];
      total += w * part[8];
    }
  }
  if (!is) return;
  const float inv = total == 0.f ? 0.f : 1.f / total;
  const uint4 v = make_uint4(pack_bf16x2(z[0] * inv, z[1] * inv), pack_bf16x2(z[2] * inv, z[3] * inv),
                             pack_bf16x2(z[4] * inv, z[5] * inv), pack_bf16x2(z[6] * inv, z[7] * inv));
  *reinterpret_cast<uint4*>(a.O + (int64_t)b * r.sb + (int64_t)(hk * G + row % G) * r.sh + (int64_t)tok * r.st + ch) = v;
  if (ch == 0 && a.lse) a.lse[((int64_t)b * r.heads + hk * G + row % G) * r.t + tok] = total == 0.f ? -INFINITY : (most + log2f(total)) * kLn2;
}

struct Plan {
  bool tiled;           // cache_tile_kernel: 64 QT rows to a tile instead of 16 QT
  int qt;
  int64_t tiles;
  TileGrid grid;
};
// Up to 32 rows of a group: tiles of 16 or 32 rows whose keys the waves share out; more: tiles of 64 or 128 rows. us, 8 heads, four
// sequences of 32 768 keys, d = 128, and sixteen of 8192, d = 64: 20 rows in tiles of 32 59 and 43, of 64 61 and 43; 40 rows in tiles
// of 64 65 and 45, of 32 87 and 68, of 128 82 and 55; 80 rows in tiles of 128 88 and 58, of 64 109 and 76. (All in 8 bits; the first in 4
// bits: 16 rows 32 us, 32 in tiles of 32 36, 64 in tiles of 64 56, 128 in tiles of 128 77.)
// `short_few`: steps up to which more rows are taken in tiles of 32 too, as long as there are two such tiles to a compute unit at most and four steps,
// one for each wave (0: never). 4 bits, 24 heads, d = 128, on 256, 512, 1024 and 2048 keys: 64 rows 9.7, 13.6, 18.0, 19.9 us in tiles of 64 and 8.5, 10.0,
// 12.9, 19.9 of 32; 500 rows on 512 and 1024 keys 19.3 and 29.9 in tiles of 128, 15.2 and 21.1 of 32; four times as many tiles 27 and 46.
Plan plan_of(const CacheDims& c, const RowDims& r, int group, int list_len, int short_few = 0) {
  Plan p;
  const int G = r.heads / c.heads_kv;
  const int per = group > 0 && group < r.t ? group : r.t;
  const int64_t rows = (int64_t)per * G;
  const int64_t steps = (int64_t)(list_len > 0 && list_len < c.max_blocks ? list_len : c.max_blocks) * (c.blk / 64);
  const int64_t of_32 = (int64_t)((r.t + per - 1) / per) * ((rows + 31) / 32) * c.batch * c.heads_kv;
  p.tiled = rows > 32 && !(steps >= 4 && steps <= short_few && of_32 <= 2 * kCus);
  p.qt = rows <= 16 || (p.tiled && rows <= 64) ? 1 : 2;
  p.grid.rows_per_tile = (p.tiled ? 64 : 16) * p.qt;
  p.grid.per_group = (int)((rows + p.grid.rows_per_tile - 1) / p.grid.rows_per_tile);
  p.grid.stored = (int)(rows < p.grid.rows_per_tile ? rows : p.grid.rows_per_tile);
  p.tiles = (int64_t)((r.t + per - 1) / per) * p.grid.per_group * c.batch * c.heads_kv;
  int64_t best = 1;
  if (p.tiled) {
    // Rounds of workgroups over the slots (two to a compute unit, three at d = 64), the last one between what it fills and whole; what one
    // takes is its steps and, in steps, its start, its end and the parts that it leaves. 312 tiles of 317 steps in 1, 2, 3, 4, 5,
    // 6, 8 parts: 512, 501, 382, 409, 442, 406, 406 us; 696 tiles of 186: 572, 531, 559, 550, 559, 583, 609.
    // Three slots at d = 64 and two: 1000 tokens of 12 heads on 30 000 keys 137 and 148 us, 64 of 16 x 8 heads on 8192 46 and 49.
    const int64_t slots = (c.d == 64 ? 3 : 2) * kCus;
    int64_t cost = -1;
    for (int64_t s = 1; s <= kMostParts && s <= (steps + 7) / 8; ++s) {
      const int64_t one = (steps + s - 1) / s + (s > 1 ? 12 : 6), all = one * (p.tiles * s + (p.tiles * s + slots - 1) / slots * slots);
      if (cost < 0 || all < cost) { cost = all; best = s; }
    }
  } else {
    // Two workgroups to a compute unit at least, and parts of at most 64 steps, 16 to a wave, so that sequences of different
    // length even out; of up to half as many more the number that fills its last round best (24 tiles of 3713 steps: 58 parts
    // 261 us, 64 parts 254); never less than a step to a wave. 256 tiles of 512 steps, ragged: 2, 4, 6, 8, 12 parts 254, 256,
    // 249, 246, 248 us; of 64 steps: 57, 59, 62, 63, 72. Up to 24 steps in one launch: the second takes longer than the
    // steps that it saves (8 tiles of 16 steps 10.2 and 8.5 us, of 24 10.4 and 10.4, of 47 10.7 and 16.0).
    const int64_t slots = 2 * kCus;
    best = (slots + p.tiles - 1) / p.tiles;
    if (best < (steps + 63) / 64) best = (steps + 63) / 64;
    int64_t top = best + best / 2;
    if (top > (steps + 3) / 4) top = (steps + 3) / 4;
    if (top > kMostParts) top = kMostParts;
    if (best > top) best = top;
    for (int64_t s = best; s <= top; ++s) {        // less of its last round empty
      const int64_t a = (p.tiles * s + slots - 1) / slots, b = (p.tiles * best + slots - 1) / slots;
      if (a * best < b * s) best = s;
    }
    if (steps <= 24 || p.tiles >= 16 * slots) best = 1;       // (many tiles even out by themselves)
  }
  p.grid.splits = (int)(best < 1 ? 1 : best);
  // never more parts than without a limit on the lists: the workspace is sized for that
  if (steps < (int64_t)c.max_blocks * (c.blk / 64)) {
    const int most = plan_of(c, r, group, 0, short_few).grid.splits;
    if (p.grid.splits > most) p.grid.splits = most;
  }
  return p;
}

// Joins the parts that a launch over `p` has left, if it was split.
template <int D>
hipError_t launch_join(const CacheDims& c, const RowDims& r, const CacheAttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.grid.splits == 1) return hipSuccess;
  int lanes = 1;
  const int64_t rows = p.tiles * p.grid.stored;
  while (lanes < p.grid.splits && lanes < 256 / (D / 8) && rows * (D / 8) * lanes < (1 << 18)) lanes *= 2;   // (many rows keep the chip busy alone)
  const int64_t per_wg = 256 / (D / 8) / lanes;
  hipLaunchKernelGGL((cache_join_kernel<D>), dim3((uint32_t)((rows + per_wg - 1) / per_wg)), dim3(256), 0, s, c, r, a, p.grid, p.tiles, lanes);
  return hipGetLastError();
}

}  // namespace
}  // namespace rsa
