// The cheap score of the blocks of an 8-bit cache and the choice of those that a group of query tokens reads.
//
// score(j) = q8 . k8_j * 2^em_j with q8 the group's summed queries and k8_j the mean key of block j, both in 8 bits with a
// power-of-two scale (that of q8 is common to a row and left out). The dot product is integer work and the scale moves no
// bit, so a score is exact, equal scores are equal, and the choice does not depend on an order of sums.
//
// One workgroup per row = (sequence, key/value head, group): the sum of the queries (fp64: exact for bf16 terms within 40
// binades of each other), the scores of all blocks as order-preserving keys, the threshold key by a histogram (keys in
// registers, each wave owning a run of blocks), and the kept blocks in ascending order. What bounds it is latency and the
// address unit: 256 rows of 512 blocks 8.3 us (its 17 MB of means would take 2.8), 696 rows of 929 19.2; the longest rows
// take sixteen waves. Where there are few rows and many blocks the scores are a launch of their own, in runs of blocks over
// many workgroups.
#include "cache_common.hpp"

namespace rsa {
namespace {

__device__ __forceinline__ uint32_t ordered_key(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float score_of(uint32_t key) {
  return __builtin_bit_cast(float, (key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}
// The value of the lane N before in its row of 16, 0 where there is none.
template <int N>
__device__ __forceinline__ int row_up(int x) { return __builtin_amdgcn_update_dpp(0, x, 0x110 + N, 0xf, 0xf, true); }
__device__ __forceinline__ double finite_or_zero(uint32_t bits16) {
  return (bits16 & 0x7f80u) == 0x7f80u ? 0.0 : (double)bf16_bits_to_float(bits16);
}
constexpr uint32_t kUnseen = 0u;                   // below every score
constexpr float kLargest = 3.4028234663852886e38f;
constexpr uint32_t kLowest = 0x00800000u;          // key of -kLargest, also of what is no number
constexpr int kRunBlocks = 1024;                   // blocks that a workgroup of the scoring launch takes

struct Row {
  int b, hk, G;
  int t0, t1;                                      // its tokens
  int t_end;                                       // the same as if every row were a query
  int seen;                                        // blocks that may be chosen: [0, seen)
  int lo_forced, hi_forced;                        // forced beside those below `first`
};
// Where a row stands, without the lengths (its t1, seen and forced blocks are set by add_lengths).
__device__ __forceinline__ Row row_of(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, int row) {
  Row w;
  const int grp = row % a.groups, bh = row / a.groups;
  w.b = bh / c.heads_kv;
  w.hk = bh % c.heads_kv;
  w.G = r.heads / c.heads_kv;
  w.t0 = grp * a.group;
  w.t_end = min(w.t0 + a.group, r.t);
  return w;
}
__device__ __forceinline__ void add_lengths(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, int kv_len, int q_len, Row& w) {
  const int shift = c.blk == 128 ? 7 : 6;          // (a shift of a negative position rounds down)
  const int64_t kv = kv_len;
  const int ql = min(q_len, r.t);
  w.t1 = min(w.t0 + a.group, ql);
  const int64_t p0 = kv - ql + w.t0, p1 = kv - ql + w.t1 - 1;              // positions of the first and the last
  int64_t seen = a.causal ? max((p1 >> shift) + 1, (int64_t)0) : (kv + c.blk - 1) >> shift;
  if (w.t1 <= w.t0 || kv <= 0) seen = 0;
  w.seen = (int)min(seen, (int64_t)c.max_blocks);
  w.lo_forced = a.last > 0 ? (int)max((int64_t)0, (p0 >> shift) - a.last + 1) : 0x7fffffff;
  w.hi_forced = a.last > 0 ? (int)(p1 >> shift) : -1;
}

template <int D>
struct QueryLds {
  double sums[256 / (D / 8)][D];
  uint32_t most[2];
  __align__(16) int8_t q8[D];
};
// A chunk of the queries of a row: eight rows of every stripe.
constexpr int kQueryRows = 8;
template <int D>
__device__ __forceinline__ void request_queries(const RowDims& r, const CacheSelectArgs& a, const Row& w, int from, uint4 (&v)[kQueryRows]) {
  constexpr int CPR = D / 8, STRIPES = 256 / CPR;
  const int cc = threadIdx.x % CPR, rows = (w.t_end - w.t0) * w.G;
  const uint16_t* Q = a.Q + (int64_t)w.b * r.sb + (int64_t)w.hk * w.G * r.sh + (int64_t)w.t0 * r.st + cc * 8;
  int i = from + (int)threadIdx.x / CPR, tok = i / w.G, head = i - tok * w.G;
  const int dt = STRIPES / w.G, dh = STRIPES - dt * w.G;       // (a division a row would take longer than the load)
#pragma unroll
  for (int u = 0; u < kQueryRows; ++u) {
    v[u] = make_uint4(0, 0, 0, 0);
    if (i < rows) v[u] = *reinterpret_cast<const uint4*>(Q + head * r.sh + tok * r.st);
    i += STRIPES;
    tok += dt;
    head += dh;
    if (head >= w.G) { head -= w.G; ++tok; }
  }
}
// The row's query in 8 bits, into L.q8 (ends with a barrier); `v`: the first chunk, requested earlier.
template <int D>
__device__ __forceinline__ void sum_queries(const RowDims& r, const CacheSelectArgs& a, const Row& w, uint4 (&v)[kQueryRows], QueryLds<D>& L) {
  constexpr int CPR = D / 8, STRIPES = 256 / CPR;
  const int tid = threadIdx.x, cc = tid % CPR;
  double acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int rows = (w.t1 - w.t0) * w.G;
  for (int from = 0; tid < 256 && from < rows; from += kQueryRows * STRIPES) {
    if (from > 0) request_queries<D>(r, a, w, from, v);
#pragma unroll
    for (int u = 0; u < kQueryRows; ++u) {
      if (from + u * STRIPES >= rows) break;
      if (from + u * STRIPES + tid / CPR >= rows) continue;               // (behind the last query)
      const uint32_t x[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[2 * e] += finite_or_zero(x[e] & 0xffffu);
        acc[2 * e + 1] += finite_or_zero(x[e] >> 16);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (tid < 256) L.sums[tid / CPR][cc * 8 + e] = acc[e];
  __syncthreads();
  if (tid < D) {
    const int stripes = min(rows, STRIPES);        // the others hold zeros
    double s = 0;
#pragma unroll 4
    for (int x = 0; x < stripes; ++x) s += L.sums[x][tid];
    // the least e with max|s| <= 127 * 2^e: by the largest exponent x (max < 2^x), and whether anything passes 127 * 2^(x-7)
    const uint32_t top = (uint32_t)(__builtin_bit_cast(uint64_t, s) >> 52) & 0x7ffu;
    const uint32_t most = (uint32_t)over_wave((int)top, MaxU32());
    if (tid % 64 == 0) L.most[tid / 64] = most;
    L.sums[0][tid] = s;                            // (column tid is this thread's own)
  }
  __syncthreads();
  if (tid < D) {
    const int x = (int)max(L.most[0], L.most[D / 64 - 1]) - 1022;
    bool over = false;
#pragma unroll
    for (int ch = tid % 64; ch < D; ch += 64) over |= fabs(L.sums[0][ch]) > ldexp(127.0, x - 7);
    const int e = max(x - 7 + (__any(over) ? 1 : 0), -100);
    L.q8[tid] = (int8_t)(int)rint(ldexp(L.sums[0][tid], -e));
  }
  __syncthreads();
}

// What a row's scores need and no length decides, requested before the lengths are here (256 rows of 512 blocks 8.3 us without and 7.9
// so, 696 of 929 19.0 and 18.6, both on one box).
template <int NI>
struct Early {
  int page[NI];
  uint4 query[kQueryRows];
};
template <int D, int NI, int W>
__device__ __forceinline__ Early<NI> request_early(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, const Row& w, int from) {
  Early<NI> v;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int m = from + (int)threadIdx.x + 64 * W * i;
    v.page[i] = m < c.max_blocks ? c.table[(int64_t)w.b * c.max_blocks + m] : -1;
  }
  if (threadIdx.x < 256) request_queries<D>(r, a, w, 0, v.query);          // four waves' work
  return v;
}

// Scores of blocks [from, to) of a row, NI to a thread, as order-preserving keys in keys[0 ..) (ends with a barrier). The loads
// take turns in the address unit of the compute unit, so there are few: pages and scales once, a block to a lane, the means 16
// channels to a lane, kRound passes requested together (pages lie anywhere: a round waits some 2500 cycles).
// Pages and scales by the lanes of each mean: 929 blocks of 696 rows 23.7 us, now 19.0.
template <int D, int NI, int W>
__device__ __forceinline__ void score_blocks(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, const Row& w, int from, int to,
                                             Early<NI>& early, QueryLds<D>& L, uint32_t* keys) {
  constexpr int kRound = W == 4 ? 16 : 8;
  constexpr int LPB = D / 16, BPP = 64 * W / LPB;  // lanes to a block, blocks to a pass
  const int tid = threadIdx.x, part = tid % LPB;
  float scale[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int m = tid + 64 * W * i, page = from + m < to && early.page[i] >= 0 && early.page[i] < c.pages ? early.page[i] : -1;
    if (from + m < to) keys[m] = (uint32_t)page;
    scale[i] = -1.f;                               // there is no page; of one that there is the scale has no sign, whatever stands in memory
    if (page >= 0) scale[i] = fabsf(c.scales[((int64_t)page * c.heads_kv + w.hk) * 4 + 2]);
  }
  __syncthreads();
  int page[kRound];
  int4 mean[kRound];
  auto request = [&](int at) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kRound; ++u) {
      const int m = at + u * BPP + tid / LPB;
      page[u] = from + m < to ? (int)keys[m] : -1;
    }
#pragma unroll
    for (int u = 0; u < kRound; ++u) {
      mean[u] = make_int4(0, 0, 0, 0);
      if (page[u] >= 0) mean[u] = *reinterpret_cast<const int4*>(c.mean + ((int64_t)page[u] * c.heads_kv + w.hk) * D + part * 16);
    }
  };
  request(0);
  sum_queries<D>(r, a, w, early.query, L);
  const int4 q = *reinterpret_cast<const int4*>(&L.q8[part * 16]);
  for (int at = 0; from + at < to; at += kRound * BPP) {
    if (at > 0) request(at);
#pragma unroll
    for (int u = 0; u < kRound; ++u) {
      const int m = at + u * BPP + tid / LPB;
      int dot = __builtin_amdgcn_sdot4(q.x, mean[u].x, 0, false);
      dot = __builtin_amdgcn_sdot4(q.y, mean[u].y, dot, false);
      dot = __builtin_amdgcn_sdot4(q.z, mean[u].z, dot, false);
      dot = __builtin_amdgcn_sdot4(q.w, mean[u].w, dot, false);
      dot += row_lane<kXor1>(dot);
      dot += row_lane<kXor2>(dot);
      if (LPB == 8) dot += row_lane<kFlip8>(dot);
      if (part == 0 && from + m < to) keys[m] = (uint32_t)dot;            // in the place of its page, which this wave has read
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int m = tid + 64 * W * i;
    if (from + m < to) {
      // 2^-22 keeps the largest scale finite; the product is exact (|dot| < 2^21)
      const float z = (float)(int)keys[m] * 0x1p-22f * scale[i];
      keys[m] = scale[i] == -1.f ? kUnseen : fabsf(z) <= kLargest ? ordered_key(z) : kLowest;
    }
  }
  __syncthreads();
}

// Scores of a run of blocks, for rows that are few.
template <int D>
__global__ __launch_bounds__(256) void cache_score_kernel(CacheDims c, RowDims r, CacheSelectArgs a, int runs) {
  __shared__ QueryLds<D> L;
  __shared__ uint32_t keys[kRunBlocks];
  const int id = xcd_run(blockIdx.x, gridDim.x), row = id / runs;
  Row w = row_of(c, r, a, row);
  const int kv_len = a.kv_len[w.b], q_len = a.q_len ? a.q_len[w.b] : r.t, from = id % runs * kRunBlocks;
  Early<kRunBlocks / 256> early = request_early<D, kRunBlocks / 256, 4>(c, r, a, w, from);
  add_lengths(c, r, a, kv_len, q_len, w);
  const int to = min(from + kRunBlocks, w.seen);
  if (from >= to) return;
  score_blocks<D, kRunBlocks / 256, 4>(c, r, a, w, from, to, early, L, keys);
  uint32_t* out = (uint32_t*)a.ws + (int64_t)row * c.max_blocks;
  for (int m = from + (int)threadIdx.x; m < to; m += 256) out[m] = keys[m - from];
}

template <int W>
struct ChoiceLds {
  __align__(16) int counts[2][W][4];
  __align__(16) int hist[256];
  int totals[3][W], n_few;
  uint32_t ends[2][W], few[64];
};
// The list of one row from the keys of its blocks, by W waves (NI keys to a thread: rows of up to 64 W NI blocks).
template <int NI, int W>
__device__ __forceinline__ void choose(const CacheSelectArgs& a, const Row& w, int row, const uint32_t* src, ChoiceLds<W>& L) {
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  int32_t* list = a.block_idx + (int64_t)row * a.list_len;
  // this wave's run of blocks, slot i of lane l being block m0 + 64 i + l
  const int m0 = wave * 64 * NI;
  uint32_t key[NI];
  unsigned long long must = 0;                     // bit i: slot i is forced
  int n_seen = 0, n_must = 0;
  uint32_t kmax = 0, nkmin = 0;                    // over the blocks that scores decide on
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int m = m0 + 64 * i + lane;
    key[i] = m < w.seen ? src[m] : kUnseen;
    const bool there = key[i] != kUnseen, forced = there && (m < a.first || (m >= w.lo_forced && m <= w.hi_forced));
    n_seen += __popcll(__ballot(there));
    n_must += __popcll(__ballot(forced));
    if (forced) {
      must |= 1ull << i;
      key[i] = kUnseen;
    }
    kmax = max(kmax, key[i]);
    nkmin = max(nkmin, key[i] != kUnseen ? ~key[i] : 0u);
  }
  kmax = (uint32_t)over_wave((int)kmax, MaxU32());
  nkmin = (uint32_t)over_wave((int)nkmin, MaxU32());
  if (tid < 256) L.hist[tid] = 0;
  if (tid == 0) L.n_few = 0;
  if (lane == 0) {
    L.totals[0][wave] = n_seen;
    L.totals[1][wave] = n_must;
    L.ends[0][wave] = kmax;
    L.ends[1][wave] = nkmin;
  }
  __syncthreads();
  // (a wave's numbers to a lane, W <= 16: over a row of lanes)
  auto of_waves = [&](const auto* x, auto op) __attribute__((always_inline)) { return over_row(lane % 16 < W ? (int)x[lane % 16] : 0, op); };
  n_seen = __builtin_amdgcn_readfirstlane(of_waves(L.totals[0], AddInt()));
  n_must = __builtin_amdgcn_readfirstlane(of_waves(L.totals[1], AddInt()));
  kmax = (uint32_t)__builtin_amdgcn_readfirstlane(of_waves(L.ends[0], MaxU32()));
  const uint32_t kmin = ~(uint32_t)__builtin_amdgcn_readfirstlane(of_waves(L.ends[1], MaxU32()));
  const int want = min(max(a.keep, n_must), n_seen);
  const int by_score = want - n_must;

  // The by_score-th largest key `tau`; kept: key > tau, and `ties` of those equal to it. First a histogram of 256 even steps
  // between the lowest and the highest score, which leaves a few keys to be ranked against each other; where it leaves more
  // than a wave has lanes (equal scores, scales far apart), bit by bit with ballot counts.
  uint32_t tau = 0xffffffffu;
  int ties = 0;
  if (by_score > 0) {
    const float smin = score_of(kmin), range = score_of(kmax) - smin;
    // Scores may be 2^-122 apart (means of 2^-100), where 255 / range passes 32 bits: the factor stays finite, and no score finds a step outside.
    const float steps = range > 0.f && range <= kLargest ? fminf(255.f / range, kLargest) : 0.f;
    auto step_of = [&](uint32_t k) __attribute__((always_inline)) { return min(max((int)((score_of(k) - smin) * steps), 0), 255); };   // monotone
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (key[i] != kUnseen) atomicAdd(&L.hist[step_of(key[i])], 1);
    __syncthreads();
    // in every wave: lane l has steps 255 - 4 l down to 252 - 4 l
    const int4 h = *reinterpret_cast<const int4*>(&L.hist[252 - 4 * lane]);
    const int four = h.x + h.y + h.z + h.w;
    int upto = four;
    upto += row_up<1>(upto);
    upto += row_up<2>(upto);
    upto += row_up<4>(upto);
    upto += row_up<8>(upto);
    const int r0 = __builtin_amdgcn_readlane(upto, 15), r1 = __builtin_amdgcn_readlane(upto, 31), r2 = __builtin_amdgcn_readlane(upto, 47);
    upto += (lane >= 16 ? r0 : 0) + (lane >= 32 ? r1 : 0) + (lane >= 48 ? r2 : 0);
    const int at = __builtin_ctzll(__ballot(upto >= by_score));          // (the last lane counts all keys)
    int above = __builtin_amdgcn_readlane(upto - four, at), step = 255 - 4 * at, n = 0;
    const int h3[4] = {__builtin_amdgcn_readlane(h.w, at), __builtin_amdgcn_readlane(h.z, at), __builtin_amdgcn_readlane(h.y, at),
                       __builtin_amdgcn_readlane(h.x, at)};
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (n == 0 && above + h3[x] >= by_score) {
        step -= x;
        n = h3[x];
      } else if (n == 0) {
        above += h3[x];
      }
    if (n <= 64) {                                 // n keys share the step that holds tau (the same in every wave)
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (key[i] != kUnseen && step_of(key[i]) == step) L.few[atomicAdd(&L.n_few, 1)] = key[i];
      __syncthreads();
      const uint32_t mine = lane < n ? L.few[lane] : kUnseen;              // (their order does not matter)
      int more = 0, same = 0;
      for (int x = 0; x < n; ++x) {
        const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)mine, x);
        more += other > mine;
        same += other == mine;
      }
      const int need = by_score - above;
      const int who = __builtin_ctzll(__ballot(lane < n && more < need && more + same >= need));
      tau = (uint32_t)__builtin_amdgcn_readlane((int)mine, who);
      ties = need - __builtin_amdgcn_readlane(more, who);
    } else {
      // from the highest bit in which keys of the row differ down; done as soon as exactly by_score keys reach a candidate
      const int vary = 32 - __builtin_clz((kmax ^ kmin) | 1u);
      tau = vary >= 32 ? 0u : (kmax >> vary) << vary;
      bool exact = false;
      int over = 0, turn = 0;                      // keys above tau's range so far
      // two bits a turn (three candidates): the turns wait for a barrier, not for the counting
      for (int bit = (vary + 1) / 2 * 2 - 2; bit >= 0 && !exact; bit -= 2, turn ^= 1) {
        int c3[3] = {0, 0, 0};
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int x = 0; x < 3; ++x) c3[x] += __popcll(__ballot(key[i] >= (tau | (uint32_t)(x + 1) << bit)));
        if (lane == 0) *reinterpret_cast<int4*>(&L.counts[turn][wave][0]) = make_int4(c3[0], c3[1], c3[2], 0);
        __syncthreads();                           // (two sets of counts: the next turn writes the other one)
#pragma unroll
        for (int x = 0; x < 3; ++x) c3[x] = __builtin_amdgcn_readfirstlane(over_row(lane % 16 < W ? L.counts[turn][lane % 16][x] : 0, AddInt()));
        const int digit = c3[2] >= by_score ? 3 : c3[1] >= by_score ? 2 : c3[0] >= by_score ? 1 : 0;
        if (digit < 3) over = c3[digit];
        tau |= (uint32_t)digit << bit;
        if (digit > 0 && c3[digit - 1] == by_score) {
          tau -= 1;
          exact = true;
        }
      }
      ties = exact ? 0 : by_score - over;          // equal to tau: the lowest blocks
    }
  }

  // kept blocks, ascending: how many before this wave, then before each slot
  int n_eq = 0;
#pragma unroll
  for (int i = 0; i < NI; ++i) n_eq += ties > 0 ? __popcll(__ballot(key[i] == tau)) : 0;
  if (lane == 0) L.totals[2][wave] = n_eq;
  __syncthreads();
  int eq_left = ties;
  for (int x = 0; x < wave; ++x) eq_left -= min(eq_left, L.totals[2][x]);
  unsigned long long out = 0;
  int n_out = 0;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const bool eq = ties > 0 && key[i] == tau;
    const unsigned long long eqs = __ballot(eq);
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(eqs >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)eqs, 0));
    const bool keep = (must >> i & 1) || (key[i] > tau) || (eq && before < eq_left);
    eq_left -= min(eq_left, (int)__popcll(eqs));
    if (keep) out |= 1ull << i;
    n_out += __popcll(__ballot(keep));
  }
  if (lane == 0) L.ends[0][wave] = (uint32_t)n_out;
  __syncthreads();
  int at = 0;
  for (int x = 0; x < wave; ++x) at += (int)L.ends[0][x];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const bool keep = out >> i & 1;
    const unsigned long long all = __ballot(keep);
    const int to = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
    if (keep && to < want) list[to] = m0 + 64 * i + lane;                  // (want <= list_len: whatever the scores, nothing lands behind the list)
    at += __popcll(all);
  }
  for (int i = want + tid; i < a.list_len; i += 64 * W) list[i] = -1;
  if (tid == 0) a.kept[row] = want;
}

// SCORED: the keys are in the workspace.
template <int D, int NI, int W, bool SCORED>
__global__ __launch_bounds__(64 * W) void cache_select_kernel(CacheDims c, RowDims r, CacheSelectArgs a) {
  __shared__ QueryLds<D> L;
  __shared__ ChoiceLds<W> choice;
  __shared__ uint32_t keys[SCORED ? 1 : 64 * W * NI];
  const int tid = threadIdx.x, row = xcd_run(blockIdx.x, gridDim.x);
  Row w = row_of(c, r, a, row);
  const int kv_len = a.kv_len[w.b], q_len = a.q_len ? a.q_len[w.b] : r.t;
  Early<SCORED ? 1 : NI> early;
  if constexpr (!SCORED) early = request_early<D, NI, W>(c, r, a, w, 0);
  add_lengths(c, r, a, kv_len, q_len, w);
  if (w.seen <= 0) {                               // nothing to choose from (the whole workgroup)
    for (int i = tid; i < a.list_len; i += 64 * W) a.block_idx[(int64_t)row * a.list_len + i] = -1;
    if (tid == 0) a.kept[row] = 0;
    return;
  }
  if constexpr (!SCORED) score_blocks<D, NI, W>(c, r, a, w, 0, w.seen, early, L, keys);
  choose<NI, W>(a, w, row, SCORED ? (const uint32_t*)a.ws + (int64_t)row * c.max_blocks : keys, choice);
}

// A launch for the scores where the rows leave most compute units idle and a row has several runs of blocks. One launch and
// two, us: 8 rows of 16 384 blocks 61 and 37, of 4096 16.8 and 15.8, of 2049 13.2 and 15.1; 64 rows of 8192 45 and 33, of 4096
// 22.4 and 19.7, of 2049 13.9 and 15.9; 120 rows of 8192 47 and 44, of 4096 24.3 and 24.2; 200 rows of 4096 28 and 33.
bool scores_apart(const CacheDims& c, int64_t rows) { return rows < 100 && c.max_blocks >= 4 * kRunBlocks; }

template <int D>
hipError_t launch_t(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.groups * c.batch * c.heads_kv;
  const dim3 grid((uint32_t)rows), block(256);
  const bool apart = a.ws && scores_apart(c, rows);
  if (apart) {
    const int runs = (c.max_blocks + kRunBlocks - 1) / kRunBlocks;
    hipLaunchKernelGGL((cache_score_kernel<D>), dim3((uint32_t)(rows * runs)), block, 0, s, c, r, a, runs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (c.max_blocks <= 4096) hipLaunchKernelGGL((cache_select_kernel<D, 4, 16, true>), grid, dim3(1024), 0, s, c, r, a);
    else hipLaunchKernelGGL((cache_select_kernel<D, 16, 16, true>), grid, dim3(1024), 0, s, c, r, a);
    return hipGetLastError();
  }
  if (c.max_blocks <= 512) hipLaunchKernelGGL((cache_select_kernel<D, 2, 4, false>), grid, block, 0, s, c, r, a);
  else if (c.max_blocks <= 1024) hipLaunchKernelGGL((cache_select_kernel<D, 4, 4, false>), grid, block, 0, s, c, r, a);
  else if (c.max_blocks <= 4096) hipLaunchKernelGGL((cache_select_kernel<D, 4, 16, false>), grid, dim3(1024), 0, s, c, r, a);
  else hipLaunchKernelGGL((cache_select_kernel<D, 16, 16, false>), grid, dim3(1024), 0, s, c, r, a);
  return hipGetLastError();
}

}  // namespace

size_t cache_select_ws_bytes(const CacheDims& c, const RowDims& r, int group) {
  const int per = group > 0 && group < r.t ? group : r.t;
  const int64_t rows = (int64_t)((r.t + per - 1) / per) * c.batch * c.heads_kv;
  return c.max_blocks <= RSA_CACHE_MAX_SELECT && scores_apart(c, rows) ? (size_t)rows * c.max_blocks * sizeof(uint32_t) : 0;
}

hipError_t launch_cache_select(const CacheDims& c, const RowDims& r, const CacheSelectArgs& a, hipStream_t s) {
  return c.d == 128 ? launch_t<128>(c, r, a, s) : launch_t<64>(c, r, a, s);
}

}  // namespace rsa
