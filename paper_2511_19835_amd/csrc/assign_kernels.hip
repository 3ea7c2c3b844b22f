// Pages for the new tokens of every sequence, from the lengths alone, so that a captured step advances its own tables.
//
// One workgroup does the part that is a chain: pages that sequences give back go on the free list in the order of the sequences
// (a prefix sum of how many each returns), then pages are taken from its end in that order (a prefix sum of how many each needs);
// a sequence whose sum is over the list's length gets none, so who is served does not depend on timing. Positions and slots of
// the new rows need only start, count and the table: the same workgroup writes few of them, many are a launch of their own.
// Bound by latency: lengths, free list, table, slot, each waiting for the one before.
#include "serve_common.hpp"

namespace rsa {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
// Rows of positions and slots that the one workgroup writes itself.
constexpr int64_t kFewRows = 8192;

// Sum of `x` over the threads up to this one; `all`: over all threads. Every thread of the workgroup calls it.
__device__ __forceinline__ int64_t prefix(int64_t x, int64_t* lds, int64_t* all) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int64_t y = __shfl_up((long long)x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                                 // (what an earlier call left in lds has been read)
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int64_t before = 0, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    const int64_t y = lds[w];
    before += w < wave ? y : 0;
    total += y;
  }
  *all = total;
  return before + x;
}

struct Want { int held, to, had, need; bool fits; };   // tokens now and then, blocks now and then; fits: within the table
__device__ __forceinline__ Want want_of(const AssignArgs& a, int b) {
  Want w;
  const int64_t cap = (int64_t)a.max_blocks * a.block;
  w.held = (int)min((int64_t)max(a.kv_len[b], 0), cap);
  const int64_t to = (int64_t)w.held + min(a.add[b], a.t);
  w.fits = to <= cap;
  w.to = (int)(w.fits ? max(to, (int64_t)0) : w.held);
  w.had = (int)(((int64_t)w.held + a.block - 1) / a.block);
  w.need = (int)(((int64_t)w.to + a.block - 1) / a.block);
  return w;
}

__device__ __forceinline__ void place(const AssignArgs& a, int b, int i, int held, int n) {
  const int64_t at = (int64_t)b * a.t + i;
  const bool is = i < n;
  const int pos = held + i;
  if (a.positions) a.positions[at] = is ? pos : -1;
  if (a.slots) {
    int64_t slot = -1;
    if (is) {
      const int page = a.table[(int64_t)b * a.max_blocks + pos / a.block];
      if (page >= 0 && page < a.pages) slot = (int64_t)page * a.block + pos % a.block;
    }
    a.slots[at] = slot;
  }
}

__global__ __launch_bounds__(kThreads) void assign_kernel(AssignArgs a) {
  __shared__ int64_t lds[kWaves];
  const int tid = threadIdx.x, lane = tid % 64;
  const int64_t rounds = ((int64_t)a.batch + kThreads - 1) / kThreads;
  const int64_t free0 = min((int64_t)max(a.free_count[0], 0), a.pages);

  // pages given back, in the order of the sequences
  int64_t freed = 0;
  for (int64_t q = 0; q < rounds; ++q) {
    const int64_t b = q * kThreads + tid;
    int lo = 0, hi = 0;                            // entries of the table that the sequence gives up; those below `own` are another's
    int own = 0;
    if (b < a.batch) {
      const Want w = want_of(a, (int)b);
      lo = w.need;
      hi = w.had;
      own = a.shared ? a.shared[b] : 0;
    }
    if (!__syncthreads_or(lo < hi)) continue;
    int64_t back = 0;
    for (unsigned long long some = __ballot(lo < hi); some; some &= some - 1) {     // a wave counts its sequences' pages one by one
      const int k = __builtin_ctzll(some);
      const int l = __shfl(lo, k), h = __shfl(hi, k), o = __shfl(own, k);
      const int32_t* row = a.table + (q * kThreads + tid - lane + k) * a.max_blocks;
      int n = 0;
      for (int e = l; e < h; e += 64) {
        const int p = e + lane < h ? row[e + lane] : -1;
        n += __popcll(__ballot(p >= 0 && p < a.pages && e + lane >= o));
      }
      if (lane == k) back = n;
    }
    int64_t all;
    const int64_t at0 = free0 + freed + prefix(back, lds, &all) - back;
    for (unsigned long long some = __ballot(lo < hi); some; some &= some - 1) {
      const int k = __builtin_ctzll(some);
      const int l = __shfl(lo, k), h = __shfl(hi, k), o = __shfl(own, k);
      int64_t at = __shfl((long long)at0, k);
      int32_t* row = a.table + (q * kThreads + tid - lane + k) * a.max_blocks;
      for (int e = l; e < h; e += 64) {
        const int p = e + lane < h ? row[e + lane] : -1;
        const bool is = p >= 0 && p < a.pages && e + lane >= o;
        const unsigned long long m = __ballot(is);
        const int64_t to = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
        if (is && to < a.pages) a.free_pages[to] = p;
        if (e + lane < h) row[e + lane] = -1;
        at += __popcll(m);
      }
    }
    freed += all;
  }
  const int64_t have = min(free0 + freed, a.pages);
  __syncthreads();                                 // the list is whole

  // pages taken, from the end of the list
  int64_t asked = 0, taken = 0;
  for (int64_t q = 0; q < rounds; ++q) {
    const int64_t b = q * kThreads + tid;
    Want w = {0, 0, 0, 0, true};
    int add = 0;
    if (b < a.batch) {
      w = want_of(a, (int)b);
      add = min(a.add[b], a.t);
    }
    const int more = max(w.need - w.had, 0);
    int64_t all;
    const int64_t upto = asked + prefix(more, lds, &all);
    const bool granted = w.fits && (more == 0 || upto <= have);
    const int64_t top = have - 1 - (upto - more);  // its first page
    const int n = granted && add > 0 ? add : 0;
    if (b < a.batch) {
      a.kv_new[b] = granted ? w.to : w.held;
      a.start[b] = add < 0 ? w.to : w.held;
      a.count[b] = n;
    }
    const bool few = granted && more <= 4;
    if (few)
      for (int e = 0; e < more; ++e) a.table[b * a.max_blocks + w.had + e] = a.free_pages[top - e];
    for (unsigned long long some = __ballot(granted && !few); some; some &= some - 1) {
      const int k = __builtin_ctzll(some);
      const int m = __shfl(more, k), had = __shfl(w.had, k);
      const int64_t from = __shfl((long long)top, k);
      int32_t* row = a.table + (q * kThreads + tid - lane + k) * a.max_blocks + had;
      for (int e = lane; e < m; e += 64) row[e] = a.free_pages[from - e];
    }
    // (needs are never negative: who is granted, those that need pages, are the first ones)
    int64_t sum;
    prefix(granted ? more : 0, lds, &sum);
    taken += sum;
    asked += all;
  }
  if (tid == 0) a.free_left[0] = (int32_t)(have - taken);
  if ((int64_t)a.batch * a.t > kFewRows) return;   // (the whole workgroup)
  __syncthreads();
  for (int u = tid; u < a.batch * a.t; u += kThreads) place(a, u / a.t, u % a.t, a.start[u / a.t], a.count[u / a.t]);
}

__global__ __launch_bounds__(256) void place_kernel(AssignArgs a) {
  const int per = (a.t + 255) / 256;
  const int b = blockIdx.x / per, i = blockIdx.x % per * 256 + threadIdx.x;
  if (i < a.t) place(a, b, i, a.start[b], a.count[b]);
}

}  // namespace

hipError_t launch_assign(const AssignArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(assign_kernel, dim3(1), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (int64_t)a.batch * a.t <= kFewRows || (!a.positions && !a.slots)) return e;
  hipLaunchKernelGGL(place_kernel, dim3((uint32_t)((int64_t)a.batch * ((a.t + 255) / 256))), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rsa
