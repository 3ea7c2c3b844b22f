// Pages for the new tokens of every sequence, from the lengths alone, so that a captured step advances its own tables.
//
// One workgroup does the part that is a chain: pages that sequences give back go on the free list in the order of the sequences
// (a prefix sum of how many each returns), then pages are taken from its end in that order (a prefix sum of how many each needs);
// a sequence whose sum is over the list's length gets none, so who is served does not depend on timing. Positions and slots of
// the new rows need only start, count and the table: the same workgroup writes few of them, many are a launch of their own.
// Bound by latency: lengths, sums, free list, table, slot, each waiting for the one before. A token for each of 32 sequences 3.0 us (5.7 with
// sums by exchanges through LDS in 64 bits and 1024 threads whatever the batch), 48 prompts of 4096 tokens 8.3 in two launches (17.0 with one
// wave for all of their pages), one of 240 000 tokens 8.2 (13.8 with one wave to a sequence).
#include "serve_common.hpp"

namespace rsa {
namespace {

constexpr int kMostThreads = 1024;
// Rows of positions and slots that the one workgroup writes itself (8000 rows: 9.8 us by itself, 7.4 with the second launch).
constexpr int64_t kFewRows = 4096;

// Sum of `x` over the lanes of the wave up to this one, by exchanges on the vector ALU.
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);        // a lane, two, four, eight to the right in rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);        // the last of a row to the next one
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);        // of the first half to the second
  return x;
}
// Sum of `x` >= 0 over the threads up to this one; `all`: over all threads. Every thread of the workgroup calls it. A table has fewer than 2^31
// entries, so a wave's sum fits 31 bits; those of the waves are added in 64.
__device__ __forceinline__ int64_t prefix(int x, int* lds, int64_t* all) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
  const int own = wave_prefix(x);
  if (waves == 1) {
    *all = __builtin_amdgcn_readlane(own, 63);
    return own;
  }
  __syncthreads();                                 // (what an earlier call left in lds has been read)
  if (lane == 63) lds[wave] = own;
  __syncthreads();
  int64_t before = 0, total = 0;
  for (int w = 0; w < waves; ++w) {
    const int y = lds[w];
    before += w < wave ? y : 0;
    total += y;
  }
  *all = total;
  return before + own;
}

struct Want { int held, to, had, need; bool fits; };   // tokens now and then, blocks now and then; fits: within the table, and in no page of others
__device__ __forceinline__ Want want_of(const AssignArgs& a, int b) {
  Want w;
  const int64_t cap = (int64_t)a.max_blocks * a.block;
  w.held = (int)min((int64_t)max(a.kv_len[b], 0), cap);
  const int64_t to = (int64_t)w.held + min(a.add[b], a.t);
  w.had = (int)(((int64_t)w.held + a.block - 1) / a.block);
  // (new tokens of a sequence that ends inside a block of its shared prefix would go into the page that others read)
  w.fits = to <= cap && !(a.shared && to > w.held && (int64_t)w.had * a.block != w.held && w.had <= a.shared[b]);
  w.to = (int)(w.fits ? max(to, (int64_t)0) : w.held);
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

__global__ __launch_bounds__(kMostThreads) void assign_kernel(AssignArgs a) {
  __shared__ int lds[kMostThreads / 64];
  __shared__ int more_of[kMostThreads], had_of[kMostThreads], held_of[kMostThreads], count_of[kMostThreads];
  __shared__ int64_t top_of[kMostThreads];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, threads = blockDim.x, waves = threads / 64;
  const int rounds = (a.batch + threads - 1) / threads;
  const int64_t free0 = min((int64_t)max(a.free_count[0], 0), a.pages);

  // pages given back, in the order of the sequences
  int64_t freed = 0;
  Want w = {0, 0, 0, 0, true};
  int add = 0;
  auto look = [&](int q) __attribute__((always_inline)) {
    const int b = q * threads + tid;
    w = {0, 0, 0, 0, true};
    add = 0;
    if (b < a.batch) {
      w = want_of(a, b);
      add = min(a.add[b], a.t);
    }
  };
  for (int q = 0; q < rounds; ++q) {
    look(q);
    const int lo = w.need, hi = w.had;             // entries of the table that the sequence gives up; those below `own` are another's
    if (!__syncthreads_or(lo < hi)) continue;
    const int own = a.shared && lo < hi ? a.shared[q * threads + tid] : 0;
    int back = 0;
    for (unsigned long long some = __ballot(lo < hi); some; some &= some - 1) {     // a wave counts its sequences' pages one by one
      const int k = __builtin_ctzll(some);
      const int l = __shfl(lo, k), h = __shfl(hi, k), o = __shfl(own, k);
      const int32_t* row = a.table + (int64_t)(q * threads + tid - lane + k) * a.max_blocks;
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
      int32_t* row = a.table + (int64_t)(q * threads + tid - lane + k) * a.max_blocks;
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
  if (freed > 0) __syncthreads();                  // the list is whole

  // pages taken, from the end of the list
  int64_t asked = 0, taken = 0;
  for (int q = 0; q < rounds; ++q) {
    const int b = q * threads + tid;
    if (rounds > 1) look(q);
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
      if (granted && more > 0 && a.shared && a.shared[b] > w.had) a.shared[b] = w.had;    // from here on the pages are its own
    }
    // Pages by whole waves, a sequence each, but for few pages to a sequence; a single new token finds its page on the way.
    const bool few = granted && more <= 4, many = granted && more > 4;
    const bool one = a.t == 1 && b < a.batch;
    int page = -1;
    if (one && n == 1 && more == 0) page = a.table[(int64_t)b * a.max_blocks + w.held / a.block];
    if (few)
      for (int e = 0; e < more; ++e) {
        const int p = a.free_pages[top - e];
        a.table[(int64_t)b * a.max_blocks + w.had + e] = p;
        if (one) page = p;
      }
    if (one) {
      if (a.positions) a.positions[b] = n == 1 ? w.held : -1;
      if (a.slots) a.slots[b] = n == 1 && page >= 0 && page < a.pages ? (int64_t)page * a.block + w.held % a.block : -1;
    }
    if (__syncthreads_or(many)) {
      more_of[tid] = many ? more : 0;
      had_of[tid] = w.had;
      top_of[tid] = top;
      __syncthreads();
      const int here = min(threads, a.batch - q * threads), share = 31 - __builtin_clz(max(waves / here, 1));      // 2^share waves to a sequence
      for (int k = wave >> share; k < here; k += waves >> share) {
        int32_t* row = a.table + (int64_t)(q * threads + k) * a.max_blocks + had_of[k];
        const int64_t from = top_of[k];
        for (int e = (wave & ((1 << share) - 1)) * 64 + lane; e < more_of[k]; e += 64 << share) row[e] = a.free_pages[from - e];
      }
      __syncthreads();
    }
    // (who is granted, of those that need pages, are the first ones)
    if (asked + all <= have) {
      taken += all;
    } else {
      int64_t sum;
      prefix(granted ? more : 0, lds, &sum);
      taken += sum;
    }
    asked += all;
    if (rounds == 1 && tid < a.batch) {
      held_of[tid] = w.held;
      count_of[tid] = n;
    }
  }
  if (tid == 0) a.free_left[0] = (int32_t)(have - taken);
  if ((int64_t)a.batch * a.t > kFewRows || a.t == 1 || (!a.positions && !a.slots)) return;       // (the whole workgroup)
  __syncthreads();
  for (int u = tid; u < a.batch * a.t; u += threads) {
    const int b = u / a.t;
    place(a, b, u % a.t, rounds == 1 ? held_of[b] : a.start[b], rounds == 1 ? count_of[b] : a.count[b]);
  }
}

__global__ __launch_bounds__(256) void place_kernel(AssignArgs a) {
  const int per = (a.t + 255) / 256;
  const int b = blockIdx.x / per, i = blockIdx.x % per * 256 + threadIdx.x;
  if (i < a.t) place(a, b, i, a.start[b], a.count[b]);
}

}  // namespace

hipError_t launch_assign(const AssignArgs& a, hipStream_t s) {
  // a thread for each sequence and for each row that the workgroup places, in whole waves
  const int64_t rows = (int64_t)a.batch * a.t, want = rows > kFewRows ? kMostThreads : a.batch > rows ? a.batch : rows;
  const int threads = want > kMostThreads ? kMostThreads : (int)((want + 63) / 64 * 64);
  hipLaunchKernelGGL(assign_kernel, dim3(1), dim3(threads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || rows <= kFewRows || a.t == 1 || (!a.positions && !a.slots)) return e;
  hipLaunchKernelGGL(place_kernel, dim3((uint32_t)((int64_t)a.batch * ((a.t + 255) / 256))), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rsa
