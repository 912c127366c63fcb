// Steps planned on the GPU: pages from a pool's free stack for new tokens, the
// step's page table, lengths, slots and positions, and pages given back.
//
// Two launches: plan_scan, one workgroup, decides whether the step fits, sums up
// the entries before each and moves the pool's lengths and stack; plan_fill
// writes the tables and tokens.  Every sum has one order, so a step's pages are
// those that a host loop over the entries would pop.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8_rows.h"
#include "wave_ops.h"

namespace cs {

struct PoolView {
  int32_t* table;
  int32_t* lengths;
  int32_t* free_pages;
  int32_t* count;
  int32_t* marks;
  int sequences, width, pages, page_log;
};

struct PlanStep {
  PoolView p;
  const int32_t* seqs;
  const int32_t* fresh;
  int batch;
  int32_t* table;
  int table_width;
  int32_t* lens;
  int32_t* starts;
  int64_t* slots;
  int32_t* positions;
  int64_t tokens;
  int32_t* status;
  int32_t* head;       // ws: [0] stack's count before the step, [1] 1 where it is planned
  int32_t* before;     // ws: [batch] new pages of the entries before
};

constexpr int kPlanThreads = 1024;
constexpr int32_t kNoMark = 0x7FFFFFFF;

__device__ __forceinline__ int pages_of(int64_t length, int page_log) {
  return (int)((length + (1 << page_log) - 1) >> page_log);
}

// Sums of the lanes before, over a workgroup of kPlanThreads; *all: of all lanes.
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* l_part, uint32_t* all) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t incl = wave_incl_scan(v, 0u, OpAdd{});
  __syncthreads();                                         // l_part is free again
  if (lane == 63) l_part[wave] = incl;
  __syncthreads();
  uint32_t base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const uint32_t s = l_part[w];
    base += w < wave ? s : 0u;
    sum += s;
  }
  *all = sum;
  return base + incl - v;
}

// A load that other lanes' atomics before the last barrier have reached.
__device__ __forceinline__ int32_t load_mark(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_mark(int32_t* p) {
  __hip_atomic_store(p, kNoMark, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Entries mark their sequences with their numbers, the lowest wins: an entry
// whose sequence bears another mark names one that an earlier entry has named.
__device__ __forceinline__ void mark_entries(const PoolView& p, const int32_t* seqs, int batch) {
  for (int i = threadIdx.x; i < batch; i += kPlanThreads) {
    const int32_t s = seqs[i];
    if (s >= 0 && s < p.sequences) atomicMin(&p.marks[s], i);
  }
  __threadfence();
  __syncthreads();
}

__global__ __launch_bounds__(kPlanThreads) void plan_scan(PlanStep a) {
  __shared__ unsigned long long l_tokens, l_pages;
  __shared__ int l_wrong;
  __shared__ uint32_t l_part[kPlanThreads / 64];
  const int tid = threadIdx.x, lg = a.p.page_log;
  if (tid == 0) {
    l_tokens = l_pages = 0;
    l_wrong = kNoMark;
  }
  mark_entries(a.p, a.seqs, a.batch);
  const int64_t most = (int64_t)min(a.p.width, a.table_width) << lg;
  const int count = min(*a.p.count, a.p.pages);
  // an entry's sequence, length before and new tokens; false where it is wrong
  auto entry = [&](int i, int32_t* s, int* old, int* n) {
    *s = a.seqs[i];
    *old = *n = 0;
    if (*s == -1) return true;
    if (*s < 0 || *s >= a.p.sequences || load_mark(&a.p.marks[*s]) != i) return false;
    *old = a.p.lengths[*s];
    *n = a.fresh[i];
    return *n >= 0 && *old >= 0 && (int64_t)*old + *n <= most;
  };
  for (int i = tid; i < a.batch; i += kPlanThreads) {
    int32_t s;
    int old, n;
    if (entry(i, &s, &old, &n)) {
      if (n > 0) {
        atomicAdd(&l_tokens, (unsigned long long)n);
        atomicAdd(&l_pages,
                  (unsigned long long)(pages_of((int64_t)old + n, lg) - pages_of(old, lg)));
      }
    } else {
      atomicMin(&l_wrong, i);
    }
  }
  __syncthreads();
  const int64_t short_tokens = (int64_t)l_tokens - a.tokens;
  const int64_t short_pages = (int64_t)l_pages - count;
  const int code = l_wrong != kNoMark ? 1 : short_tokens > 0 ? 2 : short_pages > 0 ? 3 : 0;
  const int64_t told = code == 1 ? l_wrong : code == 2 ? short_tokens : code == 3 ? short_pages : 0;
  uint32_t tokens = 0, pages = 0;                          // of the entries before
  for (int i0 = 0; i0 < a.batch; i0 += kPlanThreads) {
    const int i = i0 + tid;
    int32_t s = -1;
    int old = 0, n = 0;
    const bool there = i < a.batch;
    if (there && code == 0) entry(i, &s, &old, &n);
    const int need = pages_of((int64_t)old + n, lg) - pages_of(old, lg);
    uint32_t all_n, all_need;
    const uint32_t at = tokens + block_before((uint32_t)n, l_part, &all_n);
    const uint32_t page = pages + block_before((uint32_t)need, l_part, &all_need);
    if (there) {
      a.starts[i] = (int32_t)at;
      a.lens[i] = old + n;
      a.before[i] = (int32_t)page;
      if (s >= 0) a.p.lengths[s] = old + n;
    }
    tokens += all_n;
    pages += all_need;
  }
  for (int i = tid; i < a.batch; i += kPlanThreads) {
    const int32_t s = a.seqs[i];
    if (s >= 0 && s < a.p.sequences) store_mark(&a.p.marks[s]);
  }
  if (tid == 0) {
    a.starts[a.batch] = (int32_t)tokens;
    a.head[0] = count;
    a.head[1] = code == 0;
    *a.p.count = count - (int)pages;
    a.status[0] = code;
    a.status[1] = (int32_t)min(told, (int64_t)0x7FFFFFFF);
  }
}

// Cells of the table first, a cell to a thread, then tokens.
__global__ __launch_bounds__(256) void plan_fill(PlanStep a) {
  const int64_t id = (int64_t)workgroup() * 256 + threadIdx.x;
  const int64_t cells = (int64_t)a.batch * a.table_width;
  const int lg = a.p.page_log, count = a.head[0];
  const bool planned = a.head[1] != 0;
  auto fresh_page = [&](int entry, int x) {                // x: of the entry's new pages
    const int at = count - 1 - (a.before[entry] + x);
    return a.p.free_pages[at];
  };
  if (id < cells) {
    const int i = (int)(id / a.table_width), c = (int)(id - (int64_t)i * a.table_width);
    int32_t page = -1;
    const int32_t s = a.seqs[i];
    if (planned && s >= 0) {
      const int len = a.lens[i], n = a.starts[i + 1] - a.starts[i];
      const int held = pages_of(len - n, lg);
      if (c < held) {
        page = a.p.table[(int64_t)s * a.p.width + c];
      } else if (c < pages_of(len, lg)) {
        page = fresh_page(i, c - held);
        a.p.table[(int64_t)s * a.p.width + c] = page;
      }
    }
    a.table[id] = page;
    return;
  }
  const int64_t t = id - cells;
  if (t >= a.tokens) return;
  int64_t slot = -1;
  int32_t pos = -1;
  if (planned && t < a.starts[a.batch]) {
    int lo = 0, hi = a.batch;                              // starts[lo] <= t < starts[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.starts[mid] <= t) lo = mid;
      else hi = mid;
    }
    const int n = a.starts[lo + 1] - a.starts[lo], old = a.lens[lo] - n;
    pos = old + (int)(t - a.starts[lo]);
    const int x = pos >> lg, held = pages_of(old, lg);
    const int32_t page = x < held ? a.p.table[(int64_t)a.seqs[lo] * a.p.width + x]
                                  : fresh_page(lo, x - held);
    slot = ((int64_t)page << lg) + (pos & ((1 << lg) - 1));
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
}

// Pages past the new lengths back onto the stack: entry after entry from the
// top down, so one workgroup adds up how many there are and then moves them.
__global__ __launch_bounds__(kPlanThreads) void pool_truncate(PoolView p, const int32_t* seqs,
                                                              const int32_t* lens, int batch) {
  __shared__ uint32_t l_part[kPlanThreads / 64];
  __shared__ int l_first[kPlanThreads], l_keep[kPlanThreads], l_seq[kPlanThreads];
  const int tid = threadIdx.x, lg = p.page_log;
  mark_entries(p, seqs, batch);
  auto entry = [&](int i, int32_t* s, int* old, int* now) {
    *s = i < batch ? seqs[i] : -1;
    *old = *now = 0;
    if (*s < 0 || *s >= p.sequences || load_mark(&p.marks[*s]) != i) return false;
    *old = p.lengths[*s];
    *now = lens ? lens[i] : 0;
    if (*now < 0 || *now > *old || pages_of(*old, lg) > p.width) {
      *now = *old;
      return false;
    }
    return true;
  };
  const int count = *p.count;
  uint32_t total = 0;
  for (int i0 = 0; i0 < batch; i0 += kPlanThreads) {
    int32_t s;
    int old, now;
    uint32_t all = 0;
    const bool good = entry(i0 + tid, &s, &old, &now);
    block_before(good ? (uint32_t)(pages_of(old, lg) - pages_of(now, lg)) : 0u, l_part, &all);
    total += all;
  }
  uint32_t base = 0;
  for (int i0 = 0; i0 < batch; i0 += kPlanThreads) {
    int32_t s;
    int old, now;
    uint32_t all = 0;
    const bool good = entry(i0 + tid, &s, &old, &now);
    const int keep = pages_of(now, lg);
    const uint32_t drop = good ? (uint32_t)(pages_of(old, lg) - keep) : 0u;
    l_first[tid] = (int)block_before(drop, l_part, &all);
    l_keep[tid] = keep;
    l_seq[tid] = s;
    __syncthreads();
    for (uint32_t x = tid; x < all; x += kPlanThreads) {
      int lo = 0, hi = kPlanThreads;                       // the last entry that starts at or before x
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((uint32_t)l_first[mid] <= x) lo = mid;
        else hi = mid;
      }
      const int64_t to = (int64_t)count + total - 1 - base - x;
      const int from = l_keep[lo] + (int)(x - (uint32_t)l_first[lo]);
      if (to >= 0 && to < p.pages) p.free_pages[to] = p.table[(int64_t)l_seq[lo] * p.width + from];
    }
    if (good) p.lengths[s] = now;
    base += all;
    __syncthreads();
  }
  for (int i = tid; i < batch; i += kPlanThreads) {
    const int32_t s = seqs[i];
    if (s >= 0 && s < p.sequences) store_mark(&p.marks[s]);
  }
  if (tid == 0) *p.count = (int)min((int64_t)count + total, (int64_t)p.pages);
}

}  // namespace cs
