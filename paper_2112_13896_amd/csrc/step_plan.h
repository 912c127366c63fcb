// Steps planned on the GPU: pages from a pool's free stack for new tokens, the
// step's page table, lengths, slots and positions, and pages given back.
//
// One workgroup decides whether the step fits, sums up the entries before each
// and moves the pool's lengths and stack; the tables and tokens are written by
// it too where they are few, by a second launch where they are many.  Every sum
// has one order, so a step's pages are those that a host loop over the entries
// would pop.
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

// Sums of the threads before (modulo 2^32), over a workgroup of kPlanThreads;
// *all: of all threads, in 64 bits.  v is below 2^31.
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint64_t* l_part, uint64_t* all) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  // 64 halves of 16 bits fit 32
  const uint32_t lo = wave_incl_scan(v & 0xFFFFu, 0u, OpAdd{});
  const uint32_t hi = wave_incl_scan(v >> 16, 0u, OpAdd{});
  __syncthreads();                                         // l_part is free again
  if (lane == 63) l_part[wave] = ((uint64_t)hi << 16) + lo;
  __syncthreads();
  uint64_t base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const uint64_t s = l_part[w];
    base += w < wave ? s : 0u;
    sum += s;
  }
  *all = sum;
  return (uint32_t)base + ((hi << 16) + lo) - v;
}

// A load that other lanes' atomics before the last barrier have reached.
__device__ __forceinline__ int32_t load_mark(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_mark(int32_t* p) {
  __hip_atomic_store(p, kNoMark, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Which entries name a sequence that an earlier entry has named.  Up to a
// workgroup's threads, an entry to a thread, they meet in a table in LDS: a
// sequence's slot holds the lowest number of its entries (the scan of 1,001
// entries 11 us with it, 16 with marks in memory, whose every step waits for the
// L2 and further).
constexpr int kSlots = 2 * kPlanThreads;
struct Named {
  int32_t seq[kSlots];                                     // -1: free
  int32_t first[kSlots];
};

// (every thread of the workgroup calls this; seq -1: none)
__device__ __forceinline__ bool named_before(Named& t, int32_t seq, int entry) {
  for (int i = threadIdx.x; i < kSlots; i += kPlanThreads) {
    t.seq[i] = -1;
    t.first[i] = kNoMark;
  }
  __syncthreads();
  uint32_t at = ((uint32_t)seq * 2654435761u) % kSlots;    // (at most half of the slots are taken)
  if (seq >= 0) {
    for (;;) {
      const int32_t was = atomicCAS(&t.seq[at], -1, seq);
      if (was == -1 || was == seq) break;
      at = (at + 1) % kSlots;
    }
    atomicMin(&t.first[at], entry);
  }
  __syncthreads();
  return seq >= 0 && t.first[at] != entry;
}

// More entries mark their sequences in memory with their numbers, the lowest
// wins.
__device__ __forceinline__ void mark_entries(const PoolView& p, const int32_t* seqs, int batch) {
  for (int i = threadIdx.x; i < batch; i += kPlanThreads) {
    const int32_t s = seqs[i];
    if (s >= 0 && s < p.sequences) atomicMin(&p.marks[s], i);
  }
  __threadfence();
  __syncthreads();
}
__device__ __forceinline__ void clear_marks(const PoolView& p, const int32_t* seqs, int batch) {
  for (int i = threadIdx.x; i < batch; i += kPlanThreads) {
    const int32_t s = seqs[i];
    if (s >= 0 && s < p.sequences) store_mark(&p.marks[s]);
  }
}

// What the cells of the table and the tokens come from.
struct Planned {
  const int32_t* starts;                                   // [batch + 1]
  const int32_t* lens;                                     // [batch]
  const int32_t* before;                                   // [batch]
  int count;                                               // of the stack before the step
  bool planned;
};

__device__ __forceinline__ int32_t fresh_page(const PlanStep& a, const Planned& f, int entry,
                                              int x) {      // x: of the entry's new pages
  return a.p.free_pages[f.count - 1 - (f.before[entry] + x)];
}

__device__ __forceinline__ void plan_cell(const PlanStep& a, const Planned& f, int64_t id) {
  const int i = (int)((uint32_t)id / (uint32_t)a.table_width);
  const int c = (int)(id - (int64_t)i * a.table_width);
  int32_t page = -1;
  const int32_t s = a.seqs[i];
  if (f.planned && s >= 0) {
    const int len = f.lens[i], n = f.starts[i + 1] - f.starts[i];
    const int held = pages_of(len - n, a.p.page_log);
    if (c < held) {
      page = a.p.table[(int64_t)s * a.p.width + c];
    } else if (c < pages_of(len, a.p.page_log)) {
      page = fresh_page(a, f, i, c - held);
      a.p.table[(int64_t)s * a.p.width + c] = page;
    }
  }
  a.table[id] = page;
}

__device__ __forceinline__ void plan_token(const PlanStep& a, const Planned& f, int64_t t) {
  int64_t slot = -1;
  int32_t pos = -1;
  if (f.planned && t < f.starts[a.batch]) {
    int lo = 0, hi = a.batch;                              // starts[lo] <= t < starts[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (f.starts[mid] <= t) lo = mid;
      else hi = mid;
    }
    const int lg = a.p.page_log, n = f.starts[lo + 1] - f.starts[lo], old = f.lens[lo] - n;
    pos = old + (int)(t - f.starts[lo]);
    const int x = pos >> lg, held = pages_of(old, lg);
    const int32_t page = x < held ? a.p.table[(int64_t)a.seqs[lo] * a.p.width + x]
                                  : fresh_page(a, f, lo, x - held);
    slot = ((int64_t)page << lg) + (pos & ((1 << lg) - 1));
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
}

// plan_scan: SMALL, an entry to a thread (batch <= kPlanThreads), each read once;
// FILL, this workgroup also writes the cells and tokens.  Latency bounds it: it
// reads and writes some 30 bytes an entry.  1,001 entries take 4.0 us (11 with sums by
// 64-bit atomics in LDS); 64 entries with a token and 160 pages each 8 us, cells and
// tokens in the same launch, where each of ten rounds of cells waits for its entries'
// sequences, then for the table.  Past 1,024 entries the sequences are marked in
// memory and the entries read four times, 1,024 at a time: with the cut that takes the
// step back, a token each, 1,024 entries 18 us, 1,025 29, 5,000 79, 20,000 292,
// 100,000 1,546.
template <bool SMALL, bool FILL>
__global__ __launch_bounds__(kPlanThreads) void plan_scan(PlanStep a) {
  __shared__ int l_wrong;
  __shared__ uint64_t l_part[kPlanThreads / 64];
  __shared__ Named l_named;
  __shared__ int32_t l_starts[FILL ? kPlanThreads + 1 : 1], l_lens[FILL ? kPlanThreads : 1],
      l_before[FILL ? kPlanThreads : 1];
  const int tid = threadIdx.x, lg = a.p.page_log;
  if (tid == 0) l_wrong = kNoMark;
  const int count = min(*a.p.count, a.p.pages);
  const int64_t most = (int64_t)min(a.p.width, a.table_width) << lg;
  struct Entry {
    int32_t s;
    int old, n;
    bool wrong;
  };
  auto entry = [&](int i, bool again) {                    // again: named before
    Entry e{a.seqs[i], 0, 0, false};
    if (e.s == -1) return e;
    e.wrong = true;
    if (e.s < 0 || e.s >= a.p.sequences || again) return e;
    const int old = a.p.lengths[e.s], n = a.fresh[i];
    if (n < 0 || old < 0 || (int64_t)old + n > most) return e;
    e.old = old;
    e.n = n;
    e.wrong = false;
    return e;
  };
  auto need = [&](const Entry& e) {
    return (uint32_t)(pages_of((int64_t)e.old + e.n, lg) - pages_of(e.old, lg));
  };
  uint64_t all_tokens = 0, all_pages = 0;
  Entry mine{-1, 0, 0, false};
  uint32_t at = 0, page = 0;                               // of the entries before
  if constexpr (SMALL) {
    if (tid < a.batch) mine = entry(tid, false);
    if (named_before(l_named, mine.s >= 0 && mine.s < a.p.sequences ? mine.s : -1, tid))
      mine = Entry{mine.s, 0, 0, true};
    if (mine.wrong) atomicMin(&l_wrong, tid);
    at = block_before((uint32_t)mine.n, l_part, &all_tokens);
    page = block_before(need(mine), l_part, &all_pages);
  } else {
    mark_entries(a.p, a.seqs, a.batch);
    for (int i0 = 0; i0 < a.batch; i0 += kPlanThreads) {
      const int i = i0 + tid;
      Entry e{-1, 0, 0, false};
      if (i < a.batch) {
        const int32_t s = a.seqs[i];
        e = entry(i, s >= 0 && s < a.p.sequences && load_mark(&a.p.marks[s]) != i);
      }
      if (e.wrong) atomicMin(&l_wrong, i);
      uint64_t tokens, pages;
      block_before((uint32_t)e.n, l_part, &tokens);
      block_before(need(e), l_part, &pages);
      all_tokens += tokens;
      all_pages += pages;
    }
  }
  // (the last sum's barriers were after every entry's look at l_wrong)
  const int64_t short_tokens = (int64_t)all_tokens - a.tokens;
  const int64_t short_pages = (int64_t)all_pages - count;
  const int code = l_wrong != kNoMark ? 1 : short_tokens > 0 ? 2 : short_pages > 0 ? 3 : 0;
  const int64_t told = code == 1 ? l_wrong : code == 2 ? short_tokens : code == 3 ? short_pages : 0;
  uint32_t tokens = 0, pages = 0;                          // of the chunks before
  for (int i0 = 0; i0 < a.batch; i0 += kPlanThreads) {
    const int i = i0 + tid;
    Entry e{-1, 0, 0, false};
    const bool there = i < a.batch;
    if (SMALL) {
      if (code == 0) e = mine;
      else at = page = 0;
    } else {
      if (there && code == 0) e = entry(i, false);
      uint64_t all_n, all_need;
      at = tokens + block_before((uint32_t)e.n, l_part, &all_n);
      page = pages + block_before(need(e), l_part, &all_need);
      tokens += (uint32_t)all_n;
      pages += (uint32_t)all_need;
    }
    if (there) {
      a.starts[i] = (int32_t)at;
      a.lens[i] = e.old + e.n;
      if (e.s >= 0) a.p.lengths[e.s] = e.old + e.n;
      if (FILL) {
        l_starts[i] = (int32_t)at;
        l_lens[i] = e.old + e.n;
        l_before[i] = (int32_t)page;
      } else {
        a.before[i] = (int32_t)page;
      }
    }
  }
  if (code != 0) all_tokens = all_pages = 0;
  if (!SMALL) clear_marks(a.p, a.seqs, a.batch);
  if (tid == 0) {
    a.starts[a.batch] = (int32_t)all_tokens;
    if (FILL) {
      l_starts[a.batch] = (int32_t)all_tokens;
    } else {
      a.head[0] = count;
      a.head[1] = code == 0;
    }
    *a.p.count = count - (int)all_pages;
    a.status[0] = code;
    a.status[1] = (int32_t)min(told, (int64_t)0x7FFFFFFF);
  }
  if constexpr (FILL) {
    __syncthreads();
    // (new pages enter the pool's table here; tokens take theirs from the stack)
    const Planned f{l_starts, l_lens, l_before, count, code == 0};
    const int cells = a.batch * a.table_width;
#pragma unroll 4
    for (int id = tid; id < cells; id += kPlanThreads) plan_cell(a, f, id);
    for (int t = tid; t < (int)a.tokens; t += kPlanThreads) plan_token(a, f, t);
  }
}

// Cells of the table first, a cell to a thread, then tokens: 1,001 entries of 600
// pages with 60,000 tokens, 6 us.
__global__ __launch_bounds__(256) void plan_fill(PlanStep a) {
  const int64_t id = (int64_t)workgroup() * 256 + threadIdx.x;
  const int64_t cells = (int64_t)a.batch * a.table_width;
  const Planned f{a.starts, a.lens, a.before, a.head[0], a.head[1] != 0};
  if (id < cells) plan_cell(a, f, id);
  else if (id - cells < a.tokens) plan_token(a, f, id - cells);
}

// Pages past the new lengths back onto the stack: entry after entry from the
// top down, so one workgroup adds up how many there are and then moves them.
// SMALL as above.  2.3 us where few pages move, 7.5 for 1,001 entries, whose every
// page is looked up among the entries by halving.
template <bool SMALL>
__global__ __launch_bounds__(kPlanThreads) void pool_truncate(PoolView p, const int32_t* seqs,
                                                              const int32_t* lens, int batch) {
  __shared__ uint64_t l_part[kPlanThreads / 64];
  __shared__ int l_first[kPlanThreads], l_keep[kPlanThreads], l_seq[kPlanThreads];
  __shared__ Named l_named;
  const int tid = threadIdx.x, lg = p.page_log;
  const int count = min(*p.count, p.pages);
  struct Entry {
    int32_t s;
    int old, now;
    bool good;
  };
  auto entry = [&](int i, bool again) {
    Entry e{i < batch ? seqs[i] : -1, 0, 0, false};
    if (e.s < 0 || e.s >= p.sequences || again) return e;
    const int old = p.lengths[e.s], now = lens ? lens[i] : 0;
    if (now < 0 || now > old || pages_of(old, lg) > p.width) return e;
    return Entry{e.s, old, now, true};
  };
  auto marked = [&](int i) {
    if (i >= batch) return false;
    const int32_t s = seqs[i];
    return s >= 0 && s < p.sequences && load_mark(&p.marks[s]) != i;
  };
  Entry mine{-1, 0, 0, false};
  uint64_t total = 0;
  if constexpr (SMALL) {
    mine = entry(tid, false);
    if (named_before(l_named, mine.s >= 0 && mine.s < p.sequences ? mine.s : -1, tid))
      mine = Entry{mine.s, 0, 0, false};
  } else {
    mark_entries(p, seqs, batch);
    for (int i0 = 0; i0 < batch; i0 += kPlanThreads) {
      const Entry e = entry(i0 + tid, marked(i0 + tid));
      uint64_t all = 0;
      block_before((uint32_t)(pages_of(e.old, lg) - pages_of(e.now, lg)), l_part, &all);
      total += all;
    }
  }
  uint64_t base = 0;
  for (int i0 = 0; i0 < batch; i0 += kPlanThreads) {
    const Entry e = SMALL ? mine : entry(i0 + tid, marked(i0 + tid));
    const int keep = pages_of(e.now, lg);
    uint64_t all = 0;
    l_first[tid] = (int)block_before((uint32_t)(pages_of(e.old, lg) - keep), l_part, &all);
    l_keep[tid] = keep;
    l_seq[tid] = e.s;
    if (SMALL) total = all;
    __syncthreads();
    for (uint32_t x = tid; x < (uint32_t)all; x += kPlanThreads) {
      int lo = 0, hi = kPlanThreads;                       // the last entry to start at or before x
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((uint32_t)l_first[mid] <= x) lo = mid;
        else hi = mid;
      }
      const int64_t to = (int64_t)(count + total - 1 - base) - x;
      const int from = l_keep[lo] + (int)(x - (uint32_t)l_first[lo]);
      if (to >= 0 && to < p.pages) p.free_pages[to] = p.table[(int64_t)l_seq[lo] * p.width + from];
    }
    if (e.good) p.lengths[e.s] = e.now;
    base += all;
    __syncthreads();
  }
  if (!SMALL) clear_marks(p, seqs, batch);
  if (tid == 0) *p.count = (int)min((int64_t)(count + total), (int64_t)p.pages);
}

}  // namespace cs
