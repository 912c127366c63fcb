// C ABI entry points of what a step of serving needs beside its products:
// rotary positions, and steps planned on the GPU (declared in include/cs.h).
// Every argument is checked on the host before the first HIP call; kernels are
// enqueued on the caller's stream and nothing is allocated, freed or
// synchronised here.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "cs.h"
#include "q8_api_util.h"
#include "step_plan.h"
#include "step_rotary.h"

namespace {

constexpr int kMaxRotaryHeads = 65535, kMaxRotaryD = 1024;
constexpr int kMaxBatch = 1 << 20;
// Cells and tokens of a step that the workgroup which plans it writes itself.  One launch | two, us
// a call, eager and then recorded (16 to 600 columns, which differ by less than 1 us): 4,000 items
// 9.2 | 12.0, 5.9 | 5.9; 8,000 9.1 | 12.3, 7.8 | 6.0; 12,000 9.5 | 12.2, 8.9 | 6.0; 14,000 9.7 | 12.2,
// 9.3 | 6.1; 16,000 10.7 | 12.3, 10.4 | 6.0; 20,000 12.0 | 12.3, 11.7 | 5.9; 32,000 16.1 | 12.5, 15.8
// | 5.9.  Eager calls would draw the line at 20,000 and recorded ones at 4,000; here one kind loses
// as much as the other gains.
constexpr int64_t kFillItems = 12288;

template <typename T, int N, bool NEIGHBOURS>
int rotary_launch(cs::Rotary a, hipStream_t s) {
  constexpr int P = NEIGHBOURS ? (N > 1 ? N / 2 : 1) : N;
  const int units = a.rot / 2 / P + (a.copied ? (a.d - a.rot) / N : 0);
  // Four tokens a workgroup, so that a thread turns several units of each angle; few tokens' heads
  // are shared by as many workgroups as have a unit for every thread.
  a.per = a.tokens >= 2048 ? 4 : 1;
  const int64_t items = (int64_t)a.per * a.heads * units;
  const int64_t groups = (a.tokens + a.per - 1) / a.per;
  a.parts = (int)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 1024 / groups));
  a.by_units = cs::make_fastdiv((uint32_t)units);
  a.by_heads = cs::make_fastdiv((uint32_t)a.heads);
  a.by_parts = cs::make_fastdiv((uint32_t)a.parts);
  hipLaunchKernelGGL((cs::rotary<T, N, NEIGHBOURS>), cs::wide_grid(groups * a.parts), dim3(256),
                     (size_t)a.per * (a.rot / 2) * sizeof(float2), s, a);
  return launched();
}

int pool_view(const cs_page_pool* p, cs::PoolView* out) {
  if (!p || !p->table || !p->lengths || !p->free_pages || !p->count || !p->marks) return CS_ERR_ARG;
  if (p->sequences < 1 || p->width < 1 || p->pages < 1 || p->page < 1) return CS_ERR_ARG;
  if (!aligned(p->table, 4) || !aligned(p->lengths, 4) || !aligned(p->free_pages, 4) ||
      !aligned(p->count, 4) || !aligned(p->marks, 4))
    return CS_ERR_ARG;
  if (p->page < 16 || p->page > 1024 || (p->page & (p->page - 1)) != 0) return CS_ERR_SHAPE;
  if ((int64_t)p->sequences * p->width > kMaxCount || (int64_t)p->pages * p->page > kMaxCount ||
      (int64_t)p->width * p->page > CS_MAX_Q8_LEN)
    return CS_ERR_SHAPE;
  int lg = 4;
  while ((1 << lg) < p->page) ++lg;
  *out = {p->table, p->lengths, p->free_pages, p->count, p->marks, p->sequences, p->width,
          p->pages, lg};
  return CS_OK;
}

}  // namespace

extern "C" {

int cs_rotary(cs_dtype xt, const uint64_t* turns, int rot, int interleaved, float amplitude,
              int inverse, const int32_t* positions, int64_t tokens, int d, int q_heads,
              const void* q, int64_t ldq, int64_t hsq, void* yq, int64_t ldyq, int64_t hsyq,
              int k_heads, const void* k, int64_t ldk, int64_t hsk, void* yk, int64_t ldyk,
              int64_t hsyk, void* stream) {
  if (!is_float(xt)) return CS_ERR_DTYPE;
  if (tokens < 0 || d < 1 || q_heads < 0 || k_heads < 0 || !std::isfinite(amplitude))
    return CS_ERR_ARG;
  if (rot < 2 || rot % 2 != 0 || rot > d || d > kMaxRotaryD) return CS_ERR_SHAPE;
  if (q_heads > kMaxRotaryHeads - k_heads) return CS_ERR_SHAPE;
  const int all = q_heads + k_heads;
  if (tokens == 0 || all == 0) return CS_OK;
  if (!turns || !positions || !aligned(turns, 8) || !aligned(positions, 4)) return CS_ERR_ARG;
  if (tokens > kMaxCount / all) return CS_ERR_SHAPE;
  const int e = (int)float_size(xt);
  cs::Rotary a{};
  a.part[0] = {q, yq, ldq, hsq, ldyq, hsyq};
  a.part[1] = {k, yk, ldk, hsk, ldyk, hsyk};
  int together = 16 / e;               // elements of a load: all rows start on that many
  for (int i = 0; i < 2; ++i) {
    const int heads = i ? k_heads : q_heads;
    const cs::RotaryPart& r = a.part[i];
    if (heads == 0) continue;
    if (!r.x || !r.y || !aligned(r.x, e) || !aligned(r.y, e)) return CS_ERR_ARG;
    if (r.ldx < 0 || r.ldy < 0 || r.hsx < d || r.hsy < d || (tokens > 1 && r.ldy < d))
      return CS_ERR_SHAPE;
    if (r.x == r.y && ((tokens > 1 && r.ldx != r.ldy) || (heads > 1 && r.hsx != r.hsy)))
      return CS_ERR_ARG;
    if (r.x != r.y) a.copied = d - rot;
    auto starts = [&](const void* p, int64_t ld, int64_t hs) {
      return aligned(p, (size_t)together * e) && (tokens == 1 || ld % together == 0) &&
             (heads == 1 || hs % together == 0);
    };
    while (together > 1 && !(starts(r.x, r.ldx, r.hsx) && starts(r.y, r.ldy, r.hsy)))
      together /= 2;
  }
  const int whole = interleaved ? rot : rot / 2;
  while (together > 1 && (whole % together != 0 || (d - rot) % together != 0)) together /= 2;
  a.turns = turns;
  a.positions = positions;
  a.tokens = tokens;
  a.heads0 = q_heads;
  a.heads = all;
  a.d = d;
  a.rot = rot;
  a.amplitude = amplitude;
  a.inverse = inverse != 0;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return with_float(xt, [&](auto t) {
    using T = decltype(t);
    auto layout = [&](auto n) {
      constexpr int N = decltype(n)::value;
      return interleaved ? rotary_launch<T, N, true>(a, s) : rotary_launch<T, N, false>(a, s);
    };
    if constexpr (sizeof(T) == 2) {
      if (together == 8) return layout(std::integral_constant<int, 8>{});
    }
    if (together == 4) return layout(std::integral_constant<int, 4>{});
    if (together == 2) return layout(std::integral_constant<int, 2>{});
    return layout(std::integral_constant<int, 1>{});
  });
}

size_t cs_plan_step_workspace_bytes(int batch) {
  if (batch < 1 || batch > kMaxBatch) return 0;
  return round_up(16 + (size_t)batch * 4, 256);
}

int cs_plan_step(const cs_page_pool* pool, const int32_t* seqs, const int32_t* fresh, int batch,
                 int32_t* table, int table_width, int32_t* lens, int32_t* starts, int64_t* slots,
                 int32_t* positions, int64_t tokens, int32_t* status, void* ws, size_t ws_bytes,
                 void* stream) {
  cs::PoolView p;
  const int st = pool_view(pool, &p);
  if (st != CS_OK) return st;
  if (batch < 1 || table_width < 1 || tokens < 0) return CS_ERR_ARG;
  if (!seqs || !fresh || !table || !lens || !starts || !status || (tokens > 0 && !slots) ||
      (tokens > 0 && !positions))
    return CS_ERR_ARG;
  if (!aligned(seqs, 4) || !aligned(fresh, 4) || !aligned(table, 4) || !aligned(lens, 4) ||
      !aligned(starts, 4) || !aligned(status, 4) || !aligned(slots, 8) || !aligned(positions, 4))
    return CS_ERR_ARG;
  if (batch > kMaxBatch || (int64_t)batch * table_width > kMaxCount || tokens > kMaxCount ||
      (int64_t)table_width * pool->page > CS_MAX_Q8_LEN)
    return CS_ERR_SHAPE;
  if (!ws || !aligned(ws, 16) || ws_bytes < cs_plan_step_workspace_bytes(batch))
    return CS_ERR_WORKSPACE;
  int32_t* head = static_cast<int32_t*>(ws);
  const cs::PlanStep a{p, seqs, fresh, batch, table, table_width, lens, starts, slots, positions,
                       tokens, status, head, head + 4};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t items = (int64_t)batch * table_width + tokens;
  const bool small = batch <= cs::kPlanThreads;
  const dim3 one(1), block(cs::kPlanThreads);
  if (small && items <= kFillItems) {
    hipLaunchKernelGGL((cs::plan_scan<true, true>), one, block, 0, s, a);
    return launched();
  }
  if (small) hipLaunchKernelGGL((cs::plan_scan<true, false>), one, block, 0, s, a);
  else hipLaunchKernelGGL((cs::plan_scan<false, false>), one, block, 0, s, a);
  if (launched() != CS_OK) return CS_ERR_DEVICE;
  hipLaunchKernelGGL(cs::plan_fill, cs::wide_grid((items + 255) / 256), dim3(256), 0, s, a);
  return launched();
}

int cs_pool_truncate(const cs_page_pool* pool, const int32_t* seqs, const int32_t* lens, int batch,
                     void* stream) {
  cs::PoolView p;
  const int st = pool_view(pool, &p);
  if (st != CS_OK) return st;
  if (batch < 0) return CS_ERR_ARG;
  if (batch == 0) return CS_OK;
  if (!seqs || !aligned(seqs, 4) || !aligned(lens, 4)) return CS_ERR_ARG;
  if (batch > kMaxBatch) return CS_ERR_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 one(1), block(cs::kPlanThreads);
  if (batch <= cs::kPlanThreads)
    hipLaunchKernelGGL((cs::pool_truncate<true>), one, block, 0, s, p, seqs, lens, batch);
  else
    hipLaunchKernelGGL((cs::pool_truncate<false>), one, block, 0, s, p, seqs, lens, batch);
  return launched();
}

}  // extern "C"
