// C ABI entry points of the 4-bit cache and attention over it (declared in
// include/cs.h).  Every argument is checked on the host before the first HIP
// call; kernels are enqueued on the caller's stream and nothing is allocated,
// freed or synchronised here.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <numeric>

#include "cs.h"
#include "mx4_attention.h"
#include "mx4_rows.h"
#include "q8_api_util.h"

namespace {

int cache_view(const cs_mx4_cache* c, cs::Mx4View* out) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return CS_ERR_ARG;
  if (c->pages < 1 || c->heads < 1 || c->page < 1 || c->d < 1) return CS_ERR_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) ||
      !aligned(c->v_scale, 4))
    return CS_ERR_ARG;
  if (c->d % 16 != 0 || c->d > 256) return CS_ERR_SHAPE;
  if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1)) != 0) return CS_ERR_SHAPE;
  if ((int64_t)c->pages * c->page > kMaxCount) return CS_ERR_SHAPE;
  int lg = 4;
  while ((1 << lg) < c->page) ++lg;
  *out = {c->k, c->v, c->k_scale, c->v_scale, (int64_t)c->pages * c->page, c->heads, lg, c->d,
          (c->d + 31) / 32};
  return CS_OK;
}

// Workgroups of mx4_write and mx4_read: four wavefronts, four tokens of a head each.
dim3 cache_grid(int64_t tokens, int heads) {
  dim3 grid = cs::wide_grid(((tokens + 3) / 4 * heads + 3) / 4);
  grid.z = 2;
  return grid;
}

struct AttentionPlan {
  int per;             // rows of a workgroup: 128 (mx4_many), 32 or 16 (mx4_few)
  int64_t tiles;       // numbers of row tiles (mx4_place)
  int splits, chunk;   // parts of the key axis, positions of a part
  int most;            // parts at most, of this axis under any window and of any shorter one
  int waves;           // wavefronts of a workgroup
};

AttentionPlan attention_plan(const cs::Mx4View& c, cs_dtype qt, int tokens, int q_heads,
                             int batch, int table_width, int max_len, int window) {
  AttentionPlan p;
  const int64_t group = q_heads / c.heads, rows = tokens * group;
  // Sequences with tokens, at most.  The other entries of a padded batch have no work, and counted
  // as sequences they took the parts from those that have (three tokens over 100,000 keys each in
  // a table of 256 entries 871 us, 63 so; five over 8,192 in 64 entries 43.6, 20.7).
  const int64_t seqs = std::min(batch, tokens);
  // Rows of a sequence (bf16, d 128, eight heads; 16 | 32 | 128 rows a workgroup, us).  One
  // sequence of 32,768 keys: 32 rows 29.8 | 29.9 | 41, 64 37 | 36 | 42, 96 46 | 43 | 44, 128 51 | 48
  // | 46; three of 85,000: 20 rows 103 | 87 | 185; eight of 8,192: 32 rows 36 | 35 | 54, 64 56 | 53
  // | 60, 84 71 | 79 | 64, 128 88 | 83 | 73; 32 of 2,048: 64 rows 42 | 40 | 58, 84 60 | 63 | 58, 160
  // 91 | 96 | 93; 32 of 200: 64 rows 12.2 | 12.4 | 14.5, 96 16.6 | 18.6 | 15.5.  fp16 the same to 6
  // %.  fp32, 32 | 128 rows a workgroup, 96 rows of the four: 50 | 52, 94 | 85, 76 | 84, 25 | 21;
  // 128 rows of the first two 56 | 55, 99 | 93, 160 rows of the third 117 | 128.
  const int few = qt == CS_F32 ? 112 : 80;
  p.per = rows > few * seqs ? 128 : rows > 16 * seqs && c.d <= 128 ? 32 : 16;
  // numbers that mx4_place gives: sequences of at least a token, each with less than a tile of rows
  // that are not there, in steps of what divides both
  p.tiles = (rows + seqs * (p.per - std::gcd(group, (int64_t)p.per))) / p.per;
  int64_t len = (int64_t)table_width << c.page_log;
  if (max_len > 0) len = std::min<int64_t>(len, max_len);
  if (window > 0) len = std::min<int64_t>(len, (int64_t)window + 64);
  // As many parts as fill the card once: four workgroups a compute unit (two or three where
  // registers are more).  More make sequences of unequal length even out better, but parts have to
  // be joined: 96 sequences of up to 12,000 keys 144 us so, 140 at twice as many, 135 at three
  // times; 96 of 6,000 108 | 117 | 123; 128 of 4,500 107 | 118 | 124.  128 rows take 1.5 times as
  // long to join as a second part saves (with weights of one piece, 32 sequences of 2,048 keys: whole
  // 74 us, two parts 102; eight of 8,192 in four parts 93, in eight 79).  Short axes stay whole: the join is a launch of
  // its own (1,500 keys of one sequence 12.2 us, 14.3 in parts).
  const int64_t per_seq = (rows + seqs - 1) / seqs;
  const int64_t items = seqs * ((per_seq + p.per - 1) / p.per) * c.heads;
  const int wgs = p.per > 16 || c.d > 128 ? 2 : qt == CS_F32 ? 3 : 4;
  int64_t splits = std::min<int64_t>({256 * wgs / items, len / 256, cs::kMaxSplits});
  if (splits < (p.per == 128 ? 3 : 1) || len <= 2048) splits = 1;
  // Parts are whole steps, so a part is rounded up and there may be fewer of them than `splits`.
  // `splits` itself never grows as the axis gets shorter.
  p.most = (int)splits;
  p.chunk = (int)round_up((size_t)((len + splits - 1) / splits), 128);
  p.splits = (int)((len + p.chunk - 1) / p.chunk);
  // a workgroup or fewer a compute unit, keys whole: eight wavefronts halve its chain of steps
  const int64_t most = qt == CS_F32 || c.d > 128 ? 256 : 128;
  p.waves = p.per == 16 && p.splits == 1 && items <= most ? 8 : 4;
  return p;
}

size_t attention_part_bytes(int64_t parts, int64_t rows, int d) {
  return parts > 1 ? (size_t)parts * rows * ((size_t)d * 4 + 8) : 0;
}

bool attention_fits(const cs::Mx4View& c, int tokens, int q_heads, int table_width) {
  return q_heads % c.heads == 0 && c.heads <= 65535 && (int64_t)tokens * q_heads <= kMaxCount &&
         ((int64_t)table_width << c.page_log) <= CS_MAX_Q8_LEN;
}

}  // namespace

extern "C" {

int cs_mx4_cache_write(const cs_mx4_cache* cache, cs_dtype xt, const void* k, int64_t ldk,
                       int64_t hsk, const void* v, int64_t ldv, int64_t hsv,
                       const int64_t* slots, int64_t tokens, void* stream) {
  if (!is_float(xt)) return CS_ERR_DTYPE;
  cs::Mx4View c;
  const int st = cache_view(cache, &c);
  if (st != CS_OK) return st;
  if (tokens < 0) return CS_ERR_ARG;
  if (tokens == 0) return CS_OK;
  if (!k || !v || !slots || !aligned(k, float_size(xt)) || !aligned(v, float_size(xt)) ||
      !aligned(slots, 8))
    return CS_ERR_ARG;
  if (ldk < 0 || ldv < 0 || hsk < c.d || hsv < c.d) return CS_ERR_SHAPE;
  if (tokens > kMaxCount / c.heads) return CS_ERR_SHAPE;
  return with_float(xt, [&](auto t) {
    using T = decltype(t);
    const int64_t e = sizeof(T);
    const bool vec = aligned(k, 16) && aligned(v, 16) && ldk * e % 16 == 0 && ldv * e % 16 == 0 &&
                     hsk * e % 16 == 0 && hsv * e % 16 == 0;
    auto go = [&](auto wide) {
      hipLaunchKernelGGL((cs::mx4_write<T, decltype(wide)::value>), cache_grid(tokens, c.heads),
                         dim3(256), 0, static_cast<hipStream_t>(stream), c,
                         static_cast<const T*>(k), ldk, hsk, static_cast<const T*>(v), ldv, hsv,
                         slots, tokens, cs::make_fastdiv((uint32_t)c.heads));
      return launched();
    };
    return vec ? go(std::true_type{}) : go(std::false_type{});
  });
}

int cs_mx4_cache_read(const cs_mx4_cache* cache, const int64_t* slots, int64_t tokens, cs_dtype yt,
                      void* k, void* v, void* stream) {
  if (!is_float(yt)) return CS_ERR_DTYPE;
  cs::Mx4View c;
  const int st = cache_view(cache, &c);
  if (st != CS_OK) return st;
  if (tokens < 0) return CS_ERR_ARG;
  if (tokens == 0) return CS_OK;
  if (!k || !v || !slots || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8))
    return CS_ERR_ARG;
  if (tokens > kMaxCount / c.heads) return CS_ERR_SHAPE;
  return with_float(yt, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL((cs::mx4_read<T>), cache_grid(tokens, c.heads), dim3(256), 0,
                       static_cast<hipStream_t>(stream), c, slots, tokens,
                       cs::make_fastdiv((uint32_t)c.heads), static_cast<T*>(k),
                       static_cast<T*>(v));
    return launched();
  });
}

size_t cs_mx4_paged_attention_workspace_bytes(const cs_mx4_cache* cache, cs_dtype qt, int tokens,
                                              int q_heads, int batch, int table_width,
                                              int max_len) {
  cs::Mx4View c;
  if (!is_float(qt) || cache_view(cache, &c) != CS_OK) return 0;
  if (tokens < 1 || q_heads < 1 || batch < 1 || table_width < 1 || max_len < 0) return 0;
  if (!attention_fits(c, tokens, q_heads, table_width)) return 0;
  // the whole axis: a window or a shorter one has at most as many parts
  const AttentionPlan p = attention_plan(c, qt, tokens, q_heads, batch, table_width, max_len, 0);
  return attention_part_bytes(p.most, (int64_t)tokens * q_heads, c.d);
}

int cs_mx4_paged_attention_plan(const cs_mx4_cache* cache, cs_dtype qt, int tokens, int q_heads,
                                int batch, int table_width, int max_len, int window,
                                int64_t* info) {
  if (!info) return CS_ERR_ARG;
  if (!is_float(qt)) return CS_ERR_DTYPE;
  cs::Mx4View c;
  const int st = cache_view(cache, &c);
  if (st != CS_OK) return st;
  if (tokens < 1 || q_heads < 1 || batch < 1 || table_width < 1 || max_len < 0 || window < 0)
    return CS_ERR_ARG;
  if (!attention_fits(c, tokens, q_heads, table_width)) return CS_ERR_SHAPE;
  const AttentionPlan p = attention_plan(c, qt, tokens, q_heads, batch, table_width, max_len,
                                         window);
  info[0] = p.per;
  info[1] = p.splits;
  info[2] = p.chunk;
  info[3] = p.waves;
  info[4] = p.tiles * c.heads * p.splits;
  info[5] = (int64_t)attention_part_bytes(p.splits, (int64_t)tokens * q_heads, c.d);
  return CS_OK;
}

int cs_mx4_paged_attention(const cs_mx4_cache* cache, cs_dtype qt, const void* q, int64_t ldq,
                           int64_t hsq, int tokens, int q_heads, int batch, const int32_t* table,
                           int table_width, const int32_t* lens, const int32_t* starts,
                           int max_len, float scale, int window, void* out, void* ws,
                           size_t ws_bytes, void* stream) {
  if (!is_float(qt)) return CS_ERR_DTYPE;
  cs::Mx4View c;
  const int st = cache_view(cache, &c);
  if (st != CS_OK) return st;
  const int some = tokens > 0;                             // no tokens: no sequences needed
  if (tokens < 0 || q_heads < 1 || batch < some || table_width < some || max_len < 0 || window < 0)
    return CS_ERR_ARG;
  if (!(scale > 0.0f) || std::isinf(scale)) return CS_ERR_ARG;
  if (tokens == 0) return CS_OK;
  if (!q || !table || !lens || !starts || !out || !aligned(q, float_size(qt)) ||
      !aligned(out, 16) || !aligned(table, 4) || !aligned(lens, 4) || !aligned(starts, 4))
    return CS_ERR_ARG;
  if (ldq < 0 || hsq < c.d || !attention_fits(c, tokens, q_heads, table_width))
    return CS_ERR_SHAPE;
  const AttentionPlan p = attention_plan(c, qt, tokens, q_heads, batch, table_width, max_len,
                                          window);
  const int group = q_heads / c.heads;
  const int64_t rows = (int64_t)tokens * q_heads;
  const size_t need = std::max(
      cs_mx4_paged_attention_workspace_bytes(cache, qt, tokens, q_heads, batch, table_width,
                                             max_len),
      attention_part_bytes(p.splits, rows, c.d));
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16))) return CS_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int e = (int)float_size(qt);
  const bool vec = aligned(q, 16) && (tokens == 1 || ldq * e % 16 == 0) && hsq * e % 16 == 0;
  cs::Mx4Attention a{c, q, ldq, hsq, vec, tokens, q_heads, group, batch,
                     cs::make_fastdiv((uint32_t)group), cs::make_fastdiv((uint32_t)c.heads),
                     cs::make_fastdiv((uint32_t)p.tiles), table, table_width, lens, starts, scale,
                     std::min(window, CS_MAX_Q8_LEN), out, p.splits, p.chunk, nullptr, nullptr};
  if (p.splits > 1) {
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + (int64_t)p.splits * rows * c.d);
  }
  const int64_t blocks = p.tiles * c.heads * p.splits;
  if (blocks > kMaxCount) return CS_ERR_SHAPE;
  return with_float(qt, [&](auto t) {
    using T = decltype(t);
    const dim3 grid = cs::wide_grid(blocks);
    auto few = [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
      if (DT <= 128 && p.per == 32)
        hipLaunchKernelGGL((cs::mx4_few<T, DT <= 128 ? DT : 128, 4, 2>), grid, dim3(256), 0, s, a);
      else if (p.waves == 8)
        hipLaunchKernelGGL((cs::mx4_few<T, DT, 8, 1>), grid, dim3(512), 0, s, a);
      else
        hipLaunchKernelGGL((cs::mx4_few<T, DT, 4, 1>), grid, dim3(256), 0, s, a);
    };
    auto many = [&](auto dt) {
      constexpr int W = decltype(dt)::value, DT = W <= 64 ? 64 : W <= 128 ? 128 : 256;
      // a page that holds a step's 64 keys: one scalar address (four sequences of 700 tokens over
      // 2,700 keys 169 us, 182 and 196 with an address for every 16 keys at pages of 32 and 16)
      if (c.page_log >= 6)
        hipLaunchKernelGGL((cs::mx4_many<T, W, true>), grid, dim3(256), cs::Mx4Lds<DT>::bytes, s,
                           a);
      else
        hipLaunchKernelGGL((cs::mx4_many<T, W, false>), grid, dim3(256), cs::Mx4Lds<DT>::bytes, s,
                           a);
    };
    if (p.per < 128) with_width(c.d, few);
    else if (c.d > 64 && c.d <= 96) many(std::integral_constant<int, 96>{});
    else if (c.d > 128 && c.d <= 192) many(std::integral_constant<int, 192>{});
    else with_width(c.d, many);
    int r = launched();
    if (r == CS_OK && p.splits > 1) {
      hipLaunchKernelGGL((cs::attention_join<T, cs::Mx4View>), dim3((unsigned)rows), dim3(256), 0,
                         s, a);
      r = launched();
    }
    return r;
  });
}

}  // extern "C"
