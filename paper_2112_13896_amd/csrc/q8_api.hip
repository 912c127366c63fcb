// C ABI entry points of the 8-bit attention-layer operators (declared in
// include/cs.h).  Every argument is checked on the host before the first HIP
// call; kernels are enqueued on the caller's stream and nothing is allocated,
// freed or synchronised here.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "cs.h"
#include "q8_attention.h"
#include "q8_linear.h"
#include "q8_rows.h"

namespace {

constexpr int64_t kMaxCount = 0x7FFFFFFF;

size_t float_size(cs_dtype t) { return t == CS_F32 ? 4 : 2; }
bool is_float(cs_dtype t) { return t == CS_F32 || t == CS_F16 || t == CS_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t round_up(size_t v, size_t n) { return (v + n - 1) / n * n; }

int launched() { return hipGetLastError() == hipSuccess ? CS_OK : CS_ERR_DEVICE; }

// f(T{}) with the C++ type of a float dtype.
template <typename F>
int with_float(cs_dtype t, F f) {
  if (t == CS_F32) return f(float{});
  if (t == CS_F16) return f(_Float16{});
  return f(__bf16{});
}

// ---------------------------------------------------------------- rows
template <typename T, int WPR>
int quantise_launch(const T* x, int64_t ldx, int64_t rows, int c, int8_t* q, int64_t ldq,
                    float* scale, hipStream_t s) {
  const dim3 grid = cs::wide_grid((rows * WPR + 3) / 4), block(256);
  auto starts_on = [&](size_t n) {
    return aligned(x, n) && (rows == 1 || ldx * sizeof(T) % n == 0);
  };
  if (starts_on(16))
    hipLaunchKernelGGL((cs::quantise_rows<T, 16, WPR>), grid, block, 0, s, x, ldx, rows, c, q,
                       ldq, scale);
  else if (sizeof(T) == 4 || starts_on(4))
    hipLaunchKernelGGL((cs::quantise_rows<T, 4, WPR>), grid, block, 0, s, x, ldx, rows, c, q, ldq,
                       scale);
  else
    hipLaunchKernelGGL((cs::quantise_rows<T, (int)sizeof(T), WPR>), grid, block, 0, s, x, ldx,
                       rows, c, q, ldq, scale);
  return launched();
}

int quantise(cs_dtype xt, const void* x, int64_t ldx, int64_t rows, int c, int8_t* q, int64_t ldq,
             float* scale, hipStream_t s) {
  return with_float(xt, [&](auto t) {
    using T = decltype(t);
    const T* p = static_cast<const T*>(x);
    // a wavefront to a row | four, us: 33 x 2,048 f32 3.9 | 2.8, 777 x 1,500 4.1 | 3.5, 200 x 1,024
    // 3.1 | 2.9, 1,024 x 1,024 3.2 | 3.3, 4,096 x 1,024 4.3 | 5.6, 33 x 512 2.5 | 2.8, 8,192 x 512
    // 4.3 | 7.4, 8,192 x 2,048 15.4 | 13.8 (bf16 alike)
    if (c <= 512 || (c <= 1024 && rows > 1024))
      return quantise_launch<T, 1>(p, ldx, rows, c, q, ldq, scale, s);
    return quantise_launch<T, 4>(p, ldx, rows, c, q, ldq, scale, s);
  });
}

// ---------------------------------------------------------------- linear
// Tokens of one launch of tiles, so that it has less than 2^32 threads (further grid rows, as
// elsewhere, cost 64 x 64 tiles 0.6 of 7.3 us: another order of a step's reads and loads).
constexpr int64_t kTileRows = 1 << 28;

template <typename T, int BM, int BN, int WM, int WN, int NB>
int linear_tiles(const cs::Q8Linear& all, hipStream_t s) {
  cs::Q8Linear a = all;
  if (a.rows > kTileRows) {
    for (int64_t first = 0; first < all.rows; first += kTileRows) {
      a.x = all.x + first * all.ldx;
      a.sx = all.sx + first;
      a.y = static_cast<T*>(all.y) + first * all.ldy;
      a.rows = std::min(kTileRows, all.rows - first);
      const int st = linear_tiles<T, BM, BN, WM, WN, NB>(a, s);
      if (st != CS_OK) return st;
    }
    return CS_OK;
  }
  cs::TileOrder o;
  const int64_t tm = (a.rows + BM - 1) / BM, tn = ((int64_t)a.d_out + BN - 1) / BN;
  if (tm * tn * (BM / WM * (BN / WN) * 64) > (int64_t)UINT32_MAX) return CS_ERR_SHAPE;
  o.tiles_m = (uint32_t)tm;
  o.tiles_n = (uint32_t)tn;
  o.per_xcd = (uint32_t)(tm * tn / 8);
  o.more = (uint32_t)(tm * tn % 8);
  hipLaunchKernelGGL((cs::linear_q8_tile<T, BM, BN, WM, WN, NB>), dim3((unsigned)(tm * tn)),
                     dim3(BM / WM * (BN / WN) * 64), 0, s, a, o);
  return launched();
}

// Elements of up to 16 tokens that every workgroup of the product quantises itself, instead of a
// launch that does it once (recorded in a graph, bf16, tokens x k): 1 x 2,048 4.8 us against 7.8,
// 1 x 16,384 19.5 | 26.0, 4 x 4,096 9.3 | 9.4, 8 x 2,048 7.4 | 8.4, 16 x 1,024 7.5 | 6.8; beyond,
// 8 x 4,096 16.2 | 12.6, 16 x 2,048 10.9 | 8.9.  Calls that are not recorded save 2.7 us of the
// host's time on top.
constexpr int64_t kFusedElements = 16384;

template <typename T, typename XT, int RT>
int linear_few(const cs::Q8Linear& a, hipStream_t s) {
  constexpr int NW = 8;
  const size_t lds = sizeof(XT) > 1 ? (size_t)a.rows * round_up((size_t)a.k, 128) : 0;
  hipLaunchKernelGGL((cs::linear_q8_few<T, XT, RT, NW>), dim3((unsigned)((a.d_out + 15) / 16)),
                     dim3(NW * 64), lds, s, a);
  return launched();
}

// ---------------------------------------------------------------- cache
int cache_view(const cs_q8_cache* c, cs::CacheView* out) {
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
  *out = {c->k, c->v, c->k_scale, c->v_scale, (int64_t)c->pages * c->page, c->heads, lg, c->d};
  return CS_OK;
}

// ---------------------------------------------------------------- attention
// f(integral_constant) with the width of the kernels' registers for d channels.
template <typename F>
void with_width(int d, F f) {
  if (d <= 64) f(std::integral_constant<int, 64>{});
  else if (d <= 128) f(std::integral_constant<int, 128>{});
  else f(std::integral_constant<int, 256>{});
}

struct AttentionPlan {
  int per;             // rows of a workgroup: 128 (attention_many) or 16 (attention_few)
  int64_t tiles;       // numbers of row tiles (find_tile)
  int splits, chunk;   // parts of the key axis, positions of a part
  int most;            // parts at most, of this axis under any window and of any shorter one
  int waves;           // wavefronts of a workgroup (attention_few)
};

AttentionPlan attention_plan(const cs::CacheView& c, cs_dtype qt, int tokens, int q_heads,
                             int batch, int table_width, int max_len, int window) {
  AttentionPlan p;
  const int64_t group = q_heads / c.heads, rows = tokens * group;
  // 128 rows a workgroup from 65 rows a sequence on (bf16, d 128, eight heads; few | many):
  // 64 rows 32 | 50 us (1 x 32,768 keys), 71 | 65 (8 x 8,192), 54 | 76 (32 x 2,048), 14 | 17
  // (32 x 200); 96 rows 48 | 53, 115 | 70, 82 | 95, 20 | 20; 128 rows 49 | 40, 119 | 76
  p.per = rows > 64 * (int64_t)batch ? 128 : 16;
  p.tiles = rows / p.per + batch + 1;
  int64_t len = (int64_t)table_width << c.page_log;
  if (max_len > 0) len = std::min<int64_t>(len, max_len);
  if (window > 0) len = std::min<int64_t>(len, (int64_t)window + 64);
  // As many parts as fill the card: few rows twice, at four workgroups a compute unit (three and
  // two where fp32 queries and wide heads take more registers), so that sequences of unequal
  // length even out (64 sequences of up to 8,192 keys: 151 us filled once, 141 twice or four
  // times); many rows, whose parts cost more to join, once at one.  Keys that four wavefronts
  // pass in ten microseconds or so stay whole.
  const int64_t per_seq = (rows + batch - 1) / batch;
  const int64_t items = batch * ((per_seq + p.per - 1) / p.per) * c.heads;
  const int wgs = p.per == 128 ? 1 : 2 * (c.d > 128 ? 2 : c.d > 64 && qt == CS_F32 ? 3 : 4);
  int64_t splits = std::min<int64_t>({256 * wgs / items, len / 256, cs::kMaxSplits});
  if (splits < 1 || len <= 1024) splits = 1;
  // Parts are whole steps, so a part is rounded up and there may be fewer of them than `splits`.
  // How many fewer depends on the length (64 at most: 16,384 positions are 64, one more makes 43);
  // `splits` itself never grows as the axis gets shorter.
  p.most = (int)splits;
  p.chunk = (int)round_up((size_t)((len + splits - 1) / splits), 128);
  p.splits = (int)((len + p.chunk - 1) / p.chunk);
  // a workgroup or fewer a compute unit, keys whole: eight wavefronts halve its chain of steps
  // (four | eight, one new token, 8 cache heads of 128: 1 x 700 keys 11.1 | 9.7 us, 8 x 900 13.5 |
  // 11.6, fp32 32 x 1,000 26.1 | 18.4, heads of 256 31.9 | 26.8; but bf16 32 x 1,000 20.7 | 21.7,
  // 96 x 200 14.1 | 17.6)
  const int64_t most = qt == CS_F32 || c.d > 128 ? 256 : 128;
  p.waves = p.splits == 1 && items <= most ? 8 : 4;
  return p;
}

size_t attention_part_bytes(int64_t parts, int64_t rows, int d) {
  return parts > 1 ? (size_t)parts * rows * ((size_t)d * 4 + 8) : 0;
}

bool attention_fits(const cs::CacheView& c, int tokens, int q_heads, int table_width) {
  return q_heads % c.heads == 0 && c.heads <= 65535 && (int64_t)tokens * q_heads <= kMaxCount &&
         ((int64_t)table_width << c.page_log) <= CS_MAX_Q8_LEN;
}

}  // namespace

extern "C" {

int cs_quantise_rows(cs_dtype xt, const void* x, int64_t ldx, int64_t rows, int c, int8_t* q,
                     int64_t ldq, float* scale, void* stream) {
  if (!is_float(xt)) return CS_ERR_DTYPE;
  if (rows < 0 || c < 1) return CS_ERR_ARG;
  if (rows == 0) return CS_OK;
  if (!x || !q || !scale || !aligned(x, float_size(xt)) || !aligned(scale, 4)) return CS_ERR_ARG;
  if (ldx < c || ldq < c || rows > kMaxCount) return CS_ERR_SHAPE;
  return quantise(xt, x, ldx, rows, c, q, ldq, scale, static_cast<hipStream_t>(stream));
}

size_t cs_linear_q8_workspace_bytes(cs_dtype xt, int64_t rows, int k, int d_out) {
  if (rows < 1 || rows > kMaxCount || k < 1 || k > CS_MAX_Q8_K || d_out < 1 ||
      d_out > CS_MAX_Q8_OUT)
    return 0;
  if (!is_float(xt)) return 0;
  return round_up((size_t)rows * round_up((size_t)k, 16) + (size_t)rows * 4, 256);
}

int cs_linear_q8(cs_dtype xt, const void* x, int64_t ldx, const float* sx, int64_t rows, int k,
                 const int8_t* w, int64_t ldw, const float* sw, int d_out, const float* bias,
                 cs_dtype yt, void* y, int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
  if (!(is_float(xt) || xt == CS_I8) || !is_float(yt)) return CS_ERR_DTYPE;
  if (rows < 0 || k < 1 || d_out < 1) return CS_ERR_ARG;
  if (rows == 0) return CS_OK;
  if (!x || !w || !sw || !y || (xt == CS_I8) != (sx != nullptr)) return CS_ERR_ARG;
  if ((is_float(xt) && !aligned(x, float_size(xt))) || !aligned(y, float_size(yt)) ||
      !aligned(sx, 4) || !aligned(sw, 4) || !aligned(bias, 4))
    return CS_ERR_ARG;
  if (k > CS_MAX_Q8_K || rows > kMaxCount || ldx < k || ldw < k || ldy < d_out)
    return CS_ERR_SHAPE;
  if (d_out > CS_MAX_Q8_OUT) return CS_ERR_SHAPE;
  const size_t need = cs_linear_q8_workspace_bytes(xt, rows, k, d_out);
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16))) return CS_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int y_vec = aligned(y, 16) && ldy * (int64_t)float_size(yt) % 16 == 0;
  cs::Q8Linear a{static_cast<const int8_t*>(x), ldx, sx, rows, k, w, ldw, sw, d_out, bias, y, ldy,
                 y_vec};
  const bool w_al = aligned(w, 16) && ldw % 16 == 0 && ldw < (1 << 23);
  // A few tokens are quantised by every workgroup of the product itself.
  if (is_float(xt) && w_al && rows <= 16 && rows * k <= kFusedElements)
    return with_float(yt, [&](auto ty) {
      return with_float(xt, [&](auto tx) {
        return linear_few<decltype(ty), decltype(tx), 1>(a, s);
      });
    });
  if (is_float(xt)) {
    const int64_t ld = (int64_t)round_up((size_t)k, 16);
    int8_t* q = static_cast<int8_t*>(ws);
    float* sq = reinterpret_cast<float*>(q + rows * ld);
    const int st = quantise(xt, x, ldx, rows, k, q, ld, sq, s);
    if (st != CS_OK) return st;
    a.x = q; a.ldx = ld; a.sx = sq;
  }
  // whole 16-byte loads, offsets of a tile's rows in 32 bits
  const bool al = w_al && aligned(a.x, 16) && a.ldx % 16 == 0 && a.ldx < (1 << 23);
  return with_float(yt, [&](auto t) {
    using T = decltype(t);
    if (!al) {
      dim3 grid = cs::wide_grid((rows + 63) / 64);
      grid.z = (unsigned)(((int64_t)d_out + 63) / 64);
      hipLaunchKernelGGL((cs::linear_q8_any<T>), grid, dim3(256), 0, s, a);
      return launched();
    }
    auto tiles = [&](int bm, int bn) {
      return ((rows + bm - 1) / bm) * (((int64_t)d_out + bn - 1) / bn);
    };
    // tokens x k x d_out in us, registers alone | 64 x 64 tiles: 16 x 2,048 x 1,000 4.3 | 6.0, 16 x
    // 8,192 x 8,192 19.2 | 19.1; 32 x 2,048 x 1,000 5.4 | 6.2, 32 x 8,192 x 1,024 12.9 | 15.3, 32 x
    // 1,024 x 8,192 5.6 | 4.8, 32 x 8,192 x 8,192 26.6 | 19.2; 48 x 512 x 512 4.9 | 3.8
    if (rows <= 16) return linear_few<T, int8_t, 1>(a, s);
    if (rows <= 32 && d_out <= 2048) return linear_few<T, int8_t, 2>(a, s);
    // the largest tile of which there are enough to keep most compute units busy: 2,048 x 4,096 x
    // 4,096 40 us in 128 x 128, 59 in 64 x 64; 8,192 x 4,096 x 8,192 with its tokens quantised 321
    // in 256 x 256, 361 in 128 x 128 (before both stored whole rows; 302 now)
    if (tiles(256, 256) >= 200) return linear_tiles<T, 256, 256, 128, 64, 2>(a, s);
    if (tiles(128, 128) >= 200) return linear_tiles<T, 128, 128, 64, 64, 2>(a, s);
    return linear_tiles<T, 64, 64, 32, 32, 4>(a, s);
  });
}

int cs_cache_write(const cs_q8_cache* cache, cs_dtype xt, const void* k, int64_t ldk, int64_t hsk,
                   const void* v, int64_t ldv, int64_t hsv, const int64_t* slots, int64_t tokens,
                   void* stream) {
  if (!is_float(xt)) return CS_ERR_DTYPE;
  cs::CacheView c;
  const int st = cache_view(cache, &c);
  if (st != CS_OK) return st;
  if (tokens < 0) return CS_ERR_ARG;
  if (tokens == 0) return CS_OK;
  if (!k || !v || !slots || !aligned(k, float_size(xt)) || !aligned(v, float_size(xt)) ||
      !aligned(slots, 8))
    return CS_ERR_ARG;
  if (ldk < 0 || ldv < 0 || hsk < c.d || hsv < c.d) return CS_ERR_SHAPE;
  if (tokens > kMaxCount / c.heads) return CS_ERR_SHAPE;
  const uint32_t rows = (uint32_t)(tokens * c.heads);
  const dim3 block(256);
  dim3 grid = cs::wide_grid(((int64_t)rows + 15) / 16);
  grid.z = 2;
  return with_float(xt, [&](auto t) {
    using T = decltype(t);
    const int64_t e = sizeof(T);
    const bool vec = aligned(k, 16) && aligned(v, 16) && ldk * e % 16 == 0 && ldv * e % 16 == 0 &&
                     hsk * e % 16 == 0 && hsv * e % 16 == 0;
    const cs::FastDiv by = cs::make_fastdiv((uint32_t)c.heads);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (vec)
      hipLaunchKernelGGL((cs::cache_write<T, true>), grid, block, 0, s, c,
                         static_cast<const T*>(k), ldk, hsk, static_cast<const T*>(v), ldv, hsv,
                         slots, rows, by);
    else
      hipLaunchKernelGGL((cs::cache_write<T, false>), grid, block, 0, s, c,
                         static_cast<const T*>(k), ldk, hsk, static_cast<const T*>(v), ldv, hsv,
                         slots, rows, by);
    return launched();
  });
}

int cs_cache_read(const cs_q8_cache* cache, const int64_t* slots, int64_t tokens, cs_dtype yt,
                  void* k, void* v, void* stream) {
  if (!is_float(yt)) return CS_ERR_DTYPE;
  cs::CacheView c;
  const int st = cache_view(cache, &c);
  if (st != CS_OK) return st;
  if (tokens < 0) return CS_ERR_ARG;
  if (tokens == 0) return CS_OK;
  if (!k || !v || !slots || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8))
    return CS_ERR_ARG;
  if (tokens > kMaxCount / c.heads) return CS_ERR_SHAPE;
  const uint32_t rows = (uint32_t)(tokens * c.heads);
  const dim3 block(256);
  dim3 grid = cs::wide_grid(((int64_t)rows + 15) / 16);
  grid.z = 2;
  return with_float(yt, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL((cs::cache_read<T>), grid, block, 0, static_cast<hipStream_t>(stream), c,
                       slots, rows, cs::make_fastdiv((uint32_t)c.heads), static_cast<T*>(k),
                       static_cast<T*>(v));
    return launched();
  });
}

size_t cs_paged_attention_workspace_bytes(const cs_q8_cache* cache, cs_dtype qt, int tokens,
                                          int q_heads, int batch, int table_width, int max_len) {
  cs::CacheView c;
  if (!is_float(qt) || cache_view(cache, &c) != CS_OK) return 0;
  if (tokens < 1 || q_heads < 1 || batch < 1 || table_width < 1 || max_len < 0) return 0;
  if (!attention_fits(c, tokens, q_heads, table_width)) return 0;
  // the whole axis: a window or a shorter one has at most as many parts
  const AttentionPlan p = attention_plan(c, qt, tokens, q_heads, batch, table_width, max_len, 0);
  return attention_part_bytes(p.most, (int64_t)tokens * q_heads, c.d);
}

int cs_paged_attention_plan(const cs_q8_cache* cache, cs_dtype qt, int tokens, int q_heads,
                            int batch, int table_width, int max_len, int window, int64_t* info) {
  if (!info) return CS_ERR_ARG;
  if (!is_float(qt)) return CS_ERR_DTYPE;
  cs::CacheView c;
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
  info[3] = p.per == 16 ? p.waves : 4;
  info[4] = p.tiles * c.heads * p.splits;
  info[5] = (int64_t)attention_part_bytes(p.splits, (int64_t)tokens * q_heads, c.d);
  return CS_OK;
}

int cs_paged_attention(const cs_q8_cache* cache, cs_dtype qt, const void* q, int64_t ldq,
                       int64_t hsq, int tokens, int q_heads, int batch, const int32_t* table,
                       int table_width, const int32_t* lens, const int32_t* starts, int max_len,
                       float scale, int window, void* out, void* ws, size_t ws_bytes,
                       void* stream) {
  if (!is_float(qt)) return CS_ERR_DTYPE;
  cs::CacheView c;
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
  const size_t need = std::max(cs_paged_attention_workspace_bytes(cache, qt, tokens, q_heads, batch,
                                                                  table_width, max_len),
                               attention_part_bytes(p.splits, rows, c.d));
  if (need > 0 && (!ws || ws_bytes < need || !aligned(ws, 16))) return CS_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int e = (int)float_size(qt);
  const bool vec = aligned(q, 16) && (tokens == 1 || ldq * e % 16 == 0) && hsq * e % 16 == 0;
  cs::PagedAttention a{c, q, ldq, hsq, vec, tokens, q_heads, group, batch,
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
    const dim3 grid = cs::wide_grid(blocks), block(256);
    auto few = [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
      if (p.waves == 8)
        hipLaunchKernelGGL((cs::attention_few<T, DT, 8>), grid, dim3(512), 0, s, a);
      else
        hipLaunchKernelGGL((cs::attention_few<T, DT, 4>), grid, dim3(256), 0, s, a);
    };
    auto many = [&](auto dt) {
      constexpr int W = decltype(dt)::value, DT = W <= 64 ? 64 : W <= 128 ? 128 : 256;
      hipLaunchKernelGGL((cs::attention_many<T, W>), grid, block, cs::ManyLds<DT>::bytes, s,
                         a);
    };
    if (p.per == 16) with_width(c.d, few);
    else if (c.d > 64 && c.d <= 96) many(std::integral_constant<int, 96>{});
    else if (c.d > 128 && c.d <= 192) many(std::integral_constant<int, 192>{});
    else with_width(c.d, many);
    int r = launched();
    if (r == CS_OK && p.splits > 1) {
      hipLaunchKernelGGL((cs::attention_join<T>), dim3((unsigned)rows), block, 0, s, a);
      r = launched();
    }
    return r;
  });
}

}  // extern "C"
