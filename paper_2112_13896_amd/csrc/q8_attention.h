// Attention of new tokens over the paged int8 cache: token i of sequence b,
// at position p = len_b - n_b + i, has o = sum_j e_j v_j / sum_j e_j with
// e_j = exp(scale * q.k_j) over the positions j in (p - window, p].
//
// What both kernels below share:
//  - The rows of a cache head are the (new token, query head) pairs that read
//    it, token-major: row r is token r / group, head r % group.
//  - Products run on the f16 matrix instructions.  A code is exact in f16; a
//    query row is scaled by a power of two so that its largest element lies
//    in [2^8, 2^9), which keeps a 16-bit query exact or within 2^-25 of its
//    largest element.  fp32 queries are held as two halves (22 bits), and so
//    are the weights that multiply the values: twice the products, and an
//    error of fp32's order.
//  - Logits are formed transposed (keys x rows), so that a lane holds several
//    keys of one row: maximum and sum run mostly inside a lane, and the
//    weights are already laid out as the operand of the second product
//    (channels x rows), whose order of keys only has to agree with the
//    values' operand.
//  - With v_j = sv_j * code_j, a weight that meets the codes is e_j * sv_j.
//    To round it to f16 it is kept relative to the row's own largest: with
//    sv_j = a_j 2^E_j (1 <= a_j < 2), x_j = log2(e_j) + E_j and m the running
//    maximum of x_j over the keys the row sees, w_j = a_j 2^(x_j - m + 12) is
//    at most 2^13 and the denominator is the sum of w_j / sv_j.
//    A token with large values that a row does not see, or hardly weighs,
//    takes no precision from the others.  m follows the maximum only when that
//    is more than 4 (2^2) above it: halves have the room, and the sums so far
//    are rescaled rarely.
//  - Over values below 1e-21 or so 1 / sv could take the denominator past 32-bit
//    floats.  A row whose denominator gets large holds it times 2^-60 (SumUnit).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "q8_places.h"
#include "q8_rows.h"

namespace cs {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename View>
struct PagedAttentionOf {
  View c;
  const void* q;
  int64_t ldq, hsq;
  int q_vec;           // query heads start on 16 bytes
  int tokens, q_heads, group, batch;
  FastDiv by_group, by_heads, by_tiles;
  const int32_t* table;
  int table_width;
  const int32_t* lens;
  const int32_t* starts;
  float scale;
  int window;          // 0: none
  void* out;
  int splits, chunk;   // parts of the key axis and their length (the last takes the rest)
  float* part_o;       // [splits][tokens * q_heads][d], splits > 1
  float2* part_ml;     // [splits][tokens * q_heads]: m, l
};
typedef PagedAttentionOf<CacheView> PagedAttention;

// Workgroups go to the eight XCDs in turn: heads vary fastest, so that the
// tiles and parts that read one head's keys meet in few L2s (with eight heads,
// or a multiple, in one).
template <typename View>
__device__ __forceinline__ bool place(const PagedAttentionOf<View>& a, int* head, int* tile,
                                      int* split) {
  const uint32_t id = workgroup(), rest = fdiv(id, a.by_heads);
  *head = (int)(id - rest * a.by_heads.d);
  const uint32_t s = fdiv(rest, a.by_tiles);
  *tile = (int)(rest - s * a.by_tiles.d);
  *split = (int)s;
  return *split < a.splits;
}

// A tile of `per` rows of one sequence.  Sequence b's tiles have the numbers
// from starts[b] * group / per + b on, which leaves room for its last, partial
// one; the sequence of a tile is the number of sequences b >= 1 whose first
// tile is not past it, counted 64 at a time (one load's latency, where a
// binary search has one per level).  The few numbers without rows leave at
// once.  Tokens past the last sequence are a sequence of length 0.
struct RowTile {
  int b, token0, n;    // sequence, its first new token, its new tokens
  int row0, rows;      // first row of the tile in the sequence, the sequence's rows
  int len;             // positions
};

template <typename View>
__device__ __forceinline__ bool find_tile(const PagedAttentionOf<View>& a, int tile, int per,
                                          RowTile* t) {
  auto base = [&](int b, int start) { return (int)((int64_t)start * a.group / per) + b; };
  const int lane = threadIdx.x % 64;
  int b = 0;
  for (int b0 = 1; b0 <= a.batch; b0 += 64) {
    const int i = min(b0 + lane, a.batch);
    const bool past = b0 + lane > a.batch || base(i, a.starts[i]) > tile;
    const uint64_t later = __builtin_amdgcn_ballot_w64(past);
    b += later ? __builtin_ctzll(later) : 64;
    if (later) break;
  }
  const int start = a.starts[b];
  t->b = b;
  t->token0 = min(max(start, 0), a.tokens);
  const int end = b == a.batch ? a.tokens : min(max(a.starts[b + 1], 0), a.tokens);
  t->n = max(end - t->token0, 0);
  t->rows = t->n * a.group;
  t->row0 = (tile - base(b, start)) * per;
  t->len = b == a.batch ? 0 : min(max(a.lens[b], 0), a.table_width << a.c.page_log);
  return t->row0 >= 0 && t->row0 < t->rows;
}

// Position of a sequence's new token; those before the sequence's first
// position see nothing, wherever they are.
__device__ __forceinline__ int position(const RowTile& t, int token) {
  return max(t.len - t.n + token, -1);
}

// Positions [lo, hi) that some row of tokens t0 .. t1 of the tile sees.
template <typename View>
__device__ __forceinline__ void tile_keys(const PagedAttentionOf<View>& a, const RowTile& t,
                                          int t0, int t1, int* lo, int* hi) {
  const int p0 = position(t, t0), p1 = position(t, t1);
  *hi = p1 + 1;
  *lo = a.window > 0 ? max(p0 - a.window + 1, 0) : 0;
}

// Four codes (a dword) as two pairs of halves code * 2^-9: the byte with its
// sign bit turned is code + 128; alone in a half it is a denormal number,
// (code + 128) 2^-24, and one fused multiply-add takes it to code * 2^-9,
// exactly.  `hi` and `lo` may be different dwords: that is the transposition
// of the values' bytes.
constexpr float kCodeScale = 512.0f;                       // undoes 2^-9
__device__ __forceinline__ f16x2 code_pair(uint32_t hi, uint32_t lo, uint32_t sel) {
  const uint32_t u = __builtin_amdgcn_perm(hi, lo, sel);
  f16x2 h;
  __builtin_memcpy(&h, &u, 4);
  const f16x2 up = {(_Float16)32768.0f, (_Float16)32768.0f};
  const f16x2 off = {(_Float16)-0.25f, (_Float16)-0.25f};
  return __builtin_elementwise_fma(h, up, off);
}
constexpr uint32_t kFlip = 0x80808080u;

// Eight codes of one row, in order (two dwords, flipped here).
__device__ __forceinline__ f16x8 codes_f16(uint32_t a, uint32_t b) {
  a ^= kFlip;
  b ^= kFlip;
  const f16x2 p0 = code_pair(a, a, 0x0C010C00u), p1 = code_pair(a, a, 0x0C030C02u);
  const f16x2 p2 = code_pair(b, b, 0x0C010C00u), p3 = code_pair(b, b, 0x0C030C02u);
  return f16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// Byte c of eight dwords (flipped already), in order.
template <int C>
__device__ __forceinline__ f16x8 codes_f16_across(const uint32_t (&v)[8]) {
  constexpr uint32_t sel = 0x0C000C00u | (uint32_t)C | ((uint32_t)(4 + C) << 16);
  const f16x2 p0 = code_pair(v[1], v[0], sel), p1 = code_pair(v[3], v[2], sel);
  const f16x2 p2 = code_pair(v[5], v[4], sel), p3 = code_pair(v[7], v[6], sel);
  return f16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// Reductions over the lanes that share lane % 16 (four) or lane % 32 (two).
template <typename Op>
__device__ __forceinline__ float reduce_x32(float v, Op op) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename Op>
__device__ __forceinline__ float reduce_x16_x32(float v, Op op) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return reduce_x32(op(__uint_as_float(r[0]), __uint_as_float(r[1])), op);
}
struct FMax {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct FAdd {
  __device__ float operator()(float a, float b) const { return a + b; }
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
constexpr float kNegInf = -__builtin_inff();
constexpr float kHead = 12.0f;                             // weights are scaled by 2^12
constexpr float kSlack = 2.0f;                             // and may be 2^2 times that

// max(a, b, c), NaN ignored, as one instruction whatever the compiler knows of
// its operands.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// A query row's power of two and what turns its products into log2 units.
struct RowNorm {
  int shift;     // q * 2^shift is what the products take
  float c;       // logit * log2(e) = product * ks * c
  bool bad;      // not finite: the row's outputs are NaN
};
__device__ __forceinline__ RowNorm row_norm(float amax, float scale) {
  RowNorm r;
  r.bad = !(amax < __builtin_inff());
  int ex = 0;
  if (!r.bad && amax > 0.0f) ex = __builtin_amdgcn_frexp_expf(amax) - 1;
  r.shift = 8 - ex;
  r.c = ldexpf(scale * 1.4426950408889634f * kCodeScale, ex - 8);
  return r;
}

// How a token's values enter: sv = a 2^E.  Where all of a token's values are
// zero, so are its codes, and any scale does that leaves the others room.
// Scales below kLeast stand for kLeast, so that there is a 1 / sv.
constexpr float kLeast = 0x1p-122f;
struct ValueScale {
  float e, a, r;                                           // E, a, 1 / sv
};
__device__ __forceinline__ float held_scale(float sv) {    // NaN stays
  return sv == 0.0f ? 0x1p-60f : sv < kLeast ? kLeast : sv;
}
__device__ __forceinline__ ValueScale value_scale(float sv) {
  sv = held_scale(sv);
  ValueScale v;
  const int ex = max(__builtin_amdgcn_frexp_expf(sv) - 1, -120);
  v.e = (float)ex;
  v.a = ldexpf(sv, -ex);
  v.r = ldexpf(__builtin_amdgcn_rcpf(v.a), -ex);
  return v;
}

// Adds eight weights' share to a row's denominator (r: 1 / sv).  f16 outputs
// are as fine as the rounded weights, whose errors would show: there the sum
// takes the weights as rounded, so that their quotients still sum to 1 and a
// row that one key rules has no error from its rounding (but not those that
// are too small for a half to hold: their keys' values may be small, not their
// part in the sum).
template <typename T, int NP>
__device__ __forceinline__ float add_weights(float l, const float (&w)[8], const f16x8 (&p)[NP],
                                             const float (&r)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float t = w[i];
    if (std::is_same<T, _Float16>::value && t > 0x1p-13f) t = (float)p[0][i];
    l = fmaf(t, r[i], l);
  }
  return l;
}

// The unit that a row's denominator l is held in, 1 or 2^-60, and whether a row
// of the wavefront has the latter.
constexpr float kUnit = 0x1p-60f, kLarge = 0x1p90f;
struct SumUnit {
  float g = 1.0f;
  bool any = false;
};

// A lane's l in the unit that suits its row and what a step adds to it, p (in
// units of 1; it may be infinite).  `most`: the maximum over the row's lanes.
template <typename Most>
__device__ __forceinline__ float fit_unit(SumUnit& u, float l, float p, Most most) {
  const float row_p = most(p), row_l = most(l);            // (while all lanes are there)
  const bool large = row_p > kLarge || (u.g != 1.0f && row_l > kLarge * kUnit);
  const float g = large ? kUnit : 1.0f;
  if (g != u.g) l *= large ? kUnit : 1.0f / kUnit;
  u.g = g;
  u.any = __builtin_amdgcn_ballot_w64(large) != 0;
  return l;
}

// After the last step: numerator and denominator in one unit, that of m.
template <typename V, int N>
__device__ __forceinline__ void own_unit(const SumUnit& u, float& m, V (&o)[N]) {
  if (u.g != 1.0f) m += 60.0f;
#pragma unroll
  for (int x = 0; x < N; ++x) o[x] *= u.g;
}

template <typename T>
__device__ __forceinline__ void load_q8(const T* p, int vec, float (&f)[8]) {
  if (vec) load8(p, f);
  else load8_some(p, 8, f);
}

// One row's weights as operand halves: the value, and for fp32 what it lacks.
// The empty asm keeps w a rounded 32-bit number: the compiler may otherwise
// take a product and its conversion to half in one instruction (one rounding
// instead of two) for the first half only, and where the two roundings
// differ - one number in ten thousand - the second half would not be what the
// first one lacks.
template <int NP>
__device__ __forceinline__ void split_f16(const float (&w)[8], f16x8 (&p)[NP]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float v = w[j];
    if constexpr (NP == 2) asm volatile("" : "+v"(v));
    p[0][j] = (_Float16)v;
    if constexpr (NP == 2) p[1][j] = (_Float16)(v - (float)p[0][j]);
  }
}

// What a sum of weighted codes is multiplied by.
constexpr float out_unit(const CacheView&) { return kCodeScale; }
// Whether tokens past the last sequence have no parts: their zeros are written already.
constexpr bool rest_apart(const CacheView&) { return false; }

// The wavefronts' sums of up to 16 rows, in LDS, joined in order: 16 lanes to a
// row.
template <typename T, int NW, int DP, typename View>
__device__ __forceinline__ void few_out(const PagedAttentionOf<View>& a,
                                        const float (&l_o)[NW][16][DP],
                                        const float (&l_m)[NW][16], const float (&l_l)[NW][16],
                                        const RowTile& t, int rows_end, int head, int split) {
  const int d = a.c.d;
  const int rr = threadIdx.x / 16, x0 = threadIdx.x % 16;
  if (rr >= 16 || t.row0 + rr >= rows_end) return;
  float top = kNegInf;
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, l_m[w][rr]);
  const float base = top == kNegInf ? 0.0f : top;
  float f[NW], sum = 0.0f;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    // a wavefront without a key has sums of 0; one with NaN alone among its keys m = -inf
    f[w] = exp2_fast(l_m[w][rr] - base);
    sum = fmaf(l_l[w][rr], f[w], sum);
  }
  const int orow = t.row0 + rr;
  const int otok = (int)fdiv((uint32_t)orow, a.by_group);
  const int64_t ro = (int64_t)(t.token0 + otok) * a.q_heads + head * a.group + orow -
                     otok * a.group;
  const int64_t po = (int64_t)split * a.tokens * a.q_heads + ro;
  if (a.splits > 1 && x0 == 0) a.part_ml[po] = float2{top, sum};
  const float inv = sum == 0.0f ? 0.0f : out_unit(a.c) / sum;
  for (int x = 8 * x0; x < d; x += 128) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; ++w) s = fmaf(l_o[w][rr][x + i], f[w], s);
      v[i] = a.splits > 1 ? s : s * inv;
    }
    if (a.splits > 1) store8(a.part_o + po * d + x, v);
    else store8(static_cast<T*>(a.out) + ro * d + x, v);
  }
}

// ---------------------------------------------------------------- few rows
// attention_few: up to 16 rows of a cache head (a decoding token's query
// heads, a few drafted tokens) to a workgroup of NW wavefronts, the keys read
// once.  A wavefront takes 32 keys a step, every NW-th step of the
// workgroup's part of the key axis: keys and values go from memory to
// registers (no LDS) and are turned to halves there.
// Bound by memory: 64 sequences of up to 8,192 keys, 32 query and 8 cache
// heads of 128 (623 MB), take 135 us and 6.7 to join their parts, 4.6 TB/s of
// the 5.1 of a large copy; the vector units are busy 39 % of the time.  A
// sequence alone, 700 keys, eight wavefronts: 10.6 us, latency, 0.4 of them the
// check of each step's share of the denominator (SumUnit).
// What hides the loads is other wavefronts: registers for a step in flight
// ahead (157 us), or for a second tile of rows, would halve their number (two
// long sequences of 20 rows a head: 70 us with two tiles that both read the
// keys, the second out of the L2, 88 us with one of 32 rows; both before the
// check, with it 75 for the two tiles).
// Lane = 16 h + r.  Keys: the lane has row (key) r of two tiles of 16,
// channels h DT/4 .. ; values: keys 4h .. 4h+3 of both tiles, channels r DT/16
// .. ; logits: keys 4h .. 4h+3 of both tiles for row r.
template <typename T, int DT, int NW>
__global__ __launch_bounds__(64 * NW, DT == 256 ? 2 : DT == 128 && sizeof(T) == 4 ? 3 : 4)
void attention_few(PagedAttention a) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;
  constexpr int KS = DT / 32, CT = DT / 16;
  __shared__ float l_o[NW][16][DT + 4];
  __shared__ float l_m[NW][16], l_l[NW][16];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, h = lane / 16, d = a.c.d;
  int head, tile, split;
  if (!place(a, &head, &tile, &split)) return;
  RowTile t;
  if (!find_tile(a, tile, 16, &t)) return;
  const int rows_end = min(t.rows, t.row0 + 16);
  const int tok0 = (int)fdiv((uint32_t)t.row0, a.by_group);
  const int tok1 = (int)fdiv((uint32_t)(rows_end - 1), a.by_group);
  int lo, hi;
  tile_keys(a, t, tok0, tok1, &lo, &hi);
  const int pos0 = position(t, tok0);                      // every row sees up to pos0 ...
  const int see1 = a.window > 0 ? position(t, tok1) - a.window + 1 : 0;   // ... from see1 on
  // this workgroup's part
  const int j0 = lo / 32 * 32 + split * a.chunk;
  if (split + 1 < a.splits) hi = min(hi, j0 + a.chunk);
  const int steps = hi > j0 ? (hi - j0 + 31) / 32 : 0;

  // the query rows' operand
  const int row = min(t.row0 + r, t.rows - 1);
  const int tok = (int)fdiv((uint32_t)row, a.by_group);
  const int pos = position(t, tok);                        // the row sees up to pos
  f16x8 q[NP][KS];
  float c;
  {
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(t.token0 + tok) * a.ldq +
                  (head * a.group + row - tok * a.group) * a.hsq;
    float f[KS][8];
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int ch = h * (DT / 4) + 8 * s;
      if (ch < d) load_q8(qp + ch, a.q_vec, f[s]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (ch >= d) f[s][e] = 0.0f;
        top = max(top, abs_bits(f[s][e]));
      }
    }
    // bits of magnitudes are ordered as unsigned numbers, and as floats but for NaN
    const auto s16 = __builtin_amdgcn_permlane16_swap(top, top, false, false);
    top = max(s16[0], s16[1]);
    const auto s32 = __builtin_amdgcn_permlane32_swap(top, top, false, false);
    const RowNorm nm = row_norm(__uint_as_float(max(s32[0], s32[1])), a.scale);
    c = nm.c;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f[s][e] = nm.bad ? __uint_as_float(0x7FC00000u) : ldexpf(f[s][e], nm.shift);
      f16x8 p[NP];
      split_f16<NP>(f[s], p);
#pragma unroll
      for (int n = 0; n < NP; ++n) q[n][s] = p[n];
    }
  }

  const int32_t* table = a.table + (int64_t)t.b * a.table_width;
  const int lg = a.c.page_log, in_page = (1 << lg) - 1, n_pages = (int)(a.c.slots >> lg);
  int page[2];                                             // of the two tiles of 16 keys
  auto pages = [&](int j) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      page[u] = __builtin_amdgcn_readfirstlane(table[min(j + 16 * u, hi - 1) >> lg]);
  };
  f32x4 o[CT];
#pragma unroll
  for (int x = 0; x < CT; ++x) o[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = kNegInf, l = 0.0f;
  SumUnit unit;
  if (wave < steps) pages(j0 + 32 * wave);
  for (int step = wave; step < steps; step += NW) {
    const int j = j0 + 32 * step;
    u32x4 kr[2][DT / 64];
    uint32_t vr[DT / 64][8];
    f32x4 ks[2], vs[2];
    bool ok[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ok[u] = (uint32_t)page[u] < (uint32_t)n_pages;
      // no page: any rows, which are masked
      const int64_t row0 = (((int64_t)(ok[u] ? page[u] : 0) * a.c.heads + head) << lg) +
                           ((j + 16 * u) & in_page);
      const int8_t* kp = a.c.k + row0 * d;
#pragma unroll
      for (int p = 0; p < DT / 64; ++p) {
        const int ch = h * (DT / 4) + 16 * p;              // channels past d meet zeros in q
        kr[u][p] = *reinterpret_cast<const u32x4*>(kp + (uint32_t)(r * d + (ch < d ? ch : 0)));
      }
      // scales start on 4 bytes
      __builtin_memcpy(&ks[u], __builtin_assume_aligned(a.c.ks + row0 + 4 * h, 4), 16);
      __builtin_memcpy(&vs[u], __builtin_assume_aligned(a.c.vs + row0 + 4 * h, 4), 16);
      const int ch = r * (DT / 16);                        // channels past d are not stored
      const int8_t* vp = a.c.v + row0 * d;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[DT / 64];
        __builtin_memcpy(w,
                         __builtin_assume_aligned(
                             vp + i * d + (uint32_t)(4 * h * d + (ch < d ? ch : 0)), DT / 16),
                         DT / 16);
#pragma unroll
        for (int x = 0; x < DT / 64; ++x) vr[x][4 * u + i] = w[x];
      }
    }
    if (step + NW < steps) pages(j + 32 * NW);
    f32x4 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      s[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const f16x8 kf = codes_f16(kr[u][k / 2][k % 2 * 2], kr[u][k / 2][k % 2 * 2 + 1]);
#pragma unroll
        for (int n = 0; n < NP; ++n)
          s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, q[n][k], s[u], 0, 0, 0);
      }
    }
    // logits in log2 units, plus E
    float x[8], av[8], rv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const ValueScale sv = value_scale(vs[i / 4][i % 4]);
      av[i] = sv.a;
      rv[i] = sv.r;
      x[i] = fmaf(s[i / 4][i % 4] * ks[i / 4][i % 4], c, sv.e);
    }
    // hidden keys: past the row's position (the last part's end), before its window, no page
    if (j + 31 > pos0 || j < see1 || !ok[0] || !ok[1]) {
      const int see = a.window > 0 ? pos - a.window + 1 : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = j + 16 * (i / 4) + 4 * h + i % 4;
        if (key > pos || key < see || !ok[i / 4]) {
          x[i] = kNegInf;
          av[i] = rv[i] = 0.0f;                            // (they may be NaN)
        }
      }
    }
    float top = max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), max3(m, x[6], x[7]));
    top = reduce_x16_x32(top, FMax{});
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
      const float f = top == kNegInf ? 1.0f : exp2_fast(m - top);
      l *= f;
#pragma unroll
      for (int z = 0; z < CT; ++z) o[z] *= f;
      m = top;
    }
    const float base = m == kNegInf ? 0.0f : m - kHead;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = exp2_fast(x[i] - base) * av[i];
    f16x8 p[NP];
    split_f16<NP>(w, p);
    float sum = add_weights<T, NP>(0.0f, w, p, rv);
    auto values = [&](auto cc, int xw) {
      constexpr int C = decltype(cc)::value;
      const f16x8 vf = codes_f16_across<C>(vr[xw]);
#pragma unroll
      for (int n = 0; n < NP; ++n)
        o[4 * xw + C] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p[n], o[4 * xw + C], 0, 0, 0);
    };
#pragma unroll
    for (int xw = 0; xw < DT / 64; ++xw) {
#pragma unroll
      for (int i = 0; i < 8; ++i) vr[xw][i] ^= kFlip;
      values(std::integral_constant<int, 0>{}, xw);
      values(std::integral_constant<int, 1>{}, xw);
      values(std::integral_constant<int, 2>{}, xw);
      values(std::integral_constant<int, 3>{}, xw);
    }
    if (__builtin_expect(unit.any || __builtin_amdgcn_ballot_w64(sum > kLarge), 0)) {
      l = fit_unit(unit, l, sum, [](float v) { return reduce_x16_x32(v, FMax{}); });
#pragma unroll
      for (int i = 0; i < 8; ++i) rv[i] *= unit.g;
      sum = add_weights<T, NP>(0.0f, w, p, rv);
    }
    l += sum;
  }

  // the wavefronts' sums, joined in order
  l = reduce_x16_x32(l, FAdd{});
  if (unit.any) own_unit(unit, m, o);
  if (h == 0) {
    l_m[wave][r] = m;
    l_l[wave][r] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int x = 0; x < CT; x += 4)
      *reinterpret_cast<f32x4*>(&l_o[wave][r][(4 * h + i) * CT + x]) =
          f32x4{o[x][i], o[x + 1][i], o[x + 2][i], o[x + 3][i]};
  __syncthreads();
  few_out<T>(a, l_o, l_m, l_l, t, rows_end, head, split);
}

// ---------------------------------------------------------------- many rows
// attention_many: 128 rows of a cache head to a workgroup of four wavefronts,
// 32 rows each, 64 keys a step.  A step's codes are turned to halves once for
// all four: keys [64][DT], values transposed [DT][64], both in 16-byte chunks
// whose place in a row is permuted (xor) so that the lanes that read a column
// of chunks together meet all banks; two buffers.  The next step's codes are
// turned at the start of a step, beside its first products, and the ones after
// that are then on their way in registers under all of its arithmetic; one
// barrier a step.  Two wavefronts bring the values, two the keys, by blocks of
// 16 (a piece of one page, so their addresses are scalar).  W <= DT: channels
// that are computed, d rounded up to 32.
// Four prompts of 2,048 after up to 4,096 positions, 32 query and 8 cache heads
// of 128, bf16 (409 GFLOP): 566-603 us, 680-720 TFLOP/s (1.7 % of it the check
// of a step's share of the denominator).  Bound by each
// wavefront's own stream of some 700 instructions a step: the registers allow
// two wavefronts a SIMD, and with matrix units busy for 29 % and vector units
// for 48 % of the time neither is full.  Measured by leaving work out: loads 18 %
// of the time, the first product 20, the second 15, exponentials 7, turning
// codes 4.  Slower: 32 keys a step (720 us: twice the barriers; with three
// wavefronts a SIMD registers spill, 808), the next half step's logits among
// this one's exponentials (613: spills).  fp32 queries take twice the products.
// Lane = 32 h + r.  Logits (32 keys x 32 rows): keys 8 y + 4 h .. +3 (y =
// 0..3) of row r.  So a lane's eight weights of 16 keys are those at 4 h ..
// and 8 + 4 h .., and the values' chunk g = 2 s + h of a channel holds just
// the keys 16 s + 4 h .. +3 and 16 s + 8 + 4 h .. +3.
// Here a = 1, E = log2(sv), taken once a step.
//
// Where a chunk lies (ManyPlaces): key k's chunk i (channels 8 i ..) at byte
// (k DT 2) + 16 (i ^ key_turn(k)), channel c's chunk g of values at byte 128 c +
// 16 (g ^ chunk_turn(c)).
// A step's share of the denominator is added up before its unit is known: 32
// weights of up to 2^14 over values of 2^-122 would pass 2^128.
constexpr float kUp = 0x1p24f;
template <int DT>
struct ManyLds {                                           // bytes
  static constexpr int k = 0;                              // [2][64][DT] halves
  static constexpr int v = 2 * 64 * DT * 2;                // [2][DT][64] halves
  static constexpr int ks = 2 * v;                         // [2][64] ks * c0
  static constexpr int ls = ks + 512;                      // [2][64] log2(vs)
  static constexpr int rs = ls + 512;                      // [2][64] 1 / (vs * up)
  static constexpr int up = rs + 512;                      // [2] up: 1, kUp beside a small value
  static constexpr int bytes = up + 16;
  static constexpr int buffer = ManyPlaces<DT>::buffer;    // one of two, keys or values
};

template <typename T, int W>
__global__ __launch_bounds__(256, W > 128 ? 1 : 2) void attention_many(PagedAttention a) {
  constexpr int DT = W <= 64 ? 64 : W <= 128 ? 128 : 256;
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;
  constexpr int KS = W / 16, CT = W / 32;
  using At = ManyLds<DT>;
  using Place = ManyPlaces<DT>;
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int r = lane % 32, h = lane / 32, d = a.c.d;
  int head, tile, split;
  if (!place(a, &head, &tile, &split)) return;
  RowTile t;
  // the last tiles of a sequence see most keys: first
  if (!find_tile(a, (int)a.by_tiles.d - 1 - tile, 128, &t)) return;
  const int rows_end = min(t.rows, t.row0 + 128);
  const int row = t.row0 + wave * 32 + r;
  const int row_c = min(row, t.rows - 1);
  const int tok = (int)fdiv((uint32_t)row_c, a.by_group);
  const int qh = head * a.group + row_c - tok * a.group;
  int lo, hi;
  tile_keys(a, t, (int)fdiv((uint32_t)t.row0, a.by_group),
            (int)fdiv((uint32_t)(rows_end - 1), a.by_group), &lo, &hi);
  const int pos = position(t, tok), see = a.window > 0 ? pos - a.window + 1 : 0;
  // the wavefront's rows all see up to pos0 and from see1 on
  const int w0 = min(t.row0 + wave * 32, t.rows - 1), w1 = min(w0 + 31, t.rows - 1);
  const int pos0 = position(t, (int)fdiv((uint32_t)w0, a.by_group));
  const int pos1 = position(t, (int)fdiv((uint32_t)w1, a.by_group));
  const int see1 = a.window > 0 ? pos1 - a.window + 1 : 0;
  const int j0 = lo / 64 * 64 + split * a.chunk;
  if (split + 1 < a.splits) hi = min(hi, j0 + a.chunk);
  const int steps = hi > j0 ? (hi - j0 + 63) / 64 : 0;

  // Queries whose largest element lies in [1, 2^10) are taken as they are; c0
  // is then all that turns a product into log2 units, and it is multiplied
  // into the keys' scales.  Other rows get a power of two (row_mul undoes it).
  const float c0 = a.scale * 1.4426950408889634f * kCodeScale;
  f16x8 q[NP][KS];
  float row_mul = 1.0f;
  {
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(t.token0 + tok) * a.ldq + qh * a.hsq;
    float f[KS][8];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int ch = 16 * s + 8 * h;
      load_q8(qp + (ch < d ? ch : 0), a.q_vec, f[s]);      // all loads before the first use
    }
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (16 * s + 8 * h >= d) f[s][e] = 0.0f;
        top = max(top, abs_bits(f[s][e]));
      }
    const auto s32 = __builtin_amdgcn_permlane32_swap(top, top, false, false);
    const float big = __uint_as_float(max(s32[0], s32[1]));
    const bool bad = !(big < __builtin_inff());
    int shift = 0;
    if (!bad && big > 0.0f && !(big >= 1.0f && big < 1024.0f))
      shift = 9 - __builtin_amdgcn_frexp_expf(big);
    row_mul = ldexpf(1.0f, -shift);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f[s][e] = bad ? __uint_as_float(0x7FC00000u) : ldexpf(f[s][e], shift);
      f16x8 p[NP];
      split_f16<NP>(f[s], p);
#pragma unroll
      for (int n = 0; n < NP; ++n) q[n][s] = p[n];
    }
  }
  const bool scaled = __builtin_amdgcn_ballot_w64(row_mul != 1.0f) != 0;

  // staging: this wavefront's blocks of 16 keys are 2 half and 2 half + 1
  const int32_t* table = a.table + (int64_t)t.b * a.table_width;
  const int lg = a.c.page_log, in_page = (1 << lg) - 1, n_pages = (int)(a.c.slots >> lg);
  const bool brings_values = wave < 2;
  const int half = wave % 2;
  constexpr int KB = Place::KB, PR = Place::PR, VD = Place::VD;
  const int k_key = Place::key(lane), k_ch = Place::key_channel(lane);
  const int v_ch = Place::value_channel(lane);
  // byte of a block that this lane loads first (channels past d: any)
  const uint32_t off = brings_values
                           ? Place::value_key(lane / 16 % 2, 0) * d + (v_ch < d ? v_ch : 0)
                           : k_key * d + (k_ch < d ? k_ch : 0);
  uint32_t reg[8 * VD];                                    // both blocks' keys; one's values
  float meta = 0.0f;
  bool meta_ok = false;
  int page[4];
  auto pages = [&](int j) {
#pragma unroll
    for (int b = 0; b < 4; ++b)
      page[b] = __builtin_amdgcn_readfirstlane(table[min(j + 16 * b, hi - 1) >> lg]);
  };
  // first row of block b; a page outside the cache: any rows, hidden by `meta_ok`
  auto block_row = [&](int pg, int j, int b) {
    return (((int64_t)((uint32_t)pg < (uint32_t)n_pages ? pg : 0) * a.c.heads + head) << lg) +
           ((j + 16 * b) & in_page);
  };
  auto fetch = [&](int j) {
    const int64_t at0 = block_row(half ? page[2] : page[0], j, 2 * half) * d;
    const int64_t at1 = block_row(half ? page[3] : page[1], j, 2 * half + 1) * d;
    if (brings_values) {
      const int8_t* vp = a.c.v + (lane < 32 ? at0 : at1) + off;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t w[VD];
        __builtin_memcpy(
            w, __builtin_assume_aligned(vp + (int64_t)Place::value_key(0, i) * d, 4 * VD), 4 * VD);
#pragma unroll
        for (int y = 0; y < VD; ++y) reg[8 * y + i] = w[y];
      }
    } else {
#pragma unroll
      for (int p = 0; p < 2 * KB; ++p) {
        const int8_t* kp = a.c.k + (p < KB ? at0 : at1) + p % KB * (64 / PR) * d;
        const u32x4 w = *reinterpret_cast<const u32x4*>(kp + off);
#pragma unroll
        for (int y = 0; y < 4; ++y) reg[4 * p + y] = w[y];
      }
    }
    if (!brings_values) {                                  // a lane has key `lane` of the step
      const int b = lane / 16;
      const int pg = b == 0 ? page[0] : b == 1 ? page[1] : b == 2 ? page[2] : page[3];
      const int64_t at = block_row(pg, j, b) + lane % 16;
      meta = (half ? a.c.vs : a.c.ks)[at];                 // (not touched here: that would wait)
      meta_ok = (uint32_t)pg < (uint32_t)n_pages;
    }
  };
  auto put = [&](int at, f16x8 v) { *reinterpret_cast<f16x8*>(smem + at) = v; };
  // the lane's first row in LDS and the place of its chunk there (which the rows' numbers turn)
  const int put_row = brings_values ? At::v + Place::value_row(lane)
                                    : At::k + Place::key_row(half, lane);
  const int put_bits = brings_values ? Place::value_bits(half, lane) : Place::key_bits(half, lane);
  auto stage = [&](auto par) {                             // buffer par
    constexpr int P = decltype(par)::value, kBuf = P * At::buffer;
    if (brings_values) {
#pragma unroll
      for (int y = 0; y < VD; ++y) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = reg[8 * y + i] ^ kFlip;
        auto at = [&](int c) {                             // channel v_ch + 4 y + c
          return kBuf + Place::value_put(put_row, put_bits, 4 * y + c);
        };
        put(at(0), codes_f16_across<0>(w));
        put(at(1), codes_f16_across<1>(w));
        put(at(2), codes_f16_across<2>(w));
        put(at(3), codes_f16_across<3>(w));
      }
    } else {
#pragma unroll
      for (int p = 0; p < 2 * KB; ++p) {
        put(kBuf + Place::key_put(put_row, put_bits, p, 0), codes_f16(reg[4 * p], reg[4 * p + 1]));
        put(kBuf + Place::key_put(put_row, put_bits, p, 1),
            codes_f16(reg[4 * p + 2], reg[4 * p + 3]));
      }
    }
    if (!brings_values) {
      float* to = reinterpret_cast<float*>(smem + At::ks + P * 256) + lane;
      if (half) {
        const float sv = held_scale(meta);
        const bool num = meta == meta;
        const bool small = __builtin_amdgcn_ballot_w64(sv < 0x1p-64f) != 0;
        const float up = small ? kUp : 1.0f;
        to[(At::ls - At::ks) / 4] =            // no page: weight 0
            !meta_ok ? kNegInf : num ? __builtin_amdgcn_logf(sv) : meta;
        to[(At::rs - At::ks) / 4] = num ? 1.0f / (sv * up) : 1.0f;
        if (lane == 0) *reinterpret_cast<float*>(smem + At::up + P * 4) = up;
      } else {
        to[0] = meta_ok ? meta * c0 : 0.0f;
      }
    }
  };

  f32x16 o[CT];
#pragma unroll
  for (int x = 0; x < CT; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[x][i] = 0.0f;
  float m = kNegInf, l = 0.0f;
  SumUnit unit;
  // the chunks that a lane reads: of key r, of channel r
  constexpr int KA = Place::KA;
  int k_at[KA], v_at[4];
#pragma unroll
  for (int i = 0; i < KA; ++i) k_at[i] = At::k + Place::key_column(r, h, i);
#pragma unroll
  for (int i = 0; i < 4; ++i) v_at[i] = At::v + Place::value_column(r, h, i);
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  if (steps > 0) {
    pages(j0);
    fetch(j0);
    stage(Even{});
    pages(j0 + 64);
    if (steps > 1) fetch(j0 + 64);
    pages(j0 + 128);
  }
  __syncthreads();
  auto advance = [&](auto par, auto other, int step) {
    constexpr int P = decltype(par)::value;
    const int j = j0 + 64 * step;
    if (step + 1 < steps) stage(other);
    if (step + 2 < steps) {
      fetch(j + 128);
      pages(j + 192);
    }
    f32x16 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
    // the halves of the keys in turn; fp32's products one after the other: they are longer and
    // leave fewer registers
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      const int u = NP == 1 ? i % 2 : i / KS, k = NP == 1 ? i / 2 : i % KS;
      const f16x8 kf = *reinterpret_cast<const f16x8*>(smem + P * At::buffer +
                                                       Place::key_at(k_at[k % KA], u, k));
#pragma unroll
      for (int n = 0; n < NP; ++n)
        s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, q[n][k], s[u], 0, 0, 0);
    }
    if (scaled) {
      asm volatile("");                                    // a branch, not selects
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i / 16][i % 16] *= row_mul;
    }
    const unsigned char* meta_at = smem + At::ks + P * 256 + 16 * h;
    auto meta4 = [&](int which, int y) {                   // keys 8 y + 4 h ..
      return *reinterpret_cast<const f32x4*>(meta_at + (which - At::ks) + 32 * y);
    };
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const f32x4 ks = meta4(At::ks, y), ls = meta4(At::ls, y);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s[y / 4][y % 4 * 4 + i] = fmaf(s[y / 4][y % 4 * 4 + i], ks[i], ls[i]);
    }
    if (j + 63 > pos0) {
      const int last = pos - j - 4 * h;
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (Place::logit_key(0, i) > last) s[i / 16][i % 16] = kNegInf;
    }
    if (j < see1) {
      const int first = see - j - 4 * h;
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (Place::logit_key(0, i) < first) s[i / 16][i % 16] = kNegInf;
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < 32; i += 2) top = max3(top, s[i / 16][i % 16], s[i / 16][i % 16 + 1]);
    top = reduce_x32(top, FMax{});
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
      const float f = top == kNegInf ? 1.0f : exp2_fast(m - top);
      l *= f;
#pragma unroll
      for (int y = 0; y < CT; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[y][i] *= f;
      m = top;
    }
    const float base = m == kNegInf ? 0.0f : m - kHead;
    float lp = 0.0f;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      float w[8], rv[8];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const f32x4 rs = meta4(At::rs, 2 * v + y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[4 * y + i] = exp2_fast(s[v / 2][v % 2 * 8 + 4 * y + i] - base);
          rv[4 * y + i] = rs[i];
        }
      }
      f16x8 p[NP];
      split_f16<NP>(w, p);
      lp = add_weights<T, NP>(lp, w, p, rv);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const f16x8 vf = *reinterpret_cast<const f16x8*>(smem + P * At::buffer +
                                                         Place::value_at(v_at[v], ct));
#pragma unroll
        for (int n = 0; n < NP; ++n)
          o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, p[n], o[ct], 0, 0, 0);
      }
    }
    const float up = *reinterpret_cast<const float*>(smem + At::up + P * 4);
    if (__builtin_expect(unit.any || __builtin_amdgcn_ballot_w64(lp * up > kLarge), 0))
      l = fit_unit(unit, l, lp * up, [](float v) { return reduce_x32(v, FMax{}); });
    l = fmaf(lp, up * unit.g, l);
    __syncthreads();
  };
  for (int step = 0; step < steps; step += 2) {
    advance(Even{}, Odd{}, step);
    if (step + 1 < steps) advance(Odd{}, Even{}, step + 1);
  }
  l = reduce_x32(l, FAdd{});
  if (unit.any) own_unit(unit, m, o);
  if (row >= rows_end) return;
  const int64_t ro = (int64_t)(t.token0 + tok) * a.q_heads + qh;
  const bool part = a.splits > 1;
  const int64_t po = (int64_t)split * a.tokens * a.q_heads + ro;
  if (part && h == 0) a.part_ml[po] = float2{m, l};
  const float inv = part ? 1.0f : l == 0.0f ? 0.0f : kCodeScale / l;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int ch = 32 * ct + 8 * y + 4 * h;
      if (ch >= d) continue;
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = o[ct][4 * y + i] * inv;
      if (part) {
        *reinterpret_cast<f32x4*>(a.part_o + po * d + ch) = f32x4{v[0], v[1], v[2], v[3]};
      } else {
        typedef T t4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<t4*>(static_cast<T*>(a.out) + ro * d + ch) =
            t4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
      }
    }
}

// attention_join: the parts of a row, in a fixed order, a workgroup to a row.
// Lane s of each wavefront has part s's weight; a wavefront adds up every
// fourth part, so their loads wait for nothing but each other's turn, and the
// four sums meet in LDS.
constexpr int kMaxSplits = 64;

template <typename T, typename View>
__global__ __launch_bounds__(256) void attention_join(PagedAttentionOf<View> a) {
  __shared__ f32x4 l_y[4][64];
  const int lane = threadIdx.x % 64, d = a.c.d;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t rows = (int64_t)a.tokens * a.q_heads, row = blockIdx.x;
  if (rest_apart(a.c) && row >= (int64_t)a.starts[a.batch] * a.q_heads) return;
  float2 ml = float2{kNegInf, 0.0f};
  if (lane < a.splits) ml = a.part_ml[lane * rows + row];
  float top = ml.x;
  for (int x = 32; x > 0; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
  const float base = top == kNegInf ? 0.0f : top;
  const float f = exp2_fast(ml.x - base);                  // a part without a key: 0
  float sum = ml.y * f;                                    // (while all lanes are there)
  for (int x = 32; x > 0; x /= 2) sum += __shfl_xor(sum, x);
  const int ch = 4 * lane < d ? 4 * lane : 0;
  const float* po = a.part_o + row * d + ch;
  f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = wave; s0 < a.splits; s0 += 32)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = s0 + 4 * i;
      if (s < a.splits)
        y += *reinterpret_cast<const f32x4*>(po + s * rows * d) *
             __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s));
    }
  l_y[wave][lane] = y;
  __syncthreads();
  if (wave > 0 || 4 * lane >= d) return;
  y = l_y[0][lane] + l_y[1][lane] + l_y[2][lane] + l_y[3][lane];
  y *= sum == 0.0f ? 0.0f : out_unit(a.c) / sum;
  typedef T t4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<t4*>(static_cast<T*>(a.out) + row * d + ch) =
      t4{(T)y[0], (T)y[1], (T)y[2], (T)y[3]};
}

}  // namespace cs
