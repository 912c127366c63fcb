// Attention of new tokens over the paged 4-bit cache: token i of sequence b,
// at position p = len_b - n_b + i, has o = sum_j e_j v_j / sum_j e_j with
// e_j = exp(scale * q.k_j) over the positions j in (p - window, p].
//
// Rows (new token, query head), tiles of rows, parts of the key axis and the
// places of workgroups are those of the 8-bit cache's kernels.  What differs:
//  - Keys are never converted: the matrix cores multiply 4-bit codes, with a
//    power of two for every 32 channels, as the cache holds both.  The other
//    operand has four significant bits, so a query row is the sum of pieces, each
//    what the ones before leave, in units 2^-4 of theirs (2^-5 from the fourth on,
//    where all that is left is below half a step).  The row is first scaled by a
//    power of two, so that its largest element is near the end of the first
//    piece's range.
//    bf16: two pieces in e4m3, largest element in [2^7, 2^8).  They hold the eight
//    bits of every element that is not small; e4m3's least step, 2^-9 in units of
//    2^-4, leaves at most 2^-14 of the others: 2^-21 of the largest.
//    fp16 and fp32: four and five pieces in e2m3, which the matrix cores take at
//    twice the rate; largest element in [3.5, 7).  e2m3's step is 1/8 below 2, 1/4
//    from there and 1/2 from 4 on, so the first piece leaves at most 2^-2, the second
//    (up to 4 in its units) 2^-3 of them, and the others (up to 2) 2^-4 of theirs,
//    2^-13 and 2^-18 in the end: 2^-18.8 and 2^-23.8 of the largest element.  (e4m3
//    would take three and six pieces at half the rate: the time of six and twelve of
//    these.)
//  - Values go to bf16, exactly, by the scaled conversion, and meet weights
//    e_j = 2^(x_j - m) in bf16 pieces: two (16 bits), three (24) for fp32, whatever
//    the rows of a workgroup, so that a token's result has the same bits beside a
//    prompt as alone.  (One piece where 128 rows of bf16 share a workgroup: prompts
//    570 us instead of 750, but 8 bits: off by 4e-4 of their outputs' norm, and by up
//    to 2^-9 of the values where those cancel.)  bf16 has the exponents of 32-bit
//    floats, and the cache's scales end at 2^60, so no sum over 2^30 positions
//    overflows and weights need no scaling.
//  - The running maximum m follows the rows' maximum only when that is more
//    than 4 (2^2) above it: rescaling is rare.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx4_places.h"
#include "mx4_rows.h"
#include "q8_attention.h"

namespace cs {

typedef PagedAttentionOf<Mx4View> Mx4Attention;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float out_unit(const Mx4View&) { return 1.0f; }
constexpr bool rest_apart(const Mx4View&) { return true; }

constexpr int kFp8 = 0, kFp6 = 2, kFp4 = 4;                // operand formats
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

// The pieces of queries (their format, their number, log2 of their units) and of
// weights.
template <typename T>
struct Mx4Pieces {
  static constexpr int format = kFp6, q = sizeof(T) == 4 ? 5 : 4, w = sizeof(T) == 4 ? 3 : 2;
  static constexpr int unit(int n) { return n < 3 ? -4 * n : -5 * n + 2; }
  // elements of an operand are the channels in order: `half` of them, and the second half `apart`
  static constexpr int first(int h) { return 32 * h; }
  static constexpr int apart(int) { return 16; }
};
template <>
struct Mx4Pieces<__bf16> {
  static constexpr int format = kFp8, q = 2, w = 2;
  static constexpr int unit(int n) { return -4 * n; }
  // 16 channels of the operand's first half, and 16 of its second
  static constexpr int first(int h) { return 16 * h; }
  static constexpr int apart(int channels) { return channels / 2; }
};

// What a row is multiplied by before it is cut, log2: 8-bit pieces take a largest
// element in [2^7, 2^8), 6-bit ones in [3.5, 7).
template <typename T>
__device__ __forceinline__ int mx4_shift(float big) {
  if (!(big < __builtin_inff()) || big == 0.0f) return 0;
  const int ex = __builtin_amdgcn_frexp_expf(big);
  if (Mx4Pieces<T>::format == kFp8) return 8 - ex;
  return (__builtin_amdgcn_frexp_mantf(big) < 0.875f ? 3 : 2) - ex;
}

// Piece n of 32 elements as an operand; f becomes what it leaves, in the next
// piece's units.
template <typename T>
__device__ __forceinline__ i32x8 query_piece(float (&f)[32], int n) {
  const float up = ldexpf(1.0f, Mx4Pieces<T>::unit(n) - Mx4Pieces<T>::unit(n + 1));
  i32x8 out = {0, 0, 0, 0, 0, 0, 0, 0};
  if constexpr (Mx4Pieces<T>::format == kFp8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      int w = 0;
      w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
      out[i] = w;
      f[4 * i] = up * (f[4 * i] - __builtin_amdgcn_cvt_f32_fp8(w, 0));
      f[4 * i + 1] = up * (f[4 * i + 1] - __builtin_amdgcn_cvt_f32_fp8(w, 1));
      f[4 * i + 2] = up * (f[4 * i + 2] - __builtin_amdgcn_cvt_f32_fp8(w, 2));
      f[4 * i + 3] = up * (f[4 * i + 3] - __builtin_amdgcn_cvt_f32_fp8(w, 3));
    }
  } else {
    f32x16 even, odd;                                      // (the instruction takes them in turn)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] = f[2 * i];
      odd[i] = f[2 * i + 1];
    }
    const u32x6 w = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, 1.0f);
    const f32x32 held = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(w, 1.0f);
#pragma unroll
    for (int i = 0; i < 6; ++i) out[i] = (int)w[i];
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = up * (f[i] - held[i]);
  }
  return out;
}

// Eight weights as operands; each piece is what the ones before leave.
template <int NW>
__device__ __forceinline__ void weight_pieces(const float (&w)[8], bf16x8 (&p)[NW]) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    float a = w[j], b = w[j + 1];
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      const bf16x2 t = {(__bf16)a, (__bf16)b};             // one instruction
      p[n][j] = t[0];
      p[n][j + 1] = t[1];
      if (n + 1 == NW) break;
      uint32_t bits;
      __builtin_memcpy(&bits, &t, 4);
      a -= __uint_as_float(bits << 16);
      b -= __uint_as_float(bits & 0xFFFF0000u);
    }
  }
}

// Channels 2 B and 2 B + 1 (of eight codes) of eight tokens, as two operands.
template <int B>
__device__ __forceinline__ void values_across(const uint32_t (&v)[8], const float (&scale)[8],
                                              bf16x8 (&out)[2]) {
  uint32_t c[8], lo[4], hi[4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bf16x2 t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[i], scale[i], B);
    __builtin_memcpy(&c[i], &t, 4);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
    hi[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
  }
  __builtin_memcpy(&out[0], lo, 16);
  __builtin_memcpy(&out[1], hi, 16);
}

// A page number, as a scalar load whatever lies between it and the kernel's other
// accesses (the table does not change): a vector load here would wait for all the
// keys and values that are on their way.
typedef __attribute__((address_space(4))) const int32_t* ConstantInts;
__device__ __forceinline__ int mx4_page(const int32_t* table, int i) {
  return ((ConstantInts)(uintptr_t)table)[__builtin_amdgcn_readfirstlane(i)];
}

// Whether one of a dword's bytes is 255.
__device__ __forceinline__ bool has_bad(uint32_t w) {
  return ((~w - 0x01010101u) & w & 0x80808080u) != 0;
}
__device__ __forceinline__ uint32_t byte_of(uint32_t w, int i) { return w >> (8 * i) & 0xFFu; }

// A workgroup's head, tile of `per` rows and part.  Heads vary fastest (see
// place()), then tiles, then parts, the last parts first: those are long
// sequences', and whole.  Tiles are numbered sequence after sequence, with no
// number left out, so that workgroups without rows are the last of all (at every
// fourth place, say, they leave every fourth compute unit idle: three sequences of
// 70,000 to 100,000 keys, 20 rows each, 139 us then, 85 so).  Sequences' tiles are added up 64 at a
// time.  Tokens past the last sequence have none: mx4_rest writes their zeros.
__device__ __forceinline__ bool mx4_place(const Mx4Attention& a, int per, int* head, RowTile* t,
                                          int* split) {
  const int lane = threadIdx.x % 64;
  const uint32_t id = workgroup();
  int tile = (int)fdiv(id, a.by_heads);
  *head = (int)(id - tile * a.by_heads.d);
  int start, n, tiles;                                     // of sequence b0 + lane
  auto count = [&](int b0) {                               // tiles up to the lane's sequence
    const int b = min(b0 + lane, a.batch - 1);
    start = min(max(a.starts[b], 0), a.tokens);
    const int next = min(max(a.starts[b + 1], 0), a.tokens);
    n = b0 + lane < a.batch ? max(next - start, 0) : 0;
    tiles = (int)(((int64_t)n * a.group + per - 1) / per);
    return (int)wave_incl_scan((uint32_t)tiles, 0u, OpAdd{});
  };
  *split = 0;
  if (a.splits > 1) {
    int all = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) all += __builtin_amdgcn_readlane(count(b0), 63);
    if (all == 0) return false;
    const int turn = (int)((uint32_t)tile / (uint32_t)all);
    tile -= turn * all;
    *split = a.splits - 1 - turn;
    if (*split < 0) return false;
  }
  int base = 0;                                            // tiles of the sequences before b0
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int end = base + count(b0);
    const uint64_t there = __builtin_amdgcn_ballot_w64(end > tile);
    if (there) {
      const int i = __builtin_ctzll(there);
      t->b = b0 + i;
      t->token0 = __builtin_amdgcn_readlane(start, i);
      t->n = __builtin_amdgcn_readlane(n, i);
      t->rows = t->n * a.group;
      // a sequence's last tiles see most keys: first
      t->row0 = (__builtin_amdgcn_readlane(end, i) - 1 - tile) * per;
      t->len = min(max(a.lens[t->b], 0), a.table_width << a.c.page_log);
      return true;
    }
    base = __builtin_amdgcn_readlane(end, 63);
  }
  return false;
}

// Zeros for the tokens past the last sequence (a padded batch), a row to a
// wavefront; the workgroups share them.
template <typename T>
__device__ __forceinline__ void mx4_rest(const Mx4Attention& a) {
  const int from = min(max(a.starts[a.batch], 0), a.tokens);
  const int lane = threadIdx.x % 64, waves = blockDim.x / 64;
  const int64_t end = (int64_t)a.tokens * a.q_heads, step = (int64_t)gridDim.x * gridDim.y * waves;
  for (int64_t row = (int64_t)from * a.q_heads + (int64_t)workgroup() * waves + threadIdx.x / 64;
       row < end; row += step)
    for (int x = lane; x < a.c.d; x += 64) static_cast<T*>(a.out)[row * a.c.d + x] = (T)0.0f;
}

// ---------------------------------------------------------------- few rows
// mx4_few: up to 16 RT rows of a cache head to a workgroup of NW wavefronts, the
// keys read once.  Memory bounds it: 96 sequences of up to 12,000 keys, one token
// each, eight heads of 128 channels and four query heads to each (bf16), are 638
// MB in 135 us, 4.7 TB/s of the 5.0 to 5.2 that a large copy reaches; the same
// loads with no arithmetic take 123 us and the arithmetic with no loads 103.  What
// is read once does not stay in the L2 (nontemporal: 157 us without).  With 32 rows
// (RT 2) the keys' arithmetic serves both halves: three sequences of 70,000 to
// 100,000 keys in fp16, 284 MB in 82 us, 3.5 TB/s.  There its loads alone take 47 us and
// its arithmetic alone 56, which 1.5 wavefronts a SIMD overlap too little; no part
// stands out (of 82: one of four pieces of a query 75, one of two of a weight 73,
// values not turned 79, no exponentials 80), vector instructions are 50 % of the
// SIMDs' cycles and matrix instructions 25 %.  One step's loads are on their way at a time, of all wavefronts: a
// second set in registers gained nothing (140 us, 84).
//  A wavefront takes 32 keys a step, every NW-th step of the
// workgroup's part of the key axis, straight from memory to registers.
// Lane = 16 h + r.  Keys: the lane has row (key) r of two tiles of 16, channels
// 32 h .. of each 128: an operand as it lies.  Queries: row r, channels 16 h ..
// and 64 + 16 h .. of each 128, which is where the 8-bit operand has the same
// products.  Values: keys 4 h .. 4 h + 3 of both tiles, eight channels (four
// where DT is 64, twice eight where it is 256).  Logits: keys 4 h .. 4 h + 3 of
// both tiles for row r.
template <typename T, int DT, int NW, int RT>
__global__ __launch_bounds__(64 * NW, RT == 2 || DT == 256 || sizeof(T) == 4 ? 2 : 4)
void mx4_few(Mx4Attention a) {
  using Pieces = Mx4Pieces<T>;
  constexpr int NP = Pieces::q, WP = Pieces::w;
  constexpr int KC = DT == 256 ? 2 : 1;                    // products of 128 channels
  constexpr int VC = DT == 256 ? 2 : 1;                    // loads of eight channels
  constexpr int CT = DT / 16, PER = 16 * RT;
  __shared__ float l_o[NW][16][DT + 4];
  __shared__ float l_m[NW][16], l_l[NW][16];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, h = lane / 16, d = a.c.d, groups = a.c.groups;
  mx4_rest<T>(a);
  int head, split;
  RowTile t;
  if (!mx4_place(a, PER, &head, &t, &split)) return;
  const int rows_end = min(t.rows, t.row0 + PER);
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

  // the query rows' operands
  int pos[RT];                                             // a row sees up to pos
  i32x8 q[RT][NP][KC];
  float c[RT];                                             // turns products into log2 units
  int unit0[RT];                                           // scale byte of the first piece
#pragma unroll
  for (int y = 0; y < RT; ++y) {
    const int row = min(t.row0 + 16 * y + r, t.rows - 1);
    const int tok = (int)fdiv((uint32_t)row, a.by_group);
    pos[y] = position(t, tok);
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(t.token0 + tok) * a.ldq +
                  (head * a.group + row - tok * a.group) * a.hsq;
    float f[KC][32];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 128 * k + Pieces::first(h) + Pieces::apart(128) * (i / 2) + 8 * (i % 2);
        float g[8];
        if (ch < d) load_q8(qp + ch, a.q_vec, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f[k][8 * i + e] = ch < d ? g[e] : 0.0f;
          top = max(top, abs_bits(f[k][8 * i + e]));
        }
      }
    const auto s16 = __builtin_amdgcn_permlane16_swap(top, top, false, false);
    top = max(s16[0], s16[1]);
    const auto s32 = __builtin_amdgcn_permlane32_swap(top, top, false, false);
    const float big = __uint_as_float(max(s32[0], s32[1]));
    const int shift = mx4_shift<T>(big);
    // (never 0: hidden logits are -inf times it)
    c[y] = fmaxf(ldexpf(a.scale * 1.4426950408889634f, -shift), 0x1p-126f);
    // a row that is not finite has a scale that is no number: so is all that it meets
    unit0[y] = big < __builtin_inff() ? 127 : kMx4Bad;
#pragma unroll
    for (int k = 0; k < KC; ++k) {
#pragma unroll
      for (int e = 0; e < 32; ++e) f[k][e] = ldexpf(f[k][e], shift);
#pragma unroll
      for (int n = 0; n < NP; ++n) q[y][n][k] = query_piece<T>(f[k], n);
    }
  }

  const int32_t* table = a.table + (int64_t)t.b * a.table_width;
  const int lg = a.c.page_log, in_page = (1 << lg) - 1, n_pages = (int)(a.c.slots >> lg);
  int page[2];                                             // of the two tiles of 16 keys
  auto pages = [&](int j) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      page[u] = mx4_page(table, min(j + 16 * u, hi - 1) >> lg);
  };
  // the lane's bytes in a tile: groups past the last meet zeros in q, channels past it are not
  // stored
  uint32_t k_at[KC], s_at[KC], v_at[VC], u_at[VC];
#pragma unroll
  for (int k = 0; k < KC; ++k) {
    const int g = 4 * k + h < groups ? 4 * k + h : 0;
    k_at[k] = (uint32_t)(r * 16 * groups + 16 * g);
    s_at[k] = (uint32_t)(r * groups + g);
  }
#pragma unroll
  for (int k = 0; k < VC; ++k) {
    int i = DT == 64 ? r / 2 : r + 16 * k;                 // which eight channels
    if (i >= 4 * groups) i = 0;
    v_at[k] = (uint32_t)((h * 4 * groups + i) * 16);
    u_at[k] = (uint32_t)((h * groups + i / 4) * 4);
  }
  f32x4 o[RT][CT];
  float m[RT], l[RT];                                      // m: in log2 units
#pragma unroll
  for (int y = 0; y < RT; ++y) {
    m[y] = kNegInf;
    l[y] = 0.0f;
#pragma unroll
    for (int x = 0; x < CT; ++x) o[y][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // what a lane has of a step's 32 keys
  struct Keys {
    i32x4 kr[2][KC];
    u32x4 vr[2][VC];
    uint32_t ks[2][KC], vs[2][VC];
    bool ok[2];
  };
  auto fetch = [&](Keys& g, int j) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      g.ok[u] = (uint32_t)page[u] < (uint32_t)n_pages;
      // no page: any rows, which are masked
      const int64_t row0 = (((int64_t)(g.ok[u] ? page[u] : 0) * a.c.heads + head) << lg) +
                           ((j + 16 * u) & in_page);
      const int64_t g0 = row0 * groups;
      // scalar bases and the lane's own 32-bit offsets (opaque: added up outside the loop they
      // would be a 64-bit sum for each load)
      const uint8_t *kp = a.c.k + 16 * g0, *sp = a.c.ks + g0, *vp = a.c.v + 16 * g0,
                    *up = a.c.vs + g0;
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        g.kr[u][k] = __builtin_nontemporal_load(
            reinterpret_cast<const i32x4*>(kp + (uint32_t)opaque_int((int)k_at[k])));
        g.ks[u][k] = sp[(uint32_t)opaque_int((int)s_at[k])];
      }
#pragma unroll
      for (int k = 0; k < VC; ++k) {
        g.vr[u][k] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(vp + (uint32_t)opaque_int((int)v_at[k])));
        g.vs[u][k] =
            *reinterpret_cast<const uint32_t*>(up + (uint32_t)opaque_int((int)u_at[k]));
      }
    }
  };
  auto use = [&](Keys& g, int j) __attribute__((always_inline)) {
    float x[RT][8];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int y = 0; y < RT; ++y) {
        f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < KC; ++k) {
          const i32x8 kf = {g.kr[u][k][0], g.kr[u][k][1], g.kr[u][k][2], g.kr[u][k][3], 0, 0, 0, 0};
#pragma unroll
          for (int n = NP - 1; n >= 0; --n)
            s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                kf, q[y][n][k], s, kFp4, Pieces::format, 0, (int)g.ks[u][k], 0,
                n == 0 ? unit0[y] : 127 + Pieces::unit(n));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[y][4 * u + i] = s[i];
      }
    // values that were not finite: NaN to whoever sees them, in the weight
    bool any_bad = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) any_bad = any_bad || has_bad(g.vs[u][0]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(any_bad) != 0, 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (byte_of(g.vs[i / 4][0], i % 4) == kMx4Bad)
#pragma unroll
          for (int y = 0; y < RT; ++y) x[y][i] = __uint_as_float(0x7FC00000u);
    }
    // hidden keys: past the row's position (the last part's end), before its window, no page
    if (j + 31 > pos0 || j < see1 || !g.ok[0] || !g.ok[1] ||
        __builtin_amdgcn_ballot_w64(any_bad) != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = j + 16 * (i / 4) + 4 * h + i % 4;
#pragma unroll
        for (int y = 0; y < RT; ++y) {
          const int see = a.window > 0 ? pos[y] - a.window + 1 : 0;
          if (key > pos[y] || key < see || !g.ok[i / 4]) x[y][i] = kNegInf;
        }
        // what no row sees may hold anything: a weight of 0 needs a finite value beside it (and
        // NaN rows have codes of 0)
        const uint32_t keep = 0xFFu << (8 * (i % 4));
#pragma unroll
        for (int k = 0; k < VC; ++k)
          if (byte_of(g.vs[i / 4][k], i % 4) > (uint32_t)(kMx4Most + 127))
            g.vs[i / 4][k] = (g.vs[i / 4][k] & ~keep) | (0x7F7F7F7Fu & keep);
      }
    }
    constexpr int VF = RT == 1 ? 1 : VC;                   // decoded at once
    bf16x8 vf[VF][CT / VC];
    auto decode = [&](int k) __attribute__((always_inline)) {
      uint32_t v[8];
      float scale[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = g.vr[i / 4][k][i % 4];
        if (DT == 64) v[i] >>= 16 * (r % 2);               // its four of the eight channels
        scale[i] = power_of_two((int)byte_of(g.vs[i / 4][k], i % 4));
      }
      bf16x8(&to)[CT / VC] = vf[k % VF];
      values_across<0>(v, scale, *reinterpret_cast<bf16x8(*)[2]>(&to[0]));
      values_across<1>(v, scale, *reinterpret_cast<bf16x8(*)[2]>(&to[2]));
      if constexpr (DT > 64) {
        values_across<2>(v, scale, *reinterpret_cast<bf16x8(*)[2]>(&to[4]));
        values_across<3>(v, scale, *reinterpret_cast<bf16x8(*)[2]>(&to[6]));
      }
    };
    if constexpr (RT > 1) {                                // beside the logits' products
#pragma unroll
      for (int k = 0; k < VC; ++k) decode(k);
    }
    // The maximum that a row's weights are relative to rises only where a lane's own logits are
    // more than 4 (2^2) above it; only then do the lanes of a row need one another's.
    bool rise = false;
    float top[RT];
#pragma unroll
    for (int y = 0; y < RT; ++y) {
      top[y] = max3(max3(x[y][0], x[y][1], x[y][2]), max3(x[y][3], x[y][4], x[y][5]),
                    max3(x[y][6], x[y][7], x[y][7]));
      rise = rise || top[y] * c[y] > m[y] + kSlack;
    }
    if (__builtin_amdgcn_ballot_w64(rise)) {
#pragma unroll
      for (int y = 0; y < RT; ++y) {
        const float now = fmaxf(m[y], reduce_x16_x32(top[y], FMax{}) * c[y]);
        const float f = now == kNegInf ? 1.0f : exp2_fast(m[y] - now);
        l[y] *= f;
#pragma unroll
        for (int z = 0; z < CT; ++z) o[y][z] *= f;
        m[y] = now;
      }
    }
    bf16x8 p[RT][WP];
#pragma unroll
    for (int y = 0; y < RT; ++y) {
      const float base = m[y] == kNegInf ? 0.0f : m[y];
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = exp2_fast(fmaf(x[y][i], c[y], -base));
      weight_pieces<WP>(w, p[y]);
      l[y] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    }
#pragma unroll
    for (int k = 0; k < VC; ++k) {
      if constexpr (RT == 1) decode(k);
#pragma unroll
      for (int z = 0; z < CT / VC; ++z)
#pragma unroll
        for (int y = 0; y < RT; ++y)
#pragma unroll
          for (int n = WP - 1; n >= 0; --n)
            o[y][8 * k + z] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                vf[k % VF][z], p[y][n], o[y][8 * k + z], 0, 0, 0);
    }
  };
  Keys g;
  if (wave < steps) pages(j0 + 32 * wave);
  for (int step = wave; step < steps; step += NW) {
    const int j = j0 + 32 * step;
    fetch(g, j);
    if (step + NW < steps) pages(j + 32 * NW);
    use(g, j);
  }

  // the wavefronts' sums, joined in order, 16 rows at a time
  constexpr int PL = DT == 64 ? 4 : 8;                     // channels of a lane that lie together
#pragma unroll
  for (int y = 0; y < RT; ++y) {
    if (y > 0) __syncthreads();
    const float sum = reduce_x16_x32(l[y], FAdd{});
    if (h == 0) {
      l_m[wave][r] = m[y];
      l_l[wave][r] = sum;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < CT; x += 4)
        *reinterpret_cast<f32x4*>(&l_o[wave][r][x / PL * 128 + (4 * h + i) * PL + x % PL]) =
            f32x4{o[y][x][i], o[y][x + 1][i], o[y][x + 2][i], o[y][x + 3][i]};
    __syncthreads();
    few_out<T>(a, l_o, l_m, l_l, t, rows_end, head, split);
    t.row0 += 16;
  }
}

// ---------------------------------------------------------------- many rows
// mx4_many: 128 rows of a cache head to a workgroup of four wavefronts, 32 rows
// each, 64 keys a step, two buffers (Mx4Places).  Keys' codes go to LDS as they
// are; values are turned to bf16 and transposed once for all four wavefronts.
// The next step's values are turned beside the logits' products, and the loads for
// the step after that are then on their way under the rest of the arithmetic; one
// barrier a step.  W <= DT: channels of values that are computed, d rounded up to
// 32.  WHOLE: a page holds a step's 64 keys, so that all its addresses are scalar.
// Both pipelines bound it: 5 sequences of 2,000 new tokens over up to 6,096 keys,
// 32 query heads on eight of 128 channels (bf16), 555 GFLOP in 711 to 763 us (four
// cards), 0.73 to 0.78 PFLOP/s of the 1.17 to 1.25 that a large bf16 product reaches,
// whose operands have one piece; fp16 793 to 815, fp32 1,080 to 1,106.  Matrix
// instructions are 53 % of the SIMDs' cycles and vector instructions 60 %, at 1.8
// wavefronts a SIMD.
// Measured with one piece of weights: 558 us, 42 and 52 % of the cycles.  Values
// turned by half of the wavefronts before the products, and each operand read
// right before its product: 610 us.  From there: with an eighth of the logits'
// products 531, with a quarter of the values' 544, both 472; without exponentials
// 561, without turning values 555, without loads 529.  The next step's logits formed
// beside this step's weights, with keys two steps ahead, took 657; a higher wave
// priority during the products 640.  Where pages are shorter than a step: 700 tokens
// of four sequences over 2,700 keys, the same heads, 182 us at pages of 32 and 196
// of 16 (169 where they are not).  Registers spill in <float, 256> (38, 68 where
// pages are shorter), <fp16, 256> and <fp16, 128> (13 and 4, shorter pages alone)
// and <float, 96> (2); in none for bf16.
// Lane = 32 h + r.  Logits (32 keys x 32 rows): keys 8 y + 4 h .. +3 (y = 0..3) of
// row r.  So a lane's eight weights of 16 keys are those at 4 h .. and 8 + 4 h ..,
// and the values' chunk g = 2 s + h of a channel holds just the keys 16 s + 4 h ..
// +3 and 16 s + 8 + 4 h .. +3: two blocks of four tokens of the cache.
// Queries: row r, channels 16 h .. and 32 + 16 h .. of each 64.
template <int DT>
struct Mx4Lds {                                            // bytes
  using Place = Mx4Places<DT>;
  static constexpr int k = 0;                              // [2][64][DT / 2] codes
  static constexpr int v = 2 * Place::key_bytes;           // [2][DT][64] bf16
  static constexpr int ks = v + 2 * Place::value_bytes;    // [2][words][64] scale bytes
  static constexpr int mask = ks + 2 * Place::words * 256; // [2] keys without a page, NaN values
  static constexpr int bytes = mask + 32;
};

constexpr int kVector = 0x2, kProducts = 0x8, kLdsReads = 0x100;   // kinds of instructions

template <typename T, int W, bool WHOLE>
__global__ __launch_bounds__(256, W > 128 ? 1 : 2) void mx4_many(Mx4Attention a) {
  constexpr int DT = W <= 64 ? 64 : W <= 128 ? 128 : 256;
  using Pieces = Mx4Pieces<T>;
  constexpr int NP = Pieces::q, WP = Pieces::w;
  constexpr int KS = (W + 63) / 64, CT = W / 32;
  using At = Mx4Lds<DT>;
  using Place = Mx4Places<DT>;
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int r = lane % 32, h = lane / 32, d = a.c.d, groups = a.c.groups;
  mx4_rest<T>(a);
  int head, split;
  RowTile t;
  if (!mx4_place(a, 128, &head, &t, &split)) return;
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

  i32x8 q[NP][KS];
  float c;                                                 // turns products into log2 units
  int unit0;                                               // scale byte of the first piece
  {
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(t.token0 + tok) * a.ldq + qh * a.hsq;
    float f[KS][32];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 64 * k + Pieces::first(h) + Pieces::apart(64) * (i / 2) + 8 * (i % 2);
        float g[8];
        load_q8(qp + (ch < d ? ch : 0), a.q_vec, g);       // all loads before the first use
#pragma unroll
        for (int e = 0; e < 8; ++e) f[k][8 * i + e] = g[e];
      }
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        if (64 * k + Pieces::first(h) + Pieces::apart(64) * (i / 16) + 8 * (i / 8 % 2) >= d)
          f[k][i] = 0.0f;
        top = max(top, abs_bits(f[k][i]));
      }
    const auto s32 = __builtin_amdgcn_permlane32_swap(top, top, false, false);
    const float big = __uint_as_float(max(s32[0], s32[1]));
    const int shift = mx4_shift<T>(big);
    // (never 0: hidden logits are -inf times it)
    c = fmaxf(ldexpf(a.scale * 1.4426950408889634f, -shift), 0x1p-126f);
    // a row that is not finite has a scale that is no number: so is all that it meets
    unit0 = big < __builtin_inff() ? 127 : kMx4Bad;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
#pragma unroll
      for (int e = 0; e < 32; ++e) f[k][e] = ldexpf(f[k][e], shift);
#pragma unroll
      for (int n = 0; n < NP; ++n) q[n][k] = query_piece<T>(f[k], n);
    }
  }

  // staging: pieces of keys tid, tid + 256, ..; a unit of values to SHARE threads, CH of its eight
  // channels each; wavefront 3 has a key's scales and marks to a lane
  const int32_t* table = a.table + (int64_t)t.b * a.table_width;
  const int lg = a.c.page_log, in_page = (1 << lg) - 1, n_pages = (int)(a.c.slots >> lg);
  constexpr int PIECES = (64 * Place::KC + 255) / 256;
  const bool has_keys = tid < 64 * Place::KC;              // (DT 64: half of them)
  constexpr int SHARE = 256 / DT, CH = 8 / SHARE;          // threads to a unit, channels of each
  const int unit = tid % DT, v_part = tid / DT;
  const int piece_key = Place::piece_key(tid);
  // offsets from the first key of the step where one page holds it all, else of the block of 16
  const uint32_t k_off = (uint32_t)((WHOLE ? piece_key : piece_key % 16) * 16 * groups +
                                    (tid % Place::KC < groups ? 16 * (tid % Place::KC) : 0));
  const int v_chunk = Place::unit_chunk(unit), v_eight = Place::unit_channels(unit);
  const int v_i = v_eight < 4 * groups ? v_eight : 0;
  const int v_four = (WHOLE ? v_chunk / 2 * 4 : 0) + v_chunk % 2;   // block of four tokens
  const uint32_t v_off = (uint32_t)((v_four * 4 * groups + v_i) * 16);
  const uint32_t u_off = (uint32_t)((v_four * groups + v_i / 4) * 4);
  const int s_key = WHOLE ? lane : lane % 16;
  const uint32_t s_off = (uint32_t)(s_key * groups);
  const uint32_t m_off = (uint32_t)(s_key / 4 * 4 * groups + lane % 4);
  i32x4 kr[PIECES];
  u32x4 vr[2];
  uint32_t vs[2], ks[Place::words], kb[3];
  uint32_t key_v = 0;                                      // a value scale of key `lane`
  bool key_ok = false;
  int page[4];
  auto pages = [&](int j) {
#pragma unroll
    for (int b = 0; b < (WHOLE ? 1 : 4); ++b)
      page[b] = mx4_page(table, min(j + 16 * b, hi - 1) >> lg);
  };
  auto page_of = [&](int b) {                              // of the step's block of 16 keys b
    return b == 0 ? page[0] : b == 1 ? page[1] : b == 2 ? page[2] : page[3];
  };
  // first row of block b times the row's groups; a page outside the cache: any rows, hidden
  auto block_groups = [&](int pg, int j, int b) {
    return ((((int64_t)((uint32_t)pg < (uint32_t)n_pages ? pg : 0) * a.c.heads + head) << lg) +
            ((j + 16 * b) & in_page)) * groups;
  };
  auto fetch_scales = [&](int pg, int64_t g0) __attribute__((always_inline)) {   // key `lane`
    const uint8_t* sp = a.c.ks + g0 + s_off;
    // (nothing is computed from them here: that would wait)
#pragma unroll
    for (int n = 0; n < Place::words; ++n)
      if (groups >= 4 * n + 4) __builtin_memcpy(&ks[n], sp + 4 * n, 4);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < groups % 4) kb[i] = sp[groups / 4 * 4 + i];
    key_ok = (uint32_t)pg < (uint32_t)n_pages;
    key_v = a.c.vs[g0 + m_off];
  };
  auto fetch_values = [&](int64_t g0) __attribute__((always_inline)) {
    const uint8_t* vp = a.c.v + 16 * g0 + v_off;
    const uint8_t* up = a.c.vs + g0 + u_off;
    vr[0] = *reinterpret_cast<const u32x4*>(vp);
    vr[1] = *reinterpret_cast<const u32x4*>(vp + 128 * groups);
    vs[0] = *reinterpret_cast<const uint32_t*>(up);
    vs[1] = *reinterpret_cast<const uint32_t*>(up + 8 * groups);
  };
  auto fetch = [&](int j) __attribute__((always_inline)) {
    if constexpr (WHOLE) {                                 // one page: scalar addresses
      const int64_t g0 = block_groups(page[0], j, 0);
      const uint8_t* kp = a.c.k + 16 * g0;
      if (has_keys) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
          kr[p] = *reinterpret_cast<const i32x4*>(kp + p * (256 / Place::KC * 16) * groups + k_off);
      }
      fetch_values(g0);
      if (wave == 3) fetch_scales(page[0], g0);
      return;
    }
    if (has_keys) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        // a wavefront's pieces are of one block of 16 keys, of two where DT is 64
        const int b = (piece_key + p * (256 / Place::KC)) / 16;
        const int bu = DT == 64 ? b : __builtin_amdgcn_readfirstlane(b);
        kr[p] = *reinterpret_cast<const i32x4*>(a.c.k + 16 * block_groups(page_of(bu), j, bu) +
                                                k_off);
      }
    }
    fetch_values(block_groups(page_of(v_chunk / 2), j, v_chunk / 2));
    if (wave == 3) {
      const int b = lane / 16, pg = page_of(b);
      fetch_scales(pg, block_groups(pg, j, b));
    }
  };
  int k_put[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) k_put[p] = At::k + Place::piece_put(tid + 256 * p);
  // (its channels from CH v_part on: the turn of their rows is that of the first, xor the channel)
  const int v_row = At::v + Place::unit_row(unit) + CH * v_part * 128;
  const int v_bits = Place::unit_bits(unit) ^ 16 * CH * v_part;
  auto stage_values = [&](auto par) {                      // buffer par
    constexpr int P = decltype(par)::value;
    const int bits = opaque_int(v_bits);                   // (eight addresses, not eight registers)
    uint32_t v[8];
    float scale[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = vr[i / 4][i % 4];
      if (SHARE > 1) v[i] >>= 4 * CH * v_part;
      // what no row sees may hold anything: a weight of 0 needs a finite value beside it (and
      // NaN rows have codes of 0)
      scale[i] = power_of_two((int)min(byte_of(vs[i / 4], i % 4), (uint32_t)(kMx4Most + 127)));
    }
    auto put = [&](auto b) {
      constexpr int B = decltype(b)::value;
      bf16x8 o[2];
      values_across<B>(v, scale, o);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<bf16x8*>(smem + P * Place::value_bytes +
                                   Place::value_put(v_row, bits, 2 * B + e)) = o[e];
    };
    put(std::integral_constant<int, 0>{});
    if constexpr (CH > 2) put(std::integral_constant<int, 1>{});
    if constexpr (CH > 4) put(std::integral_constant<int, 2>{});
    if constexpr (CH > 4) put(std::integral_constant<int, 3>{});
  };
  auto stage_keys = [&](auto par) {
    constexpr int P = decltype(par)::value;
    if (has_keys) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
        *reinterpret_cast<i32x4*>(smem + P * Place::key_bytes + k_put[p]) = kr[p];
    }
    if (wave == 3) {
#pragma unroll
      for (int n = 0; n < Place::words; ++n) {
        uint32_t w = 0x7F7F7F7Fu;                          // groups that there are not
        if (groups >= 4 * n + 4) {
          w = ks[n];
        } else if (groups > 4 * n) {
#pragma unroll
          for (int i = 0; i < 3; ++i)
            if (i < groups % 4) w = (w & ~(0xFFu << 8 * i)) | kb[i] << 8 * i;
        }
        *reinterpret_cast<uint32_t*>(smem + At::ks + (P * Place::words + n) * 256 + 4 * lane) = w;
      }
      const uint64_t hidden = __builtin_amdgcn_ballot_w64(!key_ok);
      const uint64_t bad = __builtin_amdgcn_ballot_w64(key_v == (uint32_t)kMx4Bad);
      if (lane == 0)
        *reinterpret_cast<i32x4*>(smem + At::mask + 16 * P) =
            i32x4{(int)hidden, (int)(hidden >> 32), (int)bad, (int)(bad >> 32)};
    }
  };

  f32x16 o[CT];
#pragma unroll
  for (int x = 0; x < CT; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[x][i] = 0.0f;
  float m = kNegInf, l = 0.0f;                             // m: in log2 units
  int k_at[KS], v_at[4];                                   // the chunks that a lane reads
#pragma unroll
  for (int i = 0; i < KS; ++i) k_at[i] = At::k + Place::key_column(r, h, i);
#pragma unroll
  for (int i = 0; i < 4; ++i) v_at[i] = At::v + Place::value_column(r, h, i);
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  if (steps > 0) {
    pages(j0);
    fetch(j0);
    stage_keys(Even{});
    stage_values(Even{});
    pages(j0 + 64);
    if (steps > 1) fetch(j0 + 64);
    pages(j0 + 128);
  }
  __syncthreads();
  auto advance = [&](auto par, auto other, int step) {
    constexpr int P = decltype(par)::value;
    const int j = j0 + 64 * step;
    stage_keys(other);                                     // (past the last step: not used)
    f32x16 s[2];
    int sa[2][Place::words];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
#pragma unroll
      for (int n = 0; n < Place::words; ++n)
        sa[u][n] = (int)(*reinterpret_cast<const uint32_t*>(
                             smem + At::ks + (P * Place::words + n) * 256 + 4 * (32 * u + r)) >>
                         8 * h);
    }
    i32x4 kc[2][KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        kc[u][k] = *reinterpret_cast<const i32x4*>(smem + P * Place::key_bytes +
                                                   Place::key_at(k_at[k], u));
    stage_values(other);
    auto logits = [&](auto kk) {
      constexpr int K = decltype(kk)::value;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const i32x8 kf = {kc[u][K][0], kc[u][K][1], kc[u][K][2], kc[u][K][3], 0, 0, 0, 0};
#pragma unroll
        for (int n = NP - 1; n >= 0; --n)
          s[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
              kf, q[n][K], s[u], kFp4, Pieces::format, K % 2 * 2, sa[u][K / 2], 0,
              n == 0 ? unit0 : 127 + Pieces::unit(n));
      }
    };
    logits(std::integral_constant<int, 0>{});
    if constexpr (KS > 1) logits(std::integral_constant<int, 1>{});
    if constexpr (KS > 2) logits(std::integral_constant<int, 2>{});
    if constexpr (KS > 3) logits(std::integral_constant<int, 3>{});
    // in this order: reads, the values' scales, and then their conversion beside the products
    __builtin_amdgcn_sched_group_barrier(kLdsReads, 2 * KS + 2 * Place::words, 0);
    __builtin_amdgcn_sched_group_barrier(kVector, 24, 0);
#pragma unroll
    for (int i = 0; i < 2 * KS * NP; ++i) {
      __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kVector, 8, 0);
    }
    asm volatile("" : "+v"(s[0]), "+v"(s[1]));             // (the products stay before the loads)
    if (step + 2 < steps) {
      fetch(j + 128);
      pages(j + 192);
    }
    const i32x4 marks = *reinterpret_cast<const i32x4*>(smem + At::mask + 16 * P);
    if (__builtin_expect(
            __builtin_amdgcn_readfirstlane(marks[0] | marks[1] | marks[2] | marks[3]) != 0, 0)) {
      // (bits of constants in the lane's own words: a bit of its own for each key would be 32 pairs
      // of registers, kept through the loop)
      uint32_t word[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) word[i] = (uint32_t)marks[i] >> opaque_int(4 * h);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int key = Place::logit_key(0, i);
        if (word[2 + key / 32] >> key % 32 & 1) s[i / 16][i % 16] = __uint_as_float(0x7FC00000u);
        if (word[key / 32] >> key % 32 & 1) s[i / 16][i % 16] = kNegInf;
      }
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
    float top = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
    for (int i = 3; i < 31; i += 2)
      top = max3(top, s[i / 16][i % 16], s[(i + 1) / 16][(i + 1) % 16]);
    top = fmaxf(top, s[1][15]);
    top = fmaxf(m, reduce_x32(top, FMax{}) * c);
    if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
      const float f = top == kNegInf ? 1.0f : exp2_fast(m - top);
      l *= f;
#pragma unroll
      for (int y = 0; y < CT; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[y][i] *= f;
      m = top;
    }
    const float base = m == kNegInf ? 0.0f : m;
    // Operands of values and weights are formed a product ahead, where registers hold two of each
    // (fp32, four sequences of 700 new tokens and 2,700 keys, ahead | not: 128 channels, of which
    // 256 registers do not, 193 | 167 us, 192 channels 324 | 335, 256 498 | 509).
    constexpr bool AHEAD = WP < 3 || W != 128;
    constexpr int SETS = AHEAD ? 2 : 1;
    bf16x8 vf[SETS][CT], p[SETS][WP];
    auto values = [&](int v) __attribute__((always_inline)) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        vf[v % SETS][ct] = *reinterpret_cast<const bf16x8*>(
            smem + P * Place::value_bytes + Place::value_at(v_at[Place::column_of(v, ct)], ct));
    };
    auto weights = [&](int v) __attribute__((always_inline)) {
      float w[8];
#pragma unroll
      for (int y = 0; y < 8; ++y)
        w[y] = exp2_fast(fmaf(s[v / 2][v % 2 * 8 + y], c, -base));
      weight_pieces<WP>(w, p[v % SETS]);
      l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    };
    if (AHEAD) {
      values(0);
      weights(0);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (!AHEAD) {
        weights(v);
        values(v);
      } else if (v < 3) {
        values(v + 1);
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int n = WP - 1; n >= 0; --n)
          o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[v % SETS][ct], p[v % SETS][n], o[ct],
                                                          0, 0, 0);
      if (AHEAD && v < 3) weights(v + 1);
    }
    if constexpr (AHEAD) {                                 // in this order
      constexpr int each = WP == 2 ? 44 : 64;   // instructions to form weights
      __builtin_amdgcn_sched_group_barrier(kLdsReads, CT, 1);
      __builtin_amdgcn_sched_group_barrier(kVector, each, 1);
#pragma unroll
      for (int v = 0; v < 3; ++v) {
        __builtin_amdgcn_sched_group_barrier(kLdsReads, CT, 1);
#pragma unroll
        for (int i = 0; i < CT * WP; ++i) {
          __builtin_amdgcn_sched_group_barrier(kProducts, 1, 1);
          __builtin_amdgcn_sched_group_barrier(kVector, each / (CT * WP), 1);
        }
      }
      __builtin_amdgcn_sched_group_barrier(kProducts, CT * WP, 1);
    }
    __syncthreads();
  };
  for (int step = 0; step < steps; step += 2) {
    advance(Even{}, Odd{}, step);
    if (step + 1 < steps) advance(Odd{}, Even{}, step + 1);
  }
  l = reduce_x32(l, FAdd{});
  if (row >= rows_end) return;
  const int64_t ro = (int64_t)(t.token0 + tok) * a.q_heads + qh;
  const bool part = a.splits > 1;
  const int64_t po = (int64_t)split * a.tokens * a.q_heads + ro;
  if (part && h == 0) a.part_ml[po] = float2{m, l};
  const float inv = part ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
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

}  // namespace cs
