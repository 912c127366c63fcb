// Attention of new tokens over the paged 4-bit cache: token i of sequence b,
// at position p = len_b - n_b + i, has o = sum_j e_j v_j / sum_j e_j with
// e_j = exp(scale * q.k_j) over the positions j in (p - window, p].
//
// Rows (new token, query head), tiles of rows, parts of the key axis and the
// places of workgroups are those of the 8-bit cache's kernels.  What differs:
//  - Keys are never converted: the matrix cores multiply 4-bit codes, with a
//    power of two for every 32 channels, as the cache holds both.  The other
//    operand is 8 bits wide (e4m3, four significant bits), so a query row is the
//    sum of pieces, each what the ones before leave, 2^-4 of them in size: two
//    pieces hold bf16 in full, three fp16, six fp32.  A row is first scaled by a
//    power of two so that its largest element lies in [2^7, 2^8); an element's
//    last piece ends at 2^-9 of its unit (e4m3's smallest step), so N pieces
//    leave 2^(-6 - 4 N) ... 2^-21 of the largest element for N = 2.
//  - Values go to bf16, exactly, by the scaled conversion, and meet weights
//    e_j = 2^(x_j - m) in bf16 pieces: two (16 bits), three for fp32.  bf16 has
//    the exponents of 32-bit floats, and the cache's scales end at 2^60, so no
//    sum over 2^30 positions overflows and weights need no scaling.
//  - The running maximum m follows the rows' maximum only when that is more
//    than 4 (2^2) above it: rescaling is rare.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx4_rows.h"
#include "q8_attention.h"

namespace cs {

typedef PagedAttentionOf<Mx4View> Mx4Attention;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float out_unit(const Mx4View&) { return 1.0f; }

constexpr int kFp8 = 0, kFp4 = 4;                          // operand formats

template <typename T>
struct Mx4Pieces {                                         // of a query, of a weight
  static constexpr int q = sizeof(T) == 4 ? 6 : sizeof(T) == 2 ? 3 : 0, w = sizeof(T) == 4 ? 3 : 2;
};
template <>
struct Mx4Pieces<__bf16> {
  static constexpr int q = 2, w = 2;
};

// 32 elements as an operand, bytes in order; f becomes 16 times what they leave.
__device__ __forceinline__ i32x8 e4m3_piece(float (&f)[32]) {
  i32x8 out;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], w, true);
    out[i] = w;
    f[4 * i] = 16.0f * (f[4 * i] - __builtin_amdgcn_cvt_f32_fp8(w, 0));
    f[4 * i + 1] = 16.0f * (f[4 * i + 1] - __builtin_amdgcn_cvt_f32_fp8(w, 1));
    f[4 * i + 2] = 16.0f * (f[4 * i + 2] - __builtin_amdgcn_cvt_f32_fp8(w, 2));
    f[4 * i + 3] = 16.0f * (f[4 * i + 3] - __builtin_amdgcn_cvt_f32_fp8(w, 3));
  }
  return out;
}

// Eight weights as operands; each piece is what the ones before leave.
template <int NW>
__device__ __forceinline__ void weight_pieces(const float (&w)[8], bf16x8 (&p)[NW]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float v = w[j];
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      p[n][j] = (__bf16)v;
      v -= (float)p[n][j];
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

// Whether one of a dword's bytes is 255.
__device__ __forceinline__ bool has_bad(uint32_t w) {
  return ((~w - 0x01010101u) & w & 0x80808080u) != 0;
}
__device__ __forceinline__ uint32_t byte_of(uint32_t w, int i) { return w >> (8 * i) & 0xFFu; }

// ---------------------------------------------------------------- few rows
// mx4_few: up to 16 rows of a cache head to a workgroup of NW wavefronts, the
// keys read once.  A wavefront takes 32 keys a step, every NW-th step of the
// workgroup's part of the key axis, straight from memory to registers.
// Lane = 16 h + r.  Keys: the lane has row (key) r of two tiles of 16, channels
// 32 h .. of each 128: an operand as it lies.  Queries: row r, channels 16 h ..
// and 64 + 16 h .. of each 128, which is where the 8-bit operand has the same
// products.  Values: keys 4 h .. 4 h + 3 of both tiles, eight channels (four
// where DT is 64, twice eight where it is 256).  Logits: keys 4 h .. 4 h + 3 of
// both tiles for row r.
template <typename T, int DT, int NW>
__global__ __launch_bounds__(64 * NW, DT == 256 || sizeof(T) == 4 ? 2 : 4)
void mx4_few(Mx4Attention a) {
  constexpr int NP = Mx4Pieces<T>::q, WP = Mx4Pieces<T>::w;
  constexpr int KC = DT == 256 ? 2 : 1;                    // products of 128 channels
  constexpr int VC = DT == 256 ? 2 : 1;                    // loads of eight channels
  constexpr int CT = DT / 16;
  __shared__ float l_o[NW][16][DT + 4];
  __shared__ float l_m[NW][16], l_l[NW][16];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane % 16, h = lane / 16, d = a.c.d, groups = a.c.groups;
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
  const int end = hi;                                      // no row sees what is from here on
  // this workgroup's part
  const int j0 = lo / 32 * 32 + split * a.chunk;
  if (split + 1 < a.splits) hi = min(hi, j0 + a.chunk);
  const int steps = hi > j0 ? (hi - j0 + 31) / 32 : 0;

  // the query rows' operand
  const int row = min(t.row0 + r, t.rows - 1);
  const int tok = (int)fdiv((uint32_t)row, a.by_group);
  const int pos = position(t, tok);                        // the row sees up to pos
  i32x8 q[NP][KC];
  float c;                                                 // turns products into log2 units
  {
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(t.token0 + tok) * a.ldq +
                  (head * a.group + row - tok * a.group) * a.hsq;
    float f[KC][32];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 128 * k + 64 * (i / 2) + 16 * h + 8 * (i % 2);
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
    const bool bad = !(big < __builtin_inff());
    const int ex = bad || big == 0.0f ? 0 : __builtin_amdgcn_frexp_expf(big);
    c = ldexpf(a.scale * 1.4426950408889634f, ex - 8);
#pragma unroll
    for (int k = 0; k < KC; ++k) {
#pragma unroll
      for (int e = 0; e < 32; ++e)
        f[k][e] = bad ? __uint_as_float(0x7FC00000u) : ldexpf(f[k][e], 8 - ex);
#pragma unroll
      for (int n = 0; n < NP; ++n) q[n][k] = e4m3_piece(f[k]);
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
  f32x4 o[CT];
#pragma unroll
  for (int x = 0; x < CT; ++x) o[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = kNegInf, l = 0.0f;
  if (wave < steps) pages(j0 + 32 * wave);
  for (int step = wave; step < steps; step += NW) {
    const int j = j0 + 32 * step;
    i32x4 kr[2][KC];
    u32x4 vr[2][VC];
    uint32_t ks[2][KC], vs[2][VC];
    bool ok[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ok[u] = (uint32_t)page[u] < (uint32_t)n_pages;
      // no page: any rows, which are masked
      const int64_t row0 = (((int64_t)(ok[u] ? page[u] : 0) * a.c.heads + head) << lg) +
                           ((j + 16 * u) & in_page);
      const int64_t g0 = row0 * groups;
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        kr[u][k] = *reinterpret_cast<const i32x4*>(a.c.k + 16 * g0 + k_at[k]);
        ks[u][k] = *(a.c.ks + g0 + s_at[k]);
      }
#pragma unroll
      for (int k = 0; k < VC; ++k) {
        vr[u][k] = *reinterpret_cast<const u32x4*>(a.c.v + 16 * g0 + v_at[k]);
        vs[u][k] = *reinterpret_cast<const uint32_t*>(a.c.vs + g0 + u_at[k]);
      }
    }
    if (step + NW < steps) pages(j + 32 * NW);
    float x[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < KC; ++k) {
        const i32x8 kf = {kr[u][k][0], kr[u][k][1], kr[u][k][2], kr[u][k][3], 0, 0, 0, 0};
#pragma unroll
        for (int n = NP - 1; n >= 0; --n)
          s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, q[n][k], s, kFp4, kFp8, 0,
                                                               (int)ks[u][k], 0, 127 - 4 * n);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * u + i] = s[i] * c;
    }
    // values that were not finite: NaN to whoever sees them, in the weight
    bool any_bad = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) any_bad = any_bad || has_bad(vs[u][0]);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(any_bad) != 0, 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (byte_of(vs[i / 4][0], i % 4) == kMx4Bad) x[i] = __uint_as_float(0x7FC00000u);
    }
    // hidden keys: past the row's position (the last part's end), before its window, no page
    if (j + 31 > pos0 || j < see1 || !ok[0] || !ok[1] ||
        __builtin_amdgcn_ballot_w64(any_bad) != 0) {
      const int see = a.window > 0 ? pos - a.window + 1 : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = j + 16 * (i / 4) + 4 * h + i % 4;
        if (key > pos || key < see || !ok[i / 4]) x[i] = kNegInf;
        // what no row sees may hold anything: a weight of 0 needs a finite value beside it
        const uint32_t keep = 0xFFu << (8 * (i % 4));
#pragma unroll
        for (int k = 0; k < VC; ++k)
          if (key >= end || !ok[i / 4] || byte_of(vs[i / 4][k], i % 4) == kMx4Bad)
            vs[i / 4][k] = (vs[i / 4][k] & ~keep) | (0x7F7F7F7Fu & keep);
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
    const float base = m == kNegInf ? 0.0f : m;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = exp2_fast(x[i] - base);
    bf16x8 p[WP];
    weight_pieces<WP>(w, p);
    l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
#pragma unroll
    for (int k = 0; k < VC; ++k) {
      uint32_t v[8];
      float scale[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = vr[i / 4][k][i % 4];
        if (DT == 64) v[i] >>= 16 * (r % 2);               // its four of the eight channels
        scale[i] = power_of_two((int)byte_of(vs[i / 4][k], i % 4));
      }
      auto products = [&](auto b) {
        constexpr int B = decltype(b)::value;
        bf16x8 vf[2];
        values_across<B>(v, scale, vf);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int n = WP - 1; n >= 0; --n)
            o[8 * k + 2 * B + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                vf[e], p[n], o[8 * k + 2 * B + e], 0, 0, 0);
      };
      products(std::integral_constant<int, 0>{});
      products(std::integral_constant<int, 1>{});
      if constexpr (DT > 64) {
        products(std::integral_constant<int, 2>{});
        products(std::integral_constant<int, 3>{});
      }
    }
  }

  // the wavefronts' sums, joined in order
  l = reduce_x16_x32(l, FAdd{});
  if (h == 0) {
    l_m[wave][r] = m;
    l_l[wave][r] = l;
  }
  constexpr int PL = DT == 64 ? 4 : 8;                     // channels of a lane that lie together
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int x = 0; x < CT; x += 4)
      *reinterpret_cast<f32x4*>(&l_o[wave][r][x / PL * 128 + (4 * h + i) * PL + x % PL]) =
          f32x4{o[x][i], o[x + 1][i], o[x + 2][i], o[x + 3][i]};
  __syncthreads();
  few_out<T>(a, l_o, l_m, l_l, t, rows_end, head, split);
}

}  // namespace cs
