// Attention of new tokens over the paged 4-bit cache: token i of sequence b,
// at position p = len_b - n_b + i, has o = sum_j e_j v_j / sum_j e_j with
// e_j = exp(scale * q.k_j) over the positions j in (p - window, p].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx4_rows.h"
#include "q8_attention.h"

namespace cs {

typedef PagedAttentionOf<Mx4View> Mx4Attention;

// Eight codes as floats.
__device__ __forceinline__ void mx4_values8(uint32_t w, float s, float (&f)[8]) {
  const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
  const auto p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
  const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
  const auto p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
  f[0] = p0[0] * s; f[1] = p0[1] * s; f[2] = p1[0] * s; f[3] = p1[1] * s;
  f[4] = p2[0] * s; f[5] = p2[1] * s; f[6] = p3[0] * s; f[7] = p3[1] * s;
}
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
  return byte == kMx4Bad ? __uint_as_float(0x7FC00000u) : power_of_two((int)byte);
}

// A row (token, query head) to a wavefront, 64 keys a step, a key to a lane for
// the logits, up to four channels to a lane for the values.
template <typename T>
__global__ __launch_bounds__(64) void mx4_attention_row(Mx4Attention a) {
  __shared__ float l_q[256];
  __shared__ float l_w[64];
  __shared__ int64_t l_row[64];
  const int lane = threadIdx.x, d = a.c.d, groups = a.c.groups;
  int head, tile, split;
  if (!place(a, &head, &tile, &split)) return;
  RowTile t;
  if (!find_tile(a, tile, 1, &t)) return;
  const int tok = (int)fdiv((uint32_t)t.row0, a.by_group);
  const int qh = head * a.group + t.row0 - tok * a.group;
  int lo, hi;
  tile_keys(a, t, tok, tok, &lo, &hi);
  const T* qp = static_cast<const T*>(a.q) + (int64_t)(t.token0 + tok) * a.ldq + qh * a.hsq;
  for (int i = lane; i < 256; i += 64) l_q[i] = i < d ? to_f32(qp[i]) : 0.0f;
  __syncthreads();
  const int32_t* table = a.table + (int64_t)t.b * a.table_width;
  const int lg = a.c.page_log, in_page = (1 << lg) - 1;
  float m = kNegInf, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int j0 = lo; j0 < hi; j0 += 64) {
    const int j = j0 + lane;
    const int32_t page = j < hi ? table[j >> lg] : -1;
    const bool ok = (uint32_t)page < (uint32_t)(a.c.slots >> lg);
    float x = kNegInf;
    int64_t at = -1;
    if (ok) {
      at = mx4_row(a.c, ((int64_t)page << lg) + (j & in_page), head);
      x = 0.0f;
      for (int i = 0; i < 4 * groups; ++i) {
        float f[8];
        mx4_values8(*reinterpret_cast<const uint32_t*>(a.c.k + at * 16 * groups + 4 * i),
                    mx4_scale(a.c.ks[at * groups + i / 4]), f);
        for (int e = 0; e < 8; ++e) x = fmaf(f[e], l_q[8 * i + e], x);
      }
      x *= a.scale * 1.4426950408889634f;
    }
    float top = fmaxf(x, m);
    for (int s = 32; s > 0; s /= 2) top = fmaxf(top, __shfl_xor(top, s));
    const float base = top == kNegInf ? 0.0f : top;
    const float f = exp2_fast(m - base);
    const float w = exp2_fast(x - base);
    float sum = w;
    for (int s = 32; s > 0; s /= 2) sum += __shfl_xor(sum, s);
    l = l * f + sum;
    m = top;
    l_w[lane] = w;
    l_row[lane] = at;
    __syncthreads();
    for (int c = 0; c < 4; ++c) o[c] *= f;
    for (int i = 0; i < 64; ++i) {
      const int64_t r = l_row[i];
      if (r < 0) continue;
      for (int c = 0; c < 4; ++c) {
        const int ch = lane + 64 * c;
        if (ch >= d) continue;
        const uint32_t byte = a.c.v[(r / 4 * (4 * groups) + ch / 8) * 16 + r % 4 * 4 + ch % 8 / 2];
        float v[8];
        mx4_values8(byte, mx4_scale(a.c.vs[(r / 4 * groups + ch / 32) * 4 + r % 4]), v);
        o[c] = fmaf(l_w[i], ch % 2 ? v[1] : v[0], o[c]);
      }
    }
    __syncthreads();
  }
  T* y = static_cast<T*>(a.out) + ((int64_t)(t.token0 + tok) * a.q_heads + qh) * d;
  for (int c = 0; c < 4; ++c)
    if (lane + 64 * c < d) y[lane + 64 * c] = (T)(l == 0.0f ? 0.0f : o[c] / l);
}

}  // namespace cs
