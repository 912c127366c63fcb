// Rows of floats to 4-bit codes with a power of two for every 32 channels, and
// the paged cache of keys and values that holds them.
//
// A group's scale is the least 2^E with max|x| <= 7 * 2^E (so that the largest
// code, 6, is never further off than half its step), E within [-60, 60]: sums
// of products of such values stay inside 32-bit floats.  Codes are the nearest
// of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code, with a sign: the
// matrix cores' own 4-bit form, which the conversion instruction rounds to.  A
// row that is not finite gets scale bytes 255 and codes 0.
//
// Layout: keys lie token by token, which is how the matrix instructions read
// them; values in blocks of four tokens, so that a lane of the attention
// kernels has four tokens' eight channels in one load of 16 bytes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastdiv.h"
#include "q8_rows.h"
#include "wave_ops.h"

namespace cs {

struct Mx4View {
  uint8_t* k;
  uint8_t* v;
  uint8_t* ks;
  uint8_t* vs;
  int64_t slots;      // pages * page
  int heads, page_log, d;
  int groups;         // of 32 channels
};

constexpr int kMx4Bad = 255, kMx4Least = -60, kMx4Most = 60;

// Index of (slot, head) among the cache's rows; a page's rows start at a
// multiple of 16, so row / 4 and row % 4 are a block of values and its token.
__device__ __forceinline__ int64_t mx4_row(const Mx4View& c, int64_t slot, int head) {
  const int64_t page = slot >> c.page_log;
  return (((page * c.heads + head) << c.page_log) | (slot & ((1 << c.page_log) - 1)));
}

// E of a group whose largest magnitude has these bits (finite): 1.75 * 2^e is
// the last that 7 * 2^(e - 2) holds.
__device__ __forceinline__ int mx4_exponent(uint32_t top) {
  const int e = (int)((top + 0x1FFFFFu) >> 23) - 129;
  return min(max(e, kMx4Least), kMx4Most);
}

__device__ __forceinline__ float power_of_two(int byte) {  // 2^(byte - 127), 1 to 254
  return __uint_as_float((uint32_t)byte << 23);
}

__device__ __forceinline__ uint32_t mx4_codes8(const float (&f)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
  return w;
}

// mx4_write and mx4_read: a row (token, head) to 16 lanes, eight channels a
// lane (two times eight past 128 channels), keys and values by blockIdx.z.  The
// four rows of a wavefront are four tokens of one head, so that its stores of
// new tokens' values, which share a block as a rule, are whole.  Memory bounds
// both: 16,384 tokens of eight heads of 128 channels in fp16 are written in 24 us
// (67 MB read and 18 written, 3.5 TB/s) and 32,768 read back in 38 (36 MB and 134,
// 4.5 TB/s); 48 tokens take 3 us either way, the time of a launch.  A lane of
// mx4_write has one load on its way, and that only once its token's slot has come:
// without the slots 17 us where it takes 19.4 (inputs in the last-level cache; bf16 the
// same, fp32 23.2 either way), with the rows' loads before the slots' test 17.5.
struct Mx4Row {
  int64_t token;
  int head;
};
__device__ __forceinline__ Mx4Row mx4_item(const FastDiv& by_heads) {
  const uint32_t item = workgroup() * 4 + threadIdx.x / 64;            // four tokens of a head
  const uint32_t four = fdiv(item, by_heads);
  return {(int64_t)four * 4 + threadIdx.x % 64 / 16, (int)(item - four * by_heads.d)};
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void mx4_write(Mx4View c, const T* __restrict__ k, int64_t ldk,
                                                 int64_t hsk, const T* __restrict__ v, int64_t ldv,
                                                 int64_t hsv, const int64_t* __restrict__ slots,
                                                 int64_t tokens, FastDiv by_heads) {
  const Mx4Row row = mx4_item(by_heads);
  if (row.token >= tokens) return;                         // whole groups of 16 lanes leave
  const int64_t slot = slots[row.token];
  if (slot < 0 || slot >= c.slots) return;
  const int lane = threadIdx.x % 16;
  const bool val = blockIdx.z != 0;
  const T* x = val ? v + row.token * ldv + row.head * hsv : k + row.token * ldk + row.head * hsk;
  float f[2][8];
  uint32_t top[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int ch = 8 * (lane + 16 * j);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[j][e] = 0.0f;
    if (ch < c.d) {
      if (VEC) load8(x + ch, f[j]);
      else load8_some(x + ch, 8, f[j]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) top[j] = max(top[j], abs_bits(f[j][e]));
    // the four lanes of a group
    top[j] = max(top[j], (uint32_t)__builtin_amdgcn_update_dpp((int)top[j], (int)top[j], 0xB1, 0xf,
                                                               0xf, false));
    top[j] = max(top[j], (uint32_t)__builtin_amdgcn_update_dpp((int)top[j], (int)top[j], 0x4E, 0xf,
                                                               0xf, false));
  }
  const bool bad = row16_reduce(max(top[0], top[1]), OpMax{}) >= 0x7F800000u;
  const int64_t at = mx4_row(c, slot, row.head);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = lane + 16 * j, g = i / 4;
    if (g >= c.groups) continue;
    const int byte = bad ? kMx4Bad : mx4_exponent(top[j]) + 127;
    const uint32_t w = bad ? 0u : mx4_codes8(f[j], power_of_two(byte));
    uint8_t *q, *s;
    if (val) {
      q = c.v + ((at / 4 * (4 * c.groups) + i) * 16 + at % 4 * 4);
      s = c.vs + ((at / 4 * c.groups + g) * 4 + at % 4);
    } else {
      q = c.k + (at * (16 * c.groups) + 4 * i);
      s = c.ks + (at * c.groups + g);
    }
    *reinterpret_cast<uint32_t*>(q) = w;
    if (i % 4 == 0) *s = (uint8_t)byte;
  }
}

// Values code * scale, rounded once; a slot outside the cache reads as zeros.
template <typename T>
__global__ __launch_bounds__(256) void mx4_read(Mx4View c, const int64_t* __restrict__ slots,
                                                int64_t tokens, FastDiv by_heads,
                                                T* __restrict__ k, T* __restrict__ v) {
  const Mx4Row row = mx4_item(by_heads);
  if (row.token >= tokens) return;
  const int lane = threadIdx.x % 16;
  const int64_t slot = slots[row.token];
  const bool val = blockIdx.z != 0, in = slot >= 0 && slot < c.slots;
  const int64_t at = in ? mx4_row(c, slot, row.head) : 0;
  T* y = (val ? v : k) + (row.token * c.heads + row.head) * c.d;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = lane + 16 * j, g = i / 4;
    if (8 * i >= c.d) continue;
    uint32_t w = 0, byte = 127;
    if (in) {
      w = *reinterpret_cast<const uint32_t*>(
          val ? c.v + ((at / 4 * (4 * c.groups) + i) * 16 + at % 4 * 4)
              : c.k + (at * (16 * c.groups) + 4 * i));
      byte = val ? c.vs[(at / 4 * c.groups + g) * 4 + at % 4] : c.ks[at * c.groups + g];
    }
    const float s = byte == kMx4Bad ? __uint_as_float(0x7FC00000u) : power_of_two((int)byte);
    float f[8];
    const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
    const auto p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const auto p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
    const auto p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    f[0] = p0[0] * s; f[1] = p0[1] * s; f[2] = p1[0] * s; f[3] = p1[1] * s;
    f[4] = p2[0] * s; f[5] = p2[1] * s; f[6] = p3[0] * s; f[7] = p3[1] * s;
    store8(y + 8 * i, f);
  }
}

}  // namespace cs
