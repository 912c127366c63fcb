// Rows of floats to int8 codes with a 32-bit scale each, and the paged cache
// of keys and values that holds them.
//
// A row's scale is s = fl32(max|x| / 127) and a code rne(fl32(x / s)) (fl32:
// rounded to 32 bits), so that equal inputs give equal codes whoever computes
// them.  A row of zeros has scale 0 and codes 0.  A row with an infinity or a
// NaN has scale NaN and codes 0: what is computed from that row is NaN, and
// no other row is touched.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cs.h"
#include "fastdiv.h"
#include "wave_ops.h"

namespace cs {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The number of a workgroup.  A dimension of a launch takes less than 2^32
// threads (more are cut to their low 32 bits): workgroups past 2^22 are spread
// over grid rows of that many (wide_grid), and those past the last have no work.
constexpr int kGridRow = 22;
__device__ __forceinline__ uint32_t workgroup() {
  return (blockIdx.y << kGridRow) + blockIdx.x;
}
inline dim3 wide_grid(int64_t workgroups) {
  const int64_t row = (int64_t)1 << kGridRow;
  return workgroups <= row ? dim3((unsigned)workgroups)
                           : dim3((unsigned)row, (unsigned)((workgroups + row - 1) / row));
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

// Eight elements as floats: two or one 16-byte loads (p 16-byte aligned), or
// one element at a time, those from `n` on as 0.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&f)[8]) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p);
    const f32x4 b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[4 + i] = b[i]; }
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    const t8 a = *reinterpret_cast<const t8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = to_f32(a[i]);
  }
}
// The same where p is aligned to ALIGN bytes only.
template <int ALIGN, typename T>
__device__ __forceinline__ void load8_at(const T* p, float (&f)[8]) {
  T t[8];
  __builtin_memcpy(t, __builtin_assume_aligned(p, ALIGN), sizeof(t));
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = to_f32(t[i]);
}
template <typename T>
__device__ __forceinline__ void load8_some(const T* p, int n, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = i < n ? to_f32(p[i]) : 0.0f;
}

// |x| as bits: ordered as numbers, infinity above all of them, NaN above that.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

struct RowScale {
  float s;      // as stored
  float div;    // as divided by: infinity where every code is 0
  float inv;
};

__device__ __forceinline__ RowScale row_scale(uint32_t amax) {
  RowScale r;
  r.s = amax >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : __uint_as_float(amax) / 127.0f;
  const bool live = r.s > 0.0f;
  r.div = live ? r.s : __uint_as_float(0x7F800000u);
  r.inv = live ? 1.0f / r.s : 0.0f;
  return r;
}

// rne(fl32(x / s)).  x * (1/s) is within 2^-22 of the quotient, relatively,
// which is at most 127: only a product within 1e-4 of half way between two
// codes (or one that is not a number, s being too small to have a
// reciprocal) needs the division, about twelve instructions, and few
// wavefronts take that branch.
__device__ __forceinline__ int row_code(float x, const RowScale& r) {
  const float y = x * r.inv;
  float c = rintf(y);
  if (!(fabsf(y - c) < 0.4999f)) {
    c = rintf(x / r.div);
    c = c == c ? fminf(fmaxf(c, -127.0f), 127.0f) : 0.0f;
  }
  return (int)c;
}

__device__ __forceinline__ u32x2 row_codes8(const float (&f)[8], const RowScale& r) {
  u32x2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w |= ((uint32_t)row_code(f[4 * h + i], r) & 0xFFu) << (8 * i);
    out[h] = w;
  }
  return out;
}

// quantise_rows: WPR wavefronts to a row, 4 / WPR rows to a workgroup of 256.
// The row's first 64 * WPR * kRowHeld vectors of eight elements stay in
// registers between the maximum and the codes, so rows up to 8,192 elements
// (WPR 4; WPR 1 takes up to 1,024) are read once; longer rows' rest is read twice.
// Bound by memory: 8,192 rows of 4,096 bf16 (101 MB) in 18.6 us, 5.4 TB/s, a
// large copy's rate; 777 rows of 1,500 bf16 in 3.8 us, latency.
constexpr int kRowHeld = 4;

// ALIGN: rows start on 16 bytes, on 4, or anywhere.
template <typename T, int ALIGN, int WPR>
__global__ __launch_bounds__(256) void quantise_rows(const T* __restrict__ x, int64_t ldx,
                                                     int64_t rows, int c, int8_t* __restrict__ q,
                                                     int64_t ldq, float* __restrict__ scale) {
  constexpr int kLanes = 64 * WPR;
  __shared__ uint32_t part[4];
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int64_t row = (int64_t)workgroup() * (4 / WPR) + group;
  const bool live = row < rows;
  const T* xr = x + (live ? row : 0) * ldx;
  const int nv = live ? c / 8 + (c % 8 != 0) : 0;          // (c + 7 may pass 2^31)
  auto fetch = [&](int v, float (&f)[8]) {
    if (c - 8 * v >= 8) load8_at<ALIGN>(xr + 8 * (int64_t)v, f);
    else load8_some(xr + 8 * (int64_t)v, c - 8 * v, f);
  };
  float f[kRowHeld][8];
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < kRowHeld; ++j) {
    const int v = lane + kLanes * j;
    if (v < nv) {
      fetch(v, f[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = max(amax, abs_bits(f[j][i]));
    }
  }
  for (int v = lane + kLanes * kRowHeld; v < nv; v += kLanes) {
    float g[8];
    fetch(v, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, abs_bits(g[i]));
  }
  amax = wave_max_u32(amax);
  if (WPR > 1) {
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = amax;
    __syncthreads();
    amax = max(max(part[0], part[1]), max(part[2], part[3]));
  }
  if (!live) return;
  const RowScale rs = row_scale(amax);
  if (lane == 0) scale[row] = rs.s;
  int8_t* qr = q + row * ldq;
  const bool wide = (reinterpret_cast<uintptr_t>(qr) & 7) == 0;
  auto put = [&](int v, const float (&g)[8]) {
    const u32x2 w = row_codes8(g, rs);
    if (wide && c - 8 * v >= 8) {
      *reinterpret_cast<u32x2*>(qr + 8 * (int64_t)v) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < c - 8 * v) qr[8 * (int64_t)v + i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
    }
  };
#pragma unroll
  for (int j = 0; j < kRowHeld; ++j)
    if (lane + kLanes * j < nv) put(lane + kLanes * j, f[j]);
  for (int v = lane + kLanes * kRowHeld; v < nv; v += kLanes) {
    float g[8];
    fetch(v, g);
    put(v, g);
  }
}

// ---------------------------------------------------------------- the cache
// Page number and offset of a slot; slots outside the cache are left out.
struct CacheView {
  int8_t* k;
  int8_t* v;
  float* ks;
  float* vs;
  int64_t slots;      // pages * page
  int heads, page_log, d;
};

// Index of (slot, head) among the cache's rows of d codes (and its scales).
__device__ __forceinline__ int64_t cache_row(const CacheView& c, int64_t slot, int head) {
  const int64_t page = slot >> c.page_log;
  return (((page * c.heads + head) << c.page_log) | (slot & ((1 << c.page_log) - 1)));
}

// cache_write and cache_read: a row (token, head) to 16 lanes, 16 rows to a
// workgroup, keys and values by blockIdx.z.  A lane has every 16th vector of
// eight elements, at most two of them (d <= 256): 16 lanes are the most that
// d = 128, the usual size, has 16-byte vectors for, and their maximum takes
// four register moves.  Bound by memory: 16,384 tokens of 8 heads of 128 f16
// written (102 MB) in 23.9 us, 4.3 TB/s; 32,768 read (205 MB) in 37.2 us, 5.5
// TB/s.  48 tokens: 3.4 and 2.8 us, latency.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void cache_write(CacheView c, const T* __restrict__ k,
                                                   int64_t ldk, int64_t hsk,
                                                   const T* __restrict__ v, int64_t ldv,
                                                   int64_t hsv, const int64_t* __restrict__ slots,
                                                   uint32_t rows, FastDiv by_heads) {
  const uint32_t row = workgroup() * 16 + threadIdx.x / 16;
  if (row >= rows) return;                                 // whole groups of 16 lanes leave
  const int lane = threadIdx.x % 16;
  const uint32_t token = fdiv(row, by_heads);
  const int head = (int)(row - token * by_heads.d);
  const int64_t slot = slots[token];
  if (slot < 0 || slot >= c.slots) return;
  const bool val = blockIdx.z != 0;
  const T* x = val ? v + token * ldv + head * hsv : k + token * ldk + head * hsk;
  const int nv = c.d / 8;
  float f[2][8];
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = lane + 16 * j;
    if (i < nv) {
      if (VEC) load8(x + 8 * i, f[j]);
      else load8_some(x + 8 * i, 8, f[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = max(amax, abs_bits(f[j][e]));
    }
  }
  amax = row16_reduce(amax, OpMax{});
  const RowScale rs = row_scale(amax);
  const int64_t at = cache_row(c, slot, head);
  if (lane == 0) (val ? c.vs : c.ks)[at] = rs.s;
  int8_t* q = (val ? c.v : c.k) + at * c.d;
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (lane + 16 * j < nv)
      *reinterpret_cast<u32x2*>(q + 8 * (lane + 16 * j)) = row_codes8(f[j], rs);
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
  if constexpr (sizeof(T) == 4) {
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = f[i]; b[i] = f[4 + i]; }
    *reinterpret_cast<f32x4*>(p) = a;
    *reinterpret_cast<f32x4*>(p + 4) = b;
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (T)f[i];
    *reinterpret_cast<t8*>(p) = a;
  }
}

// Values code * scale, rounded once; a slot outside the cache reads as zeros.
template <typename T>
__global__ __launch_bounds__(256) void cache_read(CacheView c, const int64_t* __restrict__ slots,
                                                  uint32_t rows, FastDiv by_heads,
                                                  T* __restrict__ k, T* __restrict__ v) {
  const uint32_t row = workgroup() * 16 + threadIdx.x / 16;
  if (row >= rows) return;
  const int lane = threadIdx.x % 16;
  const uint32_t token = fdiv(row, by_heads);
  const int head = (int)(row - token * by_heads.d);
  const int64_t slot = slots[token];
  const bool val = blockIdx.z != 0, in = slot >= 0 && slot < c.slots;
  const int64_t at = in ? cache_row(c, slot, head) : 0;
  const float s = in ? (val ? c.vs : c.ks)[at] : 0.0f;
  const int8_t* q = (val ? c.v : c.k) + at * c.d;
  T* y = (val ? v : k) + (int64_t)row * c.d;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = lane + 16 * j;
    if (8 * i >= c.d) continue;
    u32x2 w = {0u, 0u};
    if (in) w = *reinterpret_cast<const u32x2*>(q + 8 * i);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)(int8_t)(w[e / 4] >> (8 * (e % 4))) * s;
    store8(y + 8 * i, f);
  }
}

}  // namespace cs
