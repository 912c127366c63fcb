// y[t][n] = (sum_k x[t][k] w[n][k]) * (sx[t] * sw[n]) + bias[n] for int8 x and
// w: the sum in int32 (exact: k <= 131,072), one rounding to y's type.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8_rows.h"

namespace cs {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct Q8Linear {
  const int8_t* x;
  int64_t ldx;
  const float* sx;
  int64_t rows;
  int k;
  const int8_t* w;
  int64_t ldw;
  const float* sw;
  int d_out;
  const float* bias;
  void* y;
  int64_t ldy;
};

// 16 codes of a row from element e on; those past k read as 0.  ALIGNED: rows
// start on 16 bytes, so whole pieces are one load.
template <bool ALIGNED>
__device__ __forceinline__ i32x4 codes16(const int8_t* row, int e, int k) {
  if (ALIGNED && e + 16 <= k) return *reinterpret_cast<const i32x4*>(row + e);
  i32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (e + i < k) v[i / 4] |= (int)((uint32_t)(uint8_t)row[e + i] << (8 * (i % 4)));
  return v;
}

// A 64 x 64 tile of y to a workgroup of four wavefronts, 32 x 32 each, 64
// codes of k a step through LDS.
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void linear_q8_tile(Q8Linear a) {
  constexpr int kLd = 64 + 16;                             // a row's bytes in LDS, padded
  __shared__ __align__(16) int8_t lx[64 * kLd], lw[64 * kLd];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int64_t t0 = (int64_t)blockIdx.y * 64;
  const int n0 = blockIdx.x * 64;
  const int sr = tid / 4, sc = tid % 4 * 16;               // the piece this thread stages
  const int64_t xt = min(t0 + sr, a.rows - 1);
  const int wn = min(n0 + sr, a.d_out - 1);
  const int8_t* xr = a.x + xt * a.ldx;
  const int8_t* wr = a.w + (int64_t)wn * a.ldw;
  const int tr = wave / 2 * 32, nc = wave % 2 * 32;
  const int fr = lane % 32, fk = lane / 32 * 16;
  i32x16 acc = {};
  for (int k0 = 0; k0 < a.k; k0 += 64) {
    const i32x4 vx = codes16<ALIGNED>(xr, k0 + sc, a.k);
    const i32x4 vw = codes16<ALIGNED>(wr, k0 + sc, a.k);
    __syncthreads();
    *reinterpret_cast<i32x4*>(lx + sr * kLd + sc) = vx;
    *reinterpret_cast<i32x4*>(lw + sr * kLd + sc) = vw;
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 64; kk += 32)
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(
          *reinterpret_cast<const i32x4*>(lx + (tr + fr) * kLd + kk + fk),
          *reinterpret_cast<const i32x4*>(lw + (nc + fr) * kLd + kk + fk), acc, 0, 0, 0);
  }
  const int n = n0 + nc + lane % 32;
  if (n >= a.d_out) return;
  const float s = a.sw[n], b = a.bias ? a.bias[n] : 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t t = t0 + tr + 8 * (i / 4) + 4 * (lane / 32) + i % 4;
    if (t < a.rows)
      static_cast<T*>(a.y)[t * a.ldy + n] = (T)((float)acc[i] * (a.sx[t] * s) + b);
  }
}

}  // namespace cs
