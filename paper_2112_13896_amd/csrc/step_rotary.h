// Rotary positions: pairs of a head's channels turned by position * frequency.
//
// An angle is a 64-bit fraction of a turn: the product of the position and
// round(f / (2 pi) 2^64) modulo 2^64 is the angle modulo a turn, with no
// rounding but the frequency's own, so positions in the millions are as good as
// the first ones.  What is left after the nearest quarter turn, at most pi / 4,
// goes through the Taylor series of sine and cosine (to x^9 and x^10: next
// terms below 2^-28 of the result).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastdiv.h"
#include "q8_rows.h"

namespace cs {

struct RotaryPart {                    // one of the two tensors
  const void* x;
  void* y;
  int64_t ldx, hsx, ldy, hsy;
};

struct Rotary {
  RotaryPart part[2];
  const uint64_t* turns;
  const int32_t* positions;
  int64_t tokens;
  int heads0, heads;                   // heads of the first tensor, of both
  int d, rot, copied;                  // channels from rot on to copy (0 where y is x)
  float amplitude;
  int inverse;
  int per;                             // tokens of a workgroup
  int parts;                           // workgroups that share their heads
  FastDiv by_units, by_heads, by_parts;   // units of a head, heads, parts
};

// cos and sin of 2 pi frac / 2^64, times amplitude.
__device__ __forceinline__ float2 turn_of(uint64_t frac, float amplitude) {
  const uint32_t quarter = (uint32_t)((frac + (1ull << 61)) >> 62);
  const int64_t rest = (int64_t)(frac - ((uint64_t)quarter << 62));     // [-2^61, 2^61)
  const float x = (float)rest * (float)(6.283185307179586 / 18446744073709551616.0);
  const float z = x * x;
  float s = fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f);
  s = fmaf(z, s, 1.0f / 120.0f);
  s = fmaf(z, s, -1.0f / 6.0f);
  s = fmaf(x * z, s, x);
  float c = fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f);
  c = fmaf(z, c, -1.0f / 720.0f);
  c = fmaf(z, c, 1.0f / 24.0f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.0f);
  const float co = quarter & 1 ? s : c, si = quarter & 1 ? c : s;
  return float2{amplitude * (quarter == 1 || quarter == 2 ? -co : co),
                amplitude * (quarter >= 2 ? -si : si)};
}

template <typename T, int N>
struct RotaryVec {
  typedef T type __attribute__((ext_vector_type(N)));
};

// rotary: a workgroup has `per` tokens and, of `parts` shares of their units,
// one.  Cosines and sines of the tokens are formed once, in LDS, for all heads.
// A unit is N pairs of a head, or N channels from rot on to copy: N elements
// are 16 bytes (8 where pairs are neighbours: N / 2 pairs), or one pair.  Memory
// bounds it: 16,384 tokens of 40 heads of 128 channels in bf16, 336 MB, 65 us,
// 5.2 TB/s, as fast as a large copy; one token 2.4 us, the time of a launch.
template <typename T, int N, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rotary(Rotary a) {
  extern __shared__ __align__(16) float2 l_turn[];         // [per][rot / 2]
  const uint32_t id = workgroup(), group = fdiv(id, a.by_parts);
  const int part = (int)(id - group * a.by_parts.d);
  const int64_t first = (int64_t)group * a.per;
  if (first >= a.tokens) return;
  const int n = (int)min((int64_t)a.per, a.tokens - first), half = a.rot / 2;
  for (int i = threadIdx.x; i < n * half; i += 256) {
    const int token = i / half;
    const int32_t p = a.positions[first + token];
    const uint64_t f = a.turns[i - token * half] * (uint64_t)(uint32_t)max(p, 0);
    l_turn[i] = turn_of(a.inverse ? 0 - f : f, a.amplitude);
  }
  __syncthreads();
  const int units = (int)a.by_units.d;
  constexpr int P = NEIGHBOURS ? (N > 1 ? N / 2 : 1) : N;  // pairs of a unit
  const int turned = half / P;
  for (int i = part * 256 + threadIdx.x; i < n * a.heads * units; i += a.parts * 256) {
    const uint32_t row = fdiv((uint32_t)i, a.by_units);
    const int unit = i - (int)row * units;
    const uint32_t token = fdiv(row, a.by_heads);
    int head = (int)(row - token * a.by_heads.d);
    const RotaryPart& q = a.part[head >= a.heads0];
    if (head >= a.heads0) head -= a.heads0;
    const T* x = static_cast<const T*>(q.x) + (first + token) * q.ldx + head * q.hsx;
    T* y = static_cast<T*>(q.y) + (first + token) * q.ldy + head * q.hsy;
    const bool none = a.positions[first + token] < 0;
    typedef typename RotaryVec<T, N>::type V;
    if (unit >= turned) {                                  // copied
      const int at = a.rot + (unit - turned) * N;
      *reinterpret_cast<V*>(y + at) = *reinterpret_cast<const V*>(x + at);
      continue;
    }
    const float2* turn = l_turn + token * half + unit * P;
    if constexpr (NEIGHBOURS && N > 1) {
      const V u = *reinterpret_cast<const V*>(x + unit * N);
      V w;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        const float2 t = turn[e];
        const float x1 = to_f32(u[2 * e]), x2 = to_f32(u[2 * e + 1]);
        w[2 * e] = (T)(x1 * t.x - x2 * t.y);
        w[2 * e + 1] = (T)(x2 * t.x + x1 * t.y);
      }
      *reinterpret_cast<V*>(y + unit * N) = none ? u : w;
    } else {
      const int at1 = NEIGHBOURS ? 2 * unit : unit * N, at2 = NEIGHBOURS ? at1 + 1 : at1 + half;
      const V u1 = *reinterpret_cast<const V*>(x + at1);
      const V u2 = *reinterpret_cast<const V*>(x + at2);
      V w1, w2;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 t = turn[e];
        const float x1 = to_f32(u1[e]), x2 = to_f32(u2[e]);
        w1[e] = (T)(x1 * t.x - x2 * t.y);
        w2[e] = (T)(x2 * t.x + x1 * t.y);
      }
      *reinterpret_cast<V*>(y + at1) = none ? u1 : w1;
      *reinterpret_cast<V*>(y + at2) = none ? u2 : w2;
    }
  }
}

}  // namespace cs
