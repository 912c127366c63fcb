// Attention of new tokens over the paged int8 cache: token i of sequence b,
// at position p = len_b - n_b + i, has o = sum_j e_j v_j / sum_j e_j with
// e_j = exp(scale * q.k_j - m) over the positions j in (p - window, p].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8_rows.h"

namespace cs {

struct PagedAttention {
  CacheView c;
  const void* q;
  int64_t ldq, hsq;
  int tokens, q_heads, batch;
  const int32_t* table;
  int table_width;
  const int32_t* lens;
  const int32_t* starts;
  float scale;
  int window;          // 0: none
  void* out;
};

// The sequence that new token t belongs to: the last b with starts[b] <= t,
// `batch` for tokens past the last sequence.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int batch, int t) {
  int lo = 0, hi = batch;                                  // starts[lo] <= t < starts[hi + 1]
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (starts[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// One wavefront to a (token, query head): 64 keys at a time, a key to a lane
// for the logits, then d / 64 channels to a lane for the values.
template <typename T>
__global__ __launch_bounds__(256) void attention_row(PagedAttention a) {
  __shared__ float lq[4][256];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, d = a.c.d;
  const int64_t item = (int64_t)blockIdx.x * 4 + wave;
  if (item >= (int64_t)a.tokens * a.q_heads) return;
  const int t = (int)(item / a.q_heads), head = (int)(item % a.q_heads);
  const int kv = head / (a.q_heads / a.c.heads);
  const T* q = static_cast<const T*>(a.q) + t * a.ldq + head * a.hsq;
  for (int i = lane; i < d; i += 64) lq[wave][i] = to_f32(q[i]) * a.scale;
  wave_lds_order();
  const int b = sequence_of(a.starts, a.batch, t);
  int pos = -1;
  if (b < a.batch) {
    const int len = min(max(a.lens[b], 0), a.table_width << a.c.page_log);
    pos = len - (a.starts[b + 1] - t);
  }
  const int first = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  float m = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int j0 = first; j0 <= pos; j0 += 64) {
    const int j = j0 + lane;
    float s = -INFINITY, sv = 0.0f;
    int64_t at = 0;
    if (j <= pos) {
      const int page = a.table[(int64_t)b * a.table_width + (j >> a.c.page_log)];
      const int64_t slot = ((int64_t)page << a.c.page_log) | (j & ((1 << a.c.page_log) - 1));
      if (slot >= 0 && slot < a.c.slots) {
        at = cache_row(a.c, slot, kv);
        float dot = 0.0f;
        for (int i = 0; i < d; ++i) dot += lq[wave][i] * (float)a.c.k[at * d + i];
        s = dot * a.c.ks[at];
        sv = a.c.vs[at];
      }
    }
    float top = s;
    for (int x = 32; x > 0; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
    const float mn = fmaxf(m, top);
    const float base = mn == -INFINITY ? 0.0f : mn;
    const float e = s == -INFINITY ? 0.0f : expf(s - base), r = expf(m - base);
    float sum = e;
    for (int x = 32; x > 0; x /= 2) sum += __shfl_xor(sum, x);
    l = l * r + sum;
    m = mn;
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] *= r;
    const float pv = s == -INFINITY ? 0.0f : e * sv;
    for (int x = 0; x < 64; ++x) {
      const float p = __shfl(pv, x);
      const int64_t row = __shfl(at, x);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (lane + 64 * u < d) o[u] += p * (float)a.c.v[row * d + lane + 64 * u];
    }
  }
  T* y = static_cast<T*>(a.out) + item * d;
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (lane + 64 * u < d) y[lane + 64 * u] = (T)(l == 0.0f ? 0.0f : o[u] / l);
}

}  // namespace cs
