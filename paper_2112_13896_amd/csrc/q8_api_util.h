// What the C entry points of the attention-layer operators check and choose by.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "cs.h"

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

// f(integral_constant) with the width of the kernels' registers for d channels.
template <typename F>
void with_width(int d, F f) {
  if (d <= 64) f(std::integral_constant<int, 64>{});
  else if (d <= 128) f(std::integral_constant<int, 128>{});
  else f(std::integral_constant<int, 256>{});
}

}  // namespace
