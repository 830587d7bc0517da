// Device helpers of the decoding operators: eight values of a row at a time,
// and the way from a token's place to its page.
#pragma once

#include "decode.hpp"
#include "token_dev.hpp"

namespace dycl {
namespace k {

// 8 consecutive values of bf16 or float32 from any element on; only the first
// `count` of fewer than 8 are read (the others are 0)
template <bool F32>
__device__ __forceinline__ void read8(const void* p, int count, float* f) {
  if (count >= 8) {
    if constexpr (F32) {
      const uint4 a = load16(p), b = load16(static_cast<const char*>(p) + 16);
      const uint32_t e[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(e[j]);
    } else {
      const uint4 a = load16(p);
      const uint32_t e[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(e[j] << 16);
        f[2 * j + 1] = __uint_as_float(e[j] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      f[j] = 0.f;
      if (j < count) f[j] = F32 ? static_cast<const float*>(p)[j] : bf2f(static_cast<const uint16_t*>(p)[j]);
    }
  }
}

template <bool F32>
__device__ __forceinline__ void write8(void* p, int count, const float* f) {
  if (count >= 8) {
    if constexpr (F32) {
      store16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
      store16(static_cast<char*>(p) + 16,
              make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
    } else {
      store16(p, make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 7; ++j) {
      if (j >= count) continue;
      if constexpr (F32)
        static_cast<float*>(p)[j] = f[j];
      else
        static_cast<uint16_t*>(p)[j] = f2bf(f[j]);
    }
  }
}

// the page of place `at` of a sequence's table, or -1
__device__ __forceinline__ int64_t page_of(const PagedArgs& c, int64_t sequence, int64_t at) {
  if (sequence < 0 || sequence >= c.sequences || at < 0) return -1;
  const int64_t i = at >> c.page_shift;
  if (i >= c.max_pages) return -1;
  const int32_t page = c.tables[sequence * c.ldt + i];
  return page >= 0 && page < c.pages ? page : -1;
}

// the first value of a token of a page, in either tensor
__device__ __forceinline__ int64_t token_at(const PagedArgs& c, int64_t page, int head, int64_t slot) {
  return (((page * c.heads + head) << c.page_shift) + slot) * c.dim;
}

}  // namespace k
}  // namespace dycl
