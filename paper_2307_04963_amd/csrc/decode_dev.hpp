// Device helpers of the decoding operators: 16 bytes of a row at a time, and the way from a token's place to its page.
#pragma once

#include "decode.hpp"
#include "token_dev.hpp"

namespace dycl {
namespace k {

// What a lane moves at a time: 16 bytes of values
template <bool F32>
constexpr int kWide = F32 ? 4 : 8;

// N consecutive values (8 of bf16, 4 of either) from any element on; only the first `count` of fewer
// are read (the others are 0)
template <bool F32, int N>
__device__ __forceinline__ void read_values(const void* p, int count, float* f) {
  static_assert(F32 ? N == 4 : N == 8, "16 bytes");
  if (count >= N) {
    const uint4 a = load16(p);
    const uint32_t e[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (F32) {
        f[j] = __uint_as_float(e[j]);
      } else {
        f[2 * j] = __uint_as_float(e[j] << 16);
        f[2 * j + 1] = __uint_as_float(e[j] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      f[j] = 0.f;
      if (j < count) f[j] = F32 ? static_cast<const float*>(p)[j] : bf2f(static_cast<const uint16_t*>(p)[j]);
    }
  }
}

template <bool F32, int N>
__device__ __forceinline__ void write_values(void* p, int count, const float* f) {
  typedef uint32_t bits64 __attribute__((ext_vector_type(2), aligned(2)));
  if (count >= N) {
    if constexpr (F32)
      store16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
    else if constexpr (N == 8)
      store16(p, make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])));
    else
      *static_cast<bits64*>(p) = bits64{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
  } else {
#pragma unroll
    for (int j = 0; j < N - 1; ++j) {
      if (j >= count) continue;
      if constexpr (F32)
        static_cast<float*>(p)[j] = f[j];
      else
        static_cast<uint16_t*>(p)[j] = f2bf(f[j]);
    }
  }
}

// N values, 4 to 16 bytes of them, to any element
template <bool F32, int N>
__device__ __forceinline__ void put_values(void* p, const float* f) {
  constexpr int WORDS = F32 ? N : N / 2;
  typedef uint32_t words __attribute__((ext_vector_type(WORDS), aligned(2)));
  words w;
#pragma unroll
  for (int i = 0; i < WORDS; ++i) w[i] = F32 ? __float_as_uint(f[i]) : pack_bf16(f[F32 ? i : 2 * i], f[F32 ? i : 2 * i + 1]);
  *static_cast<words*>(p) = w;
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
